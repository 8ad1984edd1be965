"""Refusals of head norms with rotation, the loss over a vocabulary and AdamW, found on the host
before any work, and their workspaces."""
import ctypes
import math

import pytest

from paper_2406_02052_amd import _lib as L

FAR = [0x100000000000 * (i + 1) for i in range(24)]   # addresses that nothing reads, far apart


def status(call):
    with pytest.raises(L.PetraError) as e:
        call()
    return e.value.name


def heads(batch=2, length=5, h=4, kv=2, dim=64, dtype=L.PETRA_BF16, norm=L.PETRA_NORM_RMS, eps=1e-6, layout=0, pairs=32, axes=1,
          axis=(), freq=(), **strides):
    d = L.HeadsDesc(batch, length, h, kv, dim, dtype, norm, eps, layout, pairs, axes)
    for i, a in enumerate(axis):
        d.axis[i] = a
    for i, f in enumerate(freq):
        d.freq[i] = f
    for k, v in strides.items():
        setattr(d, k + "_stride", (ctypes.c_int64 * 3)(*v))
    return d


@pytest.mark.parametrize("wrong,name", [
    (dict(batch=-1), "SHAPE"), (dict(length=-1), "SHAPE"), (dict(h=0), "SHAPE"), (dict(kv=-1), "SHAPE"), (dict(h=65536), "SHAPE"),
    (dict(dim=4), "SHAPE"), (dict(dim=136), "SHAPE"), (dict(dim=60), "SHAPE"), (dict(dtype=7), "DTYPE"), (dict(norm=2), "INVALID_ARG"),
    (dict(eps=0.0), "INVALID_ARG"), (dict(eps=math.nan), "INVALID_ARG"), (dict(layout=2), "INVALID_ARG"), (dict(pairs=6), "SHAPE"),
    (dict(pairs=36), "SHAPE"), (dict(pairs=-4), "SHAPE"), (dict(axes=0), "SHAPE"), (dict(axes=5), "SHAPE"),
    (dict(axis=[1]), "INVALID_ARG"), (dict(axis=[-1]), "INVALID_ARG"), (dict(freq=[math.inf]), "INVALID_ARG"),
    (dict(freq=[math.nan]), "INVALID_ARG"), (dict(batch=2 ** 16, length=2 ** 15), "SHAPE"),
    (dict(q=(320, 64, 4)), "ALIGN"), (dict(q=(-320, 64, 16)), "SHAPE"), (dict(q=(1280, 64, 64)), "SHAPE"),
    (dict(k=(2 ** 46, 128, 64)), "SHAPE"),
], ids=str)
def test_heads_descriptions(wrong, name):
    assert status(lambda: L.petra_heads_query(heads(**wrong))) == "PETRA_ERR_" + name


def heads_forward(d, q=FAR[0], k=FAR[1], yq=FAR[2], yk=FAR[3], qn=(FAR[4], 0), kn=(FAR[5], 0), pos=FAR[6]):
    """A call that would run is given one misaligned parameter, the last to be refused for."""
    return status(lambda: L.petra_heads_forward(d, q, k, qn, kn, pos, yq, yk, 0))


def heads_backward(d, q=FAR[0], k=FAR[1], dyq=FAR[2], dyk=FAR[3], dq=FAR[4], dk=FAR[5], qn=(FAR[6], 0), kn=(FAR[7], 0),
                   dqn=(FAR[8], 0), dkn=(FAR[9], 0), pos=FAR[10]):
    """Without the workspace, which is the last check of all."""
    return status(lambda: L.petra_heads_backward(d, q, k, qn, kn, pos, dyq, dyk, dq, dk, dqn, dkn, 0, 0, 0))


def test_heads_pointers():
    d = heads()
    assert heads_forward(d, q=0) == "PETRA_ERR_INVALID_ARG"
    assert heads_forward(d, yk=0) == "PETRA_ERR_INVALID_ARG"
    assert heads_forward(d, q=FAR[0] + 8) == "PETRA_ERR_ALIGN"
    assert heads_forward(d, qn=(0, 0)) == "PETRA_ERR_INVALID_ARG"
    assert heads_forward(d, qn=(FAR[4] + 4, 0)) == "PETRA_ERR_ALIGN"
    assert heads_forward(d, kn=(FAR[5], FAR[6] + 4)) == "PETRA_ERR_ALIGN"
    assert heads_forward(d, pos=FAR[6] + 2) == "PETRA_ERR_ALIGN"
    assert heads_forward(heads(kv=0)) == "PETRA_ERR_INVALID_ARG"
    assert heads_backward(d) == "PETRA_ERR_WORKSPACE"
    assert heads_backward(d, dq=0) == "PETRA_ERR_INVALID_ARG"
    assert heads_backward(d, q=0) == "PETRA_ERR_INVALID_ARG"
    assert heads_backward(d, dqn=None) == "PETRA_ERR_INVALID_ARG"
    assert heads_backward(d, qn=None) == "PETRA_ERR_INVALID_ARG"
    assert heads_backward(d, dqn=(FAR[8], FAR[11])) == "PETRA_ERR_INVALID_ARG"
    assert heads_backward(heads(kv=0)) == "PETRA_ERR_INVALID_ARG"
    assert heads_backward(heads(kv=0), k=0, dyk=0, dk=0, kn=None, dkn=None) == "PETRA_ERR_WORKSPACE"


def test_heads_overlap():
    d = heads()
    size = 2 * 5 * 4 * 64 * 2
    assert heads_forward(d, yq=FAR[1]) == "PETRA_ERR_ALIAS"
    assert heads_forward(d, yq=FAR[0] + 16) == "PETRA_ERR_ALIAS"
    assert heads_forward(d, yk=FAR[2] + size - 16) == "PETRA_ERR_ALIAS"
    assert heads_forward(d, pos=FAR[2]) == "PETRA_ERR_ALIAS"
    assert heads_forward(d, qn=(FAR[3], 0)) == "PETRA_ERR_ALIAS"
    # in place only where the strides are the same
    w = 8 * 64
    slices = dict(q=(5 * w, w, 64), k=(5 * w, w, 64))
    assert heads_forward(heads(**slices), yq=FAR[0]) == "PETRA_ERR_ALIAS"
    assert heads_backward(d, dq=FAR[0]) == "PETRA_ERR_WORKSPACE"
    assert heads_backward(d, dq=FAR[2]) == "PETRA_ERR_WORKSPACE"
    assert heads_backward(d, dq=FAR[3]) == "PETRA_ERR_ALIAS"
    assert heads_backward(d, dq=FAR[1]) == "PETRA_ERR_ALIAS"
    assert heads_backward(d, dq=FAR[5]) == "PETRA_ERR_ALIAS"
    assert heads_backward(heads(**slices), dq=FAR[2]) == "PETRA_ERR_ALIAS"
    assert heads_backward(heads(**slices), dq=FAR[4], dk=FAR[4] + 4 * 64 * 2) == "PETRA_ERR_WORKSPACE"
    assert heads_backward(heads(**slices), dq=FAR[4], dk=FAR[4] + 3 * 64 * 2) == "PETRA_ERR_ALIAS"
    assert heads_backward(d, dqn=(FAR[6], 0)) == "PETRA_ERR_ALIAS"
    assert heads_backward(d, dqn=(FAR[0], 0)) == "PETRA_ERR_ALIAS"
    assert heads_backward(d, dqn=(FAR[9], 0)) == "PETRA_ERR_ALIAS"
    assert heads_backward(d, dqn=(FAR[4], 0)) == "PETRA_ERR_ALIAS"


def test_heads_without_tokens():
    """Nothing is enqueued; null pointers are fine."""
    d = heads(length=0)
    assert L.petra_heads_query(d) == 0
    L.petra_heads_forward(d, 0, 0, (FAR[4], 0), (FAR[5], 0), 0, 0, 0, 0)
    L.petra_heads_backward(d, 0, 0, None, None, 0, 0, 0, 0, 0, None, None, 0, 0, 0)


def vocab(rows=10, piece=0, width=64, v=100, dtype=L.PETRA_BF16, scale=1.0):
    return L.VocabDesc(rows, piece, width, v, dtype, scale)


@pytest.mark.parametrize("wrong,name", [
    (dict(rows=-1), "SHAPE"), (dict(rows=2 ** 30 + 1), "SHAPE"), (dict(piece=-1), "SHAPE"), (dict(width=0), "SHAPE"),
    (dict(width=12), "SHAPE"), (dict(width=65544), "SHAPE"), (dict(v=0), "SHAPE"), (dict(v=2 ** 20 + 1), "SHAPE"),
    (dict(dtype=2), "DTYPE"), (dict(scale=0.0), "INVALID_ARG"), (dict(scale=math.inf), "INVALID_ARG"),
    (dict(scale=math.nan), "INVALID_ARG")], ids=str)
def test_vocab_descriptions(wrong, name):
    assert status(lambda: L.petra_vocab_query(vocab(**wrong))) == "PETRA_ERR_" + name


def test_vocab_pointers_and_overlap():
    d = vocab()

    def loss(x=FAR[0], w=FAR[1], t=FAR[2], out=FAR[3], lse=FAR[4]):
        return status(lambda: L.petra_vocab_loss(d, x, w, t, out, lse, 0, 0, 0))

    def grad(x=FAR[0], w=FAR[1], t=FAR[2], weight=0, out=FAR[3], lse=FAR[4], dx=FAR[5], dw=FAR[6]):
        return status(lambda: L.petra_vocab_gradient(d, x, w, t, weight, out, lse, dx, dw, 0, 0, 0))

    assert loss() == "PETRA_ERR_WORKSPACE" and grad() == "PETRA_ERR_WORKSPACE"
    for name in ("x", "w", "out", "lse"):
        assert loss(**{name: 0}) == "PETRA_ERR_INVALID_ARG" and grad(**{name: 0}) == "PETRA_ERR_INVALID_ARG"
        assert loss(**{name: FAR[9] + 8}) == "PETRA_ERR_ALIGN"
    assert loss(t=0) == "PETRA_ERR_INVALID_ARG" and loss(t=FAR[2] + 2) == "PETRA_ERR_ALIGN"
    assert grad(dx=0) == "PETRA_ERR_INVALID_ARG" and grad(dw=0) == "PETRA_ERR_INVALID_ARG"
    assert grad(weight=FAR[7] + 2) == "PETRA_ERR_ALIGN" and grad(weight=FAR[7]) == "PETRA_ERR_WORKSPACE"
    for a, b in (("dx", "x"), ("dw", "w"), ("dw", "x"), ("out", "t"), ("lse", "out"), ("dw", "dx"), ("dx", "w")):
        at = dict(x=FAR[0], w=FAR[1], t=FAR[2], out=FAR[3], dx=FAR[5])[b]
        assert grad(**{a: at}) == "PETRA_ERR_ALIAS", (a, b)
    assert grad(weight=FAR[3]) == "PETRA_ERR_ALIAS"


def test_vocab_workspace_is_bounded():
    """The scores of a piece take a GiB at most, and a little beside: no rows x vocab tensor."""
    per_row = 2 * (-(-131072 // 256) * 4) + 8 + 4096 * 2
    at = {rows: L.petra_vocab_query(vocab(rows, 0, 4096, 131072)) for rows in (2 ** 13, 2 ** 17)}
    sums = 131072 * 4096 * 4
    for rows, (loss, grad) in at.items():
        assert grad <= 2 ** 30 + 4096 * per_row + 4 * rows + sums + 2 ** 20, rows
        assert loss <= 2 ** 31 + 4 * rows + 2 ** 24
    # e and the splits' sums of dx, 256 tiles of 256 x 256 in fp32: 64 MiB each; rows and tiles beside them
    assert L.petra_vocab_query(vocab(8192, 256, 4096, 131072))[1] < sums + 2 ** 27 + 2 ** 23
    # a piece of one size for all rows: not a whole one and a small rest
    assert L.petra_vocab_query(vocab(4097, 0, 64, 131072))[1] < 2 ** 30 * 0.6 + 131072 * 64 * 4


@pytest.mark.parametrize("dtype", [L.PETRA_BF16, L.PETRA_FP32])
def test_vocab_plans_of_extreme_sizes(dtype):
    for rows in (0, 1, 2, 255, 257, 2 ** 30):
        for piece in (0, 1, 300, 2 ** 40):
            for width in (8, 65536):
                for v in (1, 2, 2 ** 20):
                    loss, grad = L.petra_vocab_query(vocab(rows, piece, width, v, dtype))
                    assert 0 < loss and 0 < grad
    assert L.petra_vocab_loss(vocab(0), 0, FAR[0], 0, 0, 0, FAR[1], 2 ** 20, 0) is None


def adam(n=100, dtype=L.PETRA_FP32, states=L.PETRA_FP32, **more):
    d = L.AdamwDesc(more.pop("beta1", 0.9), more.pop("beta2", 0.999), more.pop("eps", 1e-8), dtype, states, 0)
    t = (L.AdamwTensor * 2)()
    for i in range(2):
        a = FAR[8 * i:8 * i + 8]
        t[i].theta, t[i].grad, t[i].m, t[i].v, t[i].m_scale, t[i].v_scale, t[i].copy, t[i].n = *a[:7], n
    for k, v in more.items():
        setattr(t[1], k, v)
    return d, t


@pytest.mark.parametrize("wrong,name", [
    (dict(beta1=1.0), "INVALID_ARG"), (dict(beta2=-0.1), "INVALID_ARG"), (dict(beta1=math.nan), "INVALID_ARG"),
    (dict(eps=0.0), "INVALID_ARG"), (dict(dtype=2), "DTYPE"), (dict(states=L.PETRA_BF16), "DTYPE"), (dict(n=-1), "SHAPE"),
    (dict(n=2 ** 43), "SHAPE")], ids=str)
def test_adamw_descriptions(wrong, name):
    d, t = adam(**wrong)
    assert status(lambda: L.petra_adamw_query(d, t, 2)) == "PETRA_ERR_" + name


def test_adamw_most_elements():
    """A workgroup a chunk: fewer chunks than a grid holds."""
    d, t = adam(n=4096 * (2 ** 23 - 1))
    assert L.petra_adamw_query(d, t, 2)[1] == 2 ** 24 - 2
    d, t = adam(n=4096 * 2 ** 23)
    assert status(lambda: L.petra_adamw_query(d, t, 2)) == "PETRA_ERR_SHAPE"


def test_owners_refuse_another_device():
    """By what they compare, without a second one."""
    import torch

    from paper_2406_02052_amd.ops import _Owner

    owner = _Owner()
    owner.workspace = torch.empty(4)
    with pytest.raises(ValueError, match="owner's device"):
        owner._need_here(None, type("Elsewhere", (), {"get_device": lambda self: 1, "device": "cuda:1"})())


def test_adamw_layout():
    d, t = adam(n=5000)
    size, chunks, ws = L.petra_adamw_query(d, t, 2)
    assert chunks == 4 and ws > 0
    table = ctypes.create_string_buffer(size + 16)
    at = -(-ctypes.addressof(table) // 16) * 16
    L.petra_adamw_layout(d, t, 2, at, size)
    assert status(lambda: L.petra_adamw_layout(d, t, 2, at, size - 1)) == "PETRA_ERR_WORKSPACE"
    for states in (L.PETRA_FP32, L.PETRA_E4M3):
        for wrong, name in ((dict(theta=0), "INVALID_ARG"), (dict(grad=FAR[20] + 8), "ALIGN"), (dict(m=0), "INVALID_ARG"),
                            (dict(v=FAR[0]), "ALIAS"), (dict(copy=FAR[20] + 4), "ALIGN"), (dict(theta=FAR[0]), "ALIAS"),
                            (dict(copy=FAR[8] + 16), "ALIAS"), (dict(weight_decay=math.nan), "INVALID_ARG")):
            d, t = adam(n=5000, states=states, **wrong)
            assert status(lambda: L.petra_adamw_layout(d, t, 2, at, size)) == "PETRA_ERR_" + name, (states, wrong)
    for wrong, name in ((dict(m_scale=0), "INVALID_ARG"), (dict(v_scale=FAR[20] + 2), "ALIGN"), (dict(m_scale=FAR[0]), "ALIAS")):
        d, t = adam(n=5000, states=L.PETRA_E4M3, **wrong)
        assert status(lambda: L.petra_adamw_layout(d, t, 2, at, size)) == "PETRA_ERR_" + name, wrong
        d, t = adam(n=5000, **wrong)
        L.petra_adamw_layout(d, t, 2, at, size)   # fp32 states have no scales
    # 8 bits are held by whole blocks: the last one may not reach into another tensor
    d, t = adam(n=100, states=L.PETRA_E4M3, m=FAR[2] + 112)
    assert status(lambda: L.petra_adamw_layout(d, t, 2, at, size)) == "PETRA_ERR_ALIAS"


def test_adamw_step_arguments():
    d, t = adam(n=5000)

    def step(desc=d, table=FAR[0], size=None, count=2, chunks=4, steps=FAR[1], lr=FAR[2], gs=0, rng=0):
        size = 2 * 96 + 4 * 4 if size is None else size
        return status(lambda: L.petra_adamw_step(desc, table, size, count, chunks, steps, lr, gs, rng, 0, 0, 0))

    assert L.petra_adamw_query(d, t, 2)[0] == 2 * 96 + 4 * 4
    assert step() == "PETRA_ERR_WORKSPACE"
    assert step(table=0) == "PETRA_ERR_INVALID_ARG" and step(table=FAR[0] + 8) == "PETRA_ERR_ALIGN"
    assert step(size=100) == "PETRA_ERR_WORKSPACE" and step(count=-1) == "PETRA_ERR_SHAPE"
    assert step(steps=0) == "PETRA_ERR_INVALID_ARG" and step(steps=FAR[1] + 4) == "PETRA_ERR_ALIGN"
    assert step(lr=0) == "PETRA_ERR_INVALID_ARG" and step(lr=FAR[2] + 2) == "PETRA_ERR_ALIGN"
    assert step(gs=FAR[3] + 2) == "PETRA_ERR_ALIGN" and step(rng=FAR[3] + 4) == "PETRA_ERR_ALIGN"
    assert step(desc=adam(states=L.PETRA_E4M3)[0]) == "PETRA_ERR_INVALID_ARG"


def test_owners_on_the_cpu_refuse():
    """Checks of the owners that need no device."""
    import torch

    from paper_2406_02052_amd import AdamW, HeadNorm, VocabLoss
    with pytest.raises(ValueError, match="norm"):
        HeadNorm(1, 1, 1, 1, 64, norm="batch", device="cpu")
    with pytest.raises(ValueError, match="layout"):
        HeadNorm(1, 1, 1, 1, 64, layout="thirds", device="cpu")
    with pytest.raises(ValueError, match="axis for each"):
        HeadNorm(1, 1, 1, 1, 64, freq=[1.0] * 8, axis=[0] * 7, device="cpu")
    with pytest.raises(ValueError, match="at most 64"):
        HeadNorm(1, 1, 1, 1, 128, freq=[1.0] * 65, device="cpu")
    op = HeadNorm(1, 2, 2, 1, 64, device="cpu")
    x = torch.zeros(1, 2, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="needs its parameters"):
        op.forward(x, x, x, x)
    with pytest.raises(ValueError, match="device tensor"):
        op.forward(x, x, x, x, q_norm=(x, None), k_norm=(x, None))
    with pytest.raises(ValueError, match="dtype"):
        VocabLoss(1, 8, 8, "fp16", device="cpu")
    op = VocabLoss(4, 8, 8, "fp32", device="cpu")
    with pytest.raises(ValueError, match="device tensor"):
        op.forward(*[torch.zeros(4, 8)] * 2, torch.zeros(4, dtype=torch.int32), *[torch.zeros(4)] * 2)
    p = [torch.zeros(4)]
    for wrong, name in ((dict(states="int8"), "states"), (dict(weight_decay=[0.1, 0.2]), "as many"), (dict(copies=[]), "as many")):
        with pytest.raises(ValueError, match=name):
            AdamW(p, p, **wrong)
    with pytest.raises(ValueError, match="at least one"):
        AdamW([], [])
    with pytest.raises(ValueError, match="device tensor"):
        AdamW(p, p)
    with pytest.raises(ValueError, match="grads"):
        AdamW(p, [torch.zeros(4, dtype=torch.float16)])
