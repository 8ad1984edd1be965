"""More refusals of the token operators' entry points, found on the host before any work."""
import ctypes
import random

import numpy as np
import pytest

from paper_2406_02052_amd import _lib as L

FAR = [0x100000000000 * (i + 1) for i in range(12)]   # addresses that nothing reads, far apart


def desc(dtype=L.PETRA_BF16, batch=2, q_len=3, kv_len=300, heads=2, kv_heads=2, dim=8, **strides):
    d = L.AttnDesc(batch, q_len, kv_len, heads, kv_heads, dim, dtype, 0, 0.125, 0.0)
    for k, v in strides.items():
        setattr(d, k + "_stride", (ctypes.c_int64 * 3)(*v))
    return d


def status(call):
    """Calls without the workspace that they need: the last check of all."""
    with pytest.raises(L.PetraError) as e:
        call()
    return e.value.name


def forward(d, o, k=None, lse=None):
    assert L.petra_attn_query(d)[0] > 0
    return status(lambda: L.petra_attn_forward(d, FAR[0], k or FAR[1], FAR[2], 0, 0, 0, o, lse or FAR[3], 0, 0, 0))


def backward(d, dq, dk, dv, q=FAR[0]):
    return status(lambda: L.petra_attn_backward(d, q, FAR[1], FAR[2], FAR[3], FAR[4], FAR[5], 0, 0, 0, dq, dk, dv, 0, 0, 0))


def test_slices_of_one_tensor_are_apart():
    """Gradients of q, k and v as slices of one [batch, tokens, heads + 2 kv_heads, dim] tensor."""
    h, kvh, dim, n = 4, 2, 64, 300
    w = (h + 2 * kvh) * dim
    st = (n * w, w, dim)
    d = desc(q_len=n, kv_len=n, heads=h, kv_heads=kvh, dim=dim, q=st, k=st, v=st)
    at = FAR[6]
    assert backward(d, at, at + h * dim * 2, at + (h + kvh) * dim * 2) == "PETRA_ERR_WORKSPACE"
    assert backward(d, at, at + (h - 1) * dim * 2, at + (h + kvh) * dim * 2) == "PETRA_ERR_ALIAS"
    assert backward(d, at, at + h * dim * 2, at + (h + kvh) * dim * 2 - 16) == "PETRA_ERR_ALIAS"
    assert backward(d, at, at + h * dim * 2, at + (h + kvh) * dim * 2, q=at) == "PETRA_ERR_ALIAS"
    # the last token's queries only, with the keys of all
    d = desc(q_len=1, kv_len=n, heads=h, kv_heads=kvh, dim=dim, q=(n * w, 0, dim), k=st, v=st)
    last = at + (n - 1) * w * 2
    assert backward(d, last, at + h * dim * 2, at + (h + kvh) * dim * 2) == "PETRA_ERR_WORKSPACE"
    assert backward(d, last, at + h * dim * 2 - 16, at + (h + kvh) * dim * 2) == "PETRA_ERR_ALIAS"


def test_strided_output_over_a_strided_input():
    w = 6 * 8
    d = desc(q_len=300, o=(300 * w, w, 8), k=(300 * w, w, 8))
    at = FAR[6]
    assert forward(d, at, at) == "PETRA_ERR_ALIAS"
    assert forward(d, at + 16, at) == "PETRA_ERR_ALIAS"
    assert forward(d, at + 32, at) == "PETRA_ERR_WORKSPACE"
    assert forward(d, at + 300 * w * 2, at) == "PETRA_ERR_ALIAS"       # the second batch row over the first's
    # the same memory by heads first and by tokens first
    d = desc(q_len=300, o=(300 * 16, 8, 300 * 8), k=(300 * 16, 16, 8))
    assert forward(d, at, at) == "PETRA_ERR_ALIAS"
    # lse in o's gaps, which its whole rows do not fit
    d = desc(q_len=300, o=(300 * w, w, 8))
    assert forward(d, at, lse=at + 32) == "PETRA_ERR_ALIAS"


def test_strides_past_the_address_space():
    for name in "qkvo":
        for st in ((2 ** 46, 16, 8), (16, 8, 2 ** 46) if name in "qo" else (2 ** 46, 2 ** 21, 8)):
            with pytest.raises(L.PetraError) as e:
                L.petra_attn_query(desc(batch=30000, heads=2, **{name: st}))
            assert e.value.name == "PETRA_ERR_SHAPE" and "address space" in str(e.value)


def _bytes(at, strides, counts, dim):
    i = [np.arange(n) * s * 2 for n, s in zip(counts, strides)]
    first = at + (i[0][:, None, None] + i[1][None, :, None] + i[2][None, None]).reshape(-1)
    return set((first[:, None] + np.arange(0, dim * 2, 16)).reshape(-1).tolist())


def test_overlap_is_that_of_the_elements():
    """Random strided pairs against their sets of addresses."""
    rng, seen = random.Random(5), {True: 0, False: 0}
    for _ in range(600):
        batch, q_len, heads = rng.randint(1, 3), rng.randint(1, 6), rng.choice((1, 2, 4))
        kv_heads = rng.choice([x for x in (1, 2, 4) if heads % x == 0])
        dim, unit = rng.choice((8, 16)), rng.choice((1, 2, 3, 5))
        counts = (batch, q_len, heads)
        # o: every dimension steps past what the smaller ones cover, in any order
        order, st, extent = rng.sample(range(3), 3), [0] * 3, dim
        for i in order:
            st[i] = -(-extent // 8) * 8 + 8 * unit * rng.randint(0, 4)
            extent += (counts[i] - 1) * st[i]
        token = dim + 8 * rng.randint(0, 8)
        kst = (8 * rng.randint(0, 900), token, rng.choice((dim, 8 * rng.randint(0, 60), token * 300)))
        if rng.random() < 0.4:   # the strides in common
            kst = (st[0], max(st[1], dim), st[2])
        d = desc(batch=batch, q_len=q_len, kv_len=300, heads=heads, kv_heads=kv_heads, dim=dim, o=st, k=kst)
        k = FAR[6]
        o = k + 16 * rng.randint(-200, 5000)
        if st == [0] * 3 or kst == (0, 0, 0):
            continue
        want = bool(_bytes(o, st, counts, dim) & _bytes(k, kst, (batch, 300, kv_heads), dim))
        assert forward(d, o, k) == ("PETRA_ERR_ALIAS" if want else "PETRA_ERR_WORKSPACE"), (counts, kv_heads, dim, st, kst, o - k)
        seen[want] += 1
    assert min(seen.values()) > 100, seen


@pytest.mark.parametrize("bad", [3.5, "4096", np.float32(16), np.array([4096]), [4096]], ids=repr)
def test_what_is_no_address_is_refused(bad):
    """A number or text that int() takes is no device address."""
    with pytest.raises(AttributeError):
        L._ptr(bad)
    with pytest.raises(AttributeError):
        L.petra_dropout(8, L.PETRA_FP32, 0.0, 1.0, bad, 0, 0, FAR[0], 0)


def test_addresses():
    class Tensor:
        def data_ptr(self):
            return 4096

    assert (L._ptr(None), L._ptr(4096), L._ptr(Tensor())) == (0, 4096, 4096)


def test_current_stream_by_the_public_call_where_torch_has_no_other(monkeypatch):
    import torch

    class Stream:
        cuda_stream = 77

    monkeypatch.setattr(torch.cuda, "current_stream", Stream)
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    assert L._stream(None) == 77
    assert L._stream(Stream()) == 77 and L._stream(5) == 5


@pytest.mark.parametrize("out", ["y", "u"])
@pytest.mark.parametrize("param", ["gate", "post.gamma", "post.beta", "pre.gamma", "pre.beta"])
def test_coupling_outputs_over_parameters(param, out):
    d = L.CouplingDesc(12, 0, 64, L.PETRA_BF16, L.PETRA_NORM_LAYER, 1e-5, 1.0, 0.0)
    at = {"x": FAR[0], "f": FAR[1], "gate": FAR[2], "post.gamma": FAR[3], "post.beta": FAR[4], "pre.gamma": FAR[5],
          "pre.beta": FAR[6], "y": FAR[7], "u": FAR[8]}
    at[out] = at[param] - 12 * 64 * 2 + 16       # the last 8 of its elements over the first of the parameter
    call = lambda: L.petra_coupling_forward(  # noqa: E731
        d, at["x"], at["f"], at["gate"], (at["post.gamma"], at["post.beta"]), (at["pre.gamma"], at["pre.beta"]), 0,
        at["y"], at["u"], 0)
    assert status(call) == "PETRA_ERR_ALIAS"
