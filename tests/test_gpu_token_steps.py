"""GPU parity of head norms with rotation, the loss over a vocabulary and AdamW with
oracle/tokens.py (fp64), at the sizes, layouts and values where they can go wrong.

Bars, normwise per output.  fp32: products and sums in fp32, 1e-5.  bf16 (2^-9 a rounding): head norms and dx of a head
round once, 2^-8 with what fp32 adds; dx of the loss rounds e and itself, 2^-8; dw e, f x and itself, 2^-7.  Parameter
gradients, losses and lse are fp32 sums of exact products: 1e-5.  AdamW is fp32 but for its bf16 copy: 1e-6 of theta, 2^-8
of the copy; states in 8 bits are exact numbers of the format, chosen by fp32 values: all but those within fp32's rounding of a
border are the oracle's."""
import math

import numpy as np
import pytest
import torch

from oracle import tokens as T

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
ONE = {"fp32": 1e-5, "bf16": 2.0 ** -8}
TWO = {"fp32": 1e-5, "bf16": 2.0 ** -7}
RNG = (0x123456789ABCDEF, (7 << 40) + 3)


def dev(a, dtype):
    return torch.tensor(a).to("cuda", TYPES[dtype])


def host(t):
    return t.detach().double().cpu().numpy()


def draw(seed, *shapes, dtype="fp32", std=1.0):
    r = np.random.RandomState(seed)
    return [host(torch.tensor(r.randn(*s) * std).to(TYPES[dtype])) for s in shapes]


def near(got, want, bar, name):
    got, want = host(got) if torch.is_tensor(got) else got, np.asarray(want)
    assert got.shape == want.shape, name
    assert np.isfinite(got).all(), name
    err, size = np.linalg.norm(got - want), np.linalg.norm(want)
    assert err <= bar * size, (name, err / max(size, 1e-300))


def nan(shape, dtype="fp32"):
    return torch.full(shape, math.nan, dtype=TYPES[dtype], device="cuda")


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


# ---- head norms and rotation -------------------------------------------------

# batch, length, heads, kv_heads, dim, pairs
HEADS = [(1, 1, 1, 1, 8, 4), (3, 1, 16, 4, 64, 32), (2, 77, 5, 5, 40, 20), (2, 130, 3, 0, 80, 40), (1, 333, 20, 1, 128, 60),
         (5, 64, 9, 2, 96, 48), (2, 50, 2, 2, 24, 12), (2, 9, 33, 7, 128, 64), (1, 4, 130, 1, 8, 0), (4, 700, 6, 2, 64, 4),
         (2, 40, 3, 2, 120, 60), (1, 5000, 2, 1, 32, 16)]


def heads_case(shape, dtype, norm, layout, axes, seed=0):
    b, n, h, kv, d, pairs = shape
    r = np.random.RandomState(seed)
    axes = min(axes, max(pairs, 1))
    axis = [int(a) for a in r.randint(0, axes, pairs)]
    if pairs:
        axis[-1] = axes - 1
    freq = [10000.0 ** (-i / pairs) for i in range(pairs)]
    pos = r.randint(-2 ** 31, 2 ** 31 - 1, (axes, b, n)) if seed % 2 else r.randint(0, 200000, (axes, b, n))
    q, k, dyq, dyk = draw(seed, (b, n, h, d), (b, n, kv, d), (b, n, h, d), (b, n, kv, d), dtype=dtype)
    params = [tuple(1 + 0.2 * x for x in draw(9, (d,), (d,))), tuple(draw(10, (d,), (d,)))]
    params = [(params[0][0], params[1][0] if norm == "layer" else None), (params[0][1], params[1][1] if norm == "layer" else None)]
    return dict(q=q, k=k, dyq=dyq, dyk=dyk, pos=pos, freq=freq, axis=axis, params=params if norm else [None, None], axes=axes)


def on_device(p):
    return None if p is None else tuple(None if t is None else dev(t, "fp32") for t in p)


def like(p):
    return None if p is None else tuple(None if t is None else torch.full_like(t, math.nan) for t in p)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("norm,layout,axes", [("rms", "halves", 1), ("layer", "halves", 3), ("rms", "neighbours", 2), (None, "halves", 4),
                                              ("layer", "neighbours", 1), (None, "neighbours", 1)])
@pytest.mark.parametrize("shape", HEADS, ids=str)
def test_heads(shape, norm, layout, axes, dtype):
    from paper_2406_02052_amd import HeadNorm

    print("case", shape, norm, layout, axes, dtype, flush=True)
    b, n, h, kv, d, pairs = shape
    c = heads_case(shape, dtype, norm, layout, axes, seed=h + axes)
    op = HeadNorm(b, n, h, kv, d, dtype, norm=norm, eps=1e-5, layout=layout, freq=c["freq"], axis=c["axis"])
    pos = i32(c["pos"][:op.axes])
    # q and k beside each other, their gradients too, results dense
    both = torch.zeros(b, n, h + kv + 1, d, dtype=TYPES[dtype], device="cuda")
    grads = torch.full_like(both, 7.0)
    q, k = both[:, :, :h], both[:, :, h:h + kv]
    q.copy_(dev(c["q"], dtype))
    k.copy_(dev(c["k"], dtype))
    qn, kn = (on_device(p) for p in c["params"])
    yq, yk = nan((b, n, h, d), dtype), nan((b, n, kv, d), dtype)
    more = ("layer" if norm == "layer" else "rms", 1e-5, c["pos"], c["freq"], c["axis"], layout)
    keys = (k, yk, kn) if kv else (None, None, None)
    op.forward(q, keys[0], yq, keys[1], q_norm=qn, k_norm=keys[2], positions=pos)
    dyq, dyk = dev(c["dyq"], dtype), dev(c["dyk"], dtype) if kv else None
    dqn, dkn = like(qn), like(keys[2])
    dq, dk = grads[:, :, :h], grads[:, :, h:h + kv] if kv else None
    op.backward(q, keys[0], dyq, dyk, dq, dk, q_norm=qn, k_norm=keys[2], dq_norm=dqn, dk_norm=dkn, positions=pos)
    torch.cuda.synchronize()
    assert (grads[:, :, h + kv:] == 7).all()
    for x, y, dy, dx, p, dp in ((c["q"], yq, c["dyq"], dq, c["params"][0], dqn), (c["k"], yk, c["dyk"], dk, c["params"][1], dkn))[:2 if kv else 1]:
        near(y, T.head_norm(x, p, *more), ONE[dtype], "y")
        want = T.head_norm(x, p, *more, dy=dy)
        near(dx, want[0], ONE[dtype], "dx")
        if norm:
            near(dp[0], want[1], 1e-5, "dgamma")
            if norm == "layer":
                near(dp[1], want[2], 1e-5, "dbeta")


def test_heads_defaults_and_token_indices():
    """Positions of None are the tokens' indices; freq of None the usual ones."""
    from paper_2406_02052_amd import HeadNorm

    b, n, h, d = 2, 37, 3, 64
    q, k = draw(1, (b, n, h, d), (b, n, h, d))
    pos = np.broadcast_to(np.arange(n), (1, b, n))
    op = HeadNorm(b, n, h, h, d, "fp32", norm=None)
    yq, yk = nan(q.shape), nan(k.shape)
    op.forward(dev(q, "fp32"), dev(k, "fp32"), yq, yk)
    freq = [10000.0 ** (-2 * i / d) for i in range(d // 2)]
    for x, y in ((q, yq), (k, yk)):
        near(y, T.rotate(x, pos, freq, [0] * 32, "halves"), 1e-6, "y")


@pytest.mark.parametrize("layout", ["halves", "neighbours"])
def test_heads_in_place(layout):
    from paper_2406_02052_amd import HeadNorm

    shape = (2, 50, 6, 2, 64, 24)
    b, n, h, kv, d, pairs = shape
    c = heads_case(shape, "bf16", "rms", layout, 1)
    op = HeadNorm(b, n, h, kv, d, "bf16", layout=layout, freq=c["freq"], axis=c["axis"])
    pos, qn, kn = i32(c["pos"]), *(on_device(p) for p in c["params"])
    t = [dev(c[x], "bf16") for x in ("q", "k", "dyq", "dyk")]
    out, new = [torch.empty_like(x) for x in t[:2]], [torch.empty_like(x) for x in t[:2]]
    dn, dn2 = [like(qn), like(kn)], [like(qn), like(kn)]
    op.forward(t[0], t[1], *out, q_norm=qn, k_norm=kn, positions=pos)
    op.backward(*t, *new, q_norm=qn, k_norm=kn, dq_norm=dn[0], dk_norm=dn[1], positions=pos)
    over = [x.clone() for x in t]
    op.backward(t[0], t[1], over[2], over[3], over[2], over[3], q_norm=qn, k_norm=kn, dq_norm=dn2[0], dk_norm=dn2[1], positions=pos)
    assert all(torch.equal(x, y) for x, y in zip(over[2:], new)) and torch.equal(dn[0][0], dn2[0][0])
    op.backward(over[0], over[1], t[2], t[3], over[0], over[1], q_norm=qn, k_norm=kn, dq_norm=dn2[0], dk_norm=dn2[1], positions=pos)
    assert all(torch.equal(x, y) for x, y in zip(over[:2], new)) and torch.equal(dn[1][0], dn2[1][0])
    over = [x.clone() for x in t]
    op.forward(over[0], over[1], over[0], over[1], q_norm=qn, k_norm=kn, positions=pos)
    assert all(torch.equal(x, y) for x, y in zip(over, out))


def test_heads_of_no_tokens_have_zero_parameter_gradients():
    from paper_2406_02052_amd import HeadNorm

    op = HeadNorm(2, 0, 3, 1, 64, "bf16", norm="layer")
    q, k = torch.empty(2, 0, 3, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(2, 0, 1, 64, dtype=torch.bfloat16, device="cuda")
    p = (torch.ones(64, device="cuda"), torch.ones(64, device="cuda"))
    d = [like(p), like(p)]
    op.forward(q, k, q, k, q_norm=p, k_norm=p)
    op.backward(q, k, q, k, q, k, q_norm=p, k_norm=p, dq_norm=d[0], dk_norm=d[1])
    assert all((t == 0).all() for x in d for t in x)


def test_heads_nan_stays_in_its_head():
    from paper_2406_02052_amd import HeadNorm

    shape = (1, 20, 6, 2, 40, 20)
    c = heads_case(shape, "fp32", "rms", "halves", 1)
    op = HeadNorm(*shape[:5], "fp32", freq=c["freq"], axis=c["axis"])
    q, k = dev(c["q"], "fp32"), dev(c["k"], "fp32")
    q[0, 3, 2, 7] = math.nan
    q[0, 9, 5] = math.inf
    yq, yk = nan(q.shape), nan(k.shape)
    qn, kn = (on_device(p) for p in c["params"])
    op.forward(q, k, yq, yk, q_norm=qn, k_norm=kn, positions=i32(c["pos"]))
    bad = torch.isnan(yq).any(3)
    assert bad[0, 3, 2] and bad[0, 9, 5] and bad.sum() == 2 and torch.isfinite(yk).all()


# ---- loss over a vocabulary ---------------------------------------------------

# rows, width, vocab, piece_rows
VOCAB = [(1, 8, 1, 0), (1, 64, 1000, 0), (8, 64, 257, 0), (3, 200, 50, 0), (257, 136, 255, 0), (64, 512, 4096, 0), (300, 72, 513, 0),
         (700, 64, 300, 256), (513, 40, 1030, 100), (1000, 256, 64, 0), (33, 1032, 129, 7), (2, 8, 2, 1)]


def vocab_case(rows, width, vocab, dtype, seed=0, std=2.5):
    r = np.random.RandomState(seed + rows)
    x, = draw(seed + 1, (rows, width), dtype=dtype)
    w, = draw(seed + 2, (vocab, width), dtype=dtype, std=std / math.sqrt(width))
    t = r.randint(0, vocab, rows)
    out = r.rand(rows) < 0.2
    out[0] = False
    t[out] = r.choice([-100, -1, vocab, 2 ** 31 - 1, -2 ** 31], out.sum())
    weight = host(torch.tensor(r.rand(rows), dtype=torch.float32))
    return x, w, t, weight


def run_vocab(x, w, t, dtype, weight=None, scale=1.0, piece=0, op=None):
    from paper_2406_02052_amd import VocabLoss

    rows, width, vocab = len(x), x.shape[1], len(w)
    op = op or VocabLoss(rows, width, vocab, dtype, scale=scale, piece_rows=piece)
    op.workspace.fill_(0xFF)      # NaN in whatever is read before it is written
    out = [nan((rows,)), nan((rows,)), nan(x.shape, dtype), nan(w.shape, dtype)]
    alone = [nan((rows,)), nan((rows,))]
    d = dev(x, dtype), dev(w, dtype), i32(t)
    op.gradient(*d, *out, weight=None if weight is None else dev(weight, "fp32"))
    op.forward(*d, *alone)
    torch.cuda.synchronize()
    return out, alone


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("rows,width,vocab,piece", VOCAB)
def test_vocab(rows, width, vocab, piece, weighted, dtype):
    print("case", rows, width, vocab, piece, weighted, dtype, flush=True)
    x, w, t, weight = vocab_case(rows, width, vocab, dtype)
    scale = 0.5 if weighted else 1.0
    out, alone = run_vocab(x, w, t, dtype, weight if weighted else None, scale, piece)
    want = T.vocab_loss(x, w, t, scale, weight if weighted else None)
    for got in (out, alone):
        # a loss is a difference of scores of fp32 products: their size is lse's
        near(got[1], want[1], 1e-5, "lse")
        assert np.abs(host(got[0]) - want[0]).max() <= 1e-5 * np.abs(want[1]).max() + 1e-6, "loss"
    if vocab == 1:       # p = 1: the gradients are nothing but roundings
        assert np.abs(host(out[2])).max() <= 1e-5 and np.abs(host(out[3])).max() <= 1e-5
        return
    near(out[2], want[2], ONE[dtype], "dx")
    near(out[3], want[3], TWO[dtype], "dw")
    assert (out[2][torch.tensor((t < 0) | (t >= vocab), device="cuda")] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("piece", [0, 64])
def test_vocab_scores_far_above_the_targets(piece, dtype):
    """Scores of some rows pass the target's by up to 2000: those tiles take references of their own."""
    rows, width, vocab = 200, 64, 700
    x, w, t, weight = vocab_case(rows, width, vocab, dtype, std=4.0)
    x[::3] *= 40.0
    x[5] *= 128.0
    x = host(dev(x, dtype))
    out, alone = run_vocab(x, w, t, dtype, weight, piece=piece)
    want = T.vocab_loss(x, w, t, 1.0, weight)
    assert want[0].max() > 500
    for got in (out, alone):
        near(got[0], want[0], 1e-5, "loss")
        near(got[1], want[1], 1e-5, "lse")
    # e of such tiles is rounded once more: dx thrice, dw four times
    near(out[2], want[2], TWO[dtype], "dx")
    near(out[3], want[3], TWO[dtype], "dw")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_vocab_confident_rows(dtype):
    """The target's score far above all others: loss and gradients go to 0, not to NaN."""
    x, w, t, _ = vocab_case(100, 64, 300, dtype)
    x = np.where(((t >= 0) & (t < 300))[:, None], 30 * w[np.clip(t, 0, 299)], x)
    x = host(dev(x, dtype))
    out, _ = run_vocab(x, w, t, dtype)
    want = T.vocab_loss(x, w, t)
    assert np.abs(host(out[0]) - want[0]).max() <= 1e-5 * np.abs(want[1]).max()
    # p - 1 is a difference of sums near 1, 2^-24 each
    assert np.abs(host(out[2]) - want[2]).max() <= 2.0 ** -8 * np.abs(want[2]).max() + 1e-6 * np.abs(w).max()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_vocab_rows_that_take_no_part_may_hold_anything(dtype):
    x, w, t, _ = vocab_case(300, 64, 513, dtype)
    out = np.flatnonzero((t < 0) | (t >= 513))
    want = T.vocab_loss(x, w, t)
    x[out] = np.array([math.nan, math.inf, -math.inf])[np.arange(len(out)) % 3][:, None]
    got, _ = run_vocab(x, w, t, dtype, piece=128)
    near(got[2], want[2], ONE[dtype], "dx")
    near(got[3], want[3], TWO[dtype], "dw")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_vocab_without_rows_that_take_part(dtype):
    x, w, t, _ = vocab_case(70, 64, 100, dtype)
    got, alone = run_vocab(x, w, np.full(70, -1), dtype)
    assert all((g == 0).all() for g in (*got, *alone))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_vocab_without_rows(dtype):
    got, _ = run_vocab(np.zeros((0, 64)), draw(1, (100, 64), dtype=dtype)[0], np.zeros(0, int), dtype)
    assert (got[3] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_vocab_nan_row_is_nan(dtype):
    x, w, t, _ = vocab_case(100, 64, 300, dtype)
    t[50] = 7
    x[50, 3] = math.nan
    got, alone = run_vocab(x, w, t, dtype)
    want = T.vocab_loss(np.delete(x, 50, 0), w, np.delete(t, 50))
    for g in (got, alone):
        assert torch.isnan(g[0][50]) and torch.isnan(g[1][50])
        near(np.delete(host(g[1]), 50), want[1], 1e-5, "lse")
    assert torch.isnan(got[2][50]).all()
    assert np.isfinite(np.delete(host(got[2]), 50, 0)).all() and torch.isnan(got[3]).any()


def test_vocab_same_results_again():
    """Split sums are joined in a fixed order."""
    x, w, t, weight = vocab_case(2000, 64, 300, "bf16")
    a, b = run_vocab(x, w, t, "bf16", weight), run_vocab(x, w, t, "bf16", weight)
    assert all(torch.equal(p, q) for p, q in zip((*a[0], *a[1]), (*b[0], *b[1])))


# ---- AdamW --------------------------------------------------------------------

SIZES = [(1,), (3,), (64,), (65, 7), (5, 33), (4096,), (4097,), (0,), (12300,), (2, 2, 2)]


def adam_case(states, grad, copies, seed=0):
    r = np.random.RandomState(seed)
    theta = [dev(r.randn(*s) * 0.1, "fp32") for s in SIZES]
    grads = [dev(r.randn(*s) * 10.0 ** r.uniform(-6, 0, s), grad) for s in SIZES]
    copy = [x.to(torch.bfloat16) for x in theta] if copies else None
    decay = [0.1 * (i % 3) for i in range(len(SIZES))]
    return theta, grads, copy, decay


def flat(t):
    return host(t).reshape(-1)


@pytest.mark.parametrize("states", ["fp32", "fp8"])
@pytest.mark.parametrize("grad,copies,scaled", [("fp32", True, False), ("bf16", False, True), ("bf16", True, False), ("fp32", False, True)])
def test_adamw(states, grad, copies, scaled):
    """Each of four steps against the oracle's, from the states that the kernel held before it."""
    from paper_2406_02052_amd import AdamW

    print("case", states, grad, copies, scaled, flush=True)
    theta, grads, copy, decay = adam_case(states, grad, copies)
    op = AdamW(theta, grads, states=states, lr=0.01, betas=(0.8, 0.99), eps=1e-6, weight_decay=decay, copies=copy)
    scale = torch.full((1,), 0.25, device="cuda") if scaled else None
    for step in range(4):
        rng = torch.tensor((RNG[0], RNG[1] + step), dtype=torch.int64, device="cuda")
        before = [flat(t) for t in theta]
        m0, v0 = host(op.m.float()), host(op.v.float())
        if states == "fp8":
            m0, v0 = m0 * np.repeat(host(op.m_scale), 64), (v0 * np.repeat(host(op.v_scale), 64)) ** 2
        op.step(rng=rng if states == "fp8" else None, grad_scale=scale)
        torch.cuda.synchronize()
        group, off, total = 0, 0, 0
        for i, (t, g, start) in enumerate(zip(theta, grads, op.starts)):
            n = t.numel()
            part = slice(start, start + n)
            want, m, v = T.adamw(before[i], flat(g), m0[part], v0[part], step + 1, 0.01, (0.8, 0.99), 1e-6, decay[i],
                                 0.25 if scaled else 1.0)
            assert np.abs(flat(t) - want).max(initial=0) <= 1e-6 * np.abs(want).max(initial=1), i
            if copies:
                assert torch.equal(copy[i], t.to(torch.bfloat16))
            if states == "fp32":
                assert np.allclose(host(op.m[part]), m, rtol=1e-6, atol=1e-12) and np.allclose(host(op.v[part]), v, rtol=1e-6, atol=1e-16)
                continue
            whole = -(-n // 64) * 64
            u = T.adamw_numbers((RNG[0], RNG[1] + step), group, whole)
            group += whole // 4
            for held, scales, value, power, un in ((op.m, op.m_scale, m, 1, u[0]), (op.v, op.v_scale, np.sqrt(v), 2, u[1])):
                _, s = T.hold(value, power, un)
                taken = host(scales[start // 64:(start + whole) // 64])
                # a block whose largest is a power of two but for fp32's rounding (0.2 of a bf16 gradient of 1.25, which is
                # 0.25 in fp32 and a little less in fp64: one in 128 blocks) may have either scale, and its numbers go by that
                top = np.abs(np.append(value, np.zeros(whole - n))).reshape(-1, 64).max(1)
                border = np.abs(np.log2(np.where(top > 0, top, 1.3)) % 1.0 - 0.5) > 0.5 - 2.0 ** -20
                assert (taken == s)[~border].all() and ((taken == s) | (taken == 2 * s) | (2 * taken == s)).all()
                q, _ = T.hold(value, power, un, scale=taken)
                got = host(held[start:start + whole].float())
                off += (np.abs(got) != q).sum()
                total += whole
                assert (np.sign(got[:n]) == np.sign(value) * (np.abs(got[:n]) > 0)).all()
        # borders within fp32's rounding of a value: 2^-22 of it, of steps of 2^-4 or more
        assert off <= 2 + total * 1e-4, (off, total)
    assert op.steps.item() == 4


def test_adamw_of_8_bits_keeps_small_changes_of_v():
    """A gradient that shrinks by half: v has to follow by a thousandth a step, which nearest rounding would not."""
    from paper_2406_02052_amd import AdamW

    n = 64 * 512
    theta, grad = torch.zeros(n, device="cuda"), torch.full((n,), 1e-3, device="cuda")
    op = AdamW([theta], [grad], states="fp8", betas=(0.9, 0.999), weight_decay=0.0)
    rng = torch.tensor([5, 0], dtype=torch.int64, device="cuda")
    want = 0.0
    for step in range(300):
        if step == 150:
            grad.mul_(0.5)
        op.step(rng=rng)
        rng[1] += 1
        want = 0.999 * want + 0.001 * float(grad[0].double()) ** 2
    v = (op.v.float() * op.v_scale.repeat_interleave(64)).double().square()
    # the mean of n unbiased roundings: each step adds at most (a sixteenth)^2 / 4 x change / step's variance, a
    # spread of a fifth of v an element and of its 181st part over 32768
    assert abs(float(v.mean()) / want - 1) < 0.01


def test_adamw_zeroes_gradients_and_follows_device_lr():
    from paper_2406_02052_amd import AdamW

    theta, grads, _, _ = adam_case("fp32", "bf16", False)
    before = [t.clone() for t in theta]
    op = AdamW(theta, grads, lr=1.0, weight_decay=0.5, zero_grads=True)
    op.lr.fill_(0.0)
    op.step()
    assert all(torch.equal(a, b) for a, b in zip(theta, before)) and all((g == 0).all() for g in grads)
    op.lr.fill_(1e-3)
    op.step()
    assert not torch.equal(theta[5], before[5])


@pytest.mark.parametrize("states", ["fp32", "fp8"])
def test_adamw_nan_gradient(states):
    """Its own element is NaN; others are not."""
    from paper_2406_02052_amd import AdamW

    theta, grads, _, _ = adam_case(states, "fp32", False)
    grads[5][100] = math.nan
    grads[6][100] = math.inf
    op = AdamW(theta, grads, states=states)
    rng = torch.tensor(RNG, dtype=torch.int64, device="cuda") if states == "fp8" else None
    for _ in range(2):
        op.step(rng=rng)
    for i, t in enumerate(theta):
        bad = ~torch.isfinite(t)
        assert bad.sum() == (i in (5, 6)) and (i not in (5, 6) or bad[100])
    for s in (op.m, op.v):
        held = s.float()
        assert (~torch.isfinite(held[op.starts[5]:op.starts[7]])).sum() == 2
        assert torch.isfinite(held[:op.starts[5]]).all() and torch.isfinite(held[op.starts[7]:]).all()


# ---- together ------------------------------------------------------------------

def test_a_training_step_of_a_token_stage():
    """Product, head norms with rotation, attention, loss, all gradients back and the update, against automatic
    differentiation of the plain formulas in 64 bits.  fp32: 1e-4 for the chain of six operators."""
    from paper_2406_02052_amd import AdamW, Attention, HeadNorm, VocabLoss

    torch.manual_seed(0)
    b, n, h, kv, d, vocab = 2, 37, 4, 2, 32, 301
    width = h * d
    x = torch.randn(b, n, width, device="cuda")
    shapes = dict(wqkv=((h + 2 * kv) * d, width), wo=(width, width), head=(vocab, width), gq=(d,), gk=(d,))
    p = {k: torch.randn(*s, device="cuda") * (s[-1] ** -0.5) + (len(s) == 1) for k, s in shapes.items()}
    t = torch.randint(-1, vocab, (b * n,), dtype=torch.int32, device="cuda")
    norm = HeadNorm(b, n, h, kv, d, "fp32", eps=1e-6)
    attend = Attention(b, n, n, h, kv, d, "fp32", causal=True)
    loss = VocabLoss(b * n, width, vocab, "fp32")
    g = {k: torch.empty_like(v) for k, v in p.items()}

    qkv = (x.reshape(-1, width) @ p["wqkv"].T).reshape(b, n, h + 2 * kv, d)
    q, k, v = qkv[:, :, :h], qkv[:, :, h:h + kv], qkv[:, :, h + kv:]
    yq, yk = torch.empty(b, n, h, d, device="cuda"), torch.empty(b, n, kv, d, device="cuda")
    norm.forward(q, k, yq, yk, q_norm=(p["gq"], None), k_norm=(p["gk"], None))
    o, lse = torch.empty_like(yq), torch.empty(b, h, n, device="cuda")
    attend.forward(yq, yk, v, o, lse)
    y = o.reshape(-1, width) @ p["wo"].T
    rows, slse, dy = torch.empty(b * n, device="cuda"), torch.empty(b * n, device="cuda"), torch.empty_like(y)
    loss.gradient(y, p["head"], t, rows, slse, dy, g["head"])
    g["wo"].copy_(dy.T @ o.reshape(-1, width))
    do = (dy @ p["wo"]).reshape(o.shape)
    dqkv = torch.empty_like(qkv)
    dq, dk, dv = dqkv[:, :, :h], dqkv[:, :, h:h + kv], dqkv[:, :, h + kv:]
    dyq, dyk = torch.empty_like(yq), torch.empty_like(yk)
    attend.backward(yq, yk, v, o, lse, do, dyq, dyk, dv)
    norm.backward(q, k, dyq, dyk, dq, dk, q_norm=(p["gq"], None), k_norm=(p["gk"], None), dq_norm=(g["gq"], None), dk_norm=(g["gk"], None))
    g["wqkv"].copy_(dqkv.reshape(b * n, -1).T @ x.reshape(-1, width))

    ref = {k: v.double().cpu().requires_grad_() for k, v in p.items()}
    xs = x.double().cpu()
    rq = (xs @ ref["wqkv"].T).reshape(b, n, h + 2 * kv, d)
    ang = torch.arange(n).double()[:, None] * torch.tensor([10000.0 ** (-2 * i / d) for i in range(d // 2)], dtype=torch.float64)
    cos, sin = ang.cos()[:, None], ang.sin()[:, None]

    def turn(z, gamma):
        z = z / (z.square().mean(-1, keepdim=True) + 1e-6).sqrt() * gamma
        a, c = z[..., :d // 2], z[..., d // 2:]
        return torch.cat([a * cos - c * sin, a * sin + c * cos], -1).transpose(1, 2)

    rk = turn(rq[:, :, h:h + kv], ref["gk"]).repeat_interleave(h // kv, 1)
    s = turn(rq[:, :, :h], ref["gq"]) @ rk.transpose(2, 3) / math.sqrt(d)
    s = s.masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), -math.inf)
    ro = s.softmax(-1) @ rq[:, :, h + kv:].transpose(1, 2).repeat_interleave(h // kv, 1)
    logits = (ro.transpose(1, 2).reshape(-1, width) @ ref["wo"].T) @ ref["head"].T
    live = (t >= 0).cpu()
    want = logits.logsumexp(1) - logits.gather(1, t.long().cpu().clamp(min=0)[:, None])[:, 0]
    (want * live).sum().div(live.sum()).backward()
    near(rows, (want * live).detach().numpy(), 1e-5, "loss")
    for name in p:
        near(g[name], ref[name].grad.numpy(), 1e-4, name)

    copies = [v.to(torch.bfloat16) for v in p.values()]
    AdamW(list(p.values()), list(g.values()), copies=copies, lr=1e-3, weight_decay=0.1).step()
    for (name, r), c in zip(ref.items(), copies):
        new, _, _ = T.adamw(r.detach().numpy(), host(g[name]), 0.0, 0.0, 1, 1e-3, (0.9, 0.999), 1e-8, 0.1)
        near(p[name], new, 1e-6, name)
        assert torch.equal(c, p[name].to(torch.bfloat16))
