"""Head norms with rotation, the loss over a vocabulary and AdamW as programs use them: captured and replayed,
two graphs of one workspace, other streams, strides that the layout leaves open, what lies beside the tensors."""
import math

import numpy as np
import pytest
import torch

from oracle import tokens as T
from test_gpu_token_steps import (ONE, RNG, TWO, adam_case, dev, draw, heads_case, host, i32, like, nan, near, on_device, run_vocab,
                                  vocab_case)

pytestmark = pytest.mark.gpu


def captured(body):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        body()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        body()
    return g


def test_replayed_steps_are_the_eager_ones():
    """Head norms forward and backward, the loss with gradients and an 8-bit AdamW step in one graph, replayed with eager
    work between; inputs, lr and random numbers change from replay to replay."""
    from paper_2406_02052_amd import AdamW, HeadNorm, VocabLoss

    b, n, h, kv, d, vocab = 2, 50, 4, 2, 64, 600
    width = h * d
    torch.manual_seed(1)
    qk = torch.empty(b, n, h + kv, d, dtype=torch.bfloat16, device="cuda")
    q, k = qk[:, :, :h], qk[:, :, h:]
    gamma = torch.ones(d, device="cuda")
    pos = torch.zeros(1, b, n, dtype=torch.int32, device="cuda")
    target = torch.zeros(b * n, dtype=torch.int32, device="cuda")
    theta = torch.randn(vocab, width, device="cuda")
    copy, grad = theta.to(torch.bfloat16), torch.zeros(vocab, width, dtype=torch.bfloat16, device="cuda")
    rng, scale = torch.zeros(2, dtype=torch.int64, device="cuda"), torch.ones(1, device="cuda")
    y = [torch.empty_like(q.contiguous()), torch.empty_like(k.contiguous())]
    rows, lse, dx = torch.empty(b * n, device="cuda"), torch.empty(b * n, device="cuda"), torch.empty_like(y[0])
    dqk, dn = torch.empty_like(qk), [torch.empty_like(gamma) for _ in range(2)]
    norm, loss = HeadNorm(b, n, h, kv, d), VocabLoss(b * n, width, vocab)
    adam = AdamW([theta], [grad], states="fp8", copies=[copy], zero_grads=True)

    def body():
        norm.forward(q, k, *y, q_norm=(gamma, None), k_norm=(gamma, None), positions=pos)
        loss.gradient(y[0].view(b * n, width), copy, target, rows, lse, dx.view(b * n, width), grad)
        norm.backward(q, k, dx, y[1], dqk[:, :, :h], dqk[:, :, h:], q_norm=(gamma, None), k_norm=(gamma, None),
                      dq_norm=(dn[0], None), dk_norm=(dn[1], None), positions=pos)
        adam.step(rng=rng, grad_scale=scale)

    state = [theta, copy, grad, adam.m.view(torch.uint8), adam.v.view(torch.uint8), adam.m_scale, adam.v_scale, adam.steps]
    results = state + [*y, rows, lse, dx, dqk, *dn]

    def inputs(i):
        torch.manual_seed(100 + i)
        qk.copy_(torch.randn_like(qk))
        pos.copy_(torch.randint(0, 1000, pos.shape, device="cuda"))
        target.copy_(torch.randint(-1, vocab, target.shape, device="cuda"))
        rng.copy_(torch.tensor([7, i]))
        scale.fill_(0.5 + i)
        adam.lr.fill_(1e-3 * (i + 1))

    inputs(0)
    graph = captured(body)
    start = [t.clone() for t in state]
    eager = []
    for i in range(4):
        inputs(i)
        body()
        torch.cuda.synchronize()
        eager.append([t.clone() for t in results])
    for t, s in zip(state, start):
        t.copy_(s)
    for i in range(4):
        inputs(i)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a.nan_to_num(), b.nan_to_num()) for a, b in zip(results, eager[i])), i
        torch.randn(1000, 1000, device="cuda").sum().item()


def test_two_graphs_share_a_workspace():
    """A workspace holds nothing between calls: graphs of one owner may be replayed in turn."""
    from paper_2406_02052_amd import VocabLoss

    op = VocabLoss(300, 64, 1000, "bf16", piece_rows=128)
    cases = [vocab_case(300, 64, 1000, "bf16", seed=s) for s in (1, 2)]
    graphs, outs = [], []
    for x, w, t, weight in cases:
        a = dev(x, "bf16"), dev(w, "bf16"), i32(t)
        o = [nan((300,)), nan((300,)), nan(x.shape, "bf16"), nan(w.shape, "bf16")]
        graphs.append((captured(lambda a=a, o=o: op.gradient(*a, *o)), a))
        outs.append(o)
    for _ in range(3):
        for g, o, (x, w, t, _) in zip(graphs, outs, cases):
            for y in o:
                y.fill_(math.nan)
            g[0].replay()
            torch.cuda.synchronize()
            want = T.vocab_loss(x, w, t)
            near(o[0], want[0], 1e-5, "loss")
            near(o[2], want[2], ONE["bf16"], "dx")
            near(o[3], want[3], TWO["bf16"], "dw")


def test_calls_on_another_stream():
    """By the current stream and by an argument; an owner may be dropped at once."""
    from paper_2406_02052_amd import AdamW, HeadNorm, VocabLoss

    x, w, t, _ = vocab_case(200, 64, 500, "fp32")
    want = T.vocab_loss(x, w, t)
    side = torch.cuda.Stream()
    a = dev(x, "fp32"), dev(w, "fp32"), i32(t)
    c = heads_case((2, 9, 4, 2, 64, 32), "fp32", "rms", "halves", 1)
    q, k, qn, kn, pos = dev(c["q"], "fp32"), dev(c["k"], "fp32"), on_device(c["params"][0]), on_device(c["params"][1]), i32(c["pos"])
    dq, dk, dqn, dkn = torch.empty_like(q), torch.empty_like(k), like(qn), like(kn)
    theta, g = torch.ones(5000, device="cuda"), torch.ones(5000, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    for how in ("current", "argument"):
        out = [nan((200,)), nan((200,)), nan(x.shape), nan(w.shape)]
        with torch.cuda.stream(side if how == "current" else torch.cuda.current_stream()):
            more = {} if how == "current" else {"stream": side}
            side.wait_stream(torch.cuda.default_stream())
            VocabLoss(200, 64, 500, "fp32").gradient(*a, *out, **more)
            HeadNorm(2, 9, 4, 2, 64, "fp32", eps=1e-5, freq=c["freq"], axis=c["axis"]).backward(
                q, k, q, k, dq, dk, q_norm=qn, k_norm=kn, dq_norm=dqn, dk_norm=dkn, positions=pos, **more)
            op = AdamW([theta], [g], lr=0.0)
            side.wait_stream(torch.cuda.current_stream())
            op.step(**more)
            del op
        junk = [torch.full((1 << 20,), math.nan, device="cuda") for _ in range(8)]   # in what was given back, if it was
        side.synchronize()
        near(out[2], want[2], ONE["fp32"], "dx")
        near(out[3], want[3], TWO["fp32"], "dw")
        near(dq, T.head_norm(c["q"], c["params"][0], "rms", 1e-5, c["pos"], c["freq"], c["axis"], "halves", dy=c["q"])[0], 1e-5, "dq")
        assert (theta == 1).all()
        del junk


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_heads_strides(dtype):
    """Heads before tokens, rows with gaps, one head's slice; what lies between stays."""
    from paper_2406_02052_amd import HeadNorm

    shape = (3, 21, 5, 2, 40, 20)
    b, n, h, kv, d, _ = shape
    c = heads_case(shape, dtype, "rms", "halves", 1)
    t = torch.float32 if dtype == "fp32" else torch.bfloat16
    op = HeadNorm(b, n, h, kv, d, dtype, eps=1e-5, freq=c["freq"], axis=c["axis"])
    qn, kn = (on_device(p) for p in c["params"])
    more = ("rms", 1e-5, c["pos"], c["freq"], c["axis"], "halves")
    first = torch.zeros(b, h, n, d, dtype=t, device="cuda").transpose(1, 2)             # heads before tokens
    gaps = torch.full((b, n + 3, kv, d + 24), 5.0, dtype=t, device="cuda")
    k = gaps[:, 2:n + 2, :, 16:d + 16]
    first.copy_(dev(c["q"], dtype))
    k.copy_(dev(c["k"], dtype))
    before = gaps.clone()
    out = torch.full((b, n, h + 2 * kv, d), 9.0, dtype=t, device="cuda")
    yk = torch.full((b, kv, n, d), 9.0, dtype=t, device="cuda").transpose(1, 2)
    op.forward(first, k, out[:, :, kv:kv + h], yk, q_norm=qn, k_norm=kn, positions=i32(c["pos"]))
    near(out[:, :, kv:kv + h], T.head_norm(c["q"], c["params"][0], *more), ONE[dtype], "q")
    near(yk, T.head_norm(c["k"], c["params"][1], *more), ONE[dtype], "k")
    assert torch.equal(gaps, before) and (out[:, :, :kv] == 9).all() and (out[:, :, kv + h:] == 9).all()
    # in place over the gaps
    op.forward(first, k, out[:, :, kv:kv + h], k, q_norm=qn, k_norm=kn, positions=i32(c["pos"]))
    assert torch.equal(k, yk)
    k.copy_(dev(c["k"], dtype))
    assert torch.equal(gaps, before)


def test_heads_broadcast_inputs():
    """An input may repeat itself: one token's queries for all tokens."""
    from paper_2406_02052_amd import HeadNorm

    b, n, h, d = 2, 11, 3, 64
    q, = draw(1, (b, 1, h, d))
    t = dev(q, "fp32").expand(b, n, h, d)
    op = HeadNorm(b, n, h, 0, d, "fp32", norm=None)
    y = nan((b, n, h, d))
    op.forward(t, None, y, None)
    freq = [10000.0 ** (-2 * i / d) for i in range(d // 2)]
    near(y, T.rotate(np.broadcast_to(q, y.shape), np.broadcast_to(np.arange(n), (1, b, n)), freq, [0] * 32, "halves"), 1e-6, "y")
    with pytest.raises(Exception, match="share memory"):
        op.backward(None, None, y, None, t, None)


def test_adamw_leaves_what_lies_beside():
    """Tensors of odd sizes in one buffer: the elements between them stay, and states past a tensor's end are zeros."""
    from paper_2406_02052_amd import AdamW

    sizes = [1, 5, 63, 65, 4095, 4097]
    for states in ("fp32", "fp8"):
        buf, gbuf = torch.full((6 * 4160,), 3.0, device="cuda"), torch.full((6 * 4160,), 2.0, device="cuda")
        cbuf = torch.full((6 * 4160,), 4.0, dtype=torch.bfloat16, device="cuda")
        part = lambda t: [t[4160 * i:4160 * i + n] for i, n in enumerate(sizes)]  # noqa: E731
        op = AdamW(part(buf), part(gbuf), states=states, copies=part(cbuf), zero_grads=True)
        op.step(rng=torch.tensor(RNG, dtype=torch.int64, device="cuda"))
        for i, n in enumerate(sizes):
            for t, v in ((buf, 3.0), (gbuf, 2.0), (cbuf, 4.0)):
                at = t[4160 * i:4160 * (i + 1)]
                assert (at[n:] == v).all() and not (at[:n] == v).any()
            end = op.starts[i + 1] if i + 1 < len(sizes) else op.m.numel()
            for s in (op.m, op.v):
                assert (s.float()[op.starts[i]:op.starts[i] + n] > 0).all() and (s.float()[op.starts[i] + n:end] == 0).all()


def test_adamw_same_results_again_and_other_offsets():
    """A step with the same rng rounds alike, with another offset otherwise."""
    from paper_2406_02052_amd import AdamW

    got = []
    for offset in (1, 1, 2):
        theta, grads, _, decay = adam_case("fp8", "fp32", False)
        op = AdamW(theta, grads, states="fp8", weight_decay=decay)
        op.step(rng=torch.tensor([3, offset], dtype=torch.int64, device="cuda"))
        got.append((op.m.view(torch.uint8), op.v.view(torch.uint8)))
    assert all(torch.equal(a, b) for a, b in zip(got[0], got[1]))
    assert not torch.equal(got[0][0], got[2][0]) and not torch.equal(got[0][1], got[2][1])


def test_adamw_late_steps_and_extreme_betas():
    """The corrections at the first step, a late one, and without averaging."""
    from paper_2406_02052_amd import AdamW

    for betas, steps in (((0.9, 0.999), 0), ((0.9, 0.999999), 0), ((0.9, 0.999), 10 ** 7), ((0.0, 0.0), 5)):
        theta, g = dev(np.linspace(-1, 1, 300), "fp32"), dev(np.linspace(2, -3, 300), "fp32")
        before = host(theta)
        op = AdamW([theta], [g], betas=betas, lr=0.1, weight_decay=0.0)
        op.steps.fill_(steps)
        op.step()
        want, _, _ = T.adamw(before, host(g), 0.0, 0.0, steps + 1, 0.1, betas, 1e-8, 0.0)
        near(theta, want, 1e-6, (betas, steps))


def test_vocab_over_32_bits_of_offset():
    """A piece whose e passes 2^31 bytes would not fit 32-bit offsets from its start: rows at the end of a GiB of e, and a w of
    more than 2^32 bytes."""
    from paper_2406_02052_amd import VocabLoss

    rows, width, vocab = 520, 2056, 2 ** 20
    g = torch.Generator("cuda").manual_seed(1)
    x = torch.randn(rows, width, generator=g, device="cuda").bfloat16()
    w = torch.empty(vocab, width, dtype=torch.bfloat16, device="cuda")
    for part in w.split(2 ** 17):
        part.copy_(torch.randn(part.shape, generator=g, device="cuda") / width ** 0.5)
    t = torch.randint(vocab, (rows,), generator=g, dtype=torch.int32, device="cuda")
    t[rows - 1] = vocab - 1
    op = VocabLoss(rows, width, vocab)
    loss, lse, dx, dw = nan((rows,)), nan((rows,)), nan(x.shape, "bf16"), nan(w.shape, "bf16")
    op.gradient(x, w, t, loss, lse, dx, dw)
    total, want = torch.zeros(rows, dtype=torch.float64, device="cuda"), torch.zeros(rows, width, dtype=torch.float64, device="cuda")
    for part in w.split(2 ** 17):   # (scores are within 10 of 0)
        e = (x.double() @ part.double().T).exp()
        total += e.sum(1)
        want += e @ part.double()
    target = w[t.long()].double()
    near(lse, total.log().cpu().numpy(), 1e-5, "lse")
    near(loss, (total.log() - (x.double() * target).sum(1)).cpu().numpy(), 1e-5, "loss")
    near(dx, ((want / total[:, None] - target) / rows).cpu().numpy(), ONE["bf16"], "dx")
    for j in (0, 12345, vocab // 2 + 1, vocab - 1, int(t[0])):
        p = (x.double() @ w[j].double() - total.log()).exp() - (t == j).double()
        near(dw[j], (p @ x.double() / rows).cpu().numpy(), TWO["bf16"], j)


def test_vocab_of_more_rows_than_a_grid_has_waves():
    """2^26 rows and some, in several pieces: rows of one of four kinds, whose results are each other's."""
    from paper_2406_02052_amd import VocabLoss

    rows, width, vocab = 2 ** 26 + 5, 8, 3
    x4, = draw(1, (4, width), dtype="bf16")
    w, = draw(2, (vocab, width), dtype="bf16")
    t4 = np.array([2, 0, -1, 1])
    kind = torch.arange(rows, device="cuda") % 4
    t = i32(t4)[kind]
    x = torch.empty(rows, width, dtype=torch.bfloat16, device="cuda")
    for to, k in zip(x.split(2 ** 22), kind.split(2 ** 22)):   # (indexing for all at once leaves all but the first 5 rows empty)
        to.copy_(dev(x4, "bf16")[k])
    op = VocabLoss(rows, width, vocab, gradients=False)
    loss, lse = nan((rows,)), nan((rows,))
    op.forward(x, dev(w, "bf16"), t, loss, lse)
    want = T.vocab_loss(x4, w, t4)
    for got, r in ((loss, want[0]), (lse, want[1])):
        r = torch.tensor(r, device="cuda")[kind]
        assert ((got.double() - r).abs() <= 1e-5 * r.abs() + 1e-6).all()


@pytest.mark.parametrize("rows,vocab,piece", [(2000, 300, 0), (1500, 1000, 700), (3000, 260, 0), (700, 257, 100), (64, 5000, 0), (5000, 300, 0)])
def test_vocab_targets_of_many_rows(rows, vocab, piece):
    """Targets that repeat (a third of all rows at one column, as of a frequent token), at the edges of groups of 256 columns and in
    several pieces.  Where rows are listed by target (16 a column at most) what rounding leaves of their terms is taken
    back and dw, whose larger part they are, is off by its own rounding and two of the smaller part: 2^-8, as dx."""
    width = 72
    x, w, t, weight = vocab_case(rows, width, vocab, "bf16", seed=3)
    r = np.random.RandomState(1)
    t[r.rand(rows) < 0.33] = 255
    t[r.rand(rows) < 0.1] = vocab - 1
    t[r.rand(rows) < 0.1] = -1
    t[:3] = 0, 256 % vocab, vocab - 1
    for wt in (None, weight):
        out, _ = run_vocab(x, w, t, "bf16", wt, piece=piece)
        want = T.vocab_loss(x, w, t, 1.0, wt)
        near(out[2], want[2], ONE["bf16"], "dx")
        near(out[3], want[3], ONE["bf16"] if (piece or rows) <= 16 * vocab else TWO["bf16"], "dw")
        again, _ = run_vocab(x, w, t, "bf16", wt, piece=piece)
        assert torch.equal(out[3], again[3])
