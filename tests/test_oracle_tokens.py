"""Pins of oracle/tokens.py: the generator's published answers, attention and the
coupling against torch's automatic differentiation in fp64 and against differences,
and what masks leave out."""
import numpy as np
import pytest
import torch

from oracle import tokens as T

R = np.random.RandomState


@pytest.mark.parametrize("rounds,want", [(7, "5f6fb709 0d893f64 4f121f81 4f730a48"),
                                         (10, "6627e8d5 e169c58d bc57ac4c 9b00dbd8")])
def test_philox_published_answers(rounds, want):
    got = T.philox(np.zeros(4, np.uint64), (0, 0), rounds)
    assert " ".join("%08x" % int(v) for v in got) == want


def test_factors_keep_their_share_and_scale():
    m = T.factor((5, 9), 0.25, (1 << 16,))
    kept = (m > 0).mean()
    assert abs(kept - 0.75) < 5 * np.sqrt(0.25 * 0.75 / m.size)
    assert np.allclose(m[m > 0], 1 / 0.75)
    a = T.factor_attention((5, 9), 0.25, 1, 2, 3, 40)
    assert a.shape == (1, 2, 3, 40) and abs((a > 0).mean() - 0.75) < 0.15
    # keys 0..3 and 8..11 are group 0 of the first row
    assert np.array_equal(a[0, 0, 0, [0, 1, 2, 3, 8, 9, 10, 11]] > 0, T.factor((5, 9), 0.25, (8,)) > 0)


def _attn_inputs(seed=0, b=3, nq=5, nk=7, h=4, kvh=2, d=8):
    r = R(seed)
    return [r.randn(b, nq, h, d), r.randn(b, nk, kvh, d), r.randn(b, nk, kvh, d), r.randn(b, nq, h, d)]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lens", [None, ([5, 3, 4], [7, 0, 2])])
def test_attention_matches_autograd(causal, lens):
    q, k, v, g = _attn_inputs()
    lq, lk = lens or ([5] * 3, [7] * 3)
    mask = T.factor_attention((1, 2), 0.3, 3, 4, 5, 7)
    got = T.attention(q, k, v, 0.4, causal, lq, lk, mask, g)
    tq, tk, tv = (torch.tensor(x, requires_grad=True) for x in (q, k, v))
    s = torch.einsum("bihd,bjhd->bhij", tq, tk.repeat_interleave(2, 2)) * 0.4
    seen = torch.tensor(np.stack([T.visible(5, 7, a, c, causal) for a, c in zip(lq, lk)]))[:, None]
    p = torch.where(seen.any(-1, keepdim=True), s.masked_fill(~seen, -1e30).softmax(-1), torch.zeros(()).double())
    o = torch.einsum("bhij,bjhd->bihd", p * torch.tensor(mask), tv.repeat_interleave(2, 2))
    dq, dk, dv = torch.autograd.grad(o, [tq, tk, tv], torch.tensor(g))
    for x, y in zip((got[0],) + got[2:], (o, dq, dk, dv)):
        assert np.allclose(x, y.detach().numpy(), atol=1e-12)
    empty = ~seen.any(-1).expand(3, 4, 5).numpy()
    assert np.isneginf(got[1][empty]).all() and np.isfinite(got[1][~empty]).all()


def test_attention_ignores_what_lies_past_the_lengths():
    q, k, v, g = _attn_inputs()
    want = T.attention(q, k, v, 0.4, True, [5, 3, 4], [7, 2, 5], None, g)
    for t, lens in ((q, [5, 3, 4]), (g, [5, 3, 4]), (k, [7, 2, 5]), (v, [7, 2, 5])):
        for b, n in enumerate(lens):
            t[b, n:] = np.nan
    for x, y in zip(T.attention(q, k, v, 0.4, True, [5, 3, 4], [7, 2, 5], None, g), want):
        assert np.array_equal(x, y)


def _differences(fun, x, d, h=1e-5):
    return (fun(x + h * d) - fun(x - h * d)) / (2 * h)


def test_attention_gradients_match_differences():
    q, k, v, g = _attn_inputs(3)
    mask = T.factor_attention((1, 2), 0.3, 3, 4, 5, 7)
    _, _, *grads = T.attention(q, k, v, 0.4, True, [5, 3, 4], [7, 2, 5], mask, g)
    for i, grad in enumerate(grads):
        d = R(9 + i).randn(*grad.shape)

        def loss(x, i=i):
            t = [q, k, v]
            t[i] = x
            return (T.attention(*t, 0.4, True, [5, 3, 4], [7, 2, 5], mask)[0] * g)[[0]].sum() \
                + (T.attention(*t, 0.4, True, [5, 3, 4], [7, 2, 5], mask)[0][1, :3] * g[1, :3]).sum() \
                + (T.attention(*t, 0.4, True, [5, 3, 4], [7, 2, 5], mask)[0][2, :4] * g[2, :4]).sum()
        assert np.isclose(_differences(loss, (q, k, v)[i], d), (grad * d).sum(), rtol=1e-6, atol=1e-8)


@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("with_u", [False, True])
def test_coupling_gradients_match_autograd_and_differences(norm, with_u):
    r = R(1)
    x, f, dy, du = (r.randn(6, 8) for _ in range(4))
    gate, post, pre = r.randn(3, 8), (r.randn(8), r.randn(8)), (r.randn(8), r.randn(8))
    mask = T.factor((3, 4), 0.3, (6, 8))
    y = T.coupling(x, f, gate, post, norm, 1e-5, 0.75, mask)
    got = T.coupling_backward(y, f, dy, gate, post, norm, 1e-5, 0.75, mask, du if with_u else None, pre)
    assert np.allclose(got["x"], x)
    names = ["x", "f", "gate", "gamma", "beta", "pg", "pb"]
    vals = [x, f, gate, post[0], post[1], pre[0], pre[1]]

    def loss(vals):
        x, f, gate, a, b, c, d = vals
        y = T.coupling(x, f, gate, (a, b), norm, 1e-5, 0.75, mask)
        return (y * dy).sum() + ((T.norm_forward(y, (c, d), norm, 1e-5) * du).sum() if with_u else 0.0)

    grads = [got["dx"], got["df"], got["dgate"], *got["dpost"], *got.get("dpre", (None, None))]
    for i, (name, grad) in enumerate(zip(names, grads)):
        if grad is None:
            continue
        d = R(20 + i).randn(*vals[i].shape)
        diff = _differences(lambda z, i=i: loss(vals[:i] + [z] + vals[i + 1:]), vals[i], d)
        assert np.isclose(diff, (grad * d).sum(), rtol=1e-6, atol=1e-8), name
    # and the norm itself against torch's
    t = torch.tensor(f)
    want = (torch.nn.functional.layer_norm(t, (8,), *map(torch.tensor, post), 1e-5) if norm == "layer"
            else torch.nn.functional.rms_norm(t, (8,), torch.tensor(post[0]), 1e-5) + torch.tensor(post[1]))
    assert np.allclose(T.norm_forward(f, post, norm, 1e-5), want.numpy(), atol=1e-12)


def test_dropout_and_its_inverse():
    x, r = R(0).randn(1001), R(1).randn(1001)
    y = T.dropout(x, 0.5, (7, 8), r)
    assert np.allclose(T.dropout(x, 0.5, (7, 8), y, -1.0), r)
    assert set(np.unique(np.round((y - r)[x != 0] / x, 9))) <= {0.0, 2.0}
