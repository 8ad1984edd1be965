"""The fp64 formulas of head norms with rotation, the loss over a vocabulary and AdamW against
differences and against what they have to keep."""
import numpy as np
import pytest

from oracle import tokens as T


def differences(f, x, g, eps=1e-6):
    """The directional derivative of sum(g f) by every element of x."""
    out = np.zeros(x.shape)
    for i in np.ndindex(x.shape):
        y = x.copy()
        y[i] += eps
        hi = (f(y) * g).sum()
        y[i] -= 2 * eps
        out[i] = (hi - (f(y) * g).sum()) / (2 * eps)
    return out


@pytest.mark.parametrize("kind", ["rms", "layer", None])
@pytest.mark.parametrize("layout", ["halves", "neighbours"])
def test_head_norm_gradients_against_differences(kind, layout):
    r = np.random.RandomState(1)
    x, dy = r.randn(2, 3, 2, 12), r.randn(2, 3, 2, 12)
    params = (1 + 0.1 * r.randn(12), 0.1 * r.randn(12)) if kind else None
    more = (kind, 1e-5, r.randint(-50, 50, (2, 2, 3)), [1.0, 0.3, 0.1, 0.01], [0, 1, 1, 0], layout)
    dx, dgamma, dbeta = T.head_norm(x, params, *more, dy=dy)
    # central differences of step h: h^2 f''' / 6 and 2^-53 |f| / h, 1e-9 and below
    np.testing.assert_allclose(dx, differences(lambda t: T.head_norm(t, params, *more), x, dy), atol=1e-7)
    if kind:
        np.testing.assert_allclose(dgamma, differences(lambda t: T.head_norm(x, (t, params[1]), *more), params[0], dy), atol=1e-7)
        np.testing.assert_allclose(dbeta, differences(lambda t: T.head_norm(x, (params[0], t), *more), params[1], dy), atol=1e-7)


def test_rotation_keeps_products_of_equal_distances():
    r = np.random.RandomState(2)
    a, b = r.randn(1, 1, 1, 8), r.randn(1, 1, 1, 8)
    freq, axis = [1.0, 0.5, 0.1, 0.01], [0] * 4
    turned = [(T.rotate(a, [[[p + 5]]], freq, axis, "halves") * T.rotate(b, [[[p]]], freq, axis, "halves")).sum()
              for p in (0, 7, -3, 2 ** 30)]
    # angles of 2^30 radians in long double, 2^-64 of them: 1e-10
    np.testing.assert_allclose(turned, turned[0], rtol=1e-8)


@pytest.mark.parametrize("weighted", [False, True])
def test_vocab_gradients_against_differences(weighted):
    r = np.random.RandomState(3)
    x, w, t = r.randn(5, 8), r.randn(7, 8), np.array([3, -1, 0, 7, 6])
    weight = r.rand(5) if weighted else None
    each = np.array([1, 0, 1, 0, 1]) * (weight if weighted else 1 / 3)
    loss, lse, dx, dw = T.vocab_loss(x, w, t, 0.7, weight)
    np.testing.assert_allclose(dx, differences(lambda a: T.vocab_loss(a, w, t, 0.7)[0], x, each), atol=1e-8)
    np.testing.assert_allclose(dw, differences(lambda a: T.vocab_loss(x, a, t, 0.7)[0], w, each), atol=1e-8)
    assert (loss[[1, 3]] == 0).all() and (lse[[1, 3]] == 0).all() and (dx[[1, 3]] == 0).all()


def test_e4m3_numbers_are_those_of_the_type():
    import torch
    of = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(T.E4M3, of)


@pytest.mark.parametrize("power", [1, 2])
def test_held_values_keep_their_mean(power):
    """Over all 2^16 numbers the mean of q^power is x^power, but for the numbers' own spacing."""
    x = np.abs(np.random.RandomState(4).randn(64)) * 10.0 ** np.linspace(0, -5, 64)
    u = np.arange(4096) / 4096.0
    total = np.zeros(64)
    for a in u:
        q, scale = T.hold(x, power, np.full(64, a))
        total += (q * scale[0]) ** power
    step = np.diff(T.E4M3 ** power)[np.searchsorted(T.E4M3, x / scale[0], side="right") - 1] * scale[0] ** power
    big = x > 2.0 ** -9 * scale[0]        # r of smaller ones stays above 0
    assert (np.abs(total / 4096 - x ** power) <= step / 4096 + 1e-12 * x ** power)[big].all()
    assert big.sum() > 32


def test_adamw_moves_against_the_gradient_by_lr():
    """The first step is lr sign(g), whatever g's size, and the decay."""
    theta, g = np.array([1.0, -2.0, 3.0]), np.array([1e-3, -5.0, 0.0])
    new, m, v = T.adamw(theta, g, 0 * g, 0 * g, 1, 0.01, (0.9, 0.999), 1e-12, 0.1)
    np.testing.assert_allclose(new, theta - 0.01 * (np.sign(g) + 0.1 * theta), rtol=1e-8)
    np.testing.assert_allclose((m, v), (0.1 * g, 0.001 * g * g))
