"""Loss over a vocabulary where the target has nearly all of the softmax: loss and gradients follow what the others have,
however little, and not the rounding of a number near 1.

Bars, relative to the sum of the magnitudes of a result's terms.  A term p_j (j no target) is off as exp(s_j - s_t) is, by
the rounding of both scores: sums of `width` products in fp32, taken by 64 lanes (width / 64 products and 6 additions one after the
other) for the target's and by the matrix unit (blocks of 16, at most 16 additions within) for the others, each addition 2^-24 of a
partial sum of at most the sum of magnitudes; a scale by log2(e) and the power of two: 3 more of the score.  The target's term is
minus the sum of the others', no worse than they are.  bf16 tensors round e, the result and (dw) f x, 2^-8 each."""
import math

import numpy as np
import pytest
import torch

from oracle import tokens as T
from test_gpu_token_steps import dev, draw, host, run_vocab

pytestmark = pytest.mark.gpu


def confident(width, vocab, dtype, seed=0):
    """Rows of 1 - p from 1e-2 to 1e-6, eight of each decade, each with a target of its own; and where the scores lie."""
    per, decades = 8, 5
    rows = per * decades
    w, = draw(seed + 1, (vocab, width), dtype=dtype, std=2.0 / math.sqrt(width))
    noise, = draw(seed + 2, (rows, width), std=0.05)
    t = np.random.RandomState(seed).permutation(vocab)[:rows]
    x = np.empty((rows, width))
    for i in range(rows):
        want = math.log(vocab) + math.log(10.0) * (2 + i // per)   # about the score of the target
        x[i] = w[t[i]] * want / (w[t[i]] @ w[t[i]]) + noise[i]
    return host(dev(x, dtype)), w, t


def terms(x, w, t, weight=None):
    """|weight (p - 1[target])|, 1 - p of the targets, and the bar of a score's exponential in this case."""
    s = x @ w.T
    p = np.exp(s - s.max(1)[:, None])
    at = np.arange(len(x)), t
    others = p.copy()
    others[at] = 0.0
    z = p.sum(1)
    g = others / z[:, None]
    rest = g.sum(1)
    g[at] = rest
    width, size = x.shape[1], np.abs(x) @ np.abs(w).T
    bar = 2.0 ** -24 * ((width / 64 + 6) * size[at].max() + (width / 16 + 16) * size.max() + 6 * np.abs(s).max())
    return g / len(x), rest, bar


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("width,vocab,piece", [(1024, 2000, 0), (256, 700, 16), (64, 300, 0)])
def test_vocab_confident_rows_by_decade(width, vocab, piece, dtype):
    x, w, t = confident(width, vocab, dtype)
    g, rest, bar = terms(x, w, t)
    assert rest.min() < 1e-5 and rest.max() > 3e-3 and bar < 1e-3   # (about the case itself)
    out, alone = run_vocab(x, w, t, dtype, piece=piece)
    want = T.vocab_loss(x, w, t)
    for got in (out, alone):
        loss = host(got[0])
        assert (loss >= 0).all()
        # log(1 + rest) of rest: no larger error; and its own rounding
        off = np.abs(loss - want[0]) / want[0]
        assert off.max() <= bar + 2.0 ** -22, off.max()
    one = 2.0 ** -8 if dtype == "bf16" else 0.0
    norms = np.linalg.norm(w, axis=1), np.linalg.norm(x, axis=1)
    for name, got, exact, size, bits in (("dx", out[2], want[2], g @ norms[0], 2 * one), ("dw", out[3], want[3], g.T @ norms[1], 3 * one)):
        off = np.linalg.norm(host(got) - exact, axis=1) / size
        assert off.max() <= 2 * bar + bits + 2.0 ** -20, (name, off.max())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_vocab_terms_of_a_row_cancel(dtype):
    """Columns that are all one vector: a row's terms sum to nothing, so its dx is only what rounding e leaves (2^-8 of the sum of
    the others', which are the target's)."""
    width, vocab, rows = 128, 500, 24
    base, = draw(3, (1, width), dtype=dtype)
    w = np.repeat(base, vocab, 0)
    x, = draw(4, (rows, width), dtype=dtype)
    t = np.arange(rows) * 20 + 3
    out, _ = run_vocab(x, w, t, dtype)
    loss = host(out[0])
    # all scores are equal but for the order of their sums
    size = np.abs(x) @ np.abs(base[0])
    bar = 2.0 ** -24 * ((width / 64 + 6 + width / 16 + 16) * size.max() + 6 * np.abs(x @ base[0]).max())
    assert np.abs(loss - math.log(vocab)).max() <= bar + 2.0 ** -20
    off = np.linalg.norm(host(out[2]), axis=1) / (np.linalg.norm(base) * (vocab - 1) / vocab / rows)
    assert off.max() <= (2.0 ** -8 if dtype == "bf16" else 0.0) + 2 * bar + 2.0 ** -20, off.max()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("where", ["row", "column"])
def test_vocab_target_scores_that_are_no_numbers(where, dtype):
    """A target's score of infinity or NaN (by its column or by the row) leaves no finite loss."""
    x, = draw(5, (40, 64), dtype=dtype)
    x[:, 5] = np.abs(x[:, 5])
    w, = draw(6, (300, 64), dtype=dtype)
    t = np.arange(40) * 7
    for bad in (math.nan, math.inf):
        y, v = x.copy(), w.copy()
        if where == "row":
            y[11, 5] = bad
        else:
            v[t[11], 5] = bad
        _, alone = run_vocab(y, v, t, dtype)
        assert not torch.isfinite(alone[0][11]) and not torch.isfinite(alone[1][11])


def test_vocab_loss_of_known_scores():
    """Two columns with scores of 0 and -c: log(1 + e^-c), from c = 0 to where it leaves fp32's normal numbers.  The scale by log2(e) is off
    by 2^-24 of c in its factor and its product each, and power, logarithm, quotient and their products by 2^-23 each."""
    c = host(torch.linspace(0.0, 86.0, 777))
    x, w = np.zeros((777, 8)), np.zeros((2, 8))
    x[:, 0], w[1, 0] = -c, 1.0
    _, alone = run_vocab(x, w, np.zeros(777, int), "fp32")
    want = np.log1p(np.exp(-c))
    off = np.abs(host(alone[0]) - want) / want
    assert (off <= 2.0 ** -23 * (c + 8)).all(), (off / (c + 8)).max() * 2 ** 23
