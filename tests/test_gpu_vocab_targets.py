"""The loss over a vocabulary with targets as text has them: few columns with most of the rows, or one with all."""
import numpy as np
import pytest
import torch

from oracle import tokens as T
from test_gpu_token_steps import ONE, TWO, dev, host, i32, nan, near, run_vocab, vocab_case

pytestmark = pytest.mark.gpu


def zipf(r, rows, vocab):
    p = 1.0 / np.arange(1, vocab + 1)
    return r.choice(vocab, rows, p=p / p.sum())


KINDS = {"uniform": lambda r, rows, vocab: r.randint(0, vocab, rows), "zipf": zipf,
         "third": lambda r, rows, vocab: np.where(r.rand(rows) < 1 / 3, 7, r.randint(0, vocab, rows)),
         "one": lambda r, rows, vocab: np.full(rows, vocab - 1)}


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("rows,width,vocab,piece", [(5000, 72, 400, 0), (700, 520, 300, 130), (33, 1032, 50, 0), (9000, 8, 3000, 0)])
def test_vocab_skewed_targets(rows, width, vocab, piece, kind):
    """Lists of one to all rows, that begin and end anywhere; twice the same.  What rounding leaves of the targets' terms is taken
    back, so that dw is off by its own rounding and by two of the terms of the others."""
    r = np.random.RandomState(rows)
    x, w, _, weight = vocab_case(rows, width, vocab, "bf16", seed=5)
    t = KINDS[kind](r, rows, vocab)
    t[r.rand(rows) < 0.05] = -1
    out, _ = run_vocab(x, w, t, "bf16", weight, piece=piece)
    want = T.vocab_loss(x, w, t, 1.0, weight)
    near(out[2], want[2], ONE["bf16"], "dx")
    near(out[3], want[3], TWO["bf16"], "dw")
    # whole columns, of which each is nearly its own rows alone
    p = np.bincount(t[t >= 0], minlength=vocab)
    for j in np.argsort(-p)[:3]:
        if p[j]:
            near(out[3][j], want[3][j], TWO["bf16"], ("dw of column", j, p[j]))
    again, _ = run_vocab(x, w, t, "bf16", weight, piece=piece)
    assert all(torch.equal(a, b) for a, b in zip(out, again))


def test_vocab_time_does_not_go_by_the_targets():
    """2048 x 1024 over 32768: the frequent tokens of a text, a third of the rows or all of them at one column take no longer
    than targets drawn evenly, but for what one card's times differ by."""
    from paper_2406_02052_amd import VocabLoss

    rows, width, vocab = 2048, 1024, 32768
    r = np.random.RandomState(1)
    x, w, _, _ = vocab_case(rows, width, vocab, "bf16")
    x, w = dev(x, "bf16"), dev(w, "bf16")
    op = VocabLoss(rows, width, vocab)
    out = [nan((rows,)), nan((rows,)), nan((rows, width), "bf16"), nan((vocab, width), "bf16")]
    took = {}
    for kind in ("uniform", "zipf", "third", "one", "uniform"):
        t = i32(KINDS[kind](r, rows, vocab))
        times = []
        for _ in range(12):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            op.gradient(x, w, t, *out)
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        took[kind] = sorted(times)[len(times) // 2]
    print("ms", took, flush=True)
    assert all(v <= 1.3 * took["uniform"] for v in took.values()), took
    assert np.isfinite(host(out[3])).all()
