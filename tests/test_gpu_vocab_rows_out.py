"""Rows that take no part in the loss have a gradient of 0 whatever the columns hold, too."""
import math

import numpy as np
import pytest
import torch

from test_gpu_token_steps import draw, run_vocab

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,vocab,piece", [(300, 513, 0), (40, 100, 16), (64, 20000, 0)])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_vocab_columns_that_are_no_numbers(bad, rows, vocab, piece, dtype):
    x, = draw(1, (rows, 72), dtype=dtype)
    w, = draw(2, (vocab, 72), dtype=dtype)
    w[vocab // 2, 9] = bad
    t = np.arange(rows) % vocab
    t[::3] = np.array([-1, vocab, -2 ** 31])[np.arange(len(t[::3])) % 3]
    out, alone = run_vocab(x, w, t, dtype, piece=piece)
    dead = torch.tensor((t < 0) | (t >= vocab), device="cuda")
    for got in (out[0], out[1], out[2], alone[0], alone[1]):
        assert (got[dead] == 0).all()
    assert not torch.isfinite(out[2][~dead]).any(0).all()   # (those of the others do not pass for numbers)
