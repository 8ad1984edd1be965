"""GPU tests of the token operators at values and sizes that their other tests leave out, against
oracle/tokens.py (fp64); helpers and bars are those of test_gpu_ops.py."""
import math

import numpy as np
import pytest
import torch

from oracle import tokens as T
from test_gpu_ops import BAR, attention, check, dev, draw, host, like, near

pytestmark = pytest.mark.gpu

# (q_len, kv_len): by 32 rows a workgroup, whose two waves share the keys, without splits and with 4, 16
# and 64; by 64 and by 128 rows without, with 5 and with 16
PLANS = [(1, 64), (2, 100), (2, 500), (1, 2000), (1, 9000), (30, 100), (100, 100), (100, 600), (100, 2000)]


def _forward(q, k, v, dtype, kvh):
    from paper_2406_02052_amd import Attention

    b, nq, h, d = q.shape
    o, lse = like(dev(q, dtype)), torch.full((b, h, nq), 7.0, device="cuda")
    Attention(b, nq, k.shape[1], h, kvh, d, dtype).forward(*(dev(x, dtype) for x in (q, k, v)), o, lse)
    torch.cuda.synchronize()
    return host(o), host(lse)


def _like_oracle(got, q, k, v, dtype):
    """NaN where the formula has it, the formula's values elsewhere."""
    with np.errstate(invalid="ignore"):
        want = T.attention(q, k, v, 1.0 / math.sqrt(q.shape[3]))
    for x, y, bar, name in zip(got, want, (BAR[dtype, "o"], 1e-5), ("o", "lse")):
        assert np.array_equal(np.isnan(x), np.isnan(y)), name
        near(np.nan_to_num(x, nan=0.0), np.nan_to_num(y, nan=0.0), bar, name, terms=1.0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("nq,nk", PLANS)
def test_attention_of_a_nan_query_is_nan(nq, nk, dtype):
    """o and lse of a query that is NaN, whatever shares its work; the others are as they should be."""
    print("case", nq, nk, dtype, flush=True)
    q, k, v = draw(nk, (2, nq, 4, 64), (2, nk, 2, 64), (2, nk, 2, 64), dtype=dtype)
    q[1, nq - 1, 2] = math.nan
    got = _forward(q, k, v, dtype, 2)
    assert np.isnan(got[0][1, nq - 1, 2]).all() and np.isnan(got[1][1, 2, nq - 1])
    _like_oracle(got, q, k, v, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("nq,nk", PLANS)
def test_attention_over_nan_keys_is_nan(nq, nk, dtype):
    """One key, and half of the keys (whole splits, or one of two waves), of one head."""
    for first, last in ((nk // 3, nk // 3 + 1), (nk // 2, nk), (0, nk // 2)):
        print("case", nq, nk, dtype, first, last, flush=True)
        q, k, v = draw(nk, (2, nq, 4, 64), (2, nk, 2, 64), (2, nk, 2, 64), dtype=dtype)
        k[0, first:last, 1] = math.nan
        got = _forward(q, k, v, dtype, 2)
        assert np.isnan(got[0][0, :, 2:]).all() and np.isnan(got[1][0, 2:]).all()
        _like_oracle(got, q, k, v, dtype)
