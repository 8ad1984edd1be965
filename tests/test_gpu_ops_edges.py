"""GPU tests of the token operators at values and sizes that their other tests leave out, against
oracle/tokens.py (fp64); helpers and bars are those of test_gpu_ops.py."""
import math

import numpy as np
import pytest
import torch

from oracle import tokens as T
from test_gpu_ops import BAR, RNG, attention, check, coupling, dev, draw, host, like, near, rng_tensor

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


# causal with more queries than keys: the first ones see none.  (batch, q_len, kv_len, heads, kv_heads, dim),
# lengths; row tiles that such queries end inside of, head groups that divide no tile, splits of rows and keys
BLIND = [((2, 70, 20, 4, 2, 64), None), ((1, 90, 37, 3, 1, 40), None), ((3, 70, 97, 4, 2, 64), ([60, 70, 33], [41, 0, 64])),
         ((1, 900, 300, 4, 1, 128), None), ((2, 33, 5, 2, 2, 32), ([33, 20], [5, 1]))]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("p", [0.0, 0.2])
@pytest.mark.parametrize("shape,lens", BLIND, ids=str)
def test_attention_queries_without_keys_may_hold_anything(shape, lens, p, dtype):
    """NaN and infinities in queries that see no key, and in their d_o, reach nothing."""
    from paper_2406_02052_amd import Attention

    print("case", shape, lens, p, dtype, flush=True)
    b, nq, nk, h, kvh, d = shape
    lq, lk = lens or ([nq] * b, [nk] * b)
    q, k, v, g = draw(nq, (b, nq, h, d), (b, nk, kvh, d), (b, nk, kvh, d), (b, nq, h, d), dtype=dtype)
    mask = T.factor_attention(RNG, p, b, h, nq, nk) if p else None
    want = T.attention(q, k, v, 1 / math.sqrt(d), True, lq, lk, mask, g)
    for i in range(b):
        blind = max(0, lq[i] - lk[i])
        assert i or blind
        for t in (q, g):
            t[i, :blind] = np.array([math.nan, math.inf, -math.inf])[np.arange(blind) % 3, None, None]
            t[i, lq[i]:] = math.nan
    t = [dev(x, dtype) for x in (q, k, v, g)]
    op = Attention(b, nq, nk, h, kvh, d, dtype, causal=True, dropout=p)
    more = dict(rng=rng_tensor() if p else None)
    if lens:
        more.update(q_lens=torch.tensor(lq, dtype=torch.int32, device="cuda"), kv_lens=torch.tensor(lk, dtype=torch.int32, device="cuda"))
    o, lse, grads = like(t[0]), torch.full((b, h, nq), math.nan, device="cuda"), [like(x) for x in t[:3]]
    op.forward(*t[:3], o, lse, **more)
    op.backward(*t[:3], o, lse, t[3], *grads, **more)
    torch.cuda.synchronize()
    check([o, lse, *grads], want, dtype)
    for x in (o, grads[0]):
        for i in range(b):
            assert (x[i, :max(0, lq[i] - lk[i])] == 0).all() and (x[i, lq[i]:] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("nk", [60, 700])
@pytest.mark.parametrize("nq", [6, 40, 200])
def test_attention_infinities_stay_out_of_rows_past_the_length(nq, nk, dtype):
    """A value that is infinite where the queries within the length see it."""
    from paper_2406_02052_amd import Attention

    print("case", nq, nk, dtype, flush=True)
    q, k, v, g = (dev(x, dtype) for x in draw(nq, (1, nq, 2, 64), (1, nk, 2, 64), (1, nk, 2, 64), (1, nq, 2, 64), dtype=dtype))
    v[0, nk // 2] = math.inf
    n = nq // 2
    lens = dict(q_lens=torch.tensor([n], dtype=torch.int32, device="cuda"))
    op = Attention(1, nq, nk, 2, 2, 64, dtype)
    o, lse, grads = like(q), torch.full((1, 2, nq), math.nan, device="cuda"), [like(x) for x in (q, k, v)]
    op.forward(q, k, v, o, lse, **lens)
    op.backward(q, k, v, o, lse, g, *grads, **lens)
    torch.cuda.synchronize()
    for x in (o, grads[0]):
        assert not torch.isfinite(x[0, :n]).any() and (x[0, n:] == 0).all()
    assert torch.isfinite(lse[:, :, :n]).all() and torch.isneginf(lse[:, :, n:]).all()


@pytest.mark.parametrize("nq,nk", [(3, 50), (40, 50), (200, 700)])
def test_attention_gradients_of_scores_that_are_all_minus_infinity(nq, nk):
    """fp32 products past the type's range: such a row has o = 0, lse = -inf and, its probabilities being
    zero, no part in dv nor, as its q and k are finite, in dq and dk."""
    from paper_2406_02052_amd import Attention

    print("case", nq, nk, flush=True)
    q, k, v, g = draw(nq, (1, nq, 2, 64), (1, nk, 2, 64), (1, nk, 2, 64), (1, nq, 2, 64))
    k[:, :, 1] = -1e18 * np.abs(k[:, :, 1])
    q[:, nq // 2:, 1] = 1e22 * (1 + np.abs(q[:, nq // 2:, 1]))     # every product below -1e39
    k[:, :, 1] -= 1e18
    q[:, :nq // 2, 1] *= 1e-18
    q, k = (host(torch.tensor(x).float()) for x in (q, k))
    keep = [x.copy() for x in (q, g)]
    for t in keep:
        t[:, nq // 2:, 1] = 0.0
    want = T.attention(keep[0], k, v, 0.125, d_o=keep[1])           # those rows' d_o as zeros: no part in dk, dv
    t = [dev(x, "fp32") for x in (q, k, v, g)]
    op = Attention(1, nq, nk, 2, 2, 64, "fp32", scale=0.125)
    o, lse, grads = like(t[0]), torch.full((1, 2, nq), math.nan, device="cuda"), [like(x) for x in t[:3]]
    op.forward(*t[:3], o, lse)
    op.backward(*t[:3], o, lse, t[3], *grads)
    torch.cuda.synchronize()
    assert (o[0, nq // 2:, 1] == 0).all() and torch.isneginf(lse[0, 1, nq // 2:]).all()
    assert (grads[0][0, nq // 2:, 1] == 0).all()
    for h in range(2):   # the heads' gradients differ by 2^60 in size
        for x, y, name in zip(grads, want[2:], ("dq", "dk", "dv")):
            near(x[:, :, h], y[:, :, h], BAR["fp32", "grad"], name)


def _busy(stream):
    """Some tens of milliseconds of products on a stream."""
    with torch.cuda.stream(stream):
        a = torch.randn(8192, 8192, device="cuda", dtype=torch.bfloat16)
        for _ in range(40):
            a = (a @ a).clamp_(-1, 1)


@pytest.mark.parametrize("which", ["attention", "coupling"])
@pytest.mark.parametrize("how", ["argument", "current"])
def test_owner_dropped_while_its_call_runs_on_another_stream(how, which):
    """Its workspace's memory is not given to the current stream before the call has ended."""
    from paper_2406_02052_amd import Attention, Coupling

    print("case", how, which, flush=True)
    s = torch.cuda.Stream()
    if which == "attention":
        t = [dev(x, "bf16") for x in draw(5, (1, 4, 8, 64), (1, 4096, 8, 64), (1, 4096, 8, 64))]
        out = [torch.empty_like(t[0]), torch.empty(1, 8, 4, device="cuda")]
        make = lambda: Attention(1, 4, 4096, 8, 8, 64)  # noqa: E731
        call = lambda op, **kw: op.forward(*t, *out, **kw)  # noqa: E731
    else:
        y, f, dy = (dev(x, "bf16") for x in draw(6, *[(700, 256)] * 3))
        gate, post = torch.ones(1, 256, device="cuda"), (torch.ones(256, device="cuda"), None)
        new = lambda: torch.empty_like(y)  # noqa: E731
        out = [new(), new(), new(), torch.empty_like(gate), torch.empty_like(post[0])]
        make = lambda: Coupling(700, 256)  # noqa: E731
        call = lambda op, **kw: op.backward(y, f, dy, gate, post, *out[:4], (out[4], None), **kw)  # noqa: E731
    call(make())
    torch.cuda.synchronize()
    want = [x.clone() for x in out]
    for x in out:
        x.zero_()
    op = make()
    assert op.ws_bytes > 0
    at, n = op.workspace.data_ptr(), op.ws_bytes
    torch.cuda.synchronize()
    _busy(s)
    if how == "argument":
        call(op, stream=s)
    else:
        with torch.cuda.stream(s):
            call(op)
    del op
    taken = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for _ in range(4)]
    assert not s.query()                 # the call still waits
    assert all(x.data_ptr() >= at + n or x.data_ptr() + n <= at for x in taken)
    torch.cuda.synchronize()
    for x, y in zip(out, want):
        assert torch.equal(x, y)


def test_current_stream_is_torchs():
    from paper_2406_02052_amd import _lib as L

    s = torch.cuda.Stream()
    assert L._stream(None) == torch.cuda.current_stream().cuda_stream
    for stream in (s, torch.cuda.ExternalStream(torch.cuda.Stream().cuda_stream), torch.cuda.default_stream()):
        with torch.cuda.stream(stream):
            assert L._stream(None) == stream.cuda_stream == torch.cuda.current_stream().cuda_stream
    assert L._stream(None) == torch.cuda.current_stream().cuda_stream


def test_attention_of_more_workgroups_than_one_launch_holds():
    """65535 batch rows of 258 tiles of queries, 2^24 workgroups of 256 lanes and more: 2^32 lanes."""
    from paper_2406_02052_amd import Attention

    b, n, d = 65535, 33000, 8
    if torch.cuda.mem_get_info()[0] < 130 << 30:
        pytest.skip("needs 130 GB of device memory")
    assert b * -(-n // 128) >= 1 << 24
    base, k, v = (dev(x, "bf16") for x in draw(1, (1, n, 1, d), (b, 1, 1, d), (b, 1, 1, d)))
    base = (base * 2).round_()                     # sums over the queries without a rounding
    q = base.expand(b, -1, -1, -1).contiguous()
    op = Attention(b, n, 1, 1, 1, d)
    o, lse = torch.full_like(q, math.nan), torch.full((b, 1, n), math.nan, device="cuda")
    op.forward(q, k, v, o, lse)
    torch.cuda.synchronize()
    for i in range(0, b, 4096):                    # one key: o = v, lse = its score
        assert (o[i:i + 4096] == v[i:i + 4096]).all()
        score = torch.matmul(k[i:i + 4096, 0, 0].float(), base[0, :, 0].float().t().contiguous()) / math.sqrt(d)
        assert (lse[i:i + 4096, 0] - score).abs().max() <= 1e-5 * max(1.0, float(score.abs().max()))
    dq, dk, dv = o, torch.full_like(k, math.nan), torch.full_like(v, math.nan)
    # d_o = o = q: D is taken from the products where one tile holds the keys.  ds = 0, dv = the sum of d_o
    dq.fill_(math.nan)
    op.backward(q, k, v, q, lse, q, dq, dk, dv)
    torch.cuda.synchronize()
    want = base.double().sum(1).to(torch.bfloat16)[0, 0]
    assert (dv[:, 0, 0] == want).all()
    for i in range(0, b, 4096):
        assert (dq[i:i + 4096].abs().amax() <= 1e-3).all()
    assert (dk.float().abs() <= 1e-2 * math.sqrt(n)).all()
    del q, o, lse, dq, op
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_coupling_joins_as_many_gates_as_there_can_be(dtype):
    """487 gates of 21 rows over workgroups of 20: each gate's gradient is joined from two of them."""
    coupling(dtype, 487 * 21, 2048, "layer", 21)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("width", [4104, 8192])
@pytest.mark.parametrize("over", [dict(), dict(norm="layer", per_gate=1, scale=0.75), dict(norm="layer", per_gate=3, p=0.1),
                                  dict(pre=False, p=0.2), dict(per_gate=150, beta=True), dict(norm="layer", pre=False, in_place=True)],
                         ids=str)
def test_coupling_of_the_widest_rows_in_several_rounds(over, width, dtype):
    """More rows than workgroups, so that each takes several."""
    print("case", over, width, dtype, flush=True)
    coupling(dtype, 300, width, **over)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dim", [32, 72, 96])
@pytest.mark.parametrize("kv_len", [1500, 9000])
def test_attention_single_tokens_over_many_splits(kv_len, dim, dtype):
    """12 and 64 splits, most of them empty for the shorter requests."""
    print("case", kv_len, dim, dtype, flush=True)
    check(*attention(dtype, 3, 1, kv_len, 4, 2, dim, True, ([1, 1, 1], [kv_len, 0, 130]), poison=True, backward=False), dtype)
    check(*attention(dtype, 1, 1, kv_len, 4, 2, dim, lens=([1], [kv_len - 77]), poison=True), dtype)


def test_attention_gradient_strides_of_dimensions_of_one_mean_nothing():
    from paper_2406_02052_amd import Attention

    b, nk, h, kvh, d = 2, 70, 4, 2, 64
    q, k, v, g = draw(9, (b, 1, h, d), (b, nk, kvh, d), (b, nk, kvh, d), (b, 1, h, d), dtype="bf16")
    want = T.attention(q, k, v, 1 / math.sqrt(d), d_o=g)
    tq, tk, tv, tg = (dev(x, "bf16") for x in (q, k, v, g))
    tg = tg.reshape(b, h, 1, d).transpose(1, 2)          # the same memory, another stride of the one token
    o, lse = torch.empty_like(tq, memory_format=torch.contiguous_format), torch.empty(b, h, 1, device="cuda")
    assert tg.shape == o.shape and tg.stride() != o.stride() and tg.is_contiguous()
    dq = torch.full((b, h, 1, d), math.nan, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    dk, dv = like(tk), like(tv)
    op = Attention(b, 1, nk, h, kvh, d)
    op.forward(tq, tk, tv, o, lse)
    op.backward(tq, tk, tv, o, lse, tg, dq, dk, dv)
    check([o, lse, dq, dk, dv], want, "bf16")
    with pytest.raises(ValueError):                      # another stride of the heads does mean something
        op.backward(tq, tk, tv, o, lse, torch.empty(b, 1, h, 2 * d, dtype=torch.bfloat16, device="cuda")[..., :d], dq, dk, dv)
