"""Operators of a reversible attention stage, as cases that can be timed and
compared: attention, attention with its backward, the coupling that joins a
residual function to a stream (norms, gate, residual scale, dropout) with its
backward, and dropout alone.

Their formulas.  Attention, for head h of batch row b and its key head h // (heads
/ kv_heads), over the visible keys j of query i (j < kv_lens[b], and where causal
j <= i + kv_lens[b] - q_lens[b]; a query at or past q_lens[b] sees none):

    s_ij = scale q_i . k_j,  lse_i = log sum_j exp s_ij,  p_ij = exp(s_ij - lse_i)
    o_i = sum_j m_ij p_ij v_j          (o_i = 0, lse_i = -inf if no key is visible)

Coupling, for the rows of a stream x and of a residual function's output f:

    y = residual_scale x + gate m norm(f; post),   u = norm(y as stored; pre)

m is 0 or 1 / keep, by dropout; its backward also rebuilds x from y.  Dropout:
y = residual + alpha m x.

Dropout decides by 16 bits of Philox-4x32 with 7 rounds (Salmon et al. 2011): the
128-bit counter is (group, offset) and the key is the seed, rng = [seed, offset]; a
group is 8 elements, element e of it takes bits 16 e .. 16 e + 15, and is kept if
they are at least round(65536 p).  The groups of a tensor are its consecutive
elements; those of attention are, for a row of (batch, head, query), the keys
16 a + 4 c + {0, 1, 2, 3, 8, 9, 10, 11} for c = 0, 1, in the order (a, c).
"""
import math

import torch

own = False

EPS = 1e-5


def _attend(name, call, dtype, batch, q_len, kv_len, heads, kv_heads, dim, causal=False, ragged=False, dropout=0.0):
    return {"name": name, "call": call, "dtype": dtype, "batch": batch, "q_len": q_len, "kv_len": kv_len,
            "heads": heads, "kv_heads": kv_heads, "dim": dim, "causal": causal, "ragged": ragged, "dropout": dropout}


def _couple(name, call, dtype, rows, width, norm="rms", per_gate=0, scale=1.0, dropout=0.0, pre=True):
    return {"name": name, "call": call, "dtype": dtype, "rows": rows, "width": width, "norm": norm,
            "rows_per_gate": per_gate, "residual_scale": scale, "dropout": dropout, "pre": pre}


def _drop(name, dtype, n, residual):
    return {"name": name, "call": "dropout", "dtype": dtype, "n": n, "residual": residual, "dropout": 0.1}


def listed():
    return [
        # one new token for each of 8 requests over what they have so far, four query
        # heads to a key head, each request at a length of its own
        _attend("attend_token_8x4097", "attend", "bf16", 8, 1, 4097, 16, 4, 64, ragged=True),
        # the forward of a long causal sequence
        _attend("attend_causal_2x4096", "attend", "bf16", 2, 4096, 4096, 16, 16, 128, causal=True),
        # queries over another sequence's keys, held in fp32, odd sizes
        _attend("attend_fp32_3x777x1023", "attend", "fp32", 3, 777, 1023, 5, 5, 40, ragged=True),
        # what a reversible stage's backward runs, forward and gradients, over the
        # tokens of 8x8 feature maps: many short sequences
        _attend("attend_vjp_128x64", "attend_vjp", "bf16", 128, 64, 64, 8, 8, 32),
        # the same for long causal sequences with shared key heads
        _attend("attend_vjp_causal_2x4096", "attend_vjp", "bf16", 2, 4096, 4096, 16, 4, 128, causal=True),
        # the same with dropout, a head width between the usual ones, ragged lengths
        _attend("attend_vjp_dropout_5x1000", "attend_vjp", "bf16", 5, 1000, 1000, 6, 2, 80, causal=True, ragged=True, dropout=0.1),
        # the coupling of one 8x8 map's tokens: a launch
        _couple("couple_64x256", "couple", "bf16", 64, 256),
        # a large micro-batch of wide tokens, in training
        _couple("couple_16384x4096", "couple", "bf16", 16384, 4096, dropout=0.1),
        # backward with a gate for each of 37 samples, layer norm, fp32
        _couple("couple_vjp_fp32_4107x1000", "couple_vjp", "fp32", 4107, 1000, "layer", 111, 0.75),
        # backward of a large micro-batch, in training
        _couple("couple_vjp_16384x2048", "couple_vjp", "bf16", 16384, 2048, dropout=0.1),
        # dropout of a small tensor whose size nothing divides
        _drop("dropout_fp32_1000003", "fp32", 1000003, False),
        # dropout of a residual function's output, joined to its stream
        _drop("dropout_134217728", "bf16", 134217728, True),
    ]


def _spread(rng, low, high):
    """A whole number from 2^low to 2^high, spread over its logarithm."""
    n = max(1, round(2 ** rng.uniform(low, high)))
    return n + 1 if n % 1024 == 0 and n % 2048 else n


def draw(rng):
    """Calls over lengths from one token to thousands, widths of 8 to 8192 and tensors
    of one element to the largest listed, odd sizes among them."""
    kind = rng.choice(("attend", "attend", "attend_vjp", "attend_vjp", "token", "couple", "couple_vjp", "dropout"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "fp32"))
    drop = rng.choice((0.0, 0.0, 0.1, 0.25))
    if kind == "dropout":
        return {"call": "dropout", "dtype": dtype, "n": _spread(rng, 0, 26.9), "residual": rng.random() < 0.5,
                "dropout": drop or 0.5}
    if kind in ("couple", "couple_vjp"):
        width = 8 * rng.choice((2 ** rng.randrange(11), 1 + 2 * _spread(rng, 0, 9)))
        rows = _spread(rng, 0, math.log2(2 ** (25 if dtype == "bf16" else 24) / width))
        per_gate = rng.choice((0, 0, 1, _spread(rng, 1, 8)))
        if per_gate:
            rows = max(1, rows // per_gate) * per_gate
        return {"call": kind, "dtype": dtype, "rows": rows, "width": width, "norm": rng.choice(("rms", "layer")),
                "rows_per_gate": per_gate, "residual_scale": rng.choice((1.0, 1.0, 0.75)), "dropout": drop,
                "pre": rng.random() < 0.75}
    dim = rng.choice((32, 40, 64, 64, 80, 96, 128, 128))
    kv_heads = rng.choice((1, 2, 3, 4, 8))
    heads = kv_heads * rng.choice((1, 1, 2, 4))
    if kind == "token":
        q_len, kv_len = rng.choice((1, 1, 1, 2, 3, 8)), _spread(rng, 0, 16)
        most = 2 ** (28 if dtype == "bf16" else 27) // (kv_heads * kv_len * dim)
    else:
        q_len = _spread(rng, 0, 12)
        kv_len = q_len if rng.random() < 0.6 else _spread(rng, 0, 12)
        limit = 2 ** (34 if dtype == "bf16" else 31)
        while heads * q_len * kv_len * dim > limit:   # many heads: shorter sequences
            q_len, kv_len = q_len // 2 + 1, kv_len // 2 + 1
        most = min(limit // (heads * q_len * kv_len * dim), 2 ** 26 // (heads * max(q_len, kv_len) * dim))
    batch = min(128, _spread(rng, 0, math.log2(max(1, most))))
    return {"call": "attend" if kind == "token" else kind, "dtype": dtype, "batch": batch, "q_len": q_len, "kv_len": kv_len,
            "heads": heads, "kv_heads": kv_heads, "dim": dim, "causal": rng.random() < 0.5, "ragged": rng.random() < 0.4,
            "dropout": drop if kind != "token" else 0.0}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _lens(case):
    """(q_lens, kv_lens): full, or spread from nothing (the second row's) to full."""
    b, q, k = case["batch"], case["q_len"], case["kv_len"]
    if not case["ragged"]:
        return [q] * b, [k] * b
    part = [1.0 if i == 0 else 0.0 if i == 1 else (i * 0.618034) % 1.0 for i in range(b)]
    return [max(1, round(q * p)) for p in part], [round(k * p) for p in part]


class _State:
    pass


def prepare(case, seed):
    g, s = torch.Generator("cuda").manual_seed(seed), _State()

    def normal(*shape, std=1.0, dtype=None):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype or _type(case))

    s.case, s.call, s.rng = case, case["call"], None
    if case["dropout"]:
        s.rng = torch.randint(2 ** 62, (2,), generator=g, device="cuda")
    if s.call.startswith("attend"):
        b, d = case["batch"], case["dim"]
        s.q = normal(b, case["q_len"], case["heads"], d)
        s.k, s.v = (normal(b, case["kv_len"], case["kv_heads"], d) for _ in range(2))
        s.scale, s.q_lens, s.kv_lens = 1.0 / math.sqrt(d), None, None
        if case["ragged"]:
            s.q_lens, s.kv_lens = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in _lens(case))
        if s.call == "attend_vjp":
            s.do = normal(b, case["q_len"], case["heads"], d)
    elif s.call.startswith("couple"):
        r, w = case["rows"], case["width"]
        gates = r // case["rows_per_gate"] if case["rows_per_gate"] else 1
        f32, layer = torch.float32, case["norm"] == "layer"
        s.f = normal(r, w, std=2.0) + (0.5 if layer else 0.0)
        s.gate = normal(gates, w, std=0.2, dtype=f32) + 0.5
        s.post, s.pre = ((1.0 + normal(w, std=0.1, dtype=f32), normal(w, std=0.1, dtype=f32) if layer else None) for _ in range(2))
        s.x = normal(r, w)
        if s.call == "couple_vjp":
            s.y, s.dy, s.du = s.x, normal(r, w, std=1e-2), normal(r, w, std=1e-2) if case["pre"] else None
    else:
        s.x = normal(case["n"])
        s.residual = normal(case["n"]) if case["residual"] else None
    if own:
        _prepare_own(s, case)
    return s


def _prepare_own(s, case):
    """The operator's handle with its workspace, and the buffers its results go to."""
    from paper_2406_02052_amd import Attention, Coupling

    if s.call.startswith("attend"):
        s.op = Attention(case["batch"], case["q_len"], case["kv_len"], case["heads"], case["kv_heads"], case["dim"],
                         case["dtype"], causal=case["causal"], scale=s.scale, dropout=case["dropout"])
        s.o, s.lse = torch.empty_like(s.q), torch.empty(case["batch"], case["heads"], case["q_len"], device="cuda")
        if s.call == "attend_vjp":
            s.dq, s.dk, s.dv = torch.empty_like(s.q), torch.empty_like(s.k), torch.empty_like(s.v)
    elif s.call.startswith("couple"):
        s.op = Coupling(case["rows"], case["width"], case["dtype"], norm=case["norm"], eps=EPS,
                        residual_scale=case["residual_scale"], dropout=case["dropout"], rows_per_gate=case["rows_per_gate"])
        new, like = torch.empty_like, lambda p: tuple(None if t is None else torch.empty_like(t) for t in p)
        if s.call == "couple":
            s.y, s.u = new(s.x), new(s.x) if case["pre"] else None
        else:
            s.x, s.dx, s.df, s.dgate = new(s.y), new(s.y), new(s.y), new(s.gate)
            s.dpost, s.dpre = like(s.post), like(s.pre) if case["pre"] else None
    else:
        s.y = torch.empty_like(s.x)


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    if s.call.startswith("attend"):
        s.op.forward(s.q, s.k, s.v, s.o, s.lse, q_lens=s.q_lens, kv_lens=s.kv_lens, rng=s.rng)
        if s.call == "attend":
            return {"o": s.o, "lse": s.lse}
        s.op.backward(s.q, s.k, s.v, s.o, s.lse, s.do, s.dq, s.dk, s.dv, q_lens=s.q_lens, kv_lens=s.kv_lens, rng=s.rng)
        return {"o": s.o, "lse": s.lse, "dq": s.dq, "dk": s.dk, "dv": s.dv}
    if s.call == "couple":
        s.op.forward(s.x, s.f, s.gate, s.post, s.y, pre=s.pre if s.u is not None else None, u=s.u, rng=s.rng)
        return {"y": s.y} if s.u is None else {"y": s.y, "u": s.u}
    if s.call == "couple_vjp":
        pre = s.pre if s.du is not None else None
        s.op.backward(s.y, s.f, s.dy, s.gate, s.post, s.x, s.dx, s.df, s.dgate, s.dpost, du=s.du, pre=pre, dpre=s.dpre, rng=s.rng)
        return _gradients(s.x, s.dx, s.df, s.dgate, s.dpost, s.dpre)
    from paper_2406_02052_amd import dropout

    dropout(s.x, s.y, s.case["dropout"], s.rng, residual=s.residual)
    return {"y": s.y}


def _gradients(x, dx, df, dgate, dpost, dpre):
    out = {"x": x, "dx": dx, "df": df, "dgate": dgate, "dpost": [t for t in dpost if t is not None]}
    return out if dpre is None else {**out, "dpre": [t for t in dpre if t is not None]}


# ---------------------------------------------------------------------------
# the plain forms, in 32 bits
# ---------------------------------------------------------------------------

_LOW = 0xFFFFFFFF


def _bits(rng, group):
    """[..., 8] 16-bit numbers of the groups in `group` (int64): Philox-4x32, 7 rounds.
    A 64-bit product wraps, which leaves both its 32-bit halves right."""
    seed, offset = rng[0], rng[1]
    c = [group & _LOW, (group >> 32) & _LOW, (offset & _LOW).expand_as(group), ((offset >> 32) & _LOW).expand_as(group)]
    k = [seed & _LOW, (seed >> 32) & _LOW]
    for _ in range(7):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((b >> 32) & _LOW) ^ c[1] ^ k[0], b & _LOW, ((a >> 32) & _LOW) ^ c[3] ^ k[1], a & _LOW]
        k = [(k[0] + 0x9E3779B9) & _LOW, (k[1] + 0xBB67AE85) & _LOW]
    return torch.stack([h for w in c for h in (w & 0xFFFF, w >> 16)], -1)


def _cut(p):
    return round(65536 * p)


def _factor(rng, p, group):
    """The factors m of the groups' elements: 0 or 1 / keep."""
    return (_bits(rng, group) >= _cut(p)).float() * (65536.0 / (65536 - _cut(p)))


def _factor_flat(rng, p, shape):
    n = math.prod(shape)
    group = torch.arange(-(-n // 8), device="cuda")
    return _factor(rng, p, group).reshape(-1)[:n].reshape(shape)


def _factor_attend(rng, p, b, h, q, k):
    blocks = -(-k // 16)
    m = _factor(rng, p, torch.arange(b * h * q * blocks * 2, device="cuda"))
    # [row, 16 keys, which 4 of 8, which 8, 4]: in the keys' own order
    m = m.reshape(b, h, q, blocks, 2, 2, 4).transpose(-2, -3)
    return m.reshape(b, h, q, blocks * 16)[..., :k]


def _heads_first(t, heads):
    t = t.float().transpose(1, 2)
    return t.repeat_interleave(heads // t.shape[1], 1).contiguous()


def _plain_attend(s):
    case, h = s.case, s.case["heads"]
    b, nq, nk = case["batch"], case["q_len"], case["kv_len"]
    q, k, v = _heads_first(s.q, h), _heads_first(s.k, h), _heads_first(s.v, h)
    i, j = torch.arange(nq, device="cuda").reshape(1, 1, nq, 1), torch.arange(nk, device="cuda").reshape(1, 1, 1, nk)
    lq, lk = ((torch.full((b,), n, device="cuda") if t is None else t.long()).reshape(b, 1, 1, 1)
              for t, n in ((s.q_lens, nq), (s.kv_lens, nk)))
    seen = (i < lq) & (j < lk)
    if case["causal"]:
        seen = seen & (j <= i + lk - lq)
    # what lies past the lengths takes no part, whatever it holds
    k, v = (torch.where((j < lk).transpose(2, 3), t, 0.0) for t in (k, v))
    q = torch.where(i < lq, q, 0.0)
    score = torch.where(seen, (q @ k.transpose(2, 3).contiguous()) * s.scale, -math.inf)
    top = score.amax(3, keepdim=True)
    e = torch.exp(score - torch.where(top > -math.inf, top, 0.0))
    total = e.sum(3, keepdim=True)
    p = e / torch.where(total > 0, total, 1.0)
    lse = (top + torch.log(total)).squeeze(3)
    m = _factor_attend(s.rng, case["dropout"], b, h, nq, nk) if case["dropout"] else None
    pm = p if m is None else p * m
    o = pm @ v
    out = {"o": o.transpose(1, 2).to(s.q.dtype), "lse": lse}
    if s.call == "attend":
        return out
    do = torch.where(i < lq, s.do.float().transpose(1, 2), 0.0).contiguous()
    dp = do @ v.transpose(2, 3).contiguous()
    if m is not None:
        dp = dp * m
    ds = p * (dp - (do * o).sum(3, keepdim=True)) * s.scale
    dq = ds @ k
    dk, dv = ds.transpose(2, 3).contiguous() @ q, pm.transpose(2, 3).contiguous() @ do
    kvh = case["kv_heads"]
    dk, dv = (t.reshape(b, kvh, h // kvh, nk, -1).sum(2) for t in (dk, dv))
    return {**out, **{n: t.transpose(1, 2).to(s.q.dtype) for n, t in (("dq", dq), ("dk", dk), ("dv", dv))}}


def _unit(t, norm):
    """(t normalised, 1 / its deviation), by rows."""
    if norm == "layer":
        t = t - t.mean(1, keepdim=True)
    r = torch.rsqrt(t.square().mean(1, keepdim=True) + EPS)
    return t * r, r


def _affine(t, p):
    return t * p[0] if p[1] is None else t * p[0] + p[1]


def _unit_back(g, n, r, norm):
    """The gradient of the rows before they were normalised to n."""
    g = g - n * (g * n).mean(1, keepdim=True) - (g.mean(1, keepdim=True) if norm == "layer" else 0.0)
    return g * r


def _plain_couple(s):
    case, norm = s.case, s.case["norm"]
    r, w = case["rows"], case["width"]
    gate = s.gate.repeat_interleave(case["rows_per_gate"] or r, 0)
    f, fr = _unit(s.f.float(), norm)
    n = _affine(f, s.post)
    m = _factor_flat(s.rng, case["dropout"], (r, w)) if case["dropout"] else None
    nm = n if m is None else n * m
    if s.call == "couple":
        y = (s.x.float() * case["residual_scale"] + gate * nm).to(s.x.dtype)
        return {"y": y, "u": _affine(_unit(y.float(), norm)[0], s.pre).to(y.dtype)} if case["pre"] else {"y": y}
    y, dy, dpre = s.y.float(), s.dy.float(), None
    if s.du is not None:
        du = s.du.float()
        yn, yr = _unit(y, norm)
        dy = dy + _unit_back(du * s.pre[0], yn, yr, norm)
        dpre = ((du * yn).sum(0), None if s.pre[1] is None else du.sum(0))
    x = (y - gate * nm) / case["residual_scale"]
    dgate = (dy * nm).reshape(s.gate.shape[0], -1, w).sum(1)
    dn = gate * dy if m is None else gate * dy * m
    dpost = ((dn * f).sum(0), None if s.post[1] is None else dn.sum(0))
    df = _unit_back(dn * s.post[0], f, fr, norm)
    t = s.y.dtype
    return _gradients(x.to(t), (dy * case["residual_scale"]).to(t), df.to(t), dgate, dpost, dpre)


def _run_plain(s):
    if s.call.startswith("attend"):
        return _plain_attend(s)
    if s.call.startswith("couple"):
        return _plain_couple(s)
    y = s.x.float() * _factor_flat(s.rng, s.case["dropout"], s.x.shape)
    return {"y": (y if s.residual is None else y + s.residual.float()).to(s.x.dtype)}


# ---------------------------------------------------------------------------
# what a call cannot do without
# ---------------------------------------------------------------------------

def _pairs(case):
    """Visible pairs of a query and a key of one head, and the queries and keys within the lengths, over the batch."""
    pairs, lens = 0, _lens(case)
    for q, k in zip(*lens):
        if case["causal"]:
            first = max(0, q - k)   # the queries before it see nothing
            pairs += (q - first) * (k - q + first + 1 + k) // 2
        else:
            pairs += q * k
    return pairs, sum(lens[0]), sum(lens[1])


def work(case):
    esz = 2 if case["dtype"] == "bf16" else 4
    if case["call"] == "dropout":
        return {"bytes": case["n"] * esz * (3 if case["residual"] else 2), "flops": 0}
    if case["call"].startswith("attend"):
        pairs, nq, nk = _pairs(case)
        d, h, kvh = case["dim"], case["heads"], case["kv_heads"]
        whole_q, whole_k = case["batch"] * case["q_len"], case["batch"] * case["kv_len"]
        read = (nq * h + 2 * nk * kvh) * d * esz
        wrote = whole_q * h * (d * esz + 4)
        if case["call"] == "attend":   # two products
            return {"bytes": read + wrote, "flops": 4 * pairs * h * d}
        # the forward's two and the backward's five
        return {"bytes": read + wrote + (nq * h + whole_q * h + 2 * whole_k * kvh) * d * esz, "flops": 14 * pairs * h * d}
    size, gates = case["rows"] * case["width"], case["rows"] // case["rows_per_gate"] if case["rows_per_gate"] else 1
    vectors = (2 if case["norm"] == "layer" else 1) * (2 if case["pre"] else 1) + gates
    if case["call"] == "couple":
        return {"bytes": size * esz * (4 if case["pre"] else 3) + 4 * vectors * case["width"], "flops": 12 * size}
    return {"bytes": size * esz * (7 if case["pre"] else 6) + 8 * vectors * case["width"], "flops": 36 * size}


# ---------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# ---------------------------------------------------------------------------

def _mul32(a, m):
    """(high, low) words of a 32-bit word times the constant m, by 16-bit digits."""
    a0, a1, m0, m1 = a & 0xFFFF, a >> 16, m & 0xFFFF, m >> 16
    mid = a1 * m0 + (a0 * m0 >> 16)
    cross = a0 * m1 + (mid & 0xFFFF)
    return a1 * m1 + (mid >> 16) + (cross >> 16), ((cross & 0xFFFF) << 16) | (a0 * m0 & 0xFFFF)


def _kept(rng, p, element_group, element):
    """Truth values of elements given by their group and their place (0 .. 7) in it."""
    seed, offset = (int(t) for t in rng.tolist())
    x0, x1 = element_group % 2 ** 32, element_group // 2 ** 32
    x2, x3 = torch.full_like(x0, offset % 2 ** 32), torch.full_like(x0, offset // 2 ** 32)
    for r in range(7):
        k0, k1 = (seed % 2 ** 32 + r * 0x9E3779B9) % 2 ** 32, (seed // 2 ** 32 + r * 0xBB67AE85) % 2 ** 32
        (h0, l0), (h1, l1) = _mul32(x0, 0xD2511F53), _mul32(x2, 0xCD9E8D57)
        x0, x1, x2, x3 = h1 ^ x1 ^ k0, l1, h0 ^ x3 ^ k1, l0
    word = torch.where(element < 4, torch.where(element < 2, x0, x1), torch.where(element < 6, x2, x3))
    return torch.where(element % 2 == 1, word // 65536, word % 65536) >= _cut(p)


def _exact_factor(rng, p, n, first=0):
    at = torch.arange(first, first + n, device="cuda")
    return _kept(rng, p, at // 8, at % 8).double() / (1.0 - _cut(p) / 65536.0)


def _exact_attend(s):
    case = s.case
    nq, nk, h, kvh = case["q_len"], case["kv_len"], case["heads"], case["kv_heads"]
    o, lse = torch.zeros(s.q.shape, dtype=torch.float64, device="cuda"), torch.full((case["batch"], h, nq), -math.inf, dtype=torch.float64, device="cuda")
    dq, dk, dv = (torch.zeros(t.shape, dtype=torch.float64, device="cuda") for t in (s.q, s.k, s.v))
    key = torch.arange(nk, device="cuda")
    for b, (lq, lk) in enumerate(zip(*_lens(case))):
        # queries first .. lq of this row see something
        first = max(0, lq - lk) if case["causal"] else 0
        if lk == 0 or first >= lq:
            continue
        for n in range(h):
            q, (k, v) = s.q[b, first:lq, n].double(), (t[b, :lk, n // (h // kvh)].double() for t in (s.k, s.v))
            a = (q @ k.T) * s.scale
            if case["causal"]:
                a.masked_fill_(torch.ones_like(a, dtype=torch.bool).triu_(first + lk - lq + 1), -math.inf)
            l = torch.logsumexp(a, 1, keepdim=True)
            p, m = torch.exp(a - l), 1.0
            if case["dropout"]:
                row = (b * h + n) * nq + torch.arange(first, lq, device="cuda")[:, None]
                kk = key[None, :lk]
                group = (row * ((nk + 15) // 16) + kk // 16) * 2 + (kk // 4) % 2
                m = _kept(s.rng, case["dropout"], group, (kk // 8) % 2 * 4 + kk % 4) / (1.0 - _cut(case["dropout"]) / 65536.0)
            lse[b, n, first:lq] = l[:, 0]
            o[b, first:lq, n] = (p * m) @ v
            if s.call == "attend_vjp":
                g = s.do[b, first:lq, n].double()
                dp = (g @ v.T) * m
                ds = p * (dp - (p * dp).sum(1, keepdim=True))
                dq[b, first:lq, n] = ds @ k * s.scale
                dk[b, :lk, n // (h // kvh)] += ds.T @ q * s.scale
                dv[b, :lk, n // (h // kvh)] += (p * m).T @ g
    return {"o": o, "lse": lse} if s.call == "attend" else {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


def _exact_norm(t, p, layer):
    var, mean = torch.var_mean(t, 1, correction=0, keepdim=True)
    t = (t - mean) / (var + EPS).sqrt() if layer else t / ((t * t).mean(1, keepdim=True) + EPS).sqrt()
    return t * p[0] + (0.0 if p[1] is None else p[1])


def _exact_couple(s):
    """Gradients by automatic differentiation of the formulas."""
    case, layer = s.case, s.case["norm"] == "layer"
    r, w = case["rows"], case["width"]
    leaf = lambda t: None if t is None else t.double().requires_grad_()  # noqa: E731
    f, gate, post, pre = leaf(s.f), leaf(s.gate), tuple(map(leaf, s.post)), tuple(map(leaf, s.pre))
    m = _exact_factor(s.rng, case["dropout"], r * w).reshape(r, w) if case["dropout"] else 1.0
    added = (_exact_norm(f, post, layer) * m).reshape(gate.shape[0], -1, w) * gate[:, None]
    added = added.reshape(r, w)
    if s.call == "couple":
        y = (s.x.double() * case["residual_scale"] + added).detach()
        return {"y": y, "u": _exact_norm(y.to(s.x.dtype).double(), pre, layer).detach()} if case["pre"] else {"y": y}
    x = ((s.y.double() - added) / case["residual_scale"]).detach()
    total, y, dpre = s.dy.double(), leaf(s.y), None
    if case["pre"]:
        g = torch.autograd.grad(_exact_norm(y, pre, layer), [y] + [t for t in pre if t is not None], s.du.double())
        total, dpre = total + g[0], g[1:]
    df, dgate, *dpost = torch.autograd.grad(added, [f, gate] + [t for t in post if t is not None], total)
    return _gradients(x, total * case["residual_scale"], df, dgate, dpost, dpre)


def exact(case, seed):
    s = prepare(case, seed)
    if s.call.startswith("attend"):
        return _exact_attend(s)
    if s.call.startswith("couple"):
        return _exact_couple(s)
    y = s.x.double() * _exact_factor(s.rng, case["dropout"], case["n"])
    return {"y": y if s.residual is None else y + s.residual.double()}
