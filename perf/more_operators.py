"""Operators of training over tokens, as cases that can be timed and compared: norms
of query and key heads with the rotation by their positions, the loss over a large
vocabulary with its gradients, and an AdamW step over many tensors.

Their formulas.  Head norms and rotation, for each head's channels x of a token:

    z = n(x) gamma (+ beta),   (y_a, y_b) = rotation of (z_a, z_b) by freq_i position[axis_i]

n is a root-mean-square norm, a layer norm or nothing.  Pair i < pairs is channels
(i, i + pairs), "halves", or (2 i, 2 i + 1), "neighbours"; others are not rotated.

Vocabulary loss, for rows x_i with targets t_i (a row whose target is no column takes no
part: its loss, lse and gradient are 0):

    s_ij = scale x_i . w_j,  lse_i = log sum_j exp s_ij,  loss_i = lse_i - s_it,  L = sum_i weight_i loss_i

weight is given, or 1 / (the rows that take part).

AdamW, t = step + 1, g = grad_scale grad:

    m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2
    theta -= lr (m / (1 - beta1^t) / (sqrt(v / (1 - beta2^t)) + eps) + weight_decay theta)

in fp32, m and v held in fp32 or, "fp8", as e4m3 numbers with a power of two as the scale of
each 64 elements: m, and r = sqrt(v).  The scale brings the block's largest value into
[128, 256).  Values are rounded up or down to neighbours lo, hi of that format by a
random number u in [0, 1): m up if u < (|m| - lo) / (hi - lo), r up if u < (v - lo^2) / (hi^2 - lo^2), so
that m and v are kept on average; r of v > 0 is at least the smallest number.  u is 16 bits of
Philox-4x32 with 7 rounds (Salmon et al. 2011), counter (group, offset), key seed, rng = [seed, offset]:
a group is 4 elements, element e of it takes bits 32 e .. 32 e + 15 for m and the 16 above for r.
A tensor's groups start at a multiple of 16.
"""
import math

import torch

own = False

EPS = 1e-6
BETA1, BETA2, ADAM_EPS = 0.9, 0.999, 1e-8


def _heads(name, call, dtype, batch, length, heads, kv_heads, dim, pairs, norm="rms", layout="halves", axes=1, far=0):
    return {"name": name, "call": call, "dtype": dtype, "batch": batch, "length": length, "heads": heads, "kv_heads": kv_heads,
            "dim": dim, "pairs": pairs, "norm": norm, "layout": layout, "axes": axes, "far": far}


def _vocab(name, call, dtype, rows, width, vocab, ignored=0.0, weighted=False):
    return {"name": name, "call": call, "dtype": dtype, "rows": rows, "width": width, "vocab": vocab, "ignored": ignored,
            "weighted": weighted}


def _adamw(name, states, tensors, total, grad="fp32", copies=True, scaled=False):
    return {"name": name, "call": "adamw", "states": states, "tensors": tensors, "total": total, "grad": grad, "copies": copies,
            "scaled": scaled}


def listed():
    return [
        # one new token for each of 8 requests, far along
        _heads("heads_token_8x1", "heads", "bf16", 8, 1, 16, 4, 64, 32, far=100000),
        # the forward of long sequences
        _heads("heads_4x4096", "heads", "bf16", 4, 4096, 16, 4, 128, 64),
        # what a reversible stage's backward runs, over frames of images: time, height and width
        _heads("heads_vjp_video_8x2048", "heads_vjp", "bf16", 8, 2048, 16, 16, 128, 60, axes=3),
        # the same in fp32, layer norm, neighbouring channels, an odd length and a head width between the usual ones
        _heads("heads_vjp_fp32_3x777", "heads_vjp", "fp32", 3, 777, 5, 5, 40, 16, norm="layer", layout="neighbours", axes=2),
        # the loss of a few rows, as at the end of a short sequence
        _vocab("loss_8x1024x32768", "loss", "bf16", 8, 1024, 32768),
        # the loss of a validation batch, a vocabulary that nothing divides
        _vocab("loss_4000x1024x50021", "loss", "bf16", 4000, 1024, 50021, ignored=0.1),
        # loss and gradients of a micro-batch
        _vocab("loss_vjp_2048x1024x32768", "loss_vjp", "bf16", 2048, 1024, 32768, ignored=0.25, weighted=True),
        # the same in fp32, odd sizes
        _vocab("loss_vjp_fp32_777x320x10007", "loss_vjp", "fp32", 777, 320, 10007, ignored=0.1),
        # loss and gradients of a large micro-batch over a large vocabulary
        _vocab("loss_vjp_8192x4096x131072", "loss_vjp", "bf16", 8192, 4096, 131072),
        # the update of a stage of many small tensors
        _adamw("adamw_300_small", "fp32", 300, 2000000),
        # the update of large tensors with bf16 gradients
        _adamw("adamw_64m_bf16_grads", "fp32", 12, 64000000, grad="bf16", scaled=True),
        # the update of large tensors with states in 8 bits
        _adamw("adamw_fp8_134m", "fp8", 40, 134000000),
    ]


def _spread(rng, low, high):
    """A whole number from 2^low to 2^high, spread over its logarithm."""
    n = max(1, round(2 ** rng.uniform(low, high)))
    return n + 1 if n % 1024 == 0 and n % 2048 else n


def draw(rng):
    """Calls over one token to tens of thousands, head widths of 8 to 128, vocabularies of 2 to
    131072 and tensors of 1 to 134 million elements, odd sizes among them."""
    kind = rng.choice(("heads", "heads_vjp", "heads_vjp", "loss", "loss_vjp", "loss_vjp", "adamw", "adamw"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "fp32"))
    if kind.startswith("heads"):
        dim = rng.choice((8, 24, 32, 40, 64, 64, 80, 96, 128, 128))
        layout = rng.choice(("halves", "halves", "neighbours"))
        pairs = rng.choice((dim // 2, dim // 2, dim // 2, max(4, dim // 16 * 4)))
        heads = rng.choice((1, 2, 3, 8, 16, 24))
        kv_heads = rng.choice((heads, 1, rng.choice((0, heads))))
        tokens = _spread(rng, 0, math.log2(2 ** (26 if dtype == "bf16" else 25) / ((heads + kv_heads) * dim)))
        batch = rng.choice((1, 2, 5, _spread(rng, 0, 6)))
        length = max(1, tokens // batch)
        return {"call": kind, "dtype": dtype, "batch": batch, "length": length, "heads": heads, "kv_heads": kv_heads, "dim": dim,
                "pairs": pairs, "norm": rng.choice(("rms", "rms", "rms", "layer", "none")), "layout": layout,
                "axes": rng.choice((1, 1, 2, 3)), "far": rng.choice((0, 0, _spread(rng, 10, 24)))}
    if kind.startswith("loss"):
        width = 8 * rng.choice((_spread(rng, 0, 9), 2 ** rng.randrange(10)))
        vocab = _spread(rng, 1, 17)
        most = (2.0 ** 41 if dtype == "bf16" else 2.0 ** 36) / (width * vocab)
        rows = _spread(rng, 0, min(14, math.log2(max(2, most))))
        return {"call": kind, "dtype": dtype, "rows": rows, "width": width, "vocab": vocab,
                "ignored": rng.choice((0.0, 0.0, 0.2, 0.6)), "weighted": rng.random() < 0.4}
    tensors = _spread(rng, 0, 9)
    return {"call": "adamw", "states": rng.choice(("fp32", "fp8")), "tensors": tensors,
            "total": max(tensors, _spread(rng, 0, 26.9)), "grad": rng.choice(("fp32", "fp32", "bf16")), "copies": rng.random() < 0.7,
            "scaled": rng.random() < 0.5}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _pairs(case):
    """(freq, axis) of each pair: the axes share the pairs evenly, each from fast to slow."""
    n, axes = case["pairs"], min(case["axes"], case["pairs"])
    axis = [i * axes // n for i in range(n)]
    return [10000.0 ** (-(i - axis.index(a)) / axis.count(a)) for i, a in enumerate(axis)], axis


def _sizes(case):
    """Elements of each tensor, from large to small, summing to about the total; the last ones are vectors."""
    n, share = case["tensors"], case["total"] / case["tensors"]
    return [max(1, round(share * (0.002 if i % 4 == 3 else 0.2 + 1.6 * ((i * 0.618034) % 1.0)))) for i in range(n)]


def _starts(sizes):
    """Where each tensor starts in one buffer of them all, and the buffer's length: multiples of 64."""
    at, starts = 0, []
    for n in sizes:
        starts.append(at)
        at += -(-n // 64) * 64
    return starts, at


class _State:
    pass


def prepare(case, seed):
    g, s = torch.Generator("cuda").manual_seed(seed), _State()

    def normal(*shape, std=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)

    s.case, s.call = case, case["call"]
    if s.call.startswith("heads"):
        b, n, h, kv, d, t = case["batch"], case["length"], case["heads"], case["kv_heads"], case["dim"], _type(case)
        # queries and keys lie in the result of one product, beside the values
        s.qkv = normal(b, n, h + 2 * kv, d, std=1.5, dtype=t) + (0.25 if case["norm"] == "layer" else 0.0)
        s.q, s.k = s.qkv[:, :, :h], s.qkv[:, :, h:h + kv] if kv else None
        s.freq, s.axis = _pairs(case)
        s.axes = max(s.axis) + 1
        at = torch.arange(n, device="cuda", dtype=torch.int32).expand(b, n)
        if s.axes == 1:
            s.positions = (at + case["far"] + torch.randint(64, (b, 1), generator=g, device="cuda", dtype=torch.int32))[None]
        else:
            side = max(1, round(n ** (1.0 / s.axes)))
            grid = [at // side ** (s.axes - 1)] + [at // side ** i % side for i in range(s.axes - 1)][::-1]
            s.positions = torch.stack(grid) + case["far"]
        s.positions = s.positions.to(torch.int32).contiguous()
        norms = [(1.0 + normal(d, std=0.1), normal(d, std=0.1) if case["norm"] == "layer" else None) for _ in range(2)]
        s.q_norm, s.k_norm = (None, None) if case["norm"] == "none" else (norms[0], norms[1] if kv else None)
        if s.call == "heads_vjp":
            s.dy_q, s.dy_k = normal(b, n, h, d, std=1e-2, dtype=t), normal(b, n, kv, d, std=1e-2, dtype=t) if kv else None
    elif s.call.startswith("loss"):
        r, w, v, t = case["rows"], case["width"], case["vocab"], _type(case)
        s.x, s.w, s.scale = normal(r, w, dtype=t), normal(v, w, std=2.5 / math.sqrt(w), dtype=t), 1.0
        s.targets = torch.randint(v, (r,), generator=g, device="cuda", dtype=torch.int32)
        out = torch.rand(r, generator=g, device="cuda") < case["ignored"]
        s.targets[out] = -100
        s.weight = torch.rand(r, generator=g, device="cuda") / r if case["weighted"] else None
    else:
        s.sizes = _sizes(case)
        s.starts, n = _starts(s.sizes)
        blocks = torch.tensor([-(-m // 64) for m in s.sizes], device="cuda")
        left = (torch.tensor(s.starts, device="cuda") + torch.tensor(s.sizes, device="cuda")).repeat_interleave(blocks)
        s.inside = (torch.arange(n, device="cuda").reshape(-1, 64) < left[:, None]).reshape(-1)
        block = torch.exp(normal(n // 64, 1)) * 1e-3
        s.theta = normal(n, std=0.02) * s.inside
        s.grad = (((normal(n // 64, 64) * block).reshape(-1)) * s.inside).to(torch.bfloat16 if case["grad"] == "bf16" else torch.float32)
        s.copy = s.theta.to(torch.bfloat16) if case["copies"] else None
        s.decay = [0.0 if i % 4 == 3 else 0.1 for i in range(len(s.sizes))]
        s.lr = torch.full((1,), 1e-3, device="cuda")
        s.grad_scale = torch.full((1,), 0.37, device="cuda") if case["scaled"] else None
        s.rng = torch.randint(2 ** 62, (2,), generator=g, device="cuda") if case["states"] == "fp8" else None
    if own:
        _prepare_own(s, case)
    elif s.call == "adamw":
        _prepare_adamw(s, case)
    return s


def _prepare_adamw(s, case):
    """What the plain form keeps: states that begin at 0, the tensors' decays by element."""
    n = s.theta.numel()
    s.step = torch.zeros(1, dtype=torch.int64, device="cuda")
    if case["states"] == "fp32":
        s.m, s.v = (torch.zeros(n, device="cuda") for _ in range(2))
    else:
        s.m, s.v = (torch.zeros(n, device="cuda").to(torch.float8_e4m3fn) for _ in range(2))
        s.m_scale, s.v_scale = (torch.zeros(n // 64, device="cuda") for _ in range(2))
    blocks = torch.tensor([-(-m // 64) for m in s.sizes], device="cuda")
    s.decay_by = torch.tensor(s.decay, device="cuda").repeat_interleave(blocks).repeat_interleave(64)


def _prepare_own(s, case):
    """The operator's handle with its workspace, and the buffers its results go to."""
    from paper_2406_02052_amd import AdamW, HeadNorm, VocabLoss

    if s.call.startswith("heads"):
        s.op = HeadNorm(case["batch"], case["length"], case["heads"], case["kv_heads"], case["dim"], case["dtype"],
                        norm=None if case["norm"] == "none" else case["norm"], eps=EPS, layout=case["layout"], freq=s.freq,
                        axis=s.axis)
        new = lambda t: None if t is None else torch.empty(t.shape, dtype=t.dtype, device="cuda")  # noqa: E731
        if s.call == "heads":
            s.yq, s.yk = new(s.q), new(s.k)
        else:
            s.dqkv = torch.zeros_like(s.qkv)
            h, kv = case["heads"], case["kv_heads"]
            s.dq, s.dk = s.dqkv[:, :, :h], s.dqkv[:, :, h:h + kv] if kv else None
            like = lambda p: None if p is None else tuple(None if t is None else torch.empty_like(t) for t in p)  # noqa: E731
            s.dq_norm, s.dk_norm = like(s.q_norm), like(s.k_norm)
    elif s.call.startswith("loss"):
        s.op = VocabLoss(case["rows"], case["width"], case["vocab"], case["dtype"], scale=s.scale)
        s.loss, s.lse = (torch.empty(case["rows"], device="cuda") for _ in range(2))
        if s.call == "loss_vjp":
            s.dx, s.dw = torch.empty_like(s.x), torch.empty_like(s.w)
    else:
        part = lambda t: None if t is None else [t[a:a + n] for a, n in zip(s.starts, s.sizes)]  # noqa: E731
        s.op = AdamW(part(s.theta), part(s.grad), states=case["states"], betas=(BETA1, BETA2), eps=ADAM_EPS,
                     weight_decay=s.decay, copies=part(s.copy))
        s.op.lr.copy_(s.lr)


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    if s.call == "heads":
        s.op.forward(s.q, s.k, s.yq, s.yk, q_norm=s.q_norm, k_norm=s.k_norm, positions=s.positions)
        return {"q": s.yq, "k": s.yk}
    if s.call == "heads_vjp":
        s.op.backward(s.q, s.k, s.dy_q, s.dy_k, s.dq, s.dk, q_norm=s.q_norm, k_norm=s.k_norm, dq_norm=s.dq_norm, dk_norm=s.dk_norm,
                      positions=s.positions)
        return _gradients(s.dq, s.dk, s.dq_norm, s.dk_norm)
    if s.call == "loss":
        s.op.forward(s.x, s.w, s.targets, s.loss, s.lse)
        return {"loss": s.loss, "lse": s.lse}
    if s.call == "loss_vjp":
        s.op.gradient(s.x, s.w, s.targets, s.loss, s.lse, s.dx, s.dw, weight=s.weight)
        return {"loss": s.loss, "lse": s.lse, "dx": s.dx, "dw": s.dw}
    s.op.step(rng=s.rng, grad_scale=s.grad_scale)
    return _updated(s, s.op.m, s.op.v, s.op.m_scale, s.op.v_scale)


def _gradients(dq, dk, dq_norm, dk_norm):
    flat = [t for p in (dq_norm, dk_norm) if p is not None for t in p if t is not None]
    return {"dq": dq, "dk": dk, "dnorm": flat}


def _updated(s, m, v, m_scale, v_scale):
    out = {"theta": s.theta, "m": m, "v": v}
    if s.copy is not None:
        out["copy"] = s.copy
    return out if m_scale is None else {**out, "m_scale": m_scale, "v_scale": v_scale}


# ---------------------------------------------------------------------------
# the plain forms, in 32 bits
# ---------------------------------------------------------------------------

def _unit(t, norm):
    """(t normalised over its channels, 1 / its deviation)."""
    if norm == "layer":
        t = t - t.mean(-1, keepdim=True)
    r = torch.rsqrt(t.square().mean(-1, keepdim=True) + EPS)
    return t * r, r


def _turns(s):
    """cos and sin of each token's pairs [batch, length, 1, pairs]; far positions need more than 32 bits."""
    freq, axis = (torch.tensor(t, device="cuda") for t in (s.freq, s.axis))
    angle = s.positions[axis].permute(1, 2, 0).double() * torch.tensor(s.freq, dtype=torch.float64, device="cuda")
    return angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]


def _rotate(z, cos, sin, layout):
    n = cos.shape[-1]
    y = z.clone()
    a, b = (slice(0, n), slice(n, 2 * n)) if layout == "halves" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    y[..., a] = z[..., a] * cos - z[..., b] * sin
    y[..., b] = z[..., a] * sin + z[..., b] * cos
    return y


def _plain_heads(s):
    case, (cos, sin) = s.case, _turns(s)

    def forward(x, p):
        if x is None:
            return None
        z = x.float()
        if p is not None:
            z = _unit(z, case["norm"])[0] * p[0] + (0.0 if p[1] is None else p[1])
        return _rotate(z, cos, sin, case["layout"]).to(x.dtype)

    def backward(x, dy, p):
        if x is None:
            return None, None
        g = _rotate(dy.float(), cos, -sin, case["layout"])
        if p is None:
            return g.to(x.dtype), None
        n, r = _unit(x.float(), case["norm"])
        dp = ((g * n).sum((0, 1, 2)), None if p[1] is None else g.sum((0, 1, 2)))
        h = g * p[0]
        dx = h - n * (h * n).mean(-1, keepdim=True) - (h.mean(-1, keepdim=True) if case["norm"] == "layer" else 0.0)
        return (dx * r).to(x.dtype), dp

    if s.call == "heads":
        return {"q": forward(s.q, s.q_norm), "k": forward(s.k, s.k_norm)}
    (dq, dq_norm), (dk, dk_norm) = backward(s.q, s.dy_q, s.q_norm), backward(s.k, s.dy_k, s.k_norm)
    return _gradients(dq, dk, dq_norm, dk_norm)


def _plain_loss(s):
    case, x, w = s.case, s.x.float(), s.w.float()
    t = s.targets.long()
    live = (t >= 0) & (t < case["vocab"])
    at = torch.where(live, t, 0)[:, None]
    logits = (x @ w.T) * s.scale
    top = logits.amax(1, keepdim=True)
    e = torch.exp(logits - top)
    total = e.sum(1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    loss = torch.where(live, lse - logits.gather(1, at)[:, 0], 0.0)
    out = {"loss": loss, "lse": torch.where(live, lse, 0.0)}
    if s.call == "loss":
        return out
    weight = s.weight if s.weight is not None else 1.0 / live.sum().clamp(min=1)
    d = e / total
    d.scatter_add_(1, at, torch.full_like(lse, -1.0)[:, None])
    d *= torch.where(live, weight * s.scale, 0.0)[:, None]
    return {**out, "dx": (d @ w).to(s.x.dtype), "dw": (d.T @ x).to(s.w.dtype)}


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


def _scale(t):
    """The power of two that brings each row's largest magnitude into [128, 256); 0 for a row of zeros."""
    top = t.abs().amax(1, keepdim=True)
    return torch.where(top > 0, torch.ldexp(torch.ones_like(top), torch.frexp(top).exponent - 8), 0.0)


def _step_of(x):
    """Distance from x to the next e4m3 number, and the number at or below x (x >= 0)."""
    ulp = torch.ldexp(torch.ones_like(x), (torch.frexp(x).exponent - 4).clamp(min=-9))
    return ulp, torch.floor(x / ulp) * ulp


def _hold(m, v, rng):
    """(m, scale, r, scale) as held in 8 bits; rows are blocks."""
    u = _bits(rng, torch.arange(m.numel() // 4, device="cuda")).reshape(-1, 64, 2).float() / 65536.0
    sm, r = _scale(m), torch.sqrt(v)
    sr = _scale(r)
    x = m.abs() / torch.where(sm > 0, sm, 1.0)
    ulp, lo = _step_of(x)
    hm = torch.copysign(torch.where(u[..., 0] * ulp < x - lo, lo + ulp, lo), m)
    # v in units of its block's scale, squared: exact, the scale is a power of two
    one = torch.where(sr > 0, sr, 1.0)
    w, (ulp, lo) = v / one / one, _step_of(r / one)
    hr = torch.where(u[..., 1] * (ulp * (2.0 * lo + ulp)) < w - lo * lo, lo + ulp, lo)
    hr = torch.where(v > 0, hr.clamp(min=2.0 ** -9), hr)
    return hm.to(torch.float8_e4m3fn), sm, hr.to(torch.float8_e4m3fn), sr


def _plain_adamw(s):
    s.step += 1
    t = s.step.double()
    c1, c2 = (-torch.expm1(t * math.log(b)) for b in (BETA1, BETA2))
    c1, c2 = c1.float(), c2.sqrt().float()
    fp8 = s.rng is not None
    m, v = s.m, s.v
    if fp8:
        m = (m.float().reshape(-1, 64) * s.m_scale[:, None]).reshape(-1)
        v = (v.float().reshape(-1, 64) * s.v_scale[:, None]).reshape(-1).square()
    g = s.grad.float()
    if s.grad_scale is not None:
        g = g * s.grad_scale
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + g * g * (1.0 - BETA2)
    s.theta -= s.lr * (m / c1 / (torch.sqrt(v) / c2 + ADAM_EPS) + s.decay_by * s.theta)
    if s.copy is not None:
        s.copy.copy_(s.theta)
    if not fp8:
        s.m.copy_(m)
        s.v.copy_(v)
        return _updated(s, s.m, s.v, None, None)
    hm, sm, hr, sr = _hold(m.reshape(-1, 64), v.reshape(-1, 64), s.rng)
    s.m, s.v, s.m_scale, s.v_scale = hm.reshape(-1), hr.reshape(-1), sm.reshape(-1), sr.reshape(-1)
    return _updated(s, s.m, s.v, s.m_scale, s.v_scale)


def _run_plain(s):
    if s.call.startswith("heads"):
        return _plain_heads(s)
    return _plain_loss(s) if s.call.startswith("loss") else _plain_adamw(s)


# ---------------------------------------------------------------------------
# what a call cannot do without
# ---------------------------------------------------------------------------

def work(case):
    if case["call"] == "adamw":
        n, fp8 = sum(_sizes(case)), case["states"] == "fp8"
        return {"bytes": n * (8 + (2 if case["grad"] == "bf16" else 4) + (4.25 if fp8 else 16) + (2 if case["copies"] else 0)),
                "flops": 15 * n}
    esz = 2 if case["dtype"] == "bf16" else 4
    if case["call"].startswith("heads"):
        n = case["batch"] * case["length"]
        size = n * (case["heads"] + case["kv_heads"]) * case["dim"]
        vjp = case["call"] == "heads_vjp"
        return {"bytes": size * esz * (3 if vjp else 2) + 4 * n * min(case["axes"], case["pairs"]) + 16 * case["dim"],
                "flops": size * (16 if vjp else 8)}
    r, w, v = case["rows"], case["width"], case["vocab"]
    vjp = case["call"] == "loss_vjp"
    return {"bytes": (r * w + v * w) * esz * (2 if vjp else 1) + 12 * r, "flops": 2 * r * w * v * (3 if vjp else 1)}


# ---------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# ---------------------------------------------------------------------------

def _exact_heads(s):
    """Rotations as products of complex numbers, gradients by automatic differentiation."""
    case, n = s.case, s.case["pairs"]
    freq = torch.tensor(s.freq, dtype=torch.float64, device="cuda")
    at = torch.stack([s.positions[a] for a in s.axis], -1)
    turn = torch.polar(torch.ones_like(at, dtype=torch.float64), at * freq)[:, :, None]

    def apply(x, p):
        if p is not None:
            var, mean = torch.var_mean(x, -1, correction=0, keepdim=True)
            x = (x - mean) / (var + EPS).sqrt() if case["norm"] == "layer" else x / ((x * x).mean(-1, keepdim=True) + EPS).sqrt()
            x = x * p[0] + (0.0 if p[1] is None else p[1])
        head, rest = x[..., :2 * n], x[..., 2 * n:]
        apart = head.unflatten(-1, (2, n)).movedim(-2, -1) if case["layout"] == "halves" else head.unflatten(-1, (n, 2))
        turned = torch.view_as_real(torch.view_as_complex(apart.contiguous()) * turn)
        turned = turned.movedim(-1, -2) if case["layout"] == "halves" else turned
        return torch.cat([turned.flatten(-2), rest], -1)

    out, norms, names = {}, [], (("q", s.q, s.q_norm), ("k", s.k, s.k_norm))
    for name, x, p in names:
        if x is None:
            out[name if s.call == "heads" else "d" + name] = None
            continue
        x = x.double().requires_grad_()
        p = None if p is None else [None if t is None else t.double().requires_grad_() for t in p]
        y = apply(x, p)
        if s.call == "heads":
            out[name] = y.detach()
            continue
        leaves = [x] + [t for t in p or [] if t is not None]
        out["d" + name], *dp = torch.autograd.grad(y, leaves, (s.dy_q if name == "q" else s.dy_k).double())
        norms += dp
    return out if s.call == "heads" else {**out, "dnorm": norms}


def _exact_loss(s):
    case, v = s.case, s.case["vocab"]
    x, w, t = s.x.double(), s.w.double(), s.targets.tolist()
    rows = torch.tensor([i for i, a in enumerate(t) if 0 <= a < v], device="cuda", dtype=torch.int64)
    cols = torch.tensor([a for a in t if 0 <= a < v], device="cuda", dtype=torch.int64)
    loss, lse, dx, dw = (torch.zeros(n, dtype=torch.float64, device="cuda") for n in ((case["rows"],), (case["rows"],), x.shape, w.shape))
    for part, cut in zip(rows.split(2048), cols.split(2048)):
        logits = torch.mm(x[part], w.t()).mul_(s.scale)
        l = torch.logsumexp(logits, 1)
        lse[part], loss[part] = l, l - logits[torch.arange(len(part), device="cuda"), cut]
        if s.call == "loss_vjp":
            p = logits.sub_(l[:, None]).exp_()
            p[torch.arange(len(part), device="cuda"), cut] -= 1.0
            p *= (s.weight.double()[part, None] if s.weight is not None else 1.0 / len(rows)) * s.scale
            dx[part] = torch.mm(p, w)
            dw += torch.mm(p.t(), x[part])
    return {"loss": loss, "lse": lse} if s.call == "loss" else {"loss": loss, "lse": lse, "dx": dx, "dw": dw}


def _mul32(a, m):
    """(high, low) words of a 32-bit word times the constant m, by 16-bit digits."""
    a0, a1, m0, m1 = a & 0xFFFF, a >> 16, m & 0xFFFF, m >> 16
    mid = a1 * m0 + (a0 * m0 >> 16)
    cross = a0 * m1 + (mid & 0xFFFF)
    return a1 * m1 + (mid >> 16) + (cross >> 16), ((cross & 0xFFFF) << 16) | (a0 * m0 & 0xFFFF)


def _numbers(rng, n):
    """Two 16-bit numbers of each of n elements, in [0, 1)."""
    seed, offset = (int(t) for t in rng.tolist())
    at = torch.arange(n, device="cuda")
    x0, x1 = at // 4 % 2 ** 32, at // 4 // 2 ** 32
    x2, x3 = torch.full_like(x0, offset % 2 ** 32), torch.full_like(x0, offset // 2 ** 32)
    for r in range(7):
        k0, k1 = (seed % 2 ** 32 + r * 0x9E3779B9) % 2 ** 32, (seed // 2 ** 32 + r * 0xBB67AE85) % 2 ** 32
        (h0, l0), (h1, l1) = _mul32(x0, 0xD2511F53), _mul32(x2, 0xCD9E8D57)
        x0, x1, x2, x3 = h1 ^ x1 ^ k0, l1, h0 ^ x3 ^ k1, l0
    word = torch.where(at % 4 < 2, torch.where(at % 2 == 0, x0, x1), torch.where(at % 2 == 0, x2, x3))
    return word % 65536 / 65536.0, word // 65536 / 65536.0


def _exact_adamw(s):
    """The first step from states of 0.  The numbers of the format are looked up in a table of them all; scales
    have no value of their own apart from the numbers they belong to."""
    case, n = s.case, s.theta.numel()
    g = s.grad.double() * (1.0 if s.grad_scale is None else s.grad_scale.double())
    m, v = (1.0 - BETA1) * g, (1.0 - BETA2) * g ** 2
    decay = torch.zeros(n, dtype=torch.float64, device="cuda")
    for a, size, d in zip(s.starts, s.sizes, s.decay):
        decay[a:a + size] = d
    theta = s.theta.double()
    theta = theta - s.lr.double() * (m / (1.0 - BETA1) / ((v / (1.0 - BETA2)).sqrt() + ADAM_EPS) + decay * theta)
    out = {"theta": theta} if s.copy is None else {"theta": theta, "copy": theta}
    if case["states"] == "fp32":
        return {**out, "m": m, "v": v}
    table = torch.arange(127, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).double()
    u, root = _numbers(s.rng, n), v.sqrt()

    def held(t, power, u):
        """|t| rounded so that its `power` is kept on average, in units of its block's scale."""
        top = t.reshape(-1, 64).amax(1)
        unit = torch.where(top > 0, 2.0 ** (torch.floor(torch.log2(top.clamp(min=1e-300))) - 7), 1.0).repeat_interleave(64)
        t = t / unit
        lo = torch.searchsorted(table, t, right=True) - 1
        a, b = table[lo] ** power, table[lo + 1] ** power
        return torch.where(u * (b - a) < t ** power - a, table[lo + 1], table[lo])

    r = held(root, 2, u[1])
    return {**out, "m": held(m.abs(), 1, u[0]) * m.sign(), "v": torch.where(root > 0, r.clamp(min=2.0 ** -9), r),
            "m_scale": None, "v_scale": None}


def exact(case, seed):
    s = prepare(case, seed)
    if s.call.startswith("heads"):
        return _exact_heads(s)
    return _exact_loss(s) if s.call.startswith("loss") else _exact_adamw(s)
