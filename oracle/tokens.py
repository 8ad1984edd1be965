"""Operators of stages over tokens in fp64 (numpy): dropout's generator, attention,
the gated norm coupling, head norms with rotation and the loss over a vocabulary with
their gradients, and AdamW, each from its formula."""
import numpy as np


# ---- dropout ---------------------------------------------------------------

def philox(counter, key, rounds=7):
    """Philox-4x32 (Salmon et al. 2011): counter [..., 4], key [2] words -> [..., 4]."""
    c = [np.asarray(counter)[..., i].astype(np.uint64) for i in range(4)]
    k = [int(key[0]), int(key[1])]
    low, sh = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(rounds):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> sh) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> sh) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, -1)


def group_bits(rng, group):
    """The eight 16-bit numbers of each group: [..., 8]."""
    seed, offset = (int(v) % 2 ** 64 for v in rng)
    group = np.asarray(group, np.uint64)
    c = np.stack([group & np.uint64(0xFFFFFFFF), group >> np.uint64(32),
                  np.full_like(group, offset & 0xFFFFFFFF), np.full_like(group, offset >> 32)], -1)
    w = philox(c, (seed & 0xFFFFFFFF, seed >> 32))
    return np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], -1).reshape(*group.shape, 8)


def cut(p):
    return round(65536 * p)


def factor(rng, p, shape):
    """0 or 1 / share kept, for the elements of a tensor."""
    n = int(np.prod(shape, dtype=np.int64))
    bits = group_bits(rng, np.arange(-(-n // 8))).reshape(-1)[:n].reshape(shape)
    return (bits >= cut(p)) / (1.0 - cut(p) / 65536.0)


def factor_attention(rng, p, batch, heads, q_len, kv_len):
    """The same for the probabilities [batch, heads, q_len, kv_len]."""
    j = np.arange(kv_len)
    row = np.arange(batch * heads * q_len).reshape(batch, heads, q_len, 1)
    group = (row * (-(-kv_len // 16)) + j // 16) * 2 + (j % 16 // 4) % 2
    bits = np.take_along_axis(group_bits(rng, group), np.broadcast_to(
        (j % 16 // 8) * 4 + j % 4, group.shape)[..., None], -1)[..., 0]
    return (bits >= cut(p)) / (1.0 - cut(p) / 65536.0)


def dropout(x, p, rng, residual=None, alpha=1.0):
    m = factor(rng, p, x.shape)
    y = alpha * np.where(m > 0, x * m, 0.0)
    return y if residual is None else y + residual


# ---- attention --------------------------------------------------------------

def visible(q_len, kv_len, lq, lk, causal):
    i, j = np.arange(q_len)[:, None], np.arange(kv_len)[None]
    seen = (i < lq) & (j < lk)
    return seen & (j <= i + lk - lq) if causal else seen


def attention(q, k, v, scale, causal=False, q_lens=None, kv_lens=None, mask=None, d_o=None):
    """[batch, len, heads, dim] arrays; mask: dropout's factors.  (o, lse), and with d_o
    also (dq, dk, dv)."""
    b, nq, h, _ = q.shape
    nk, kvh = k.shape[1:3]
    o, lse = np.zeros(q.shape), np.full((b, h, nq), -np.inf)
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for n in range(b):
        lq = nq if q_lens is None else min(max(int(q_lens[n]), 0), nq)
        lk = nk if kv_lens is None else min(max(int(kv_lens[n]), 0), nk)
        seen = visible(lq, lk, lq, lk, causal)
        rows = seen.any(1)
        if not rows.any():
            continue
        for g in range(h):
            e = g // (h // kvh)
            # the lengths cut the tensors: what lies past them has no part
            qq, kk, vv = q[n, :lq, g], k[n, :lk, e], v[n, :lk, e]
            s = np.where(seen, scale * (qq @ kk.T), -np.inf)
            top = np.where(rows, s.max(1, initial=-np.inf), 0.0)[:, None]
            p = np.exp(s - top)
            total = p.sum(1, keepdims=True)
            p = p / np.where(total > 0, total, 1.0)
            lse[n, g, :lq][rows] = (top + np.log(np.where(total > 0, total, 1.0)))[rows, 0]
            m = 1.0 if mask is None else mask[n, g, :lq, :lk]
            o[n, :lq, g] = (p * m) @ vv
            if d_o is None:
                continue
            gg = d_o[n, :lq, g]
            dp = m * (gg @ vv.T)
            ds = scale * p * (dp - (p * dp).sum(1, keepdims=True))
            dq[n, :lq, g] = ds @ kk
            dk[n, :lk, e] += ds.T @ qq
            dv[n, :lk, e] += (p * m).T @ gg
    return (o, lse) if d_o is None else (o, lse, dq, dk, dv)


# ---- coupling ---------------------------------------------------------------

def unit(z, norm, eps):
    z = z - z.mean(1, keepdims=True) if norm == "layer" else z
    r = 1.0 / np.sqrt((z * z).mean(1, keepdims=True) + eps)
    return z * r, r


def affine(z, p):
    return z * p[0] + (0.0 if p[1] is None else p[1])


def unit_backward(h, z, r, norm):
    h = h - z * (h * z).mean(1, keepdims=True) - (h.mean(1, keepdims=True) if norm == "layer" else 0.0)
    return r * h


def coupling(x, f, gate, post, norm, eps, scale, mask=None):
    """y; gate [gates, width] shared by consecutive rows."""
    g = np.repeat(gate, x.shape[0] // gate.shape[0], 0)
    return scale * x + g * affine(unit(f, norm, eps)[0], post) * (1.0 if mask is None else mask)


def norm_forward(x, pre, norm, eps):
    return affine(unit(x, norm, eps)[0], pre)


def coupling_backward(y, f, dy, gate, post, norm, eps, scale, mask=None, du=None, pre=None):
    """dict of x, dx, df, dgate, dpost and, with du, dpre."""
    out, t, w = {}, dy, y.shape[1]
    if du is not None:
        yn, r = unit(y, norm, eps)
        t = t + unit_backward(du * pre[0], yn, r, norm)
        out["dpre"] = ((du * yn).sum(0), du.sum(0))
    out["dx"] = scale * t
    if f is None:
        return out
    m = 1.0 if mask is None else mask
    g = np.repeat(gate, y.shape[0] // max(1, gate.shape[0]), 0)
    fn, r = unit(f, norm, eps)
    n = affine(fn, post) * m
    dn = g * t * m
    out.update(x=(y - g * n) / scale, df=unit_backward(dn * post[0], fn, r, norm),
               dgate=(t * n).reshape(gate.shape[0], -1, w).sum(1), dpost=((dn * fn).sum(0), dn.sum(0)))
    return out


# ---- head norms and rotation -------------------------------------------------

def rotate(z, positions, freq, axis, layout):
    """z [batch, len, heads, dim], positions [axes][batch, len]."""
    y, n = np.array(z, float), len(freq)
    for i in range(n):
        a, b = (i, i + n) if layout == "halves" else (2 * i, 2 * i + 1)
        # whole turns apart in long double: far positions keep their fraction
        t = np.asarray(positions[axis[i]], np.longdouble) * np.longdouble(freq[i])
        t = np.remainder(t, 2 * np.longdouble("3.14159265358979323846264338327950288")).astype(float)[:, :, None]
        y[..., a] = z[..., a] * np.cos(t) - z[..., b] * np.sin(t)
        y[..., b] = z[..., a] * np.sin(t) + z[..., b] * np.cos(t)
    return y


def head_norm(x, params, kind, eps, positions, freq, axis, layout, dy=None):
    """y, or with dy (dx, dgamma, dbeta); params (gamma, beta or None), or None for no norm."""
    if params is None:
        return rotate(x, positions, freq, axis, layout) if dy is None else (
            rotate(dy, positions, [-f for f in freq], axis, layout), None, None)
    z = x - x.mean(-1, keepdims=True) if kind == "layer" else x
    r = 1.0 / np.sqrt((z * z).mean(-1, keepdims=True) + eps)
    z = z * r
    gamma, beta = params
    if dy is None:
        return rotate(z * gamma + (0.0 if beta is None else beta), positions, freq, axis, layout)
    g = rotate(dy, positions, [-f for f in freq], axis, layout)
    h = g * gamma
    dx = h - z * (h * z).mean(-1, keepdims=True)
    if kind == "layer":
        dx = dx - h.mean(-1, keepdims=True)
    return r * dx, (g * z).sum((0, 1, 2)), None if beta is None else g.sum((0, 1, 2))


# ---- loss over a vocabulary ---------------------------------------------------

def vocab_loss(x, w, targets, scale=1.0, weight=None):
    """loss, lse, dx, dw of sum(weight loss); rows whose target is no column take no part."""
    rows, vocab = len(x), len(w)
    live = np.array([0 <= t < vocab for t in targets], bool)
    at = np.flatnonzero(live)
    loss, lse, dx = np.zeros(rows), np.zeros(rows), np.zeros(x.shape)
    dw = np.zeros(w.shape)
    if len(at):
        t = np.asarray(targets)[at]
        s = scale * (x[at] @ w.T)
        top = s.max(1)
        lse[at] = top + np.log(np.exp(s - top[:, None]).sum(1))
        loss[at] = lse[at] - s[np.arange(len(at)), t]
        p = np.exp(s - lse[at, None])
        p[np.arange(len(at)), t] -= 1.0
        p *= scale * (np.full(len(at), 1.0 / len(at)) if weight is None else np.asarray(weight)[at])[:, None]
        dx[at], dw = p @ w, p.T @ x[at]
    return loss, lse, dx, dw


# ---- AdamW --------------------------------------------------------------------

E4M3 = np.array([0.0] + [i / 8 * 2.0 ** -6 for i in range(1, 8)]
                + [(1 + i / 8) * 2.0 ** e for e in range(-6, 9) for i in range(8)][:119])


def adamw(theta, grad, m, v, t, lr, betas, eps, decay, grad_scale=1.0):
    """theta, m, v after step t (from 1)."""
    g = grad_scale * grad
    m = betas[0] * m + (1 - betas[0]) * g
    v = betas[1] * v + (1 - betas[1]) * g * g
    step = m / (1 - betas[0] ** t) / (np.sqrt(v / (1 - betas[1] ** t)) + eps)
    return theta - lr * (step + decay * theta), m, v


def hold(x, power, u, scale=None):
    """|x| by blocks of 64 (padded with zeros) in e4m3 with a power of two as the scale (or the one
    that is given): (numbers, scales).  u in [0, 1) decides between neighbours such that x^power is
    kept on average."""
    n = len(x)
    a = np.zeros(-(-n // 64) * 64)
    a[:n] = np.abs(x)
    blocks = a.reshape(-1, 64)
    top = blocks.max(1)
    if scale is None:
        scale = np.where(top > 0, 2.0 ** (np.floor(np.log2(np.where(top > 0, top, 1.0))) - 7), 0.0)
    y = blocks / np.where(scale > 0, scale, 1.0)[:, None]
    lo = np.searchsorted(E4M3, y, side="right") - 1
    b0, b1 = E4M3[lo] ** power, E4M3[lo + 1] ** power
    up = np.asarray(u).reshape(y.shape) * (b1 - b0) < y ** power - b0
    q = E4M3[lo + up]
    if power == 2:
        q = np.where(y > 0, np.maximum(q, E4M3[1]), q)
    return q.reshape(-1), scale


def adamw_numbers(rng, first_group, n):
    """The two random numbers of each of n elements (a multiple of 4) from a group of 4 on."""
    bits = group_bits(rng, first_group + np.arange(n // 4)).reshape(-1, 2)
    return bits[:, 0] / 65536.0, bits[:, 1] / 65536.0
