"""A reversible attention block from the token operators: two streams, no stored activations.

    y1 = s x1 + g1 drop(n(F(x2))),   y2 = s x2 + g2 drop(n(G(y1)))

F is causal attention with dropout on its probabilities (its projections by torch's products), G
a two-layer network; the coupling's kernel also forms the norm that the next function reads.
The backward keeps y1, y2, the parameters and 16 bytes of {seed, offset} per dropout: it runs G
and F again, rebuilds x2 and x1 from y2 and y1 and gives the gradients of both streams and of
every parameter.

    python examples/reversible_attention.py [--batch B --tokens N --width C --heads H --kv-heads K]

prints how far the rebuilt streams and a directional derivative are from what they should be.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2406_02052_amd import Attention, Coupling  # noqa: E402


class Block:
    def __init__(self, batch, tokens, width, heads, kv_heads, dtype="bf16", dropout=0.1, scale=1.0, seed=0):
        self.dims = (batch, tokens, heads, kv_heads, width // heads)
        self.rows, self.width, self.dropout = batch * tokens, width, dropout
        self.type = torch.bfloat16 if dtype == "bf16" else torch.float32
        dim = width // heads
        self.attention = Attention(batch, tokens, tokens, heads, kv_heads, dim, dtype, causal=True, dropout=dropout)
        self.coupling = Coupling(self.rows, width, dtype, residual_scale=scale, dropout=dropout)
        g = torch.Generator("cuda").manual_seed(seed)

        def weight(n_in, n_out):
            return torch.randn(n_in, n_out, generator=g, device="cuda") / math.sqrt(n_in)

        one = torch.ones(width, device="cuda")
        self.params = {"qkv": weight(width, (heads + 2 * kv_heads) * dim), "out": weight(width, width),
                       "up": weight(width, 2 * width), "down": weight(2 * width, width)}
        for f in "FG":
            self.params.update({f + ".gate": one.clone()[None] * 0.5, f + ".post": one.clone(), f + ".pre": one.clone()})
        self.seed = seed

    def rngs(self, step):
        """{seed, offset} of the three dropouts of one micro-batch's step."""
        return [torch.tensor([self.seed, 3 * step + i], dtype=torch.int64, device="cuda") for i in range(3)] \
            if self.dropout else [None] * 3

    def new(self):
        return torch.empty(self.rows, self.width, dtype=self.type, device="cuda")

    def _w(self, name):
        return self.params[name].to(self.type)

    def _norm(self, f, which):
        return (self.params[f + "." + which], None)

    # -- the residual functions, from u = n(stream) to their output ----------
    def F(self, u, rng):
        b, n, h, k, d = self.dims
        qkv = (u @ self._w("qkv")).view(b, n, h + 2 * k, d)      # one tensor: q, k and v are its slices
        q, kk, v = qkv[:, :, :h], qkv[:, :, h:h + k], qkv[:, :, h + k:]
        o, lse = torch.empty(b, n, h, d, dtype=self.type, device="cuda"), torch.empty(b, h, n, device="cuda")
        self.attention.forward(q, kk, v, o, lse, rng=rng)
        return o.view(self.rows, self.width) @ self._w("out"), (u, qkv, o, lse)

    def F_backward(self, df, saved, rng, grads):
        b, n, h, k, d = self.dims
        u, qkv, o, lse = saved
        grads["out"] = o.view(self.rows, self.width).float().t() @ df.float()
        do = (df @ self._w("out").t().contiguous()).view(b, n, h, d)
        dqkv = torch.empty_like(qkv)
        parts = [t for x in (qkv, dqkv) for t in (x[:, :, :h], x[:, :, h:h + k], x[:, :, h + k:])]
        self.attention.backward(*parts[:3], o, lse, do, *parts[3:], rng=rng)
        dqkv = dqkv.view(self.rows, -1)
        grads["qkv"] = u.float().t() @ dqkv.float()
        return dqkv @ self._w("qkv").t().contiguous()

    def G(self, u):
        a = u @ self._w("up")
        return torch.relu(a) @ self._w("down"), (u, a)

    def G_backward(self, dg, saved, grads):
        u, a = saved
        grads["down"] = torch.relu(a).float().t() @ dg.float()
        da = (dg @ self._w("down").t().contiguous()) * (a > 0)
        grads["up"] = u.float().t() @ da.float()
        return da @ self._w("up").t().contiguous()

    # -- the block ----------------------------------------------------------
    def forward(self, x1, x2, step=0):
        r, c = self.rngs(step), self.coupling
        u2, u1, y1, y2 = (self.new() for _ in range(4))
        c.forward(x2, pre=self._norm("F", "pre"), u=u2)
        c.forward(x1, self.F(u2, r[0])[0], self.params["F.gate"], self._norm("F", "post"), y1,
                  pre=self._norm("G", "pre"), u=u1, rng=r[1])     # y1 and the norm that G reads
        c.forward(x2, self.G(u1)[0], self.params["G.gate"], self._norm("G", "post"), y2, rng=r[2])
        return y1, y2

    def backward(self, y1, y2, dy1, dy2, step=0):
        """(x1, x2, dx1, dx2, gradients by name); y1 and y2 are all that is left of the forward."""
        r, c, grads = self.rngs(step), self.coupling, {}
        new_norm = lambda: (torch.empty(self.width, device="cuda"), None)  # noqa: E731
        norms = {k: new_norm() for k in ("F.post", "F.pre", "G.post", "G.pre")}
        gates = {f: torch.empty_like(self.params[f + ".gate"]) for f in "FG"}
        u1, x2, dx2, dg = (self.new() for _ in range(4))
        c.forward(y1, pre=self._norm("G", "pre"), u=u1)
        g, saved = self.G(u1)
        c.backward(y2, g, dy2, self.params["G.gate"], self._norm("G", "post"), x2, dx2, dg, gates["G"], norms["G.post"],
                   rng=r[2])
        du1 = self.G_backward(dg, saved, grads)
        u2, x1, dx1, df = (self.new() for _ in range(4))
        c.forward(x2, pre=self._norm("F", "pre"), u=u2)
        f, saved = self.F(u2, r[0])
        # y1 is read twice, as the stream and through G's norm: both gradients in one pass
        c.backward(y1, f, dy1, self.params["F.gate"], self._norm("F", "post"), x1, dx1, df, gates["F"], norms["F.post"],
                   du=du1, pre=self._norm("G", "pre"), dpre=norms["G.pre"], rng=r[1])
        du2 = self.F_backward(df, saved, r[0], grads)
        # and x2 through F's norm: dx2 += (dn/dx2)^T du2, by the coupling without a function at scale 1
        total = self.new()
        Coupling(self.rows, self.width, "bf16" if self.type is torch.bfloat16 else "fp32").backward(
            x2, None, dx2, None, None, None, total, None, None, None, du=du2, pre=self._norm("F", "pre"),
            dpre=norms["F.pre"])
        grads.update({f + ".gate": gates[f] for f in "FG"}, **{k: v[0] for k, v in norms.items()})
        return x1, x2, dx1, total, grads


def check(block, seed=1):
    """(error of the rebuilt streams, error of the derivative along their gradient), both relative."""
    g = torch.Generator("cuda").manual_seed(seed)

    def draw():
        return torch.randn(block.rows, block.width, generator=g, device="cuda").to(block.type)

    x1, x2, dy1, dy2 = (draw() for _ in range(4))
    y1, y2 = block.forward(x1, x2)
    b1, b2, dx1, dx2, _ = block.backward(y1, y2, dy1, dy2)
    rebuilt = max(float((b - x).float().norm() / x.float().norm()) for b, x in ((b1, x1), (b2, x2)))
    # the derivative of sum(y dy) by a step that moves the streams by a hundredth of their size
    step = 0.01 * float(x1.float().norm() / dx1.float().norm())

    def loss(s):
        z1, z2 = block.forward(*((x.float() + s * d.float()).to(block.type) for x, d in ((x1, dx1), (x2, dx2))))
        return float((z1.double() * dy1.double()).sum() + (z2.double() * dy2.double()).sum())

    want = float(dx1.double().square().sum() + dx2.double().square().sum())
    return rebuilt, abs((loss(step) - loss(-step)) / (2 * step) - want) / want


def main():
    p = argparse.ArgumentParser()
    for name, value in (("batch", 4), ("tokens", 256), ("width", 256), ("heads", 4), ("kv-heads", 2)):
        p.add_argument("--" + name, type=int, default=value)
    p.add_argument("--dtype", choices=("bf16", "fp32"), default="bf16")
    a = p.parse_args()
    block = Block(a.batch, a.tokens, a.width, a.heads, a.kv_heads, a.dtype)
    rebuilt, derivative = check(block)
    print(f"rebuilt streams off by {rebuilt:.2e}, derivative along the gradient off by {derivative:.2e}")


if __name__ == "__main__":
    main()
