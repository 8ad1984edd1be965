"""The example's block: its streams are rebuilt from its output, and its gradients are those of
automatic differentiation of the same block in fp64, masks from the oracle's generator."""
import math
import os
import sys

import numpy as np
import pytest
import torch

from oracle import tokens as T

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def plain(block, x1, x2, p):
    """The block in fp64 by torch's operations, on the CPU."""
    b, n, h, k, d = block.dims
    masks = [torch.ones(())] * 3
    if block.dropout:
        rngs = [r.tolist() for r in block.rngs(0)]
        masks = [torch.tensor(T.factor_attention(rngs[0], block.dropout, b, h, n, n))] \
            + [torch.tensor(T.factor(r, block.dropout, (block.rows, block.width))) for r in rngs[1:]]

    def norm(x, gamma):
        return x / (x.square().mean(1, keepdim=True) + 1e-5).sqrt() * gamma

    qkv = (norm(x2, p["F.pre"]) @ p["qkv"]).view(b, n, h + 2 * k, d).transpose(1, 2)
    q, kk, v = qkv[:, :h], qkv[:, h:h + k].repeat_interleave(h // k, 1), qkv[:, h + k:].repeat_interleave(h // k, 1)
    s = (q @ kk.transpose(2, 3)) / math.sqrt(d)
    s = s.masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), -math.inf)
    o = (s.softmax(3) * masks[0]) @ v
    f = o.transpose(1, 2).reshape(block.rows, block.width) @ p["out"]
    scale = block.coupling.desc.residual_scale
    y1 = scale * x1 + p["F.gate"] * norm(f, p["F.post"]) * masks[1]
    g = torch.relu(norm(y1, p["G.pre"]) @ p["up"]) @ p["down"]
    return y1, scale * x2 + p["G.gate"] * norm(g, p["G.post"]) * masks[2]


@pytest.mark.parametrize("dtype,sizes,dropout,scale", [
    ("fp32", (2, 70, 96, 4, 2), 0.2, 1.0), ("fp32", (1, 33, 64, 2, 1), 0.0, 0.75), ("bf16", (2, 130, 256, 4, 2), 0.1, 1.0)])
def test_block_rebuilds_its_input_and_differentiates(dtype, sizes, dropout, scale):
    """Bars: fp32, some ten products and norms in a row, 1e-4.  bf16: 2^-9 for a rebuilt stream, twice
    and with G's error, 2^-7; a relu turns where its input's error, some 2^-8 of its size, passes zero,
    so about 2^-8 of them do, which changes a gradient by the root of that, 6 %: twice that."""
    import reversible_attention as R

    block = R.Block(*sizes, dtype=dtype, dropout=dropout, scale=scale)
    r = np.random.RandomState(0)
    host = [torch.tensor(r.randn(block.rows, block.width)).to(block.type).double() for _ in range(4)]
    x1, x2, dy1, dy2 = (t.to("cuda", block.type) for t in host)
    y1, y2 = block.forward(x1, x2)
    got = block.backward(y1, y2, dy1, dy2)
    leaves = {n: t.cpu().double().requires_grad_() for n, t in block.params.items()}
    h1, h2 = host[0].requires_grad_(), host[1].requires_grad_()
    w1, w2 = plain(block, h1, h2, leaves)
    want = torch.autograd.grad((w1, w2), [h1, h2] + list(leaves.values()), (host[2], host[3]))

    def rel(a, b):
        return float((a.detach().cpu().double() - b.detach()).norm() / b.detach().norm())

    errors = {"y1": rel(y1, w1), "y2": rel(y2, w2), "x1": rel(got[0], h1), "x2": rel(got[1], h2),
              "dx1": rel(got[2], want[0]), "dx2": rel(got[3], want[1])}
    errors.update({n: rel(got[4][n].reshape(w.shape), w) for n, w in zip(leaves, want[2:])})
    print(errors, flush=True)
    for n, e in errors.items():
        assert e <= (1e-4 if dtype == "fp32" else 2.0 ** -7 if n[0] in "xy" else 0.125), (n, e)


def test_example_checks_itself():
    """fp32: a central difference over a hundredth of the streams' size is off by its third-order term."""
    import reversible_attention as R

    rebuilt, derivative = R.check(R.Block(2, 70, 96, 4, 2, "fp32"))
    assert rebuilt <= 1e-5 and derivative <= 0.02
