"""Owners of the workspaces of the token operators around the C ABI: attention,
the coupling of a residual function to its stream, and dropout.

Marshalling only, as in stage.py.  Tensors are the caller's; their types, shapes
and strides are checked here, everything else by the library.  A workspace holds
nothing between calls, but calls of one owner that overlap in time (on other
streams) need an owner each.  An owner may be dropped while its calls still run:
its workspace's memory is not given out again before the streams they were put on
have passed them.  A stream that is given as a bare handle can't be waited for so;
there the owner has to stay until the work is done.
"""
from __future__ import annotations

import math

from . import _lib as L


def _types(dtype: str):
    import torch
    if dtype not in ("bf16", "fp32"):
        raise ValueError(f"dtype must be 'bf16' or 'fp32', got {dtype!r}")
    return (L.PETRA_BF16, torch.bfloat16) if dtype == "bf16" else (L.PETRA_FP32, torch.float32)


def _need(t, name: str, dtype, shape, dense: bool = True) -> None:
    if t.dtype is not dtype or t.shape != shape or not t.is_cuda:
        raise ValueError(f"{name}: need a device tensor {shape} of {dtype}, got {tuple(t.shape)} "
                         f"of {t.dtype} on {t.device}")
    if dense and not t.is_contiguous():
        raise ValueError(f"{name}: need a contiguous tensor, got strides {t.stride()}")


def _need_rng(rng) -> None:
    import torch
    if (rng.dtype is not torch.int64 or rng.numel() != 2 or not rng.is_contiguous()
            or not rng.is_cuda):
        raise ValueError("rng: need a device int64 tensor [seed, offset]")


class _Owner:
    """A workspace, and the streams that have used it."""

    def _own(self, ws_bytes: int, device) -> None:
        import torch
        self.ws_bytes = ws_bytes
        self.workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=device)
        # the allocator knows the stream that memory is taken on, and no other
        self.streams = set()
        if self.workspace.is_cuda:
            self.streams.add(torch.cuda.current_stream(self.workspace.device).cuda_stream)

    def _on(self, stream) -> int:
        """The stream's handle; tells the allocator of a stream that is new to the workspace."""
        handle = L._stream(stream)
        if handle not in self.streams and not isinstance(stream, int):
            import torch
            self.workspace.record_stream(torch.cuda.current_stream() if stream is None else stream)
            self.streams.add(handle)
        return handle


class Attention(_Owner):
    """Attention of [batch, q_len, heads, head_dim] over [batch, kv_len, kv_heads, head_dim]
    tensors (any strides of the first three dimensions; channels contiguous)."""

    def __init__(self, batch: int, q_len: int, kv_len: int, heads: int, kv_heads: int,
                 head_dim: int, dtype: str = "bf16", causal: bool = False,
                 scale: float | None = None, dropout: float = 0.0, device: str = "cuda"):
        import torch
        code, self.tdtype = _types(dtype)
        self.q_shape = (batch, q_len, heads, head_dim)
        self.kv_shape = (batch, kv_len, kv_heads, head_dim)
        self.lse_shape = (batch, heads, q_len)
        self.desc = L.AttnDesc(batch, q_len, kv_len, heads, kv_heads, head_dim, code, int(causal),
                               1.0 / math.sqrt(head_dim) if scale is None else scale, dropout)
        self.form = None
        self.itype, self.ftype = torch.int32, torch.float32
        self.fwd_bytes, self.bwd_bytes = L.petra_attn_query(self.desc)
        self._own(max(self.fwd_bytes, self.bwd_bytes), device)

    def _lay(self, q, k, v, o, lse, q_lens, kv_lens, rng) -> None:
        """Checks the tensors and puts their strides into the description.  What was checked
        last (types, shapes and strides) is not checked again."""
        form = (q.shape, k.shape, v.shape, o.shape, lse.shape, q.stride(), k.stride(), v.stride(),
                o.stride(), lse.stride(), q.dtype, k.dtype, v.dtype, o.dtype, lse.dtype, q.is_cuda,
                k.is_cuda, v.is_cuda, o.is_cuda, lse.is_cuda)
        if form != self.form:
            self._check(q, k, v, o, lse)
            self.form = form
        for t, name in ((q_lens, "q_lens"), (kv_lens, "kv_lens")):
            if t is not None:
                _need(t, name, self.itype, self.q_shape[:1])
        if rng is not None:
            _need_rng(rng)

    def _check(self, q, k, v, o, lse) -> None:
        self.form = None
        for t, name, shape in ((q, "q", self.q_shape), (k, "k", self.kv_shape),
                               (v, "v", self.kv_shape), (o, "o", self.q_shape)):
            _need(t, name, self.tdtype, shape, dense=False)
            st = t.stride()
            if st[3] != 1 and t.shape[3] > 1:
                raise ValueError(f"{name}: channels must be contiguous, got strides {st}")
            # the stride of a dimension of one means nothing
            st = tuple(s if n > 1 else 0 for s, n in zip(st[:3], t.shape[:3]))
            # the description takes three zeros for a contiguous tensor: those of one
            # vector that all positions share cannot be told apart from that
            if st == (0, 0, 0) and math.prod(t.shape[:3]) > 1:
                raise ValueError(f"{name}: all positions share one vector")
            setattr(self.desc, name + "_stride", (L.ctypes.c_int64 * 3)(*st))
        _need(lse, "lse", self.ftype, self.lse_shape)

    def forward(self, q, k, v, o, lse, q_lens=None, kv_lens=None, rng=None, stream=None) -> None:
        """Writes o [batch, q_len, heads, head_dim] and lse (fp32 [batch, heads, q_len])."""
        self._lay(q, k, v, o, lse, q_lens, kv_lens, rng)
        L.petra_attn_forward(self.desc, q, k, v, q_lens, kv_lens, rng, o, lse, self.workspace,
                             self.ws_bytes, self._on(stream))

    def backward(self, q, k, v, o, lse, d_o, dq, dk, dv, q_lens=None, kv_lens=None, rng=None,
                 stream=None) -> None:
        """Writes dq, dk, dv from the forward's o and lse and the gradient d_o of o."""
        self._lay(q, k, v, o, lse, q_lens, kv_lens, rng)
        for t, name, like in ((d_o, "d_o", o), (dq, "dq", q), (dk, "dk", k), (dv, "dv", v)):
            _need(t, name, self.tdtype, like.shape, dense=False)
            st, want = t.stride(), like.stride()
            if st != want and any(x != y for x, y, n in zip(st, want, t.shape) if n > 1):
                raise ValueError(f"{name}: need strides {want}, got {st}")
        L.petra_attn_backward(self.desc, q, k, v, o, lse, d_o, q_lens, kv_lens, rng, dq, dk, dv,
                              self.workspace, self.ws_bytes, self._on(stream))


class Coupling(_Owner):
    """y = residual_scale x + gate m n(f; post), u = n(y; pre) over [rows, width] tensors, and its
    backward, which also rebuilds x.  post and pre are (gamma, beta or None), fp32."""

    def __init__(self, rows: int, width: int, dtype: str = "bf16", norm: str = "rms",
                 eps: float = 1e-5, residual_scale: float = 1.0, dropout: float = 0.0,
                 rows_per_gate: int = 0, device: str = "cuda"):
        import torch
        if norm not in ("rms", "layer"):
            raise ValueError(f"norm must be 'rms' or 'layer', got {norm!r}")
        code, self.tdtype = _types(dtype)
        self.shape, self.ftype = (rows, width), torch.float32
        self.desc = L.CouplingDesc(rows, rows_per_gate, width, code,
                                   L.PETRA_NORM_RMS if norm == "rms" else L.PETRA_NORM_LAYER,
                                   eps, residual_scale, dropout)
        self.gate_shape = (rows // rows_per_gate if rows_per_gate else 1, width)
        self._own(L.petra_coupling_query(self.desc), device)

    def _check(self, acts, gates, norms, rng) -> None:
        """acts: (name, tensor) of activations; gates and norms likewise; None is left out."""
        for name, t in acts:
            if t is not None:
                _need(t, name, self.tdtype, self.shape)
        for name, t in gates:
            if t is not None:
                _need(t, name, self.ftype, self.gate_shape)
        for name, p in norms:
            if p is not None:
                _need(p[0], name, self.ftype, self.shape[1:])
                if p[1] is not None:
                    _need(p[1], name, self.ftype, self.shape[1:])
        if rng is not None:
            _need_rng(rng)

    def forward(self, x, f=None, gate=None, post=None, y=None, pre=None, u=None, rng=None,
                stream=None) -> None:
        """Writes y and, with pre, u.  Without f only u = n(x; pre)."""
        self._check((("x", x), ("f", f), ("y", y), ("u", u)), (("gate", gate),),
                    (("post", post), ("pre", pre)), rng)
        L.petra_coupling_forward(self.desc, x, f, gate, post, pre, rng, y, u, stream)

    def backward(self, y, f, dy, gate, post, x, dx, df, dgate, dpost, du=None, pre=None,
                 dpre=None, rng=None, stream=None) -> None:
        """Writes x (rebuilt; may be None), dx, df and the parameters' gradients.  With f, gate,
        post and what belongs to them None: only dx and dpre."""
        self._check((("y", y), ("f", f), ("dy", dy), ("du", du), ("x", x), ("dx", dx),
                     ("df", df)), (("gate", gate), ("dgate", dgate)),
                    (("post", post), ("pre", pre), ("dpost", dpost), ("dpre", dpre)), rng)
        L.petra_coupling_backward(self.desc, y, f, dy, du, gate, post, pre, rng, x, dx, df, dgate,
                                  dpost, dpre, self.workspace, self.ws_bytes, self._on(stream))


def dropout(x, y, p: float, rng, residual=None, alpha: float = 1.0, stream=None) -> None:
    """y = residual + alpha m x, m of rng = [seed, offset] (device int64)."""
    import torch
    if x.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError(f"x: need bfloat16 or float32, got {x.dtype}")
    for t, name in ((x, "x"), (y, "y"), (residual, "residual")):
        if t is not None:
            _need(t, name, x.dtype, x.shape)
    if rng is not None:
        _need_rng(rng)
    L.petra_dropout(x.numel(), L.PETRA_BF16 if x.dtype is torch.bfloat16 else L.PETRA_FP32, p,
                    alpha, x, residual, rng, y, stream)
