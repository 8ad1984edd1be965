"""Owners of the workspaces of the token operators around the C ABI: attention,
the coupling of a residual function to its stream, dropout, the norms and rotation
of heads, the loss over a vocabulary and AdamW.

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
        self._need_stream(stream)
        handle = L._stream(stream)
        if handle not in self.streams and not isinstance(stream, int):
            import torch
            for t in self._owned():
                t.record_stream(torch.cuda.current_stream() if stream is None else stream)
            self.streams.add(handle)
        return handle

    def _need_stream(self, stream) -> None:
        """A stream that is given is one of the owner's device.  (Its handle does not tell: that of
        the default stream is the same for every device.)"""
        index = self.workspace.get_device()
        if getattr(stream, "device_index", index) != index:
            raise ValueError(f"need a stream of the owner's device {self.workspace.device}, "
                             f"got {stream}")

    def _owned(self):
        """The owner's memory that its calls use."""
        return (self.workspace,)

    def _need_here(self, *tensors) -> None:
        """The tensors, and the current device, whose stream runs the call, are the owner's."""
        index = self.workspace.get_device()
        for t in tensors:
            if t is not None and t.get_device() != index:
                raise ValueError(f"need all tensors on the owner's device {self.workspace.device}, "
                                 f"got one on {t.device}")
        if L._device() != index:
            raise ValueError(f"the current device is {L._device()}, the owner's "
                             f"{self.workspace.device}")


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
        self._need_stream(stream)
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


_NONE = (None, None)


class HeadNorm(_Owner):
    """Norms of query and key heads with the rotation by their tokens' positions, over
    [batch, length, heads, head_dim] and [batch, length, kv_heads, head_dim] tensors (any strides
    of the first three dimensions; channels contiguous).

    freq: radians a position of each pair of channels, by default 10000^(-i / (head_dim / 2)) for
    i < head_dim / 2, () for no rotation; axis: the axis of positions of each pair (default 0).
    layout: the pairs are channels (i, i + pairs), 'halves', or (2 i, 2 i + 1), 'neighbours'.
    kv_heads = 0: queries only."""

    def __init__(self, batch: int, length: int, heads: int, kv_heads: int, head_dim: int,
                 dtype: str = "bf16", norm: str | None = "rms", eps: float = 1e-6,
                 layout: str = "halves", freq=None, axis=None, device: str = "cuda"):
        import torch
        code, self.tdtype = _types(dtype)
        if norm not in ("rms", "layer", None):
            raise ValueError(f"norm must be 'rms', 'layer' or None, got {norm!r}")
        if layout not in ("halves", "neighbours"):
            raise ValueError(f"layout must be 'halves' or 'neighbours', got {layout!r}")
        if freq is None:
            freq = [10000.0 ** (-2.0 * i / head_dim) for i in range(head_dim // 2)]
        freq = [float(f) for f in freq]
        axis = [0] * len(freq) if axis is None else [int(a) for a in axis]
        if len(freq) > L.PETRA_HEAD_PAIRS or len(axis) != len(freq):
            raise ValueError(f"need an axis for each of at most {L.PETRA_HEAD_PAIRS} frequencies, "
                             f"got {len(axis)} and {len(freq)}")
        self.norm = norm
        self.axes = max(axis, default=0) + 1
        self.shapes = ((batch, length, heads, head_dim), (batch, length, kv_heads, head_dim))
        self.param_shape, self.positions_shape = (head_dim,), (self.axes, batch, length)
        self.itype, self.ftype = torch.int32, torch.float32
        self.desc = L.HeadsDesc(batch, length, heads, kv_heads, head_dim, code,
                                L.PETRA_NORM_LAYER if norm == "layer" else L.PETRA_NORM_RMS, eps,
                                L.PETRA_PAIRS_HALVES if layout == "halves" else
                                L.PETRA_PAIRS_NEIGHBOURS, len(freq), self.axes)
        for i, (f, a) in enumerate(zip(freq, axis)):
            self.desc.freq[i], self.desc.axis[i] = f, a
        self.form = None
        self._own(L.petra_heads_query(self.desc), device)

    @staticmethod
    def _form(tensors):
        return [(t.shape, t.stride(), t.dtype, t.get_device()) if t is not None else None
                for t in tensors]

    def _lay(self, back, acts, params, positions) -> None:
        """Checks the tensors and puts their strides into the description.  acts: q and k (back:
        their gradients too, at the end) and what is laid out like the results; params: the
        norms' and (back) their gradients'.  What was checked last (types, shapes and strides) is
        not checked again."""
        form = (back, L._device(), self._form(acts + params + (positions,)))
        if self.form == form:
            return
        self.form = None
        names = ("dq", "dk", "dyq", "dyk", "q", "k") if back else ("q", "k", "yq", "yk")
        fields = ("q_stride", "k_stride", "yq_stride", "yk_stride")
        for i, (t, name) in enumerate(zip(acts, names)):
            if t is None and (self.shapes[i % 2][2] == 0 or i >= 4):
                continue   # (the library needs q and k where there is a norm)
            if t is None:
                raise ValueError(f"{name}: need a tensor")
            _need(t, name, self.tdtype, self.shapes[i % 2], dense=False)
            if i < 4:
                setattr(self.desc, fields[i], self._strides(t, name))
            elif any(x != y for x, y, n in zip(t.stride(), acts[i - 4].stride(), t.shape) if n > 1):
                raise ValueError(f"{name}: need the strides of its gradient "
                                 f"{acts[i - 4].stride()}, got {t.stride()}")
        for t, name in zip(params, ("q_norm", "q_norm", "k_norm", "k_norm", "dq_norm", "dq_norm",
                                    "dk_norm", "dk_norm")):
            if t is not None:
                if self.norm is None:
                    raise ValueError(f"{name}: this owner has no norm")
                _need(t, name, self.ftype, self.param_shape)
        if positions is not None:
            _need(positions, "positions", self.itype, self.positions_shape)
        self._need_here(*acts, *params, positions)
        self.form = form

    @staticmethod
    def _strides(t, name: str):
        st = t.stride()
        if st[3] != 1 and t.shape[3] > 1:
            raise ValueError(f"{name}: channels must be contiguous, got strides {st}")
        st = tuple(s if n > 1 else 0 for s, n in zip(st[:3], t.shape[:3]))
        # (three zeros are a contiguous tensor's in the description)
        if st == (0, 0, 0) and math.prod(t.shape[:3]) > 1:
            raise ValueError(f"{name}: all positions share one vector")
        return (L.ctypes.c_int64 * 3)(*st)

    def forward(self, q, k, yq, yk, q_norm=None, k_norm=None, positions=None, stream=None) -> None:
        """Writes yq and yk.  q_norm and k_norm: (gamma, beta or None), fp32; positions: int32
        [axes, batch, length] (None: a token's index)."""
        self._need_stream(stream)
        self._need_norms(q_norm, k_norm)
        self._lay(False, (q, k, yq, yk), (q_norm or _NONE) + (k_norm or _NONE), positions)
        L.petra_heads_forward(self.desc, q, k, q_norm, k_norm, positions, yq, yk, stream)

    def backward(self, q, k, dyq, dyk, dq, dk, q_norm=None, k_norm=None, dq_norm=None,
                 dk_norm=None, positions=None, stream=None) -> None:
        """Writes dq, dk (strides of q and k) and the norms' parameters' gradients.  Without a
        norm q and k may be None."""
        self._need_norms(q_norm, k_norm)
        self._lay(True, (dq, dk, dyq, dyk, q, k), (q_norm or _NONE) + (k_norm or _NONE)
                  + (dq_norm or _NONE) + (dk_norm or _NONE), positions)
        L.petra_heads_backward(self.desc, q, k, q_norm, k_norm, positions, dyq, dyk, dq, dk,
                               dq_norm, dk_norm, self.workspace, self.ws_bytes, self._on(stream))

    def _need_norms(self, q_norm, k_norm) -> None:
        if self.norm is not None and (q_norm is None or (k_norm is None and self.shapes[1][2])):
            raise ValueError(f"q_norm, k_norm: a {self.norm} norm needs its parameters")


class VocabLoss(_Owner):
    """Softmax cross entropy of scale x w^T over a vocabulary, without its logits: x [rows, width],
    w [vocab, width], targets int32 [rows] (any that is no column takes its row out).

    piece_rows: rows whose scores are held at a time, for less memory (0: within 1 GiB).
    gradients=False: a workspace for the loss alone."""

    def __init__(self, rows: int, width: int, vocab: int, dtype: str = "bf16", scale: float = 1.0,
                 piece_rows: int = 0, gradients: bool = True, device: str = "cuda"):
        import torch
        code, self.tdtype = _types(dtype)
        self.x_shape, self.w_shape, self.row_shape = (rows, width), (vocab, width), (rows,)
        self.itype, self.ftype = torch.int32, torch.float32
        self.desc = L.VocabDesc(rows, piece_rows, width, vocab, code, scale)
        self.loss_bytes, self.gradient_bytes = L.petra_vocab_query(self.desc)
        self._own(max(self.loss_bytes, self.gradient_bytes) if gradients else self.loss_bytes,
                  device)

    def _check(self, x, w, targets, loss, lse) -> None:
        _need(x, "x", self.tdtype, self.x_shape)
        _need(w, "w", self.tdtype, self.w_shape)
        _need(targets, "targets", self.itype, self.row_shape)
        _need(loss, "loss", self.ftype, self.row_shape)
        _need(lse, "lse", self.ftype, self.row_shape)
        self._need_here(x, w, targets, loss, lse)

    def forward(self, x, w, targets, loss, lse, stream=None) -> None:
        """Writes loss and lse, fp32 [rows]."""
        self._check(x, w, targets, loss, lse)
        L.petra_vocab_loss(self.desc, x, w, targets, loss, lse, self.workspace, self.ws_bytes,
                           self._on(stream))

    def gradient(self, x, w, targets, loss, lse, dx, dw, weight=None, stream=None) -> None:
        """Writes loss, lse and the gradients of sum(weight * loss); weight: fp32 [rows] (None:
        1 / the rows that take part)."""
        self._check(x, w, targets, loss, lse)
        _need(dx, "dx", self.tdtype, self.x_shape)
        _need(dw, "dw", self.tdtype, self.w_shape)
        if weight is not None:
            _need(weight, "weight", self.ftype, self.row_shape)
        self._need_here(dx, dw, weight)
        L.petra_vocab_gradient(self.desc, x, w, targets, weight, loss, lse, dx, dw,
                               self.workspace, self.ws_bytes, self._on(stream))


class AdamW(_Owner):
    """An AdamW step over many tensors: params (fp32) and their grads (fp32 or bf16, all of one
    type), which the owner keeps.

    A step works on the memory that the tensors had when the owner was made, and the owner keeps
    that.  It does not follow a tensor that is given other memory (`p.data = ...`): each step
    looks at 8 of the tensors in turn and refuses one that has moved, now and from then on.  m,
    v and their scales are copied into, not replaced.  Storage that is resized away under the
    owner is not seen in time.

    states: 'fp32', or 'fp8' for 8 bits an element.  m and v (fp8: r = sqrt(v), as
    float8_e4m3fn, with m_scale and v_scale for each 64 elements) are one tensor each for all, each
    parameter's from a multiple of 64 on: m[starts[i]:starts[i] + n].  lr (fp32) and steps
    (int64) are device tensors of one element, for the caller to set.  weight_decay: one for all, or
    one for each.  copies: bf16 tensors that follow their parameters (None: none).  zero_grads: each
    step sets the gradients to 0."""

    def __init__(self, params, grads, states: str = "fp32", lr: float = 1e-3,
                 betas=(0.9, 0.999), eps: float = 1e-8, weight_decay=0.01, copies=None,
                 zero_grads: bool = False):
        import torch
        if states not in ("fp32", "fp8"):
            raise ValueError(f"states must be 'fp32' or 'fp8', got {states!r}")
        self.params, self.grads = list(params), list(grads)
        self.copies = [None] * len(self.params) if copies is None else list(copies)
        try:
            decay = [float(d) for d in weight_decay]
        except TypeError:
            decay = [float(weight_decay)] * len(self.params)
        if not self.params:
            raise ValueError("params: need at least one tensor")
        if not len(self.params) == len(self.grads) == len(self.copies) == len(decay):
            raise ValueError(f"need as many of each: {len(self.params)} params, {len(self.grads)} "
                             f"grads, {len(self.copies)} copies, {len(decay)} weight decays")
        device, gtype = self.params[0].device, self.grads[0].dtype
        if gtype not in (torch.float32, torch.bfloat16):
            raise ValueError(f"grads: need float32 or bfloat16, got {gtype}")
        for i, (p, g, c) in enumerate(zip(self.params, self.grads, self.copies)):
            _need(p, f"params[{i}]", torch.float32, p.shape)
            _need(g, f"grads[{i}]", gtype, p.shape)
            if c is not None:
                _need(c, f"copies[{i}]", torch.bfloat16, p.shape)
            if any(t is not None and t.device != device for t in (p, g, c)):
                raise ValueError(f"params[{i}]: need all tensors on {device}")
        fp8, at = states == "fp8", 0
        self.starts = []
        for p in self.params:
            self.starts.append(at)
            at += -(-p.numel() // 64) * 64
        # (zeros of a type with no fill of its own)
        self.m, self.v = (torch.zeros(at, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn)
                          if fp8 else torch.zeros(at, device=device) for _ in range(2))
        self.m_scale, self.v_scale = ((torch.zeros(at // 64, device=device) for _ in range(2))
                                      if fp8 else (None, None))
        self.lr = torch.full((1,), lr, device=device)
        self.steps = torch.zeros(1, dtype=torch.int64, device=device)
        self.fp8, self.ftype, self.itype = fp8, torch.float32, torch.int64
        self.desc = L.AdamwDesc(betas[0], betas[1], eps,
                                L.PETRA_BF16 if gtype is torch.bfloat16 else L.PETRA_FP32,
                                L.PETRA_E4M3 if fp8 else L.PETRA_FP32, int(zero_grads))
        self.count = len(self.params)
        tensors = (L.AdamwTensor * self.count)()
        size = 1 if fp8 else 4
        # scales of a tensor begin at any multiple of 4 bytes in theirs: blocks of 64
        for t, p, g, c, d, start in zip(tensors, self.params, self.grads, self.copies, decay,
                                        self.starts):
            t.theta, t.grad, t.n, t.weight_decay = p.data_ptr(), g.data_ptr(), p.numel(), d
            t.m, t.v = self.m.data_ptr() + size * start, self.v.data_ptr() + size * start
            if fp8:
                t.m_scale = self.m_scale.data_ptr() + start // 64 * 4
                t.v_scale = self.v_scale.data_ptr() + start // 64 * 4
            t.copy = None if c is None else c.data_ptr()
        self.table_bytes, self.chunks, ws_bytes = L.petra_adamw_query(self.desc, tensors,
                                                                      self.count)
        table = torch.empty(max(self.table_bytes, 1), dtype=torch.uint8)
        L.petra_adamw_layout(self.desc, tensors, self.count, table, self.table_bytes)
        self.table = table.to(device)
        self._keep()
        self._own(ws_bytes, device)

    def _keep(self) -> None:
        """What the table points to, whatever becomes of the caller's tensors: (name, the tensor,
        one of the same memory, its address) of each, and the states."""
        self._laid = [(f"{name}[{i}]", t, t.detach(), t.data_ptr())
                      for name, of in (("params", self.params), ("grads", self.grads),
                                       ("copies", self.copies))
                      for i, t in enumerate(of) if t is not None]
        self._states = self.m, self.v, self.m_scale, self.v_scale
        self._state_memory = [t.detach() for t in self._states if t is not None]
        self._turn, self._set = 0, (self.lr, self.steps)

    def _need_laid(self) -> None:
        """The table's memory is still the tensors': of the states, and of the next of the others (an
        address takes 0.1 us to ask for, all of 300 tensors would take longer than their step)."""
        m, v, m_scale, v_scale = self._states
        if not (self.m is m and self.v is v and self.m_scale is m_scale and self.v_scale is v_scale):
            name = next(n for n, t in zip(("m", "v", "m_scale", "v_scale"), self._states)
                        if getattr(self, n) is not t)
            raise ValueError(f"{name}: has been replaced, copy into it instead")
        turn = self._turn
        for name, t, _, at in self._laid[turn:turn + 8]:
            if t.data_ptr() != at:
                raise ValueError(f"{name}: its memory is not what was laid out, make a new owner")
        self._turn = turn + 8 if turn + 8 < len(self._laid) else 0

    def _owned(self):
        return [self.workspace, self.table, self.lr, self.steps, *self._state_memory,
                *(laid[2] for laid in self._laid)]

    def step(self, rng=None, grad_scale=None, stream=None) -> None:
        """Updates params, copies and states; rng (device int64 [seed, offset], for fp8): another
        offset each step; grad_scale: a device fp32 factor of all gradients."""
        if rng is not None:
            _need_rng(rng)
        if grad_scale is not None:
            _need(grad_scale, "grad_scale", self.ftype, (1,))
        _need(self.lr, "lr", self.ftype, (1,))
        _need(self.steps, "steps", self.itype, (1,))
        self._need_here(rng, grad_scale, self.lr, self.steps)
        self._need_laid()
        if self.lr is not self._set[0] or self.steps is not self._set[1]:
            self.streams.clear()   # (tells the allocator of them)
            self._set = (self.lr, self.steps)
        L.petra_adamw_step(self.desc, self.table, self.table_bytes, self.count, self.chunks,
                           self.steps, self.lr, grad_scale, rng, self.workspace, self.ws_bytes,
                           self._on(stream))
