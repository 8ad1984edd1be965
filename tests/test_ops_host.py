"""Refusals of the token operators' entry points: found on the host, before any work."""
import ctypes

import pytest

from paper_2406_02052_amd import _lib as L

A, B, C, D, E, F, G, H = (0x10000000 * (i + 1) for i in range(8))   # addresses that nothing reads


def _attn(**over):
    d = dict(batch=2, q_len=5, kv_len=7, heads=4, kv_heads=2, head_dim=64, dtype=L.PETRA_BF16, causal=0,
             scale=0.125, dropout=0.0)
    st = {k: over.pop(k) for k in list(over) if k.endswith("_stride")}
    d.update(over)
    desc = L.AttnDesc(*d.values())
    for k, v in st.items():
        setattr(desc, k, (ctypes.c_int64 * 3)(*v))
    return desc


def _refused(status, call, *args):
    with pytest.raises(L.PetraError) as e:
        call(*args)
    assert e.value.name == status, str(e.value)
    assert str(e.value) and L.petra_last_error()


@pytest.mark.parametrize("over,status", [
    (dict(heads=3), "PETRA_ERR_SHAPE"), (dict(kv_heads=0), "PETRA_ERR_SHAPE"), (dict(head_dim=12), "PETRA_ERR_SHAPE"),
    (dict(head_dim=136), "PETRA_ERR_SHAPE"), (dict(head_dim=0), "PETRA_ERR_SHAPE"), (dict(batch=-1), "PETRA_ERR_SHAPE"),
    (dict(batch=40000), "PETRA_ERR_SHAPE"), (dict(kv_len=2 ** 30 + 1), "PETRA_ERR_SHAPE"),
    (dict(q_len=2 ** 30), "PETRA_ERR_SHAPE"), (dict(dtype=2), "PETRA_ERR_DTYPE"),
    (dict(scale=0.0), "PETRA_ERR_INVALID_ARG"), (dict(scale=float("nan")), "PETRA_ERR_INVALID_ARG"),
    (dict(scale=-1.0), "PETRA_ERR_INVALID_ARG"), (dict(dropout=1.0), "PETRA_ERR_INVALID_ARG"),
    (dict(dropout=-0.1), "PETRA_ERR_INVALID_ARG"), (dict(dropout=float("nan")), "PETRA_ERR_INVALID_ARG"),
    (dict(dropout=1 - 2.0 ** -18), "PETRA_ERR_INVALID_ARG"),
    (dict(q_stride=(1280, 256, 60)), "PETRA_ERR_ALIGN"), (dict(q_stride=(1280, -256, 64)), "PETRA_ERR_SHAPE"),
    (dict(k_stride=(2 ** 25, 2 ** 22, 64)), "PETRA_ERR_SHAPE"), (dict(o_stride=(1280, 0, 64)), "PETRA_ERR_SHAPE"),
    (dict(o_stride=(1280, 128, 64)), "PETRA_ERR_SHAPE")])
def test_attention_descriptions(over, status):
    _refused(status, L.petra_attn_query, _attn(**over))


def test_attention_broadcast_inputs_are_read_but_not_written():
    d = _attn(k_stride=(0, 128, 64))
    L.petra_attn_query(d)
    _refused("PETRA_ERR_SHAPE", L.petra_attn_backward, d, A, B, C, D, E, F, 0, 0, 0, G, H, A + 0x1000000, 0x90000000,
             1 << 20, 0)


def test_attention_pointers():
    d = _attn()
    fwd, bwd = L.petra_attn_query(d)

    def run(q=A, k=B, v=C, o=D, lse=E, ws=F, n=1 << 30, lens=0, rng=0, desc=d):
        L.petra_attn_forward(desc, q, k, v, lens, 0, rng, o, lse, ws, n, 0)

    for name in ("q", "k", "v", "o", "lse"):
        _refused("PETRA_ERR_INVALID_ARG", lambda name=name: run(**{name: 0}))
        _refused("PETRA_ERR_ALIGN", lambda name=name: run(**{name: 0x7000008}))
    _refused("PETRA_ERR_ALIGN", lambda: run(lens=0x7000002))
    _refused("PETRA_ERR_ALIAS", lambda: run(o=A))
    _refused("PETRA_ERR_ALIAS", lambda: run(o=B + 16))
    _refused("PETRA_ERR_ALIAS", lambda: run(lse=D + 64))
    _refused("PETRA_ERR_INVALID_ARG", lambda: run(desc=_attn(dropout=0.5)))
    _refused("PETRA_ERR_ALIGN", lambda: run(desc=_attn(dropout=0.5), rng=0x7000004))
    long = _attn(batch=1, q_len=1, kv_len=1 << 16)
    assert L.petra_attn_query(long)[0] > 0
    _refused("PETRA_ERR_WORKSPACE", lambda: run(desc=long, ws=0, n=0, k=B, v=0x30000000000, o=0x40000000000,
                                                lse=0x50000000000))
    with pytest.raises(L.PetraError) as e:
        L.petra_attn_backward(d, A, B, C, D, E, F, 0, 0, 0, G, H, H, 0x90000000, 1 << 20, 0)
    assert e.value.name == "PETRA_ERR_ALIAS"
    _refused("PETRA_ERR_WORKSPACE", L.petra_attn_backward, d, A, B, C, D, E, F, 0, 0, 0, G, H, 0x90000000, 0xa0000000,
             bwd - 1, 0)


def _coupling(**over):
    d = dict(rows=12, rows_per_gate=0, width=64, dtype=L.PETRA_BF16, norm=L.PETRA_NORM_RMS, eps=1e-5,
             residual_scale=1.0, dropout=0.0)
    d.update(over)
    return L.CouplingDesc(*d.values())


@pytest.mark.parametrize("over,status", [
    (dict(rows=-1), "PETRA_ERR_SHAPE"), (dict(rows=2 ** 31), "PETRA_ERR_SHAPE"), (dict(rows_per_gate=5), "PETRA_ERR_SHAPE"),
    (dict(rows_per_gate=-1), "PETRA_ERR_SHAPE"), (dict(width=60), "PETRA_ERR_SHAPE"), (dict(width=8200), "PETRA_ERR_SHAPE"),
    (dict(width=0), "PETRA_ERR_SHAPE"), (dict(dtype=5), "PETRA_ERR_DTYPE"), (dict(norm=2), "PETRA_ERR_INVALID_ARG"),
    (dict(eps=0.0), "PETRA_ERR_INVALID_ARG"), (dict(eps=float("nan")), "PETRA_ERR_INVALID_ARG"),
    (dict(residual_scale=0.0), "PETRA_ERR_INVALID_ARG"), (dict(dropout=1.5), "PETRA_ERR_INVALID_ARG")])
def test_coupling_descriptions(over, status):
    _refused(status, L.petra_coupling_query, _coupling(**over))


def test_coupling_pointers():
    d, norm = _coupling(), (G, None)

    def fwd(x=A, f=B, gate=C, post=norm, pre=norm, rng=0, y=D, u=E, desc=d):
        L.petra_coupling_forward(desc, x, f, gate, post, pre, rng, y, u, 0)

    for name in ("x", "gate", "y"):
        _refused("PETRA_ERR_INVALID_ARG", lambda name=name: fwd(**{name: 0}))
        _refused("PETRA_ERR_ALIGN", lambda name=name: fwd(**{name: 0x7000008}))
    _refused("PETRA_ERR_INVALID_ARG", lambda: fwd(post=None))
    _refused("PETRA_ERR_INVALID_ARG", lambda: fwd(pre=None))
    _refused("PETRA_ERR_INVALID_ARG", lambda: fwd(f=0))
    _refused("PETRA_ERR_INVALID_ARG", lambda: fwd(f=0, y=0, gate=0, post=None, u=0, pre=None))
    _refused("PETRA_ERR_ALIAS", lambda: fwd(y=B))
    _refused("PETRA_ERR_ALIAS", lambda: fwd(y=A + 16))
    _refused("PETRA_ERR_ALIAS", lambda: fwd(u=A))
    _refused("PETRA_ERR_ALIAS", lambda: fwd(u=D))
    _refused("PETRA_ERR_INVALID_ARG", lambda: fwd(desc=_coupling(dropout=0.5)))

    need = L.petra_coupling_query(d)

    def bwd(y=A, f=B, dy=C, du=D, gate=E, post=norm, pre=norm, rng=0, x=F, dx=H, df=0x90000000, dgate=0xa0000000,
            dpost=(0xb0000000, None), dpre=(0xc0000000, None), ws=0xd0000000, n=need, desc=d):
        L.petra_coupling_backward(desc, y, f, dy, du, gate, post, pre, rng, x, dx, df, dgate, dpost, dpre, ws, n, 0)

    for name in ("y", "f", "dy", "du", "gate", "dx", "df", "dgate"):
        _refused("PETRA_ERR_INVALID_ARG", lambda name=name: bwd(**{name: 0}))
    for name, val in (("post", None), ("pre", None), ("dpost", None), ("dpre", None), ("dpost", (G + 64, G + 128))):
        _refused("PETRA_ERR_INVALID_ARG", lambda name=name, val=val: bwd(**{name: val}))
    _refused("PETRA_ERR_ALIAS", lambda: bwd(dx=A))
    _refused("PETRA_ERR_ALIAS", lambda: bwd(df=C))
    _refused("PETRA_ERR_ALIAS", lambda: bwd(x=H))
    _refused("PETRA_ERR_ALIAS", lambda: bwd(dgate=E))
    _refused("PETRA_ERR_ALIAS", lambda: bwd(dpre=(0xb0000000, None)))
    _refused("PETRA_ERR_WORKSPACE", lambda: bwd(n=need - 1))


def test_dropout_refusals():
    def run(n=100, dtype=1, p=0.5, alpha=1.0, x=A, r=0, rng=B, y=C):
        L.petra_dropout(n, dtype, p, alpha, x, r, rng, y, 0)

    _refused("PETRA_ERR_SHAPE", lambda: run(n=-1))
    _refused("PETRA_ERR_DTYPE", lambda: run(dtype=3))
    _refused("PETRA_ERR_INVALID_ARG", lambda: run(p=1.0))
    _refused("PETRA_ERR_INVALID_ARG", lambda: run(alpha=float("inf")))
    _refused("PETRA_ERR_INVALID_ARG", lambda: run(rng=0))
    _refused("PETRA_ERR_INVALID_ARG", lambda: run(x=0))
    _refused("PETRA_ERR_ALIGN", lambda: run(y=0x7000002))
    _refused("PETRA_ERR_ALIAS", lambda: run(y=A + 16))
    _refused("PETRA_ERR_ALIAS", lambda: run(r=C + 16))


def test_nothing_to_do_is_no_error():
    L.petra_dropout(0, 1, 0.5, 1.0, 0, 0, A, 0, 0)
    L.petra_attn_forward(_attn(batch=0), 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0)
    L.petra_attn_forward(_attn(q_len=0), 0, B, C, 0, 0, 0, 0, 0, 0, 0, 0)
    L.petra_coupling_forward(_coupling(rows=0), 0, 0, 0, None, None, 0, 0, 0, 0)


def test_null_description():
    lib = L.load()
    n = ctypes.c_size_t()
    assert lib.petra_attn_query(None, ctypes.byref(n), ctypes.byref(n)) == 1
    assert lib.petra_coupling_query(None, ctypes.byref(n)) == 1
