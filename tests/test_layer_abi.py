"""Refusals of the entry points around the attention, on the CPU: fake device
addresses that are never dereferenced, every call with an argument that the
checks must reject (skipped where a GPU is visible)."""
from __future__ import annotations

import ctypes

import pytest

from paper_2411_01738_amd import _lib
from tests.test_abi import P, needs_no_gpu

pytestmark = needs_no_gpu


HIP = -8


def _i32(*x):
    return (ctypes.c_int32 * len(x))(*x)


def _i64(*x):
    return (ctypes.c_int64 * len(x))(*x)


def _scaling(kind=0, factor=1.0, orig=0.0, fast=32.0, slow=1.0, magnitude=1.0):
    return ctypes.byref(_lib.RopeScaling(kind, factor, orig, fast, slow, magnitude))


@pytest.mark.parametrize("change,code", [
    (dict(pos=None), -1), (dict(pos=P(0) + 8), -5), (dict(cos=None), -1), (dict(cos=P(0)), -6), (dict(sin=P(1) + 64), -6),
    (dict(dtype=0), -2), (dict(n=-1), -3), (dict(n=1 << 31), -3), (dict(axes=0), -4), (dict(axes=5), -4), (dict(dims=None), -1),
    (dict(dims=_i32(16, 7)), -3), (dict(dims=_i32(16, 0)), -3), (dict(dims=_i32(200, 200)), -3), (dict(theta=0.0), -4),
    (dict(theta=float("nan")), -4), (dict(sc=_scaling(4)), -4), (dict(sc=_scaling(1, 0.0)), -4), (dict(sc=_scaling(2, -1.0)), -4),
    (dict(sc=_scaling(2, 2.0), dims=_i32(16, 2)), -3), (dict(sc=_scaling(3, 2.0)), -4), (dict(sc=_scaling(3, 2.0, 100.0, 1.0, 1.0)), -4),
    (dict(sc=_scaling(0, magnitude=float("inf"))), -4)])
def test_table(change, code):
    a = dict(pos=P(0), dtype=2, n=100, axes=2, dims=_i32(16, 48), theta=1e4, sc=None, cos=P(1), sin=P(2))
    a.update(change)
    L = _lib.lib()
    assert L.xdit_rope_table(*a.values()) == code and L.xdit_last_error()


def test_empty_table():
    assert _lib.lib().xdit_rope_table(None, 2, 0, 1, _i32(64), 1e4, None, None, None) == 0


# x, cos, sin, y, strides, B, N, H, d, rot, per batch, layout, transpose, dtype
@pytest.mark.parametrize("change,code", [
    (dict(x=None), -1), (dict(cos=None), -1), (dict(sin=None), -1), (dict(y=None), -1), (dict(x=P(0) + 8), -5), (dict(y=P(0) + 16), -6),
    (dict(y=P(1)), -6), (dict(dtype=3), -2), (dict(d=96), -7), (dict(B=-1), -3), (dict(N=1 << 31), -3), (dict(B=1 << 16, N=1 << 16), -3),
    (dict(H=70000), -3), (dict(rot=0), -3), (dict(rot=12), -3), (dict(rot=72), -3), (dict(layout=2), -4),
    (dict(strides=_i64(2048, 128, 64, 2048, 128, 32)), -6),      # heads of y on top of each other
    (dict(strides=_i64(2048, 128, 64, 2048, 64, 64)), -6),       # tokens of y on top of each other
    (dict(strides=_i64(2048, 128, 64, 2048, 0, 64)), -6), (dict(strides=_i64(2048, 128, 68, 2048, 128, 64)), -5),
    (dict(strides=_i64(2048, -128, 64, 2048, 128, 64)), -5), (dict(strides=_i64(1 << 60, 128, 64, 2048, 128, 64)), -3),
    (dict(y=P(0) + 2 * 128, strides=_i64(2048, 128, 64, 2048, 128, 64)), -6),   # shifted by a token
    (dict(y=P(0) + 2 * 64, strides=_i64(4096, 256, 64, 4096, 256, 64)), -6)])   # by a head of two
def test_rope(change, code):
    a = dict(x=P(0), cos=P(1), sin=P(2), y=P(3), strides=None, B=2, N=16, H=2, d=64, rot=64, pb=0, layout=0, tr=0, dtype=0)
    a.update(change)
    L = _lib.lib()
    assert L.xdit_rope(*a.values()) == code and L.xdit_last_error()


def _qk(**kw):
    p = _lib.Qk(2, 16, 2, 2, 64, 0, 1, 1e-6, P(20), P(21), None, None, 1, 0, 32, P(22), P(23), 0, None)
    for n, v in kw.items():
        setattr(p, n, v)
    return p


QK = [(dict(batch=-1), -3), (dict(q_heads=-1), -3), (dict(k_heads=70000), -3), (dict(head_dim=80), -7), (dict(dtype=2), -2),
      (dict(weight_dtype=2), -2), (dict(norm=3), -4), (dict(norm=-1), -4), (dict(norm=0), -4), (dict(eps=-1e-6), -4),
      (dict(eps=float("nan")), -4), (dict(eps=1e300), -4), (dict(bq=P(24)), -4), (dict(layout=7), -4), (dict(rot_dim=20), -3),
      (dict(rot_dim=0), -3), (dict(cos=None), -1), (dict(sin=P(23) + 4), -5), (dict(wq=P(20) + 2), -5)]


@pytest.mark.parametrize("change,code", QK)
def test_qk_parameters(change, code):
    L = _lib.lib()
    p = _qk(**change)
    assert L.xdit_qk_norm_rope(ctypes.byref(p), P(0), P(1), P(2), P(3)) == code and L.xdit_last_error()
    assert L.xdit_qk_norm_rope_bwd(ctypes.byref(p), P(0), P(1), P(2), P(3), P(4), P(5), None, None, None, None, None, 0) == code


def test_qk_tensors():
    L = _lib.lib()
    f = lambda p, *t: L.xdit_qk_norm_rope(None if p is None else ctypes.byref(p), *t)
    assert f(None, P(0), P(1), P(2), P(3)) == -1
    assert f(_qk(), P(0), None, P(2), P(3)) == -1
    assert f(_qk(), P(0), P(1), P(1), P(3)) == -6          # q_out on k
    assert f(_qk(), P(0), P(1), P(2), P(2)) == -6
    assert f(_qk(), P(0), P(1), P(2), P(0)) == -6          # k_out on q
    assert f(_qk(), P(0), P(1), P(22), P(3)) == -6         # on the table
    assert f(_qk(), P(0), P(1), P(20) - 64, P(3)) == -6    # on a weight
    # one fused buffer of q, k and v rows: in place is fine up to the launch, a head's shift is not
    row = 6 * 64
    fused = _i64(*[16 * row, row, 64] * 4)
    p = _qk(strides=ctypes.cast(fused, ctypes.POINTER(ctypes.c_int64)))
    assert f(p, P(0), P(0) + 256, P(0) + 128, P(0) + 256) == -6
    assert f(p, P(0), P(0) + 256, P(0), P(0) + 128) == -6
    assert f(p, P(0), P(0) + 256, P(0) + 2 * row - 128, P(0) + 256) == -6   # from the last head into the next row
    # q, k, v of [B, 3, H, N, d], of [B, N, H, 3, d], every other token; H = 2, N = 16: elements shared by one
    for strides, ok, bad in (([3 * 2 * 16 * 64, 64, 16 * 64], 2 * 16 * 64, 2 * 16 * 64 - 64), ([16 * 6 * 64, 6 * 64, 3 * 64], 64, 3 * 64),
                             ([32 * 2 * 64, 4 * 64, 64], 2 * 64, 64)):
        p = _qk(strides=ctypes.cast(_i64(*strides * 4), ctypes.POINTER(ctypes.c_int64)))
        assert f(p, P(0), P(0) + 2 * bad, P(0), P(0) + 2 * bad) == -6
        assert f(p, P(0), P(0) + 2 * ok, P(0), P(0) + 2 * ok) == HIP   # to the launch, which has no device
    # nothing to do
    assert f(_qk(batch=0), None, None, None, None) == 0


def test_qk_gradients():
    L = _lib.lib()
    need = L.xdit_qk_norm_rope_bwd_workspace_bytes(2, 16, 2, 2, 64, 0)
    assert need > 0 and L.xdit_qk_norm_rope_bwd_workspace_bytes(2, 16, 2, 2, 65, 0) == -1
    assert L.xdit_qk_norm_rope_bwd_workspace_bytes(2, 1 << 31, 2, 2, 64, 0) == -1

    def f(p=None, t=(P(0), P(1), P(2), P(3), P(4), P(5)), g=(P(6), P(7), None, None), ws=P(8), n=need):
        return L.xdit_qk_norm_rope_bwd(ctypes.byref(p or _qk()), *t, *g, ws, n)

    assert f(ws=None) == -4 and f(n=need - 1) == -4 and f(ws=P(8) + 8) == -5
    assert f(g=(P(6), P(7), P(9), None)) == -4                    # an RMS norm's bias
    assert f(g=(P(6), P(6), None, None)) == -6 and f(g=(P(6) + 2, P(7), None, None)) == -5
    assert f(g=(P(0), P(7), None, None)) == -6 and f(ws=P(4)) == -6 and f(g=(P(8), P(7), None, None)) == -6
    assert f(t=(P(0), P(1), P(2), P(3), P(1), P(5))) == -6        # dq on k
    assert f(t=(P(0), P(1), P(2), P(3), P(3), P(5))) == -6        # dq on dk_out
    assert f(t=(P(0), P(1), P(2), P(3), P(4), P(4))) == -6
    assert f(t=(P(0), P(1), None, P(3), P(4), P(5))) == -1
    assert f(_qk(k_heads=0), t=(P(0), None, P(2), None, P(4), None), g=(P(6), P(7), None, None)) == -3
    none = _qk(norm=0, wq=None, wk=None)
    assert f(none) == -4                                           # weights' gradients without a norm


BWD = dict(q=P(0), k=P(1), v=P(2), out=P(3), lse=P(4), dout=P(5), dlse=P(6), dq=P(7), dk=P(8), dv=P(9), accum=0, ws=P(10), n=1 << 30,
           B=1, Nq=300, Nk=200, H=2, d=64, dtype=0)


@pytest.mark.parametrize("change,code", [
    *[({n: None}, -1) for n in ("q", "k", "v", "out", "lse", "dout", "dq", "dk", "dv")], (dict(q=P(0) + 8), -5), (dict(lse=P(4) + 2), -5),
    (dict(dlse=P(6) + 1), -5), (dict(ws=P(10) + 128), -5), (dict(ws=None), -4), (dict(n=100), -4), (dict(accum=4), -4), (dict(accum=-1), -4),
    (dict(B=-1), -3), (dict(Nq=1 << 31), -3), (dict(Nk=1 << 24), -3), (dict(d=96), -7), (dict(dtype=2), -2),
    (dict(dq=P(0)), -6), (dict(dq=P(3)), -6), (dict(dk=P(8), dv=P(8)), -6), (dict(dv=P(2) + 16), -6), (dict(dk=P(5)), -6), (dict(dq=P(6)), -6),
    (dict(ws=P(7)), -6), (dict(ws=P(4)), -6),
    # float32 sums reach twice as far as bf16 gradients
    (dict(dq=P(8) - 300 * 2 * 64 * 2, accum=1), -6), (dict(dk=P(9) - 200 * 2 * 64 * 2, accum=2), -6)])
def test_attention_gradients(change, code):
    L = _lib.lib()
    assert L.xdit_chunk_attn_bwd(*{**BWD, **change}.values()) == code and L.xdit_last_error()


def test_attention_gradients_of_nothing():
    L = _lib.lib()
    none = {n: None for n in ("q", "k", "v", "out", "lse", "dout", "dlse", "dq", "dk", "dv", "ws")}
    assert L.xdit_chunk_attn_bwd(*{**BWD, **none, "B": 0}.values()) == 0
    assert L.xdit_chunk_attn_bwd(*{**BWD, **none, "Nq": 0, "Nk": 0}.values()) == 0


def test_workspace_of_the_attention_gradients():
    """Two float32 per query row, and the partials of cut sweeps: none where the
    workgroups are many."""
    L = _lib.lib()
    f = L.xdit_chunk_attn_bwd_workspace_bytes
    assert f(2, 1024, 1024, 16, 72, 0) == 8 * 2 * 16 * 1024
    assert f(1, 4224, 4224, 24, 128, 0) == 8 * 24 * 4224
    assert f(1, 1, 4429, 24, 64, 0) > 8 * 24 and f(1, 4429, 1, 24, 64, 0) > 8 * 24 * 4429
    assert f(0, 10, 10, 2, 64, 0) == 0 and f(1, 0, 10, 2, 64, 0) >= 0
    assert f(1, 10, 10, 2, 96, 0) == -1 and f(1, -1, 10, 2, 64, 0) == -1


def test_workspace_of_many_batches():
    """A call of more than 2^24 - 1 workgroups runs as several launches of whole
    batches, which share the workspace: it holds those of one.  16 heads of one
    query and one key are 32 workgroups, so 524287 batches at a time."""
    f = _lib.lib().xdit_chunk_attn_bwd_workspace_bytes
    one = f(524287, 1, 1, 16, 64, 0)
    assert 8 * 16 * 524287 <= one < 8 * 16 * 524287 + 256
    for B in (524288, 2 * 524287 + 3):
        assert f(B, 1, 1, 16, 64, 0) == one
    assert f(524286, 1, 1, 16, 64, 0) < one


def test_stage_step_qk():
    L = _lib.lib()

    def f(qk, **kw):
        a = dict(x=P(0), wq=P(1), wk=P(2), wv=P(3), wo=P(4), kv=P(5), off=0, len=8, q=P(6), k=P(7), v=P(8), o=P(9), y=P(10), B=1, N=16,
                 H=2, d=64, C=128, dtype=0)
        a.update(kw)
        return L.xdit_stage_step_qk(None if qk is None else ctypes.byref(qk), *a.values())

    good = dict(batch=1, tokens=8)
    assert f(None) == -1
    for bad in (dict(batch=2), dict(tokens=9), dict(q_heads=1), dict(k_heads=0), dict(head_dim=128), dict(dtype=1)):
        assert f(_qk(**{**good, **bad})) == -3
    assert f(_qk(**good, norm=0)) == -4 and f(_qk(**good, rot_dim=12)) == -3
    assert f(_qk(**good, cos=P(9))) == -6 and f(_qk(**good, wq=P(5))) == -6 and f(_qk(**good, wk=P(6))) == -6
    assert f(_qk(**good), q=P(6), k=P(6)) == -6 and f(_qk(**good), dtype=1) == -7


@pytest.mark.parametrize("bad", [dict(layout="other"), dict(layout=0), dict(norm="other"), dict(norm=None)])
def test_stage_step_names(bad):
    """A wrong name is refused before anything else, also where nothing is
    rotated or normalised."""
    import paper_2411_01738_amd as xd

    with pytest.raises(xd.XditError, match=f"{list(bad)[0]} = "):
        xd.xdit_stage_step(None, None, None, None, None, None, 0, None, None, None, None, None, **bad)
