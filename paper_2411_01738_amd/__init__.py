"""MI355X (gfx950) DiT attention hot path of xDiT (arXiv 2411.01738).

Thin binding over the C ABI of libxdit.so (include/xdit.h): each function
takes torch tensors that already live on the GPU, checks that they are dense,
reads their sizes, passes raw device pointers and torch's current stream, and
raises XditError when the library rejects the call.  All arithmetic runs in
the library's HIP kernels; there is no host or PyTorch fallback.  Calls go
through _binding (csrc/binding.cpp), which does the same checks in native
code; a call that it does not take, for one whose arguments are wrong, goes
through the checks below, which say why.

Layouts: activations [B, N, H, d]; K/V buffer [2, B, N, H, d]; LSE [B, H, Nq]
float32.  dtypes: bfloat16 or float32 (LSE always float32).
"""
from __future__ import annotations

import ctypes
import warnings

from ._lib import (LAYOUTS, NORMS, SCALINGS, XDIT_ACCUM_DKV, XDIT_ACCUM_DQ, XDIT_BF16, XDIT_F32, XDIT_I64, XDIT_MAX_AXES, XDIT_MAX_PARTIALS,
                   XDIT_MAX_RANGES, XDIT_MAX_SPLITS, Qk, RopeScaling, XditError, check, lib)

__all__ = ["xdit_patch_attn", "xdit_patch_attn_ranges", "xdit_chunk_attn",
           "xdit_chunk_attn_accum", "xdit_chunk_attn_accum_split", "xdit_chunk_attn_split",
           "xdit_patch_attn_split", "xdit_chunk_attn_split_noalloc",
           "split_workspace_bytes", "xdit_lse_merge",
           "xdit_kv_update", "xdit_stage_step", "xdit_rope_table", "xdit_rope", "xdit_qk_norm_rope",
           "xdit_qk_norm_rope_bwd", "qk_norm_rope_bwd_workspace_bytes", "xdit_chunk_attn_bwd",
           "chunk_attn_bwd_workspace_bytes", "set_stream", "XditError", "XDIT_MAX_PARTIALS", "XDIT_MAX_RANGES",
           "version"]


def _torch():
    import torch
    return torch


_native = None  # the _binding module; False: not built


def _load_native():
    global _native
    torch = _torch()
    lib()  # says what is missing if nothing is built
    _native = False
    try:
        from . import _binding
        _binding.init(torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream)
        _native = _binding
    except AttributeError:  # a torch without GPU support: no call gets past the checks
        pass
    except ImportError as e:
        warnings.warn(f"the torch binding does not load ({e}): calls go through ctypes, at several times the host "
                      "time; build it with `python -m paper_2411_01738_amd.build`", RuntimeWarning, stacklevel=3)
    return _native


def _done(rc) -> bool:
    """Whether the native path took the call; raises if the library rejected it."""
    if rc is None:
        return False
    check(rc)
    return True


def _dtype_code(t) -> int:
    torch = _torch()
    if t.dtype == torch.bfloat16:
        return XDIT_BF16
    if t.dtype == torch.float32:
        return XDIT_F32
    raise XditError(-2, f"unsupported dtype {t.dtype}")


def _dense(t, name: str, ndim: int):
    if t is None:
        return None
    if not t.is_cuda:
        raise XditError(-1, f"{name} must be a GPU tensor")
    if t.dim() != ndim:
        raise XditError(-3, f"{name} must have {ndim} dims, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise XditError(-5, f"{name} must be contiguous")
    return t


def _buffer(kv_buf):
    _dense(kv_buf, "kv_buf", 5)
    if kv_buf.shape[0] < 2:
        raise XditError(-3, f"kv_buf must be [2, B, N, H, d] (K's plane, then V's), got {tuple(kv_buf.shape)}")


def _ptr(t) -> int | None:
    return None if t is None else t.data_ptr()


def _use_current_stream() -> None:
    lib().xdit_set_stream(_torch().cuda.current_stream().cuda_stream)


def set_stream(stream) -> None:
    """Route later calls of this thread to `stream` (a torch.cuda.Stream or a raw
    hipStream_t handle).  The functions below always use torch's current stream."""
    handle = getattr(stream, "cuda_stream", stream)
    check(lib().xdit_set_stream(handle))


def version() -> str:
    return lib().xdit_version().decode()


def xdit_patch_attn(q, kv_buf, patch_off: int, patch_len: int, fresh_k, fresh_v, out) -> None:
    """PipeFusion patch step: write fresh_k/fresh_v into rows
    [patch_off, patch_off+patch_len) of kv_buf [2,B,N,H,d] (in place), then
    out = attention(q, updated K, updated V) for the patch's queries
    q [B,patch_len,H,d]."""
    nat = _native if _native is not None else _load_native()
    if nat and _done(nat.patch(q, kv_buf, patch_off, patch_len, fresh_k, fresh_v, out)):
        return
    _buffer(kv_buf)
    for t, n in ((q, "q"), (fresh_k, "fresh_k"), (fresh_v, "fresh_v"), (out, "out")):
        _dense(t, n, 4)
    _, B, N, H, d = kv_buf.shape
    for t, n in ((q, "q"), (fresh_k, "fresh_k"), (fresh_v, "fresh_v"), (out, "out")):
        if tuple(t.shape) != (B, patch_len, H, d):
            raise XditError(-3, f"{n} has shape {tuple(t.shape)}, expected {(B, patch_len, H, d)}")
        if t.dtype != kv_buf.dtype:
            raise XditError(-2, f"{n} dtype {t.dtype} differs from kv_buf's {kv_buf.dtype}")
    _use_current_stream()
    check(lib().xdit_patch_attn(_ptr(q), _ptr(kv_buf), int(patch_off), int(patch_len),
                                _ptr(fresh_k), _ptr(fresh_v), _ptr(out), B, N, H, d,
                                _dtype_code(kv_buf)))


def _patch_args(q, kv_buf, ranges, fresh_k, fresh_v, out, lse):
    _buffer(kv_buf)
    for t, n in ((q, "q"), (fresh_k, "fresh_k"), (fresh_v, "fresh_v"), (out, "out")):
        _dense(t, n, 4)
    _dense(lse, "lse", 3)
    _, B, N, H, d = kv_buf.shape
    nr = len(ranges)
    F = sum(int(r[1]) for r in ranges)
    Nq = q.shape[1]
    for t, n, rows in ((q, "q", Nq), (out, "out", Nq), (fresh_k, "fresh_k", F),
                       (fresh_v, "fresh_v", F)):
        if t is None:
            if B * rows * H * d > 0:
                raise XditError(-1, f"{n} is required")
            continue
        if tuple(t.shape) != (B, rows, H, d):
            raise XditError(-3, f"{n} has shape {tuple(t.shape)}, expected {(B, rows, H, d)}")
        if t.dtype != kv_buf.dtype:
            raise XditError(-2, f"{n} dtype {t.dtype} differs from kv_buf's {kv_buf.dtype}")
    if lse is not None:
        torch = _torch()
        if lse.dtype != torch.float32 or tuple(lse.shape) != (B, H, Nq):
            raise XditError(-3, f"lse must be float32 [B,H,Nq] = {(B, H, Nq)}")
    offs = (ctypes.c_int64 * max(nr, 1))(*[int(r[0]) for r in ranges])
    lens = (ctypes.c_int64 * max(nr, 1))(*[int(r[1]) for r in ranges])
    return ((_ptr(q), Nq, _ptr(kv_buf), nr, offs, lens, _ptr(fresh_k), _ptr(fresh_v), _ptr(out), _ptr(lse)),
            (B, N, H, d, _dtype_code(kv_buf)))


def xdit_patch_attn_ranges(q, kv_buf, ranges, fresh_k, fresh_v, out, lse=None) -> None:
    """General patch step: write fresh_k/fresh_v [B, F, H, d] into the row
    ranges [(off, len), ...] of kv_buf [2,B,N,H,d] (range 0's rows first; F =
    sum of the lengths), then out = attention(q, updated K, updated V) for the
    queries q [B,Nq,H,d] and, if given, lse [B,H,Nq] (natural log)."""
    nat = _native if _native is not None else _load_native()
    if nat and _done(nat.patch_ranges(q, kv_buf, ranges, fresh_k, fresh_v, out, lse)):
        return
    tensors, sizes = _patch_args(q, kv_buf, ranges, fresh_k, fresh_v, out, lse)
    _use_current_stream()
    check(lib().xdit_patch_attn_ranges(*tensors, *sizes))


def _chunk_args(q, k, v, out, lse):
    for t, n in ((q, "q"), (k, "k"), (v, "v"), (out, "out")):
        _dense(t, n, 4)
    _dense(lse, "lse", 3)
    B, Nq, H, d = q.shape
    Nk = k.shape[1]
    if tuple(k.shape) != (B, Nk, H, d) or tuple(v.shape) != (B, Nk, H, d):
        raise XditError(-3, f"k/v shapes {tuple(k.shape)}/{tuple(v.shape)} do not match q")
    if tuple(out.shape) != (B, Nq, H, d):
        raise XditError(-3, "out shape differs from q")
    for t, n in ((k, "k"), (v, "v"), (out, "out")):
        if t.dtype != q.dtype:
            raise XditError(-2, f"{n} dtype differs from q's")
    if lse is not None:
        torch = _torch()
        if lse.dtype != torch.float32 or tuple(lse.shape) != (B, H, Nq):
            raise XditError(-3, f"lse must be float32 [B,H,Nq] = {(B, H, Nq)}")
    return (_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), B, Nq, Nk, H, d, _dtype_code(q))


def xdit_chunk_attn(q, k, v, out, lse=None) -> None:
    """Chunk attention: out = attention(q, k, v) and, if given,
    lse [B,H,Nq] = log-sum-exp of the scaled scores (natural log)."""
    nat = _native if _native is not None else _load_native()
    if nat and _done(nat.chunk(q, k, v, out, lse, False)):
        return
    args = _chunk_args(q, k, v, out, lse)
    _use_current_stream()
    check(lib().xdit_chunk_attn(*args))


def split_workspace_bytes(q, kv_len: int, splits: int = 0) -> int:
    """Bytes of workspace the *_split calls need for queries shaped like q
    [B,Nq,H,d] over kv_len keys (0 when no split happens)."""
    B, Nq, H, d = q.shape
    n = lib().xdit_split_workspace_bytes(B, Nq, int(kv_len), H, d, _dtype_code(q), int(splits))
    if n < 0:
        raise XditError(-3, "xdit_split_workspace_bytes rejected the sizes")
    return int(n)


def _workspace(ws):
    if ws is None:
        return None, 0
    if not ws.is_cuda or not ws.is_contiguous():
        raise XditError(-5, "workspace must be a dense GPU tensor")
    return ws.data_ptr(), ws.numel() * ws.element_size()


def xdit_chunk_attn_split(q, k, v, out, lse=None, splits: int = 0, workspace=None) -> None:
    """xdit_chunk_attn with each query tile's keys split `splits` ways (0: the
    library chooses); workspace: a GPU tensor of split_workspace_bytes bytes."""
    nat = _native if _native is not None else _load_native()
    if nat and _done(nat.chunk_split(q, k, v, out, lse, splits, workspace, False)):
        return
    args = _chunk_args(q, k, v, out, lse)
    wp, wb = _workspace(workspace)
    _use_current_stream()
    check(lib().xdit_chunk_attn_split(*args[:5], int(splits), wp, wb, *args[5:]))


def xdit_chunk_attn_split_noalloc(q, k, v, out, lse=None, splits: int = 0) -> None:
    """xdit_chunk_attn_split with the partials kept in the library's fixed
    per-GPU scratch array (no workspace, nothing allocated)."""
    args = _chunk_args(q, k, v, out, lse)
    _use_current_stream()
    check(lib().xdit_chunk_attn_split_noalloc(*args[:5], int(splits), *args[5:]))


def xdit_patch_attn_split(q, kv_buf, ranges, fresh_k, fresh_v, out, lse=None, splits: int = 0,
                          workspace=None) -> None:
    """xdit_patch_attn_ranges with the keys split `splits` ways (0: the
    library chooses); workspace as for xdit_chunk_attn_split."""
    nat = _native if _native is not None else _load_native()
    if nat and _done(nat.patch_split(q, kv_buf, ranges, fresh_k, fresh_v, out, lse, splits, workspace)):
        return
    tensors, sizes = _patch_args(q, kv_buf, ranges, fresh_k, fresh_v, out, lse)
    wp, wb = _workspace(workspace)
    _use_current_stream()
    check(lib().xdit_patch_attn_split(*tensors, int(splits), wp, wb, *sizes))


def xdit_chunk_attn_accum(q, k, v, out, lse) -> None:
    """Ring step: merge attention(q, k, v) into the running (out, lse) in
    place.  lse = -inf marks an empty running state (out then ignored)."""
    nat = _native if _native is not None else _load_native()
    if nat and _done(nat.chunk(q, k, v, out, lse, True)):
        return
    if lse is None:
        raise XditError(-1, "the running lse is required")
    args = _chunk_args(q, k, v, out, lse)
    _use_current_stream()
    check(lib().xdit_chunk_attn_accum(*args))


def xdit_chunk_attn_accum_split(q, k, v, out, lse, splits: int = 0, workspace=None) -> None:
    """xdit_chunk_attn_accum with each query tile's keys split `splits` ways
    (0: the library chooses); workspace as for xdit_chunk_attn_split."""
    nat = _native if _native is not None else _load_native()
    if nat and _done(nat.chunk_split(q, k, v, out, lse, splits, workspace, True)):
        return
    if lse is None:
        raise XditError(-1, "the running lse is required")
    args = _chunk_args(q, k, v, out, lse)
    wp, wb = _workspace(workspace)
    _use_current_stream()
    check(lib().xdit_chunk_attn_accum_split(*args[:5], int(splits), wp, wb, *args[5:]))


def xdit_lse_merge(outs, lses, n: int, out, lse_out=None) -> None:
    """Merge n chunk partials (outs[r] [B,Nq,H,d], lses[r] [B,H,Nq] float32)
    into out, and the merged log-sum-exp into lse_out if given."""
    nat = _native if _native is not None else _load_native()
    if nat and _done(nat.merge(outs, lses, n, out, lse_out)):
        return
    n = int(n)
    if n < 1 or n > len(outs) or n > len(lses):
        raise XditError(-4, f"n = {n} does not match {len(outs)} outs / {len(lses)} lses")
    _dense(out, "out", 4)
    _dense(lse_out, "lse_out", 3)
    B, Nq, H, d = out.shape
    torch = _torch()
    for r in range(n):
        _dense(outs[r], f"outs[{r}]", 4)
        _dense(lses[r], f"lses[{r}]", 3)
        if tuple(outs[r].shape) != (B, Nq, H, d) or outs[r].dtype != out.dtype:
            raise XditError(-3, f"outs[{r}] does not match out")
        if tuple(lses[r].shape) != (B, H, Nq) or lses[r].dtype != torch.float32:
            raise XditError(-3, f"lses[{r}] must be float32 {(B, H, Nq)}")
    if lse_out is not None and (tuple(lse_out.shape) != (B, H, Nq) or lse_out.dtype != torch.float32):
        raise XditError(-3, f"lse_out must be float32 {(B, H, Nq)}")
    optrs = (ctypes.c_void_p * n)(*[outs[r].data_ptr() for r in range(n)])
    lptrs = (ctypes.c_void_p * n)(*[lses[r].data_ptr() for r in range(n)])
    _use_current_stream()
    check(lib().xdit_lse_merge(optrs, lptrs, n, _ptr(out), _ptr(lse_out), B, Nq, H, d,
                               _dtype_code(out)))


def xdit_kv_update(kv_buf, patch_off: int, patch_len: int, fresh_k, fresh_v) -> None:
    """Copy fresh K/V [B,patch_len,H,d] into rows [patch_off, patch_off+patch_len)
    of kv_buf [2,B,N,H,d], bit for bit."""
    nat = _native if _native is not None else _load_native()
    if nat and _done(nat.update(kv_buf, patch_off, patch_len, fresh_k, fresh_v)):
        return
    _buffer(kv_buf)
    _dense(fresh_k, "fresh_k", 4)
    _dense(fresh_v, "fresh_v", 4)
    _, B, N, H, d = kv_buf.shape
    for t, nm in ((fresh_k, "fresh_k"), (fresh_v, "fresh_v")):
        if tuple(t.shape) != (B, patch_len, H, d) or t.dtype != kv_buf.dtype:
            raise XditError(-3, f"{nm} must be {(B, patch_len, H, d)} of kv_buf's dtype")
    _use_current_stream()
    check(lib().xdit_kv_update(_ptr(kv_buf), int(patch_off), int(patch_len), _ptr(fresh_k),
                               _ptr(fresh_v), B, N, H, d, _dtype_code(kv_buf)))


def xdit_stage_step(x, wq, wk, wv, wo, kv_buf, patch_off: int, q, k, v, o, y, *, norm: str = "none", eps: float = 1e-6,
                    norm_wq=None, norm_wk=None, norm_bq=None, norm_bk=None, cos=None, sin=None,
                    layout: str = "interleaved") -> None:
    """One PipeFusion stage micro-step at one attention layer: q/k/v = x
    W{q,k,v} (x [B,L,C], W [C,H*d]), the patch step over kv_buf [2,B,N,H,d]
    at rows [patch_off, patch_off+L) with fresh K/V (k, v) and output o, then
    y = o wo (wo [H*d,C]).  q, k, v, o [B,L,H,d] and y [B,L,C] are written.
    With a norm or a rotary table, q and k are normalised and rotated as by
    xdit_qk_norm_rope between the projections and the patch step: cos, sin
    hold the patch's rows, [L, r] or [B, L, r]."""
    _choice(NORMS, "norm", norm)
    _choice(LAYOUTS, "layout", layout)
    _buffer(kv_buf)
    _, B, N, H, d = kv_buf.shape
    _dense(x, "x", 3)
    L, C = x.shape[1], x.shape[2]
    if x.shape[0] != B:
        raise XditError(-3, f"x must be [B, L, C] with B = {B}")
    for t, nm, shp in ((wq, "wq", (C, H * d)), (wk, "wk", (C, H * d)), (wv, "wv", (C, H * d)),
                       (wo, "wo", (H * d, C)), (y, "y", (B, L, C))):
        _dense(t, nm, len(shp))
        if tuple(t.shape) != shp or t.dtype != x.dtype:
            raise XditError(-3, f"{nm} must be {shp} of x's dtype")
    for t, nm in ((q, "q"), (k, "k"), (v, "v"), (o, "o")):
        _dense(t, nm, 4)
        if tuple(t.shape) != (B, L, H, d) or t.dtype != x.dtype:
            raise XditError(-3, f"{nm} must be {(B, L, H, d)} of x's dtype")
    if kv_buf.dtype != x.dtype:
        raise XditError(-3, "kv_buf must have x's dtype")
    if norm != "none" or any(t is not None for t in (norm_wq, norm_wk, norm_bq, norm_bk, cos, sin)):
        p = _qk(q, k, [], norm, eps, norm_wq, norm_wk, norm_bq, norm_bk, cos, sin, layout)
        p.strides = None  # dense, as checked above
        _use_current_stream()
        check(lib().xdit_stage_step_qk(ctypes.byref(p), _ptr(x), _ptr(wq), _ptr(wk), _ptr(wv), _ptr(wo), _ptr(kv_buf),
                                       int(patch_off), L, _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(y), B, N, H, d, C,
                                       _dtype_code(x)))
        return
    _use_current_stream()
    check(lib().xdit_stage_step(_ptr(x), _ptr(wq), _ptr(wk), _ptr(wv), _ptr(wo), _ptr(kv_buf),
                                int(patch_off), L, _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(y), B,
                                N, H, d, C, _dtype_code(x)))


# -- queries and keys between their projection and the attention ----------------
def _choice(table: dict, what: str, name):
    code = table.get(name) if isinstance(name, str) else None
    if code is None:
        raise XditError(-4, f"{what} = {name!r}, expected one of {', '.join(table)}")
    return code


def _on_device(t, name: str):
    """A GPU tensor of the current device, whose stream the call goes to."""
    if not t.is_cuda:
        raise XditError(-1, f"{name} must be a GPU tensor")
    if t.device.index != _torch().cuda.current_device():
        raise XditError(-5, f"{name} is on {t.device}, not on the current device")


def _vector(t, name: str, n: int, dtypes):
    """A dense [n] tensor of one of the types, or None."""
    if t is None:
        return
    _on_device(t, name)
    if tuple(t.shape) != (n,) or not t.is_contiguous() or t.dtype not in dtypes:
        raise XditError(-3, f"{name} must be a dense [{n}] tensor of {' or '.join(str(x) for x in dtypes)}")


def _head_views(tensors):
    """Sizes (B, N, d) and strides of [B, N, H, d] tensors whose heads lie
    contiguous: (tensor, name, shape it must have or None) each; a None tensor
    has strides 0."""
    strides = []
    for t, name, shape, dtype in tensors:
        if t is None:
            strides += [0, 0, 0]
            continue
        _on_device(t, name)
        if t.dim() != 4:
            raise XditError(-3, f"{name} must have 4 dims, got {tuple(t.shape)}")
        if t.stride(3) != 1:
            raise XditError(-5, f"{name}: the elements of a head must be contiguous")
        if tuple(t.shape) != tuple(shape):
            raise XditError(-3, f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
        if t.dtype != dtype:
            raise XditError(-2, f"{name} dtype {t.dtype} differs from {dtype}")
        strides += t.stride()[:3]
    return (ctypes.c_int64 * len(strides))(*strides)


def _table(cos, sin, B: int, N: int):
    """(rot_dim, table per batch) of a rotary table, [N, r] or [B, N, r]."""
    if cos is None and sin is None:
        return 0, 0
    torch = _torch()
    for t, n in ((cos, "cos"), (sin, "sin")):
        if t is None:
            raise XditError(-1, "cos and sin go together")
        _on_device(t, n)
        if t.dtype != torch.float32 or not t.is_contiguous() or tuple(t.shape[:-1]) not in ((N,), (B, N)):
            raise XditError(-3, f"{n} must be a dense float32 [{N}, rot / 2] or [{B}, {N}, rot / 2], got {tuple(t.shape)}")
    if cos.shape != sin.shape:
        raise XditError(-3, "cos and sin differ in shape")
    return 2 * cos.shape[-1], int(cos.dim() == 3)


def xdit_rope_table(pos, dims, cos, sin, theta: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                    orig_len: float = 0.0, fast: float = 32.0, slow: float = 1.0, magnitude: float = 1.0) -> None:
    """cos, sin [N, sum(dims) / 2] float32 of the angles of positions pos
    [N, len(dims)] (int64, or float32 for fractional ones): axis a turns
    dims[a] / 2 pairs at theta^(-2i / dims[a]).  scaling: "none", "linear" (all
    frequencies / factor), "ntk" (theta grown so that the slowest pair is
    divided by factor) or "ramp" (by a pair's turns within orig_len: kept from
    `fast` turns on, / factor up to `slow`); magnitude multiplies the table."""
    nat = _native if _native is not None else _load_native()
    if nat and _done(nat.rope_table(pos, dims, cos, sin, theta, scaling, factor, orig_len, fast, slow, magnitude)):
        return
    torch = _torch()
    dims = [int(x) for x in dims]
    if not 1 <= len(dims) <= XDIT_MAX_AXES:
        raise XditError(-4, f"{len(dims)} axes outside [1, {XDIT_MAX_AXES}]")
    _on_device(pos, "pos")
    if pos.dtype not in (torch.int64, torch.float32):
        raise XditError(-2, f"positions are int64 or float32, not {pos.dtype}")
    if pos.dim() != 2 or pos.shape[1] != len(dims) or not pos.is_contiguous():
        raise XditError(-3, f"pos must be a dense [N, {len(dims)}] tensor, got {tuple(pos.shape)}")
    n, cols = pos.shape[0], sum(dims) // 2
    for t, name in ((cos, "cos"), (sin, "sin")):
        _on_device(t, name)
        if t.dtype != torch.float32 or tuple(t.shape) != (n, cols) or not t.is_contiguous():
            raise XditError(-3, f"{name} must be a dense float32 [{n}, {cols}] tensor")
    sc = RopeScaling(_choice(SCALINGS, "scaling", scaling), float(factor), float(orig_len), float(fast), float(slow),
                     float(magnitude))
    d = (ctypes.c_int32 * len(dims))(*dims)
    _use_current_stream()
    check(lib().xdit_rope_table(_ptr(pos), XDIT_I64 if pos.dtype == torch.int64 else XDIT_F32, n, len(dims), d, float(theta),
                                ctypes.byref(sc), _ptr(cos), _ptr(sin)))


def xdit_rope(x, cos, sin, y, layout: str = "interleaved", transpose: bool = False) -> None:
    """y = x [B, N, H, d] with the first 2 * cos.shape[-1] elements of each head
    rotated by its row's angles (cos, sin [N, r] or [B, N, r]); pairs of
    neighbours ("interleaved") or (i, i + r) ("half").  transpose: turned back,
    the gradient.  x and y may be strided (each head contiguous); y may be x."""
    nat = _native if _native is not None else _load_native()
    if nat and _done(nat.rope(x, cos, sin, y, layout, transpose)):
        return
    lay = _choice(LAYOUTS, "layout", layout)
    if x.dim() != 4:
        raise XditError(-3, f"x must have 4 dims, got {tuple(x.shape)}")
    code = _dtype_code(x)
    strides = _head_views([(x, "x", x.shape, x.dtype), (y, "y", x.shape, x.dtype)])
    B, N, H, d = x.shape
    if cos is None or sin is None:
        raise XditError(-1, "cos and sin are required")
    rot, per_batch = _table(cos, sin, B, N)
    _use_current_stream()
    check(lib().xdit_rope(_ptr(x), _ptr(cos), _ptr(sin), _ptr(y), strides, B, N, H, d, rot, per_batch, lay, int(transpose),
                          code))


def _qk(q, k, others, norm, eps, wq, wk, bq, bk, cos, sin, layout):
    """The parameters of a call on queries and keys; others: (tensor, name,
    whether of q's shape) in argument order."""
    torch = _torch()
    if q.dim() != 4 or (k is not None and k.dim() != 4):
        raise XditError(-3, "q and k must have 4 dims")
    B, N, H, d = q.shape
    Hk = 0 if k is None else k.shape[2]
    code = _dtype_code(q)
    views = [(q, "q", q.shape, q.dtype), (k, "k", (B, N, Hk, d), q.dtype)]
    for t, name, as_q in others:
        if t is None and (as_q or Hk):
            raise XditError(-1, f"{name} is required")
        views.append((t, name, (B, N, H if as_q else Hk, d), q.dtype))
    strides = _head_views(views)
    weights = [(wq, "wq"), (wk, "wk"), (bq, "bq"), (bk, "bk")]
    types = {t.dtype for t, _ in weights if t is not None}
    for t, name in weights:
        _vector(t, name, d, (torch.bfloat16, torch.float32))
    if len(types) > 1:
        raise XditError(-2, "weights and biases of one call have one type")
    rot, per_batch = _table(cos, sin, B, N)
    return Qk(B, N, H, Hk, d, code, _choice(NORMS, "norm", norm), float(eps), _ptr(wq), _ptr(wk), _ptr(bq), _ptr(bk),
              XDIT_BF16 if torch.bfloat16 in types else XDIT_F32, _choice(LAYOUTS, "layout", layout), rot, _ptr(cos),
              _ptr(sin), per_batch, strides)


def xdit_qk_norm_rope(q, k, q_out, k_out, norm: str = "rms", eps: float = 1e-6, wq=None, wk=None, bq=None, bk=None,
                      cos=None, sin=None, layout: str = "interleaved") -> None:
    """Queries q [B, N, H, d] and keys k [B, N, Hk, d] (or None) normalised per
    head ("rms" or "layer", weights [d] and, for "layer", biases [d] of their own,
    bfloat16 or float32; "none": not normalised) and rotated as by xdit_rope (no table: not rotated).
    Tensors may be strided (each head contiguous): views of one fused
    projection's output; q_out may be q and k_out k."""
    nat = _native if _native is not None else _load_native()
    if nat and _done(nat.qk_norm_rope(q, k, q_out, k_out, norm, eps, wq, wk, bq, bk, cos, sin, layout)):
        return
    p = _qk(q, k, [(q_out, "q_out", True), (k_out, "k_out", False)], norm, eps, wq, wk, bq, bk, cos, sin, layout)
    _use_current_stream()
    check(lib().xdit_qk_norm_rope(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(q_out), _ptr(k_out)))


def qk_norm_rope_bwd_workspace_bytes(q, k) -> int:
    """Bytes of workspace that xdit_qk_norm_rope_bwd needs for the weights'
    gradients of q [B, N, H, d] and k (or None)."""
    B, N, H, d = q.shape
    n = lib().xdit_qk_norm_rope_bwd_workspace_bytes(B, N, H, 0 if k is None else k.shape[2], d, _dtype_code(q))
    if n < 0:
        raise XditError(-3, "xdit_qk_norm_rope_bwd_workspace_bytes rejected the sizes")
    return int(n)


def xdit_qk_norm_rope_bwd(q, k, dq_out, dk_out, dq, dk, norm: str = "rms", eps: float = 1e-6, wq=None, wk=None, cos=None,
                          sin=None, layout: str = "interleaved", dwq=None, dwk=None, dbq=None, dbk=None,
                          workspace=None) -> None:
    """Gradients of xdit_qk_norm_rope: dq, dk of its inputs q and k, given the
    gradients dq_out, dk_out of its outputs; and, where given, the float32
    gradients [d] of weights (dwq, dwk) and, for "layer", biases (dbq, dbk),
    for which a workspace of qk_norm_rope_bwd_workspace_bytes bytes is needed.
    dq may be dq_out or q, dk likewise."""
    nat = _native if _native is not None else _load_native()
    if nat and _done(nat.qk_norm_rope_bwd(q, k, dq_out, dk_out, dq, dk, norm, eps, wq, wk, cos, sin, layout, dwq, dwk, dbq,
                                          dbk, workspace)):
        return
    torch = _torch()
    p = _qk(q, k, [(dq_out, "dq_out", True), (dk_out, "dk_out", False), (dq, "dq", True), (dk, "dk", False)], norm, eps, wq,
            wk, None, None, cos, sin, layout)
    for t, name in ((dwq, "dwq"), (dwk, "dwk"), (dbq, "dbq"), (dbk, "dbk")):
        _vector(t, name, q.shape[3], (torch.float32,))
    if workspace is not None:
        _on_device(workspace, "workspace")
    wp, wb = _workspace(workspace)
    _use_current_stream()
    check(lib().xdit_qk_norm_rope_bwd(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(dq_out), _ptr(dk_out), _ptr(dq), _ptr(dk),
                                      _ptr(dwq), _ptr(dwk), _ptr(dbq), _ptr(dbk), wp, wb))


# -- the attention's gradients --------------------------------------------------
def chunk_attn_bwd_workspace_bytes(q, kv_len: int) -> int:
    """Bytes of workspace that xdit_chunk_attn_bwd needs for queries shaped like
    q [B, Nq, H, d] over kv_len keys."""
    B, Nq, H, d = q.shape
    n = lib().xdit_chunk_attn_bwd_workspace_bytes(B, Nq, int(kv_len), H, d, _dtype_code(q))
    if n < 0:
        raise XditError(-3, "xdit_chunk_attn_bwd_workspace_bytes rejected the sizes")
    return int(n)


def xdit_chunk_attn_bwd(q, k, v, out, lse, dout, dq, dk, dv, dlse=None, accum_dq: bool = False, accum_dkv: bool = False,
                        workspace=None) -> None:
    """Gradients dq [B, Nq, H, d], dk, dv [B, Nk, H, d] of xdit_chunk_attn's
    inputs, given its out and lse, the gradient dout of out and, if any, dlse of
    lse; or, given the out and lse of all chunks of a sequence and their dout,
    this chunk's dk and dv and its part of dq.  accum_dq: dq is a float32 sum
    that the part is added to; accum_dkv: dk and dv are.  workspace: a GPU
    tensor of chunk_attn_bwd_workspace_bytes bytes."""
    nat = _native if _native is not None else _load_native()
    if nat and _done(nat.chunk_bwd(q, k, v, out, lse, dout, dq, dk, dv, dlse, accum_dq, accum_dkv, workspace)):
        return
    torch = _torch()
    args = _chunk_args(q, k, v, out, lse)
    if lse is None:
        raise XditError(-1, "lse is required")
    B, Nq, H, d = q.shape
    for t, n, like, accum in ((dout, "dout", q, False), (dq, "dq", q, accum_dq), (dk, "dk", k, accum_dkv),
                              (dv, "dv", k, accum_dkv)):
        if t is None:
            raise XditError(-1, f"{n} is required")
        _dense(t, n, 4)
        if tuple(t.shape) != tuple(like.shape):
            raise XditError(-3, f"{n} has shape {tuple(t.shape)}, expected {tuple(like.shape)}")
        if t.dtype != (torch.float32 if accum else q.dtype):
            raise XditError(-2, f"{n} has dtype {t.dtype}, expected {torch.float32 if accum else q.dtype}")
    _dense(dlse, "dlse", 3)
    if dlse is not None and (dlse.dtype != torch.float32 or tuple(dlse.shape) != (B, H, Nq)):
        raise XditError(-3, f"dlse must be float32 [B,H,Nq] = {(B, H, Nq)}")
    for t, n in ((q, "q"), (k, "k"), (v, "v"), (out, "out"), (lse, "lse"), (dout, "dout"), (dq, "dq"), (dk, "dk"), (dv, "dv"),
                 (dlse, "dlse"), (workspace, "workspace")):
        if t is not None:
            _on_device(t, n)
    wp, wb = _workspace(workspace)
    _use_current_stream()
    check(lib().xdit_chunk_attn_bwd(*args[:5], _ptr(dout), _ptr(dlse), _ptr(dq), _ptr(dk), _ptr(dv),
                                    (XDIT_ACCUM_DQ if accum_dq else 0) | (XDIT_ACCUM_DKV if accum_dkv else 0), wp, wb,
                                    *args[5:]))
