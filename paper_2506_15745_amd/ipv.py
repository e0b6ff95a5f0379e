"""Python binding of ``libipv.so`` (ctypes; argument marshalling only).

Every function here passes device pointers of torch tensors, sizes and the
current HIP stream to the C ABI declared in ``include/ipv.h``; all of the
pass's work runs in the library's HIP kernels. Importing works anywhere, but
the first call loads ``libipv.so`` and raises :class:`IpvError` when it has
not been built -- there is no fallback implementation.

Tensor layouts (all contiguous, on the same GPU):
  K, V        [B, L, H, S, D]  torch.bfloat16 or torch.float32
  frame_idx   [B, L, H, S]     torch.int32
  patch_idx   [B, L, H, S]     torch.int32
  tar, van    [B, L, H, S]     torch.float32
  keep_idx    [B, L, H, C]     torch.int32
  pool_size   [B, L]           torch.int32
The paged cache (:class:`PagePool`, ``ipv_page_write``, ``ipv_page_read``,
``ipv_attend``) takes rows and queries of any strides whose last dimension is
contiguous; its layouts stand at those functions.
"""
from __future__ import annotations

import ctypes
import functools
import os
from array import array

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libipv.so")

OK, ERR_NULL, ERR_ALIGN, ERR_SHAPE, ERR_DTYPE, ERR_BUDGET, ERR_ARG, ERR_WORKSPACE, ERR_HIP = range(9)
BF16, F32 = 0, 1
DEV_BAD_PATCH, DEV_BAD_FRAMES, DEV_RECENT_OVER, DEV_BAD_KEEP, DEV_NAN, DEV_WAIT_TIMEOUT, DEV_BAD_PAGE = 1, 2, 4, 8, 16, 32, 64
# `mode` bits: reversed TaR / VaN stages, consecutive-frame TaR, head-shared
# selection, Uniform Select (frames at regular intervals, no scores)
TAR_REVERSE, VAN_REVERSE, TAR_ADJACENT, HEAD_SHARED, UNIFORM_SELECT = 1, 2, 4, 8, 16

# page formats (a pool's K and V: bf16, fp32, e4m3 or e2m1 elements with a scale for each 32)
PAGES_BF16, PAGES_F32, PAGES_FP8, PAGES_FP4 = range(4)
SCALE_BLOCK = 32

PAGED_EXPORTS = ("ipv_page_write", "ipv_page_read", "ipv_attend_workspace_bytes", "ipv_attend", "ipv_qkv_write",
                 "ipv_block_bounds", "ipv_blocks_workspace_bytes", "ipv_block_select", "ipv_attend_blocks", "ipv_page_compact",
                 "ipv_page_copy")
EXPORTS = PAGED_EXPORTS + (
           "ipv_workspace_bytes", "ipv_tar_scores", "ipv_van_scores", "ipv_select", "ipv_compact",
           "ipv_compress", "ipv_compress_timed", "ipv_compress_noalloc", "ipv_append", "ipv_ckv_step", "ipv_ckv_stream",
           "ipv_clear_device_errors",
           "ipv_read_device_errors", "ipv_status_str")


class IpvError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__("%s: %s (status %d)" % (what, status_str(status), status))


class Shape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("streams", "layers", "kv_heads", "head_dim", "capacity", "grid_h", "grid_w", "dtype")]


class PageShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("pages", "layers", "kv_heads", "page_rows", "head_dim", "format")]


class Events(ctypes.Structure):
    """hipEvent_t handles recorded at the pass's step boundaries (see ipv.h)."""
    _fields_ = [("at", ctypes.c_void_p * 6)]

    def __init__(self, *handles):
        super().__init__()
        for i, h in enumerate(handles):
            self.at[i] = h


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded library (raises IpvError if it is not built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise IpvError(ERR_HIP, "libipv.so is not built (run paper_2506_15745_amd.build)")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, f64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_double, ctypes.c_size_t
        sp = ctypes.POINTER(Shape)
        L.ipv_workspace_bytes.argtypes = [sp, ctypes.POINTER(ctypes.c_size_t)]
        u32 = ctypes.c_uint32
        ns = ctypes.POINTER(i32)  # host array of B row counts
        L.ipv_tar_scores.argtypes = [sp, vp, vp, vp, ns, i32, u32, vp, vp, sz, vp]
        L.ipv_van_scores.argtypes = [sp, vp, vp, vp, ns, vp, vp, vp, vp, sz, vp]
        L.ipv_select.argtypes = [sp, vp, vp, vp, ns, i32, f64, i32, u32, vp, vp, sz, vp]
        L.ipv_compact.argtypes = [sp, vp, vp, vp, vp, ns, vp, i32, vp, sz, vp]
        L.ipv_compress.argtypes = [sp, vp, vp, vp, vp, ns, i32, f64, i32, u32, vp, vp, vp, vp, vp, sz, vp]
        L.ipv_compress_timed.argtypes = [sp, vp, vp, vp, vp, ns, i32, f64, i32, u32, vp, vp, vp, vp, vp, sz, vp,
                                         ctypes.POINTER(Events)]
        L.ipv_compress_noalloc.argtypes = [sp, vp, vp, vp, vp, ns, i32, f64, i32, u32, vp, vp, vp, vp, vp, vp]
        L.ipv_append.argtypes = [sp, vp, vp, vp, vp, ns, vp, vp, i32, i32, i32, vp]
        L.ipv_ckv_step.argtypes = [sp, vp, vp, vp, vp, ns, vp, vp, i32, i32, i32, i32, i32, f64, i32, u32, vp, vp, vp,
                                   vp, vp, sz, ns, ns, vp]
        L.ipv_ckv_stream.argtypes = [sp, vp, vp, vp, vp, ns, vp, vp, i32, i32, i32, i32, i32, f64, i32, u32, vp, vp,
                                     vp, vp, vp, sz, ns, vp]
        L.ipv_clear_device_errors.argtypes = [vp, sz, vp]
        L.ipv_read_device_errors.argtypes = [vp, sz, vp, ctypes.POINTER(ctypes.c_uint32)]
        L.ipv_status_str.argtypes = [ctypes.c_int]
        L.ipv_status_str.restype = ctypes.c_char_p
        for name in EXPORTS[len(PAGED_EXPORTS):-1]:
            getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


_paged_lib = None


def _paged() -> ctypes.CDLL:
    """The library with the paged cache's calls described."""
    global _paged_lib
    L = lib()
    if _paged_lib is not L:
        vp, i32, f64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_double, ctypes.c_size_t
        ps = ctypes.POINTER(PageShape)
        rows = [ps, vp, vp, vp, vp, vp, i32, i32, vp, vp, i32, i32, vp, vp, i32, vp, vp, i32, vp, sz, vp]
        L.ipv_page_write.argtypes = rows
        L.ipv_page_read.argtypes = rows
        L.ipv_attend_workspace_bytes.argtypes = [ps, i32, i32, i32, ctypes.POINTER(ctypes.c_size_t)]
        L.ipv_attend.argtypes = [ps, vp, vp, vp, vp, vp, i32, i32, vp, vp, vp, i32, vp, vp, i32, i32, f64, i32, i32, vp,
                                 vp, vp, vp, sz, vp]
        L.ipv_qkv_write.argtypes = [ps, vp, vp, vp, vp, vp, i32, vp, i32, i32, vp, vp, i32, vp, vp, i32, vp, vp, vp, i32, vp, vp, f64,
                                    vp, i32, vp, vp, vp, sz, vp]
        L.ipv_block_bounds.argtypes = [ps, vp, vp, vp, i32, vp, i32, i32, vp, vp, i32, i32, vp, sz, vp]
        L.ipv_blocks_workspace_bytes.argtypes = [ps, i32, i32, i32, i32, i32, i32, ctypes.POINTER(ctypes.c_size_t)]
        L.ipv_block_select.argtypes = [ps, vp, i32, vp, i32, i32, vp, vp, vp, i32, vp, vp, i32, i32, i32, i32, i32, vp, vp, sz, vp]
        L.ipv_attend_blocks.argtypes = [ps, vp, vp, vp, vp, vp, i32, vp, i32, i32, vp, vp, vp, i32, vp, vp, i32, i32, f64, i32, i32,
                                        i32, vp, vp, vp, vp, vp, sz, vp]
        L.ipv_page_compact.argtypes = [ps, vp, vp, vp, vp, vp, i32, vp, i32, vp, i32, i32, vp, vp, i32, vp, vp, i32, vp, sz, vp]
        L.ipv_page_copy.argtypes = [ps, vp, vp, vp, vp, vp, i32, vp, vp, i32, i32, vp, sz, vp]
        for name in PAGED_EXPORTS:
            getattr(L, name).restype = ctypes.c_int
        _paged_lib = L
    return L


def status_str(status: int) -> str:
    if _lib is None and not os.path.exists(LIB_PATH):
        return "status %d" % status
    return lib().ipv_status_str(status).decode()


def _check(rc: int, what: str):
    if rc != OK:
        raise IpvError(rc, what)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise IpvError(ERR_DTYPE, "K/V dtype %s" % t.dtype)


def shape_of(K: torch.Tensor, grid_h: int, grid_w: int) -> Shape:
    if K.dim() != 5:
        raise IpvError(ERR_SHAPE, "K must be [B, L, H, S, D]")
    B, L, H, S, D = K.shape
    return Shape(B, L, H, D, S, grid_h, grid_w, _dtype_code(K))


@functools.lru_cache(maxsize=256)
def _shape(B, L, H, D, S, grid_h, grid_w, dtype) -> Shape:
    """A Shape for the library to read (shared: never handed to a caller)."""
    return Shape(B, L, H, D, S, grid_h, grid_w, dtype)


def _ptr(t):
    if t is None:
        return None
    if t.is_cuda and t.is_contiguous():
        return t.data_ptr()
    if t.device.type != "cuda":
        raise IpvError(ERR_ARG, "tensors must be in GPU memory (got %s)" % t.device)
    if not t.is_contiguous():
        raise IpvError(ERR_SHAPE, "tensors must be contiguous")
    return t.data_ptr()


def _expect(what, t, shape, dtype, device, optional=False):
    """Refuse a companion tensor whose shape, dtype or device does not match
    the cache: the library only sees pointers, so a smaller buffer would be
    written past its end."""
    if t is None:
        if optional:
            return
        raise IpvError(ERR_NULL, "%s is required" % what)
    if t.dtype is dtype and t.shape == shape and t.device == device:
        return
    if t.dtype != dtype:
        raise IpvError(ERR_DTYPE, "%s must be %s (got %s)" % (what, dtype, t.dtype))
    if tuple(t.shape) != tuple(shape):
        raise IpvError(ERR_SHAPE, "%s must have shape %s (got %s)" % (what, tuple(shape), tuple(t.shape)))
    if t.device != device:
        raise IpvError(ERR_ARG, "%s is on %s, the cache on %s" % (what, t.device, device))


def _check_meta(K, frame_idx, patch_idx):
    """frame_idx / patch_idx: int32 [B, L, H, S] beside K [B, L, H, S, D]."""
    rows = tuple(K.shape[:4])
    _expect("frame_idx", frame_idx, rows, torch.int32, K.device)
    _expect("patch_idx", patch_idx, rows, torch.int32, K.device)


def _check_scores(ref, device, tar=None, van=None, optional=False):
    """tar / van: fp32 [B, L, H, S]."""
    _expect("tar", tar, ref, torch.float32, device, optional)
    _expect("van", van, ref, torch.float32, device, optional)


def _check_keep(keep_idx, rows, budget, device, optional=False):
    """keep_idx: int32 [B, L, H, budget]."""
    _expect("keep_idx", keep_idx, tuple(rows[:3]) + (int(budget),), torch.int32, device, optional)


def _check_ws(ws, device, optional=False):
    if ws is None:
        if optional:
            return
        raise IpvError(ERR_WORKSPACE, "a workspace is required")
    if ws.device != device:
        raise IpvError(ERR_ARG, "the workspace is on %s, the cache on %s" % (ws.device, device))


def _ws_bytes(ws):
    return 0 if ws is None else ws.numel() * ws.element_size()


def _check_cache(K, V, frame_idx, patch_idx):
    """V like K; the metadata beside them."""
    _expect("V", V, tuple(K.shape), K.dtype, K.device)
    _check_meta(K, frame_idx, patch_idx)


def _check_pass_buffers(K, V, frame_idx, patch_idx, tar, van, keep_idx, budget, ws, optional=False,
                        need_ws=True, mode=0):
    """Every buffer of a whole pass against the cache K [B, L, H, S, D];
    optional: the score, keep and workspace buffers may be None (the
    continual-compression calls need them only when a pass runs)."""
    _check_cache(K, V, frame_idx, patch_idx)
    _check_scores(K.shape[:4], K.device, tar, van, optional or bool(mode & UNIFORM_SELECT))
    _check_keep(keep_idx, K.shape, budget, K.device, optional)
    if need_ws:
        _check_ws(ws, K.device, optional)


# A call's host time is its checks: 21 us for ipv_ckv_step when every tensor's
# shape, dtype and device went through _expect and the pointers through _ptr, 12.6 us
# with the whole set read once here. (A frame's append takes 8 us on the GPU.)
def _pass_ptrs(K, V, frame_idx, patch_idx, tar, van, keep_idx, budget, ws, grid_h, grid_w):
    """(shape, device, K, V, frame_idx, patch_idx, tar, van, keep_idx, ws) as
    the library takes them, or None when a check fails or a buffer is missing:
    the checks one by one then say whether that is an error and which."""
    if (V is None or frame_idx is None or patch_idx is None or tar is None or van is None or keep_idx is None or ws is None
            or type(grid_h) is not int or type(grid_w) is not int):  # _shape keeps results by value: 4.0 is equal to 4
        return None
    kd, dev, kv = K.dtype, K.get_device(), K.shape
    code = BF16 if kd is torch.bfloat16 else F32 if kd is torch.float32 else -1
    if code < 0 or dev < 0 or len(kv) != 5:
        return None
    B, L, H, S, D = kv
    rows, i32, f32 = (B, L, H, S), torch.int32, torch.float32
    if (V.dtype is kd and frame_idx.dtype is i32 and patch_idx.dtype is i32 and tar.dtype is f32 and van.dtype is f32
            and keep_idx.dtype is i32 and V.shape == kv and frame_idx.shape == rows and patch_idx.shape == rows
            and tar.shape == rows and van.shape == rows and keep_idx.shape == (B, L, H, int(budget))
            and V.get_device() == dev and frame_idx.get_device() == dev and patch_idx.get_device() == dev
            and tar.get_device() == dev and van.get_device() == dev and keep_idx.get_device() == dev
            and ws.get_device() == dev and K.is_cuda and K.is_contiguous() and V.is_contiguous()
            and frame_idx.is_contiguous() and patch_idx.is_contiguous() and tar.is_contiguous()
            and van.is_contiguous() and keep_idx.is_contiguous() and ws.is_contiguous()):
        return (_shape(B, L, H, D, S, grid_h, grid_w, code), dev, K.data_ptr(), V.data_ptr(), frame_idx.data_ptr(),
                patch_idx.data_ptr(), tar.data_ptr(), van.data_ptr(), keep_idx.data_ptr(), ws.data_ptr())
    return None


def _checked_ptrs(K, V, frame_idx, patch_idx, tar, van, keep_idx, budget, ws, grid_h, grid_w, mode, optional=False):
    """(shape, K, V, frame_idx, patch_idx, tar, van, keep_idx, ws), every check made."""
    got = _pass_ptrs(K, V, frame_idx, patch_idx, tar, van, keep_idx, budget, ws, grid_h, grid_w)
    if got is not None:
        return got[:1] + got[2:]
    s = shape_of(K, grid_h, grid_w)
    _check_pass_buffers(K, V, frame_idx, patch_idx, tar, van, keep_idx, budget, ws, optional=optional, mode=mode)
    return (s, _ptr(K), _ptr(V), _ptr(frame_idx), _ptr(patch_idx), _ptr(tar), _ptr(van), _ptr(keep_idx), _ptr(ws))


def _check_new_rows(K, K_new, V_new):
    """K_new / V_new: [B, L, H, rows, D] with the cache's dtype."""
    if K_new.dtype != K.dtype or V_new.dtype != K.dtype:
        raise IpvError(ERR_DTYPE, "K_new/V_new must have the cache's dtype")
    if K_new.shape != V_new.shape or K_new.dim() != 5 or K_new.shape[:3] != K.shape[:3] \
            or K_new.shape[4] != K.shape[4]:
        raise IpvError(ERR_SHAPE, "K_new/V_new must be [B, L, H, rows, D] like the cache")


def counts(n_tokens, streams: int):
    """Host array of per-stream row counts from an int (every stream) or a sequence."""
    if isinstance(n_tokens, int):
        vals = [n_tokens] * streams
    else:
        vals = [int(v) for v in n_tokens]
        if len(vals) != streams:
            raise IpvError(ERR_SHAPE, "n_tokens needs one count per stream (%d)" % streams)
    return (ctypes.c_int32 * streams)(*vals)


def _stream(stream):
    if stream is None:
        if torch.cuda.is_initialized():  # the handle of torch.cuda.current_stream(), without the object
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def workspace_bytes(shape: Shape) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().ipv_workspace_bytes(ctypes.byref(shape), ctypes.byref(out)), "ipv_workspace_bytes")
    return out.value


def alloc_workspace(shape: Shape, device) -> torch.Tensor:
    """A zeroed workspace tensor (uint8) for calls on `shape`."""
    return torch.zeros(workspace_bytes(shape), dtype=torch.uint8, device=device)


def ipv_tar_scores(K, frame_idx, patch_idx, n_tokens, recent_frames, tar, ws, grid_h, grid_w, stream=None, mode=0):
    s = shape_of(K, grid_h, grid_w)
    _check_meta(K, frame_idx, patch_idx)
    _expect("tar", tar, K.shape[:4], torch.float32, K.device)
    _check_ws(ws, K.device)
    _check(lib().ipv_tar_scores(ctypes.byref(s), _ptr(K), _ptr(frame_idx), _ptr(patch_idx), counts(n_tokens, s.streams),
                                recent_frames, mode, _ptr(tar), _ptr(ws), _ws_bytes(ws), _stream(stream)),
           "ipv_tar_scores")


def ipv_van_scores(V, frame_idx, patch_idx, n_tokens, cv_tau, van, pool_size, ws, grid_h, grid_w, stream=None):
    s = shape_of(V, grid_h, grid_w)
    _check_meta(V, frame_idx, patch_idx)
    _expect("van", van, V.shape[:4], torch.float32, V.device)
    _expect("pool_size", pool_size, V.shape[:2], torch.int32, V.device, optional=True)
    _check_ws(ws, V.device)
    tau = None if cv_tau is None else (ctypes.c_double * 3)(*cv_tau)
    _check(lib().ipv_van_scores(ctypes.byref(s), _ptr(V), _ptr(frame_idx), _ptr(patch_idx), counts(n_tokens, s.streams),
                                None if tau is None else ctypes.addressof(tau), _ptr(van), _ptr(pool_size),
                                _ptr(ws), _ws_bytes(ws), _stream(stream)), "ipv_van_scores")


def ipv_select(tar, van, frame_idx, n_tokens, budget, alpha, recent_frames, keep_idx, ws, grid_h, grid_w,
               head_dim=128, dtype=BF16, stream=None, mode=0):
    """The select step needs only the slice geometry: (B, L, H, S) from
    frame_idx and the patch grid; head_dim/dtype only size the workspace.
    With UNIFORM_SELECT in mode, tar and van may be None."""
    if frame_idx.dim() != 4:
        raise IpvError(ERR_SHAPE, "frame_idx must be [B, L, H, S]")
    B, L, H, S = frame_idx.shape
    s = Shape(B, L, H, head_dim, S, grid_h, grid_w, dtype)
    _expect("frame_idx", frame_idx, frame_idx.shape, torch.int32, frame_idx.device)
    _check_scores(frame_idx.shape, frame_idx.device, tar, van, optional=bool(mode & UNIFORM_SELECT))
    _check_keep(keep_idx, frame_idx.shape, budget, frame_idx.device)
    _check_ws(ws, frame_idx.device)
    _check(lib().ipv_select(ctypes.byref(s), _ptr(tar), _ptr(van), _ptr(frame_idx), counts(n_tokens, B), budget,
                            float(alpha), recent_frames, mode, _ptr(keep_idx), _ptr(ws), _ws_bytes(ws),
                            _stream(stream)),
           "ipv_select")


def ipv_compact(K, V, frame_idx, patch_idx, n_tokens, keep_idx, budget, ws, grid_h, grid_w, stream=None):
    s = shape_of(K, grid_h, grid_w)
    _check_cache(K, V, frame_idx, patch_idx)
    _check_keep(keep_idx, K.shape, budget, K.device)
    _check_ws(ws, K.device)
    _check(lib().ipv_compact(ctypes.byref(s), _ptr(K), _ptr(V), _ptr(frame_idx), _ptr(patch_idx),
                             counts(n_tokens, s.streams),
                             _ptr(keep_idx), budget, _ptr(ws), _ws_bytes(ws), _stream(stream)),
           "ipv_compact")


def ipv_compress(K, V, frame_idx, patch_idx, n_tokens, budget, alpha, recent_frames, cv_tau, tar, van, keep_idx,
                 ws, grid_h, grid_w, stream=None, mode=0):
    s, k, v, fr, pa, tr, vn, keep, w = _checked_ptrs(K, V, frame_idx, patch_idx, tar, van, keep_idx, budget, ws, grid_h,
                                                     grid_w, mode)
    tau = None if cv_tau is None else (ctypes.c_double * 3)(*cv_tau)
    _check(lib().ipv_compress(ctypes.byref(s), k, v, fr, pa, counts(n_tokens, s.streams), budget, float(alpha),
                              recent_frames, mode, None if tau is None else ctypes.addressof(tau), tr, vn, keep, w,
                              _ws_bytes(ws), _stream(stream)), "ipv_compress")


def ipv_compress_timed(K, V, frame_idx, patch_idx, n_tokens, budget, alpha, recent_frames, cv_tau, tar, van,
                       keep_idx, ws, grid_h, grid_w, events: Events, stream=None, mode=0):
    s = shape_of(K, grid_h, grid_w)
    _check_pass_buffers(K, V, frame_idx, patch_idx, tar, van, keep_idx, budget, ws, mode=mode)
    tau = None if cv_tau is None else (ctypes.c_double * 3)(*cv_tau)
    _check(lib().ipv_compress_timed(ctypes.byref(s), _ptr(K), _ptr(V), _ptr(frame_idx), _ptr(patch_idx),
                                    counts(n_tokens, s.streams),
                                    budget, float(alpha), recent_frames, mode,
                                    None if tau is None else ctypes.addressof(tau), _ptr(tar), _ptr(van),
                                    _ptr(keep_idx), _ptr(ws), _ws_bytes(ws), _stream(stream), ctypes.byref(events)),
           "ipv_compress_timed")


def ipv_compress_noalloc(K, V, frame_idx, patch_idx, n_tokens, budget, alpha, recent_frames, cv_tau, tar, van,
                         keep_idx, grid_h, grid_w, device_errors=None, stream=None, mode=0):
    """ipv_compress with the library's own per-GPU workspace (no workspace
    argument, nothing allocated by the call); device_errors: an int32/uint32
    device tensor of one element that receives the pass's error word, or None."""
    s = shape_of(K, grid_h, grid_w)
    _check_pass_buffers(K, V, frame_idx, patch_idx, tar, van, keep_idx, budget, None, need_ws=False, mode=mode)
    if device_errors is not None and (device_errors.numel() != 1 or device_errors.element_size() != 4
                                      or device_errors.device != K.device):
        raise IpvError(ERR_SHAPE, "device_errors must be one 4-byte element on the cache's device")
    tau = None if cv_tau is None else (ctypes.c_double * 3)(*cv_tau)
    _check(lib().ipv_compress_noalloc(ctypes.byref(s), _ptr(K), _ptr(V), _ptr(frame_idx), _ptr(patch_idx),
                                      counts(n_tokens, s.streams), budget, float(alpha), recent_frames, mode,
                                      None if tau is None else ctypes.addressof(tau), _ptr(tar), _ptr(van),
                                      _ptr(keep_idx), _ptr(device_errors), _stream(stream)),
           "ipv_compress_noalloc")


def ipv_append(K, V, frame_idx, patch_idx, n_tokens, K_new, V_new, frame_id, first_patch, grid_h, grid_w,
               stream=None):
    """Append K_new/V_new ([B, L, H, rows, D]) after row n_tokens[b] of every
    slice of stream b; returns the new row count(s) (an int for an int
    n_tokens, else a list)."""
    s = shape_of(K, grid_h, grid_w)
    _check_cache(K, V, frame_idx, patch_idx)
    _check_new_rows(K, K_new, V_new)
    rows = K_new.shape[3]
    ns = counts(n_tokens, s.streams)
    _check(lib().ipv_append(ctypes.byref(s), _ptr(K), _ptr(V), _ptr(frame_idx), _ptr(patch_idx), ns,
                            _ptr(K_new), _ptr(V_new), rows, frame_id, first_patch, _stream(stream)), "ipv_append")
    return n_tokens + rows if isinstance(n_tokens, int) else [v + rows for v in ns]


def ipv_ckv_step(K, V, frame_idx, patch_idx, n_tokens, K_new, V_new, frame_id, first_patch, mem_cap, budget,
                 alpha, recent_frames, cv_tau, tar, van, keep_idx, ws, grid_h, grid_w, stream=None, mode=0):
    """Append, then compress to `budget` every stream that holds >= mem_cap
    rows. Returns (row counts, whether each stream's pass ran): ints for an
    int n_tokens (every stream then behaves alike), else lists."""
    got = _pass_ptrs(K, V, frame_idx, patch_idx, tar, van, keep_idx, budget, ws, grid_h, grid_w)
    new = K_new.shape if got is not None else ()
    if (len(new) == 5 and V_new.shape == new and K_new.dtype is K.dtype and V_new.dtype is K.dtype
            and (new[0], new[1], new[2], new[4]) == (got[0].streams, got[0].layers, got[0].kv_heads, got[0].head_dim)
            and K_new.get_device() == got[1] and V_new.get_device() == got[1] and K_new.is_contiguous()
            and V_new.is_contiguous()):
        s, _, k, v, fr, pa, tr, vn, keep, w = got
        kn, vnew = K_new.data_ptr(), V_new.data_ptr()
    else:
        s = shape_of(K, grid_h, grid_w)
        _check_cache(K, V, frame_idx, patch_idx)
        _check_new_rows(K, K_new, V_new)
        s, k, v, fr, pa, tr, vn, keep, w = _checked_ptrs(K, V, frame_idx, patch_idx, tar, van, keep_idx, budget, ws,
                                                         grid_h, grid_w, mode, optional=True)
        new, kn, vnew = K_new.shape, _ptr(K_new), _ptr(V_new)
    tau = None if cv_tau is None else (ctypes.c_double * 3)(*cv_tau)
    out = (ctypes.c_int32 * s.streams)
    n_out, comp = out(), out()
    _check(lib().ipv_ckv_step(ctypes.byref(s), k, v, fr, pa, counts(n_tokens, s.streams), kn, vnew, new[3], frame_id,
                              first_patch, mem_cap, budget, float(alpha), recent_frames, mode,
                              None if tau is None else ctypes.addressof(tau), tr, vn, keep, w, _ws_bytes(ws), n_out,
                              comp, _stream(stream)), "ipv_ckv_step")
    if isinstance(n_tokens, int):
        return n_out[0], bool(comp[0])
    return list(n_out), [bool(c) for c in comp]


def ipv_ckv_stream(K, V, frame_idx, patch_idx, n_tokens, frames_K, frames_V, first_frame_id, mem_cap, budget,
                   alpha, recent_frames, cv_tau, tar, van, keep_idx, ws, grid_h, grid_w, stream=None, mode=0):
    """Frames frames_K/V[f] ([F, B, L, H, rows, D]) through ipv_ckv_step one
    after another in one library call. Returns (row counts, passes per
    stream): ints for an int n_tokens, else lists."""
    s = shape_of(K, grid_h, grid_w)
    _check_cache(K, V, frame_idx, patch_idx)
    if frames_K.dtype != K.dtype or frames_V.dtype != K.dtype:
        raise IpvError(ERR_DTYPE, "frames_K/V must have the cache's dtype")
    if frames_K.shape != frames_V.shape or frames_K.dim() != 6 or frames_K.shape[1:4] != K.shape[:3] \
            or frames_K.shape[5] != K.shape[4]:
        raise IpvError(ERR_SHAPE, "frames_K/V must be [F, B, L, H, rows, D] like the cache")
    s, k, v, fr, pa, tr, vn, keep, w = _checked_ptrs(K, V, frame_idx, patch_idx, tar, van, keep_idx, budget, ws, grid_h,
                                                     grid_w, mode, optional=True)
    tau = None if cv_tau is None else (ctypes.c_double * 3)(*cv_tau)
    ns = counts(n_tokens, s.streams)
    passes = (ctypes.c_int32 * s.streams)()
    _check(lib().ipv_ckv_stream(ctypes.byref(s), k, v, fr, pa, ns, _ptr(frames_K), _ptr(frames_V), frames_K.shape[0],
                                frames_K.shape[4], first_frame_id, mem_cap, budget, float(alpha), recent_frames, mode,
                                None if tau is None else ctypes.addressof(tau), tr, vn, keep, w, _ws_bytes(ws), passes,
                                _stream(stream)), "ipv_ckv_stream")
    if isinstance(n_tokens, int):
        return ns[0], passes[0]
    return list(ns), list(passes)


def ipv_clear_device_errors(ws, stream=None):
    _check(lib().ipv_clear_device_errors(_ptr(ws), _ws_bytes(ws), _stream(stream)), "ipv_clear_device_errors")


def ipv_read_device_errors(ws, stream=None) -> int:
    out = ctypes.c_uint32(0)
    _check(lib().ipv_read_device_errors(_ptr(ws), _ws_bytes(ws), _stream(stream), ctypes.byref(out)),
           "ipv_read_device_errors")
    return out.value


# ---------------------------------------------------------------- paged cache
class PagePool:
    """Pages of cache rows: K, V [P, L, H, T, X] in GPU memory, contiguous, X = D
    elements of bf16 or fp32, or with K_scales, V_scales (uint8 [P, L, H, T,
    D / 32]) D bytes of e4m3 or D / 2 bytes of e2m1 elements (torch.uint8). A
    cache K, V [B, L, H, S, D] of this module is a pool of B pages of S rows (its
    calls then take page_table None)."""

    def __init__(self, K, V, K_scales=None, V_scales=None):
        if K.dim() != 5:
            raise IpvError(ERR_SHAPE, "K must be [P, L, H, T, X]")
        P, L, H, T, X = K.shape
        _expect("V", V, K.shape, K.dtype, K.device)
        if K.dtype == torch.uint8:
            if K_scales is None or V_scales is None:
                raise IpvError(ERR_NULL, "8- and 4-bit pages need K_scales and V_scales")
            if K_scales.dim() != 5:
                raise IpvError(ERR_SHAPE, "K_scales must be [P, L, H, T, D / 32]")
            D = K_scales.shape[4] * SCALE_BLOCK
            if X not in (D, D // 2):
                raise IpvError(ERR_SHAPE, "rows of %d bytes do not go with %d scales" % (X, K_scales.shape[4]))
            fmt = PAGES_FP8 if X == D else PAGES_FP4
            for what, t in (("K_scales", K_scales), ("V_scales", V_scales)):
                _expect(what, t, (P, L, H, T, D // SCALE_BLOCK), torch.uint8, K.device)
        else:
            if K_scales is not None or V_scales is not None:
                raise IpvError(ERR_ARG, "bf16 and fp32 pages have no scales")
            fmt, D = _dtype_code(K), X
        self._tensors = K, V, K_scales, V_scales
        self.format, self.head_dim, self.device = fmt, D, K.device
        self.dtype = torch.float32 if fmt == PAGES_F32 else torch.bfloat16  # of queries and outputs
        self.shape = PageShape(P, L, H, T, D, fmt)
        self._dev = K.get_device()
        self._args = (ctypes.byref(self.shape), _ptr(K), _ptr(V), _ptr(K_scales), _ptr(V_scales))

    # not to be replaced: their addresses are made into arguments once
    K = property(lambda self: self._tensors[0])
    V = property(lambda self: self._tensors[1])
    K_scales = property(lambda self: self._tensors[2])
    V_scales = property(lambda self: self._tensors[3])

    @classmethod
    def empty(cls, pages, layers, kv_heads, page_rows, head_dim, format, device="cuda"):  # noqa: A002
        """A pool of zeroed pages."""
        rows = (pages, layers, kv_heads, page_rows)
        if format in (PAGES_BF16, PAGES_F32):
            kind = torch.bfloat16 if format == PAGES_BF16 else torch.float32
            return cls(*(torch.zeros(rows + (head_dim,), dtype=kind, device=device) for _ in range(2)))
        if format not in (PAGES_FP8, PAGES_FP4):
            raise IpvError(ERR_DTYPE, "page format %r" % (format,))
        width = (head_dim, head_dim, head_dim // SCALE_BLOCK, head_dim // SCALE_BLOCK) if format == PAGES_FP8 else \
            (head_dim // 2, head_dim // 2, head_dim // SCALE_BLOCK, head_dim // SCALE_BLOCK)
        return cls(*(torch.zeros(rows + (w,), dtype=torch.uint8, device=device) for w in width))


# What these calls cost on the host is their checks and conversions: counts go through
# array (a third of a ctypes array's time), stride arrays are kept by value, and a
# pool's own arguments are made with it.
def _host_counts(values, streams, what):
    """A host array with one count per stream, from an int or a sequence."""
    try:
        if isinstance(values, int):
            return array("i", (values,) * streams)
        if len(values) != streams:
            raise IpvError(ERR_SHAPE, "%s needs one count per stream (%d)" % (what, streams))
        return array("i", values)
    except OverflowError:
        raise IpvError(ERR_SHAPE, "%s holds a count of more than 32 bits" % what) from None


def _query_counts(q_rows, streams, most):
    """A host array of each stream's queries (None: all). The library sees one at the least as the most that there are: tensors
    of none are checked here."""
    rows = _host_counts(most if q_rows is None else q_rows, streams, "q_rows")
    if most == 0 and any(rows):
        raise IpvError(ERR_SHAPE, "more queries than the tensor's 0")
    return rows


_I32 = 2**31


def _whole32(what, *values):
    """Refuse what ctypes would cut to its low 32 bits."""
    for v in values:
        if not -_I32 <= v < _I32:
            raise IpvError(ERR_ARG, "%s: %d has more than 32 bits" % (what, v))


def _table(pool, table, streams):
    """(pointer, columns) of a page table [B, cols], or of none (stream b's rows are page b)."""
    if table is None:
        return None, 1
    shape = table.shape
    if table.dtype is not torch.int32 or len(shape) != 2 or shape[0] != streams:
        raise IpvError(ERR_SHAPE, "page_table must be int32 [%d, columns]" % streams)
    if table.get_device() != pool._dev:
        raise IpvError(ERR_ARG, "page_table is on %s, the pool on %s" % (table.device, pool.device))
    return _ptr(table), shape[1]


@functools.lru_cache(maxsize=256)
def _stride_array(strides, sizes):
    """Strides (elements) of all but the last dimension, which must be contiguous; 0 for a dimension of one."""
    if strides[-1] != 1:
        raise IpvError(ERR_SHAPE, "the last dimension of rows and queries must be contiguous")
    return (ctypes.c_int64 * (len(sizes) - 1))(*[st if n > 1 else 0 for st, n in zip(strides[:-1], sizes)])


def _not_expanded(what, strides, sizes):
    """Refuse a result's place whose elements are the same memory."""
    if any(st == 0 and n > 1 for st, n in zip(strides, sizes)):
        raise IpvError(ERR_SHAPE, "%s is written and must not be an expanded tensor" % what)


def _same_gpu(pool, ws, **tensors):
    dev = pool.K.get_device()
    for what, t in tensors.items():
        if t is not None and t.get_device() != dev:
            raise IpvError(ERR_ARG, "%s is on %s, the pool on %s" % (what, t.device, pool.device))
    if ws is None:
        raise IpvError(ERR_WORKSPACE, "a workspace is required")
    if ws.get_device() != dev:
        raise IpvError(ERR_ARG, "the workspace is on %s, the pool on %s" % (ws.device, pool.device))


def alloc_page_workspace(device) -> torch.Tensor:
    """A zeroed workspace for ipv_page_write and ipv_page_read (the device error word)."""
    return torch.zeros(256, dtype=torch.uint8, device=device)


def attend_workspace_bytes(pool: PagePool, streams: int, q_heads: int, max_rows: int) -> int:
    _whole32("ipv_attend_workspace_bytes", streams, q_heads, max_rows)
    out = ctypes.c_size_t(0)
    _check(_paged().ipv_attend_workspace_bytes(pool._args[0], streams, q_heads, max_rows, ctypes.byref(out)),
           "ipv_attend_workspace_bytes")
    return out.value


def alloc_attend_workspace(pool: PagePool, streams: int, q_heads: int, max_rows: int) -> torch.Tensor:
    """A workspace for ipv_attend calls of at most these sizes: zeros where it has to be."""
    ws = torch.empty(attend_workspace_bytes(pool, streams, q_heads, max_rows), dtype=torch.uint8, device=pool.device)
    ws[:4352] = 0
    return ws


def _page_rows(name, pool, page_table, first_row, K, V, ws, rows, first_layer, rotary, stream):
    shape, dev, table, cols, angles = K.shape, pool._dev, None, 1, 0
    if len(shape) != 5 or V.shape != shape or shape[2] != pool.shape.kv_heads or shape[4] != pool.head_dim:
        raise IpvError(ERR_SHAPE, "K and V must be [B, layers, %d, rows, %d]" % (pool.shape.kv_heads, pool.head_dim))
    if V.dtype is not K.dtype:
        raise IpvError(ERR_DTYPE, "K and V must have one dtype")
    B, L, _, N, D = shape
    strides = _stride_array(k_strides := K.stride(), shape)
    if V.stride() != k_strides and list(_stride_array(V.stride(), shape)) != list(strides):
        raise IpvError(ERR_SHAPE, "K and V must have the same strides")
    if 0 in k_strides and name == "ipv_page_read":
        _not_expanded("K, V", k_strides, shape)
    if rows is None:
        rows = N
    elif (rows if isinstance(rows, int) else max(rows, default=0)) > N:
        raise IpvError(ERR_SHAPE, "more rows than the tensor's %d" % N)
    if rotary is not None:
        if rotary.dtype is not torch.float32 or rotary.dim() != 3 or tuple(rotary.shape[1:]) != (D // 2, 2):
            raise IpvError(ERR_SHAPE, "rotary must be fp32 [positions, %d, 2]" % (D // 2))
        angles = rotary.shape[0]
    if page_table is not None:
        table, cols = _table(pool, page_table, B)
    if ws is None or ws.get_device() != dev or K.get_device() != dev or V.get_device() != dev or \
            (rotary is not None and rotary.get_device() != dev):
        _same_gpu(pool, ws, K=K, V=V, rotary=rotary)
    first, counts_ = _host_counts(first_row, B, "first_row"), _host_counts(rows, B, "rows")
    if not -_I32 <= first_layer < _I32:
        _whole32("first_layer", first_layer)
    at = _ptr(ws)  # also stands for tensors without elements, whose own addresses are null
    rc = getattr(_paged(), name)(*pool._args, table, cols, B, first.buffer_info()[0], counts_.buffer_info()[0], first_layer, L,
                                 K.data_ptr() or at, V.data_ptr() or at, _dtype_code(K), strides,
                                 None if rotary is None else _ptr(rotary) or at, angles, at, ws.nbytes, _stream(stream))
    if rc != OK:
        _check(rc, name)


def ipv_page_write(pool, page_table, first_row, K, V, ws, rows=None, first_layer=0, rotary=None, stream=None):
    """Rows K/V ([B, layers, H, rows, D], bf16 or fp32) of layers first_layer, ...
    into the pool at positions first_row[b], first_row[b] + 1, ... (ints, or a
    sequence with one per stream; rows: all, or how many of each stream);
    rotary (fp32 [positions, D / 2, 2], cosine and sine) turns the keys to
    their positions. page_table: int32 [B, columns], or None."""
    _page_rows("ipv_page_write", pool, page_table, first_row, K, V, ws, rows, first_layer, rotary, stream)


def ipv_page_read(pool, page_table, first_row, K, V, ws, rows=None, first_layer=0, rotary=None, stream=None):
    """Rows of the pool into K/V (as for ipv_page_write), keys turned back where rotary is given."""
    _page_rows("ipv_page_read", pool, page_table, first_row, K, V, ws, rows, first_layer, rotary, stream)


def ipv_attend(pool, page_table, n_tokens, q_first, layer, q, out, ws, q_rows=None, scale=None, window=0, sinks=0,
               lse=None, stream=None):
    """Attention of q ([B, q_heads, M, D], in the pool's dtype) over the first
    n_tokens[b] rows of one layer, into out (the same shape); query i of stream b
    stands at position q_first[b] + i and sees the rows up to there, with a
    window only the last `window` of them and the first `sinks` rows. scale:
    1 / sqrt(D) if None. q_rows: queries of each stream (M if None). lse: fp32
    [B, q_heads, M] that receives the logarithm of each softmax's sum, or None."""
    shape, dev, table, cols = q.shape, pool._dev, None, 1
    if len(shape) != 4 or shape[3] != pool.head_dim:
        raise IpvError(ERR_SHAPE, "q must be [B, q_heads, rows, %d]" % pool.head_dim)
    if q.dtype is not pool.dtype or out.dtype is not pool.dtype:
        raise IpvError(ERR_DTYPE, "q and out must be %s" % pool.dtype)
    if out.shape != shape:
        raise IpvError(ERR_SHAPE, "out must have q's shape")
    B, A, M, D = shape
    if lse is not None:
        _expect("lse", lse, (B, A, M), torch.float32, pool.device)
    if page_table is not None:
        table, cols = _table(pool, page_table, B)
    if ws is None or ws.get_device() != dev or q.get_device() != dev or out.get_device() != dev:
        _same_gpu(pool, ws, q=q, out=out)
    n, first = _host_counts(n_tokens, B, "n_tokens"), _host_counts(q_first, B, "q_first")
    rows = _query_counts(q_rows, B, M)
    q_strides, out_strides = q.stride(), out.stride()
    q_at = _stride_array(q_strides, shape)
    if 0 in out_strides:
        _not_expanded("out", out_strides, shape)
    if not (-_I32 <= layer < _I32 and -_I32 <= window < _I32 and -_I32 <= sinks < _I32):
        _whole32("layer, window, sinks", layer, window, sinks)
    at = _ptr(ws)  # also stands for tensors without elements, whose own addresses are null
    rc = _paged().ipv_attend(*pool._args, table, cols, B, n.buffer_info()[0], first.buffer_info()[0], rows.buffer_info()[0],
                             layer, q.data_ptr() or at, q_at, A, M or 1, D ** -0.5 if scale is None else scale, window, sinks,
                             out.data_ptr() or at, q_at if out_strides == q_strides else _stride_array(out_strides, shape),
                             None if lse is None else _ptr(lse), at, ws.nbytes, _stream(stream))
    if rc != OK:
        _check(rc, "ipv_attend")


def _pool_stream(pool, stream):
    """The stream (the current one if None), which must be the pool's GPU's, that GPU being the current one."""
    if not torch.cuda.is_initialized():
        return _stream(stream)
    device = torch._C._cuda_getDevice()
    if device != pool._dev or (stream is not None and stream.device.index != device):
        raise IpvError(ERR_ARG, "the pool is on %s, the current device is %d, the stream %s" % (pool.device, device, stream))
    return torch._C._cuda_getCurrentRawStream(device) if stream is None else stream.cuda_stream


class BlockBounds:
    """Bounds of the keys of every block of `block_rows` rows of a pool's pages (a multiple of
    16 that divides their rows): values [P, L, H, T / block_rows, 2, D] in the pool's dtype, each
    channel's lowest and highest element (zeros until they are made)."""

    def __init__(self, pool: PagePool, block_rows: int, values=None):
        s = pool.shape
        if block_rows < 16 or block_rows % 16 or s.page_rows % block_rows:
            raise IpvError(ERR_SHAPE, "blocks of %d rows in pages of %d" % (block_rows, s.page_rows))
        shape = (s.pages, s.layers, s.kv_heads, s.page_rows // block_rows, 2, pool.head_dim)
        if values is None:
            values = torch.zeros(shape, dtype=pool.dtype, device=pool.device)
        _expect("values", values, shape, pool.dtype, pool.device)
        self.pool, self.block_rows, self._values, self._at = pool, block_rows, values, _ptr(values)

    # not to be replaced: its address is made into an argument once
    values = property(lambda self: self._values)


def _bounds_args(pool, bounds):
    if bounds is None:
        return None, 0
    if bounds.pool is not pool:
        raise IpvError(ERR_ARG, "bounds of another pool")
    return bounds._at, bounds.block_rows


def _float_row(what, t, n, pool):
    """(pointer of) an fp32 row of n elements, or None."""
    if t is None:
        return None
    if t.dtype is not torch.float32 or t.shape != (n,) or t.get_device() != pool._dev:
        _expect(what, t, (n,), torch.float32, pool.device)
    return _ptr(t)


def _angle_args(pool, rotary, at):
    """(pointer, positions) of a table of angles, or of none."""
    if rotary is None:
        return None, 0
    shape = rotary.shape
    if rotary.dtype is not torch.float32 or len(shape) != 3 or shape[1] * 2 != pool.head_dim or shape[2] != 2:
        raise IpvError(ERR_SHAPE, "rotary must be fp32 [positions, %d, 2]" % (pool.head_dim // 2))
    if rotary.get_device() != pool._dev:
        raise IpvError(ERR_ARG, "rotary is on %s, the pool on %s" % (rotary.device, pool.device))
    return _ptr(rotary) or at, shape[0]


@functools.lru_cache(maxsize=256)
def _token_strides(q, k, v, out, shape, kv):
    """Stride arrays of q, of k and v, and of q_out."""
    arrays = _stride_array(q, shape), _stride_array(k, kv), _stride_array(out, shape)
    if list(_stride_array(v, kv)) != list(arrays[1]):
        raise IpvError(ERR_SHAPE, "k and v must have the same strides")
    _not_expanded("q_out", out, shape)
    return arrays


def ipv_qkv_write(pool, page_table, first_row, layer, q, k, v, q_out, ws, rows=None, q_norm=None, k_norm=None, eps=1e-6, rotary=None,
                  bounds=None, stream=None):
    """New tokens of one layer: queries q [B, q_heads, M, D] and keys and values k, v [B, H, M, D]
    (bf16 or fp32, any strides with the last dimension contiguous, k's and v's the same) of tokens at positions
    first_row[b], first_row[b] + 1, ... Each head of the queries and of the keys is divided by the root of its
    mean square plus eps and multiplied by q_norm or k_norm (fp32 [D]; None: not), then turned to its position by
    rotary (fp32 [positions, D / 2, 2], or None). Queries go to q_out (the pool's dtype; q itself where it is that),
    keys and values into the pages; bounds (BlockBounds, or None) of the blocks written to are brought up to date. rows: all
    M, or how many of each stream."""
    shape, kv, dev, table, cols = q.shape, k.shape, pool._dev, None, 1
    if len(shape) != 4 or shape[3] != pool.head_dim:
        raise IpvError(ERR_SHAPE, "q must be [B, q_heads, rows, %d]" % pool.head_dim)
    B, A, M, D = shape
    if kv != (B, pool.shape.kv_heads, M, D) or v.shape != kv:
        raise IpvError(ERR_SHAPE, "k and v must be [%d, %d, %d, %d]" % (B, pool.shape.kv_heads, M, D))
    kind = q.dtype
    if k.dtype is not kind or v.dtype is not kind:
        raise IpvError(ERR_DTYPE, "q, k and v must have one dtype")
    if q_out.shape != shape:
        raise IpvError(ERR_SHAPE, "q_out must have q's shape")
    if q_out.dtype is not pool.dtype:
        raise IpvError(ERR_DTYPE, "q_out must be %s" % pool.dtype)
    q_at, k_at, out_at = _token_strides(q.stride(), k.stride(), v.stride(), q_out.stride(), shape, kv)
    if rows is None:
        rows = M
    elif (rows if isinstance(rows, int) else max(rows, default=0)) > M:
        raise IpvError(ERR_SHAPE, "more rows than the tensor's %d" % M)
    if page_table is not None:
        table, cols = _table(pool, page_table, B)
    if ws is None or ws.get_device() != dev or q.get_device() != dev or k.get_device() != dev or v.get_device() != dev or \
            q_out.get_device() != dev:
        _same_gpu(pool, ws, q=q, k=k, v=v, q_out=q_out)
    first, counts_ = _host_counts(first_row, B, "first_row"), _host_counts(rows, B, "rows")
    if not -_I32 <= layer < _I32:
        _whole32("layer", layer)
    at = _ptr(ws)  # also stands for tensors without elements, whose own addresses are null
    angles, positions = _angle_args(pool, rotary, at)
    bound, block_rows = _bounds_args(pool, bounds)
    rc = _paged().ipv_qkv_write(*pool._args, bound, block_rows, table, cols, B, first.buffer_info()[0], counts_.buffer_info()[0], layer,
                                q.data_ptr() or at, q_at, A, k.data_ptr() or at, v.data_ptr() or at, k_at,
                                BF16 if kind is torch.bfloat16 else _dtype_code(q),
                                _float_row("q_norm", q_norm, D, pool), _float_row("k_norm", k_norm, D, pool), eps, angles, positions,
                                q_out.data_ptr() or at, out_at, at, ws.nbytes, _pool_stream(pool, stream))
    if rc != OK:
        _check(rc, "ipv_qkv_write")


def ipv_block_bounds(pool, page_table, first_row, rows, bounds, ws, first_layer=0, layers=None, stream=None):
    """The bounds (BlockBounds) of every block that holds one of the positions first_row[b], ...,
    first_row[b] + rows[b] - 1, made from its rows before first_row[b] + rows[b] (ints, or sequences with one per
    stream; without a page_table both ints mean all of the pool's pages), of layers first_layer, ... (layers: how many; None: all)."""
    if page_table is not None:
        table, cols = _table(pool, page_table, page_table.shape[0])
        B = page_table.shape[0]
    else:
        table, cols, B = None, 1, next((len(x) for x in (first_row, rows) if not isinstance(x, int)), pool.shape.pages)
    _same_gpu(pool, ws)
    first, counts_ = _host_counts(first_row, B, "first_row"), _host_counts(rows, B, "rows")
    layers = pool.shape.layers - first_layer if layers is None else layers
    _whole32("first_layer, layers", first_layer, layers)
    if bounds is None:
        raise IpvError(ERR_NULL, "bounds are required")
    bound, block_rows = _bounds_args(pool, bounds)
    _check(_paged().ipv_block_bounds(pool._args[0], pool._args[1], pool._args[3], bound, block_rows, table, cols, B,
                                     first.buffer_info()[0], counts_.buffer_info()[0], first_layer, layers, _ptr(ws), ws.nbytes,
                                     _pool_stream(pool, stream)), "ipv_block_bounds")


def blocks_workspace_bytes(pool: PagePool, block_rows: int, streams: int, q_heads: int, max_rows: int, top: int, max_tokens: int) -> int:
    _whole32("ipv_blocks_workspace_bytes", block_rows, streams, q_heads, max_rows, top, max_tokens)
    out = ctypes.c_size_t(0)
    _check(_paged().ipv_blocks_workspace_bytes(pool._args[0], block_rows, streams, q_heads, max_rows, top, max_tokens, ctypes.byref(out)),
           "ipv_blocks_workspace_bytes")
    return out.value


def alloc_blocks_workspace(bounds: BlockBounds, streams: int, q_heads: int, max_rows: int, top: int, max_tokens: int) -> torch.Tensor:
    """A workspace for ipv_block_select and ipv_attend_blocks calls of at most these sizes (top: blocks a query; max_tokens:
    rows of a stream): zeros where it has to be."""
    pool = bounds.pool
    ws = torch.empty(blocks_workspace_bytes(pool, bounds.block_rows, streams, q_heads, max_rows, top, max_tokens), dtype=torch.uint8,
                     device=pool.device)
    ws[:4352] = 0
    return ws


def _lists(pool, blocks, B, M):
    """(pointer, entries) of lists of blocks [B, H, M, top]."""
    shape = blocks.shape
    if blocks.dtype is not torch.int32 or len(shape) != 4 or shape[:3] != (B, pool.shape.kv_heads, M):
        raise IpvError(ERR_SHAPE, "blocks must be int32 [%d, %d, %d, entries]" % (B, pool.shape.kv_heads, M))
    if blocks.get_device() != pool._dev:
        raise IpvError(ERR_ARG, "blocks is on %s, the pool on %s" % (blocks.device, pool.device))
    return _ptr(blocks), shape[3]


def ipv_block_select(pool, page_table, bounds, n_tokens, q_first, layer, q, blocks, ws, q_rows=None, first_blocks=0, last_blocks=1,
                     stream=None):
    """For each query of q ([B, q_heads, M, D], the pool's dtype; query i of stream b at position q_first[b] + i) and KV
    head the blocks, among those that hold one of the first n_tokens[b] rows up to the query, whose bounds allow the largest
    sum of its heads' scores: into blocks, int32 [B, H, M, top], in ascending order, then -1. The first first_blocks and the
    last last_blocks of them are always picked. q_rows: queries of each stream (M if None)."""
    shape, dev, table, cols = q.shape, pool._dev, None, 1
    if len(shape) != 4 or shape[3] != pool.head_dim:
        raise IpvError(ERR_SHAPE, "q must be [B, q_heads, rows, %d]" % pool.head_dim)
    if q.dtype is not pool.dtype:
        raise IpvError(ERR_DTYPE, "q must be %s" % pool.dtype)
    B, A, M, _ = shape
    if page_table is not None:
        table, cols = _table(pool, page_table, B)
    if bounds is None:
        raise IpvError(ERR_NULL, "bounds are required")
    bound, block_rows = _bounds_args(pool, bounds)
    listed, top = _lists(pool, blocks, B, M)
    _same_gpu(pool, ws, q=q)
    n, first = _host_counts(n_tokens, B, "n_tokens"), _host_counts(q_first, B, "q_first")
    rows = _query_counts(q_rows, B, M)
    _whole32("layer, first_blocks, last_blocks", layer, first_blocks, last_blocks)
    at = _ptr(ws)
    _check(_paged().ipv_block_select(pool._args[0], bound, block_rows, table, cols, B, n.buffer_info()[0], first.buffer_info()[0],
                                     rows.buffer_info()[0], layer, q.data_ptr() or at, _stride_array(q.stride(), shape), A, M or 1,
                                     first_blocks, last_blocks, top, listed or at, at, ws.nbytes, _pool_stream(pool, stream)), "ipv_block_select")


def ipv_attend_blocks(pool, page_table, n_tokens, q_first, layer, q, blocks, out, ws, bounds=None, block_rows=None, q_rows=None,
                      scale=None, first_blocks=0, last_blocks=1, lse=None, stream=None):
    """Attention as ipv_attend's over the rows of the blocks that blocks (int32 [B, H, M, top]) lists for each query and KV
    head. With bounds the lists are made first, as ipv_block_select does, and left in blocks; without, they are
    read as they are (in any order, negative entries and blocks past the query adding nothing) and block_rows says how many
    rows a block has."""
    shape, dev, table, cols = q.shape, pool._dev, None, 1
    if len(shape) != 4 or shape[3] != pool.head_dim:
        raise IpvError(ERR_SHAPE, "q must be [B, q_heads, rows, %d]" % pool.head_dim)
    if q.dtype is not pool.dtype or out.dtype is not pool.dtype:
        raise IpvError(ERR_DTYPE, "q and out must be %s" % pool.dtype)
    if out.shape != shape:
        raise IpvError(ERR_SHAPE, "out must have q's shape")
    B, A, M, D = shape
    if lse is not None:
        _expect("lse", lse, (B, A, M), torch.float32, pool.device)
    if page_table is not None:
        table, cols = _table(pool, page_table, B)
    bound, rows_of = _bounds_args(pool, bounds)
    if bounds is None:
        if block_rows is None:
            raise IpvError(ERR_ARG, "without bounds block_rows is required")
        _whole32("block_rows", block_rows)
        rows_of = block_rows
    elif block_rows is not None and block_rows != rows_of:
        raise IpvError(ERR_ARG, "bounds are of blocks of %d rows" % rows_of)
    listed, top = _lists(pool, blocks, B, M)
    if ws is None or ws.get_device() != dev or q.get_device() != dev or out.get_device() != dev:
        _same_gpu(pool, ws, q=q, out=out)
    n, first = _host_counts(n_tokens, B, "n_tokens"), _host_counts(q_first, B, "q_first")
    rows = _query_counts(q_rows, B, M)
    q_strides, out_strides = q.stride(), out.stride()
    q_at = _stride_array(q_strides, shape)
    if 0 in out_strides:
        _not_expanded("out", out_strides, shape)
    if not (-_I32 <= layer < _I32 and -_I32 <= first_blocks < _I32 and -_I32 <= last_blocks < _I32):
        _whole32("layer, first_blocks, last_blocks", layer, first_blocks, last_blocks)
    at = _ptr(ws)  # also stands for tensors without elements, whose own addresses are null
    rc = _paged().ipv_attend_blocks(*pool._args, bound, rows_of, table, cols, B, n.buffer_info()[0], first.buffer_info()[0],
                                    rows.buffer_info()[0], layer, q.data_ptr() or at, q_at, A, M or 1,
                                    D ** -0.5 if scale is None else scale, first_blocks, last_blocks, top, listed or at,
                                    out.data_ptr() or at, q_at if out_strides == q_strides else _stride_array(out_strides, shape),
                                    None if lse is None else _ptr(lse) or at, at, ws.nbytes, _pool_stream(pool, stream))
    if rc != OK:
        _check(rc, "ipv_attend_blocks")


def ipv_page_compact(pool, page_table, new_table, n_tokens, keep_idx, ws, rows=None, rotary=None, bounds=None, stream=None):
    """Row j < rows[b] (all C if None) of every slice of stream b, in the pages of new_table[b], becomes row keep_idx[b, l, h, j]
    (int32 [B, L, H, C], as ipv_select writes it) of the n_tokens[b] rows in the pages of page_table[b], which may not be
    among the new ones. With rotary keys are turned from the position that they had to the one that they get; bounds
    (BlockBounds, or None) of the new blocks are made. Without rows (C = 0 as well) the call does nothing."""
    s, shape, table, cols = pool.shape, keep_idx.shape, None, 1
    if keep_idx.dtype is not torch.int32 or len(shape) != 4 or tuple(shape[1:3]) != (s.layers, s.kv_heads):
        raise IpvError(ERR_SHAPE, "keep_idx must be int32 [B, %d, %d, C]" % (s.layers, s.kv_heads))
    B, C = shape[0], shape[3]
    if page_table is not None:
        table, cols = _table(pool, page_table, B)
    if new_table is None:
        raise IpvError(ERR_NULL, "new_table is required")
    new, new_cols = _table(pool, new_table, B)
    _same_gpu(pool, ws, keep_idx=keep_idx)
    n, counts_ = _host_counts(n_tokens, B, "n_tokens"), _host_counts(C if rows is None else rows, B, "rows")
    if C == 0 and any(counts_):
        raise IpvError(ERR_SHAPE, "more rows than keep_idx's 0")
    at = _ptr(ws)  # also stands for a tensor without elements, whose own address is null
    angles, positions = _angle_args(pool, rotary, at)
    bound, block_rows = _bounds_args(pool, bounds)
    rc = _paged().ipv_page_compact(*pool._args, bound, block_rows, table, cols, new, new_cols, B, n.buffer_info()[0], _ptr(keep_idx) or at,
                                   C or 1, counts_.buffer_info()[0], angles, positions, at, ws.nbytes, _pool_stream(pool, stream))
    if rc != OK:
        _check(rc, "ipv_page_compact")


def ipv_page_copy(pool, from_pages, to_pages, ws, rows=None, bounds=None, stream=None):
    """Pages from_pages[i] onto to_pages[i] (int32 [N], on the pool's GPU), or the first `rows` rows of their slices, with
    their scales and bounds (BlockBounds, or None). No page may be written twice, or written and read by one call (but that
    one copied onto itself is left alone)."""
    for what, t in (("from_pages", from_pages), ("to_pages", to_pages)):
        if t.dtype is not torch.int32 or t.dim() != 1 or t.shape != from_pages.shape:
            raise IpvError(ERR_SHAPE, "%s must be int32 [N]" % what)
    _same_gpu(pool, ws, from_pages=from_pages, to_pages=to_pages)
    rows = pool.shape.page_rows if rows is None else rows
    _whole32("rows", rows)
    at = _ptr(ws)
    bound, block_rows = _bounds_args(pool, bounds)
    rc = _paged().ipv_page_copy(*pool._args, bound, block_rows, _ptr(from_pages) or at, _ptr(to_pages) or at, from_pages.shape[0], rows,
                                at, ws.nbytes, _pool_stream(pool, stream))
    if rc != OK:
        _check(rc, "ipv_page_copy")


class PageTables:
    """Which pages of a pool its streams have: `table` (int32 [streams, columns], on the pool's GPU, -1 where a stream has no
    page) is what the other calls take. Streams may share pages (fork); a shared one is copied before a stream writes to it
    (reserve). A page that goes back can be handed out again at once, so the calls that use them run on one HIP stream, these
    methods on it as the current one, outside of captures: they write the table, whose memory stays the same."""

    def __init__(self, pool: PagePool, streams: int, columns: int):
        if streams < 1 or columns < 1:
            raise IpvError(ERR_SHAPE, "a table of %d streams and %d columns" % (streams, columns))
        self.pool, self.columns = pool, columns
        self.pages = [[] for _ in range(streams)]  # of each stream, in order
        self._users = [0] * pool.shape.pages
        self._free = list(range(pool.shape.pages - 1, -1, -1))
        self._table = torch.full((streams, columns), -1, dtype=torch.int32, device=pool.device)

    table = property(lambda self: self._table)
    free_pages = property(lambda self: len(self._free))

    def _columns_of(self, end):
        cols = -(-end // self.pool.shape.page_rows)
        if cols > self.columns:
            raise IpvError(ERR_SHAPE, "%d rows take %d pages, the table has %d columns" % (end, cols, self.columns))
        return cols

    def _stream_of(self, *streams):
        for b in streams:
            if not 0 <= b < len(self.pages):
                raise IpvError(ERR_ARG, "stream %d of %d" % (b, len(self.pages)))

    def _have(self, wanted):
        if wanted > len(self._free):
            raise IpvError(ERR_ARG, "%d pages wanted, %d are free" % (wanted, len(self._free)))

    def _take(self):
        page = self._free.pop()
        self._users[page] = 1
        return page

    def _give_back(self, pages):
        for page in pages:
            self._users[page] -= 1
            if self._users[page] == 0:
                self._free.append(page)

    def _int32(self, values):
        return torch.tensor(values, dtype=torch.int32).to(self.pool.device)

    def _publish(self):
        self._table.copy_(torch.tensor([x + [-1] * (self.columns - len(x)) for x in self.pages], dtype=torch.int32))

    def reserve(self, first_row, rows, ws, bounds=None):
        """Pages for the rows[b] rows from first_row[b] on of every stream, and for all before them: new ones where it has none;
        where it shares one that holds some of these rows, a copy (with bounds, if given) of its own. Without enough
        free pages nothing changes and the call raises."""
        streams, T = len(self.pages), self.pool.shape.page_rows
        first, rows = _host_counts(first_row, streams, "first_row"), _host_counts(rows, streams, "rows")
        own, missing, users = [], [0] * streams, {}  # (stream, column) of shared pages; pages behind those of a stream; users left
        for b, pages in enumerate(self.pages):
            if first[b] < 0 or rows[b] < 0:
                raise IpvError(ERR_SHAPE, "negative rows")
            if rows[b] == 0:
                continue
            cols = self._columns_of(first[b] + rows[b])
            missing[b] = max(cols - len(pages), 0)
            for c in range(first[b] // T, min(cols, len(pages))):
                left = users.get(pages[c], self._users[pages[c]])
                if left > 1:
                    own.append((b, c))
                    users[pages[c]] = left - 1
        self._have(len(own) + sum(missing))
        if own:
            new = self._free[len(self._free) - len(own):][::-1]
            ipv_page_copy(self.pool, self._int32([self.pages[b][c] for b, c in own]), self._int32(new), ws, bounds=bounds)
            for b, c in own:
                self._give_back([self.pages[b][c]])
                self.pages[b][c] = self._take()
        for b, pages in enumerate(self.pages):
            pages.extend([self._take() for _ in range(missing[b])])
        if own or any(missing):
            self._publish()

    def fork(self, stream, to, n_tokens):
        """Stream `to` has the pages of the first n_tokens rows of `stream`, instead of those that it had. Bounds of the last
        block are still those of all the rows that are there, which selection for `to` sees (no score comes out too low) until
        rows are written to that block (ipv_qkv_write makes them anew) or, in a page of its own (reserve), ipv_block_bounds does."""
        self._stream_of(stream, to)
        cols = self._columns_of(n_tokens)
        if n_tokens < 0 or cols > len(self.pages[stream]):
            raise IpvError(ERR_SHAPE, "stream %d has no %d rows" % (stream, n_tokens))
        shared = self.pages[stream][:cols]
        for page in shared:
            self._users[page] += 1
        self._give_back(self.pages[to])
        self.pages[to] = shared
        self._publish()

    def free(self, stream, n_tokens=0):
        """The pages behind the first n_tokens rows of a stream go back. Bounds of the last block that is left are those of all
        the rows that are there, as after fork."""
        self._stream_of(stream)
        if n_tokens < 0:
            raise IpvError(ERR_SHAPE, "negative rows")
        cols = -(-n_tokens // self.pool.shape.page_rows)
        self._give_back(self.pages[stream][cols:])
        del self.pages[stream][cols:]
        self._publish()

    def compact(self, streams, n_tokens, keep_idx, ws, rows=None, rotary=None, bounds=None):
        """ipv_page_compact of these streams, keep_idx [len(streams), L, H, C], into pages of their own; those that they had go
        back. It takes free pages for all new rows first; without enough, or with more rows (n_tokens) than a stream has pages
        for, nothing changes and the call raises."""
        self._stream_of(*streams)
        if len(set(streams)) != len(streams):
            raise IpvError(ERR_ARG, "a stream is named twice")
        if not streams:
            return
        held = _host_counts(n_tokens, len(streams), "n_tokens")
        counts_ = _host_counts(keep_idx.shape[-1] if rows is None else rows, len(streams), "rows")
        if min(counts_) < 0 or min(held) < 0:
            raise IpvError(ERR_SHAPE, "negative rows")
        for b, n in zip(streams, held):
            if n > len(self.pages[b]) * self.pool.shape.page_rows:
                raise IpvError(ERR_SHAPE, "stream %d has no %d rows" % (b, n))
        cols = [self._columns_of(r) for r in counts_]
        self._have(sum(cols))
        had = [self.pages[b] for b in streams]
        fresh = iter(self._free[len(self._free) - sum(cols):][::-1])
        new = [[next(fresh) for _ in range(c)] for c in cols]
        at = [self._int32([x + [-1] * (self.columns - len(x)) for x in pages]) for pages in (had, new)]
        ipv_page_compact(self.pool, at[0], at[1], n_tokens, keep_idx, ws, rows=rows, rotary=rotary, bounds=bounds)
        for b, x in zip(streams, new):
            self.pages[b] = [self._take() for _ in x]
        for pages in had:
            self._give_back(pages)
        self._publish()


class Compressor:
    """Buffers for repeated passes over caches of one shape.

    Holds the score, keep-index and workspace tensors so a pass allocates
    nothing; ``compress`` runs the whole pass on the current stream.
    """

    def __init__(self, K: torch.Tensor, grid_h: int, grid_w: int, budget: int):
        self.grid_h, self.grid_w, self.budget = grid_h, grid_w, budget
        self.shape = shape_of(K, grid_h, grid_w)
        B, L, H, S, D = K.shape
        dev = K.device
        self.tar = torch.zeros((B, L, H, S), dtype=torch.float32, device=dev)
        self.van = torch.zeros((B, L, H, S), dtype=torch.float32, device=dev)
        self.keep_idx = torch.zeros((B, L, H, budget), dtype=torch.int32, device=dev)
        self.ws = alloc_workspace(self.shape, dev)

    def compress(self, K, V, frame_idx, patch_idx, n_tokens, alpha, recent_frames, cv_tau=None, stream=None,
                 mode=0):
        ipv_compress(K, V, frame_idx, patch_idx, n_tokens, self.budget, alpha, recent_frames, cv_tau, self.tar,
                     self.van, self.keep_idx, self.ws, self.grid_h, self.grid_w, stream, mode)

    def device_errors(self) -> int:
        return ipv_read_device_errors(self.ws)
