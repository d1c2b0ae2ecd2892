"""ctypes binding of libmw.so (include/mw.h).  Argument marshalling only.

Every function here forwards torch tensors' device pointers and the current
HIP stream to the C ABI; all arithmetic runs in the library's HIP kernels.
There is no fallback: if the library is missing or a call fails, an
exception is raised.
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import math
import operator
import os

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libmw.so")

MW_OK = 0
MW_EINVAL = -1
MW_EUNSUPPORTED = -2
MW_EALIGN = -3
MW_EFULL = -4
MW_EEMPTY = -5
MW_EHIP = -6
MW_QUEUED_CAUSAL = 0
MW_QUEUED_ISOLATED = 1
MW_MAX_WINDOW = 64
MW_MAX_QUEUED = 64
MW_MAX_SLOTS = 128
MW_PAGE_BLOCK = 64
MW_MAX_SEQS = 256
MW_MAX_ROPE_BANDS = 4
MW_MAX_ROPE_PAIRS = 64

STATUS_NAMES = {0: "MW_OK", -1: "MW_EINVAL", -2: "MW_EUNSUPPORTED", -3: "MW_EALIGN", -4: "MW_EFULL",
                -5: "MW_EEMPTY", -6: "MW_EHIP"}


class MWError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{STATUS_NAMES.get(code, code)}: {msg}")
        self.code = code


class mw_kvcache(ctypes.Structure):
    _fields_ = [("k_slots", ctypes.c_void_p), ("v_slots", ctypes.c_void_p),
                ("S", ctypes.c_int), ("B", ctypes.c_int), ("H", ctypes.c_int), ("L", ctypes.c_int),
                ("D", ctypes.c_int), ("head", ctypes.c_int64), ("tail", ctypes.c_int64),
                ("k_sink", ctypes.c_void_p), ("v_sink", ctypes.c_void_p), ("sink_len", ctypes.c_int),
                ("elem_bytes", ctypes.c_int), ("k_scale", ctypes.c_float), ("v_scale", ctypes.c_float),
                ("rope_total", ctypes.c_int64), ("rope_offset", ctypes.c_int), ("rope_count", ctypes.c_int),
                ("rope_theta", ctypes.c_float), ("rope_set", ctypes.c_int),
                ("rope_at_commit", ctypes.c_int64 * MW_MAX_SLOTS)]


class mw_kvpages(ctypes.Structure):
    _fields_ = [("k_pages", ctypes.c_void_p), ("v_pages", ctypes.c_void_p), ("k_scales", ctypes.c_void_p),
                ("v_scales", ctypes.c_void_p), ("table", ctypes.c_void_p), ("lens", ctypes.c_void_p),
                ("host", ctypes.c_void_p), ("P", ctypes.c_int), ("H", ctypes.c_int), ("L", ctypes.c_int),
                ("D", ctypes.c_int), ("N", ctypes.c_int), ("W", ctypes.c_int)]


class mw_rope(ctypes.Structure):
    _fields_ = [("dim_offset", ctypes.c_int), ("dim_count", ctypes.c_int), ("theta", ctypes.c_float)]


class mw_rope_band(ctypes.Structure):
    _fields_ = [("dim_offset", ctypes.c_int), ("dim_count", ctypes.c_int), ("theta", ctypes.c_double), ("axis", ctypes.c_int),
                ("factor", ctypes.c_double), ("trained_len", ctypes.c_double), ("turns_lo", ctypes.c_double),
                ("turns_hi", ctypes.c_double)]


class mw_rope_bands(ctypes.Structure):
    _fields_ = [("n_bands", ctypes.c_int), ("n_pairs", ctypes.c_int), ("n_axes", ctypes.c_int), ("halves", ctypes.c_int),
                ("gain", ctypes.c_float), ("dim_offset", ctypes.c_int * MW_MAX_ROPE_BANDS),
                ("dim_count", ctypes.c_int * MW_MAX_ROPE_BANDS), ("axis", ctypes.c_uint8 * MW_MAX_ROPE_PAIRS),
                ("freq", ctypes.c_double * MW_MAX_ROPE_PAIRS)]


class mw_packed(ctypes.Structure):
    _fields_ = [("cu_q", ctypes.c_void_p), ("cu_k", ctypes.c_void_p), ("plan", ctypes.c_void_p), ("N", ctypes.c_int),
                ("total_q", ctypes.c_int), ("total_k", ctypes.c_int), ("H", ctypes.c_int), ("Hkv", ctypes.c_int),
                ("D", ctypes.c_int), ("chunk_len", ctypes.c_int), ("backward", ctypes.c_int)]


class mw_strides(ctypes.Structure):
    _fields_ = [("b", ctypes.c_int64), ("h", ctypes.c_int64), ("t", ctypes.c_int64)]


class mw_sched_config(ctypes.Structure):
    _fields_ = [("window", ctypes.c_int), ("stride", ctypes.c_int), ("n_chunks", ctypes.c_int),
                ("cache_chunks", ctypes.c_int), ("frames_per_chunk", ctypes.c_int), ("sink_frames", ctypes.c_int),
                ("shift", ctypes.c_double), ("n_bins", ctypes.c_int)]


class mw_sched_tick(ctypes.Structure):
    _fields_ = [("tick", ctypes.c_int64), ("first", ctypes.c_int), ("n_active", ctypes.c_int),
                ("updates_per_chunk", ctypes.c_int),
                ("tau", ctypes.c_double * MW_MAX_QUEUED), ("dtau", ctypes.c_double * MW_MAX_QUEUED),
                ("n_commit", ctypes.c_int), ("n_evict", ctypes.c_int), ("rope_shift", ctypes.c_int),
                ("cache_live", ctypes.c_int), ("pos_first", ctypes.c_int)]


# Exported symbols and their signatures (mirrors include/mw.h).
_vp, _i, _f, _sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
_ip = ctypes.POINTER(ctypes.c_int)
_cache_p = ctypes.POINTER(mw_kvcache)
_str_p = ctypes.POINTER(mw_strides)
_pages_p = ctypes.POINTER(mw_kvpages)
_seq_p = ctypes.POINTER(ctypes.c_int32)
_packed_p = ctypes.POINTER(mw_packed)
_bands_p = ctypes.POINTER(mw_rope_bands)
SIGNATURES = {
    "mw_last_error": ([], ctypes.c_char_p),
    "mw_version": ([], _i),
    "mw_block_causal_attn_fwd": ([_vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _f, _vp], _i),
    "mw_block_causal_attn_bwd_workspace_size": ([_i, _i, _i, _i], _sz),
    "mw_block_causal_attn_bwd": ([_vp] * 9 + [_vp, _sz, _i, _i, _i, _i, _i, _f, _vp], _i),
    "mw_kvcache_init": ([_cache_p, _vp, _vp, _i, _i, _i, _i, _i], _i),
    "mw_kvcache_append": ([_cache_p, _vp, _vp, _vp], _i),
    "mw_kvcache_evict": ([_cache_p, _i], _i),
    "mw_kvcache_set_sink": ([_cache_p, _vp, _vp, _i], _i),
    "mw_kvcache_rope_shift": ([_cache_p, _i, ctypes.POINTER(mw_rope), _vp], _i),
    "mw_kvcache_live": ([_cache_p], _i),
    "mw_kvcache_slot_of": ([_cache_p, ctypes.c_int64], _i),
    "mw_chunk_attn_cached_workspace_size": ([_cache_p, _i, _i, _i], _sz),
    "mw_chunk_attn_cached_plan": ([_cache_p, _i, _i, _i, _i, _sz, _ip, _ip], _i),
    "mw_chunk_attn_cached": ([_vp, _vp, _vp, _i, _i, _cache_p, _i, _i, _vp, _vp, _f, _vp, _sz, _vp], _i),
    "mw_block_causal_attn_fwd_strided": ([_vp, _vp, _vp, _vp, _vp, _str_p, _i, _i, _i, _i, _i, _f, _vp], _i),
    "mw_block_causal_attn_bwd_strided": ([_vp] * 9 + [_vp, _sz, _str_p, _i, _i, _i, _i, _i, _f, _vp], _i),
    "mw_block_causal_attn_bwd_noalloc": ([_vp] * 9 + [_i, _i, _i, _i, _i, _f, _vp], _i),
    "mw_kvcache_append_strided": ([_cache_p, _vp, _vp, _str_p, _vp], _i),
    "mw_chunk_attn_cached_strided": ([_vp, _vp, _vp, _i, _i, _cache_p, _i, _i, _vp, _vp, _f, _vp, _sz, _str_p,
                                      _vp], _i),
    "mw_quantize_fp8": ([_vp, _str_p, _vp, _i, _i, _i, _i, _f, _vp], _i),
    "mw_kvcache_init_fp8": ([_cache_p, _vp, _vp, _i, _i, _i, _i, _i, _f, _f], _i),
    "mw_chunk_attn_cached_fp8": ([_vp, _vp, _vp, _i, _i, _cache_p, _i, _i, _vp, _vp, _f, _f, _vp, _sz, _str_p, _vp],
                                 _i),
    "mw_cross_attn_workspace_size": ([_i] * 6, _sz),
    "mw_cross_attn_fwd": ([_vp] * 6 + [_str_p] + [_i] * 6 + [_f, _vp, _sz, _vp], _i),
    "mw_cross_attn_bwd_workspace_size": ([_i] * 6, _sz),
    "mw_cross_attn_bwd": ([_vp] * 11 + [_sz, _str_p] + [_i] * 6 + [_f, _vp], _i),
    "mw_kvpages_host_bytes": ([_i, _i, _i], _sz),
    "mw_kvpages_init": ([_pages_p] + [_vp] * 7 + [_sz] + [_i] * 6, _i),
    "mw_kvpages_len": ([_pages_p, _i], _i),
    "mw_kvpages_n_free": ([_pages_p], _i),
    "mw_kvpages_page_of": ([_pages_p, _i, _i], _i),
    "mw_kvpages_append": ([_pages_p, _seq_p, _i, _vp, _vp, _str_p, _i, _vp], _i),
    "mw_kvpages_fork": ([_pages_p, _i, _i, _vp], _i),
    "mw_kvpages_copy": ([_pages_p, _i, _i, _vp], _i),
    "mw_kvpages_free": ([_pages_p, _seq_p, _i, _vp], _i),
    "mw_kvpages_evict": ([_pages_p, _i, _i, _i, _vp], _i),
    "mw_kvpages_compact": ([_pages_p, _vp], _i),
    "mw_chunk_attn_paged_workspace_size": ([_pages_p, _seq_p] + [_i] * 4, _sz),
    "mw_chunk_attn_paged": ([_vp] * 3 + [_i, _i, _pages_p, _seq_p] + [_i] * 3 + [_vp, _vp, _f, _vp, _sz, _str_p, _vp], _i),
    "mw_packed_plan_bytes": ([_i] * 8, _sz),
    "mw_packed_init": ([_packed_p, _vp, _vp, _vp, _sz] + [_i] * 8 + [_vp], _i),
    "mw_packed_attn_workspace_size": ([_packed_p], _sz),
    "mw_packed_attn_fwd": ([_vp] * 3 + [_packed_p, _vp, _vp, _f, _vp, _sz, _str_p, _vp], _i),
    "mw_packed_attn_bwd_workspace_size": ([_packed_p], _sz),
    "mw_packed_attn_bwd": ([_vp] * 6 + [_packed_p] + [_vp] * 3 + [_f, _vp, _sz, _str_p, _vp], _i),
    "mw_rope_bands_init": ([_bands_p, ctypes.POINTER(mw_rope_band), _i, _i, _f], _i),
    "mw_rope_apply": ([_vp] * 4 + [_bands_p, _vp, _i, _str_p, ctypes.c_int64, _i, _str_p] + [_i] * 5 + [_vp], _i),
    "mw_kvpages_weigh_workspace_size": ([_pages_p, _seq_p, _i, _i, _i], _sz),
    "mw_kvpages_weigh": ([_pages_p, _seq_p, _i, _vp, _vp, _i, _i, _vp, _i, _f, _vp, _sz, _str_p, _vp], _i),
    "mw_kvpages_evict_weighted_workspace_size": ([_pages_p, _seq_p, _i, _i, _i], _sz),
    "mw_kvpages_evict_weighted": ([_pages_p, _seq_p, _i, _vp, _i, _i, _i, _vp, _sz, _vp], _i),
    "mw_sched_num_ticks": ([ctypes.POINTER(mw_sched_config)], ctypes.c_int64),
    "mw_sched_plan": ([ctypes.POINTER(mw_sched_config), ctypes.c_int64, ctypes.POINTER(mw_sched_tick)], _i),
}

_lib = None


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libmw.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"libmw.so not found at {path}: build it with "
                           f"`python -m paper_2608_01127_amd.build` (no CPU fallback exists)")
    lib = ctypes.CDLL(path)
    for name, (args, res) in SIGNATURES.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = res
    _lib = lib
    return lib


def _check(code: int) -> int:
    if code < 0:
        msg = load().mw_last_error().decode(errors="replace")
        raise MWError(code, msg)
    return code


# ----------------------------------------------------------------------------- torch glue

def _torch():
    import torch
    return torch


def _stream_handle(device) -> int:
    """Handle of the current HIP stream of `device` (a device or its index)."""
    torch = _torch()
    index = device if isinstance(device, int) else device.index
    if index is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream(device).cuda_stream
    return torch._C._cuda_getCurrentRawStream(index)  # current_stream() without its Stream object: 0.1 for 1.1 us


def _ptr(t) -> int:
    return 0 if t is None else t.data_ptr()


def _bf16_4d(name, t, view: bool = False):
    """bf16 [B,H,T,D] on a GPU; contiguous, or (view=True) any view whose last
    dimension is contiguous (the library checks the remaining strides)."""
    torch = _torch()
    if t.dtype != torch.bfloat16:
        raise TypeError(f"{name} must be bfloat16, got {t.dtype}")
    if t.dim() != 4:
        raise ValueError(f"{name} must be [B,H,T,D], got shape {tuple(t.shape)}")
    if view:
        if t.shape[-1] > 1 and t.stride(-1) != 1:
            raise ValueError(f"{name} must have a contiguous last (head) dimension")
    elif not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be on a GPU device")


def _u8_4d(name, t):
    """e4m3 codes as a contiguous uint8 [B,H,T,D] tensor on a GPU."""
    torch = _torch()
    if t.dtype != torch.uint8:
        raise TypeError(f"{name} must hold e4m3 codes as uint8, got {t.dtype}")
    if t.dim() != 4 or not t.is_contiguous() or t.device.type != "cuda":
        raise ValueError(f"{name} must be a contiguous [B,H,T,D] tensor on a GPU")


@functools.lru_cache(maxsize=512)
def _strides_array(*strides):
    arr = (mw_strides * len(strides))()
    for i, s in enumerate(strides):
        arr[i] = mw_strides(s[0], s[1], s[2])
    return arr


def _strides(*ts):
    """mw_strides array (B, H, T element strides) of the given [B,H,T,D] views.  The arrays are kept
    by their values (the library only reads them): filling one takes 0.6 us a tensor."""
    return _strides_array(*[t.stride() for t in ts])


def _plain_views(ts, shape, ref) -> bool:
    """Whether every tensor is a bf16 [B,H,T,D] view of `shape` on the GPU of `ref` with a contiguous
    last dimension: what the checks below find one by one, in a sixth of their time.  A call
    whose tensors are not goes through them, for their errors."""
    try:
        index = ref.get_device()
    except AttributeError:  # no tensor
        return False
    if index < 0 or len(shape) != 4:
        return False
    bf16 = _torch().bfloat16
    for t in ts:
        if t.dtype is not bf16 or t.shape != shape or t.get_device() != index or t.stride()[-1] != 1:
            return False
    return True


def _check_lse(lse, shape, dev) -> None:
    """An lse output (or None): fp32, contiguous, of the given shape, on `dev`."""
    if lse is None:
        return
    torch = _torch()
    if lse.dtype != torch.float32 or tuple(lse.shape) != tuple(shape) or not lse.is_contiguous():
        raise ValueError(f"lse must be a contiguous fp32 tensor of shape {tuple(shape)}, got "
                         f"{lse.dtype} {tuple(lse.shape)}")
    if lse.device != dev:
        raise ValueError("lse must be on the device of the inputs")


def _same_device(*ts):
    dev = ts[0].device
    for t in ts:
        if t is not None and t.device != dev:
            raise ValueError("all tensors must be on the same device")
    return dev


def mw_block_causal_attn_fwd(q, k, v, chunk_len: int, scale=None, out=None, lse=None):
    """Block-causal attention forward.  q, k, v: bf16 [B,H,T,D] (views with a
    contiguous head dimension are read in place).  Returns (o, lse)."""
    torch = _torch()
    plain = _plain_views((q, k, v) if out is None else (q, k, v, out), q.shape, q)
    if not plain:
        for n, t in (("q", q), ("k", k), ("v", v)):
            _bf16_4d(n, t, view=True)
        if k.shape != q.shape or v.shape != q.shape:
            raise ValueError("q, k, v must have the same shape")
        _same_device(q, k, v)
    B, H, T, D = q.shape
    dev = q.device
    scale = 1.0 / math.sqrt(D) if scale is None else float(scale)
    o = torch.empty_like(q) if out is None else out
    lse = torch.empty((B, H, T), dtype=torch.float32, device=dev) if lse is None else lse
    if not plain:
        _bf16_4d("out", o, view=True)
        if o.shape != q.shape:
            raise ValueError("out must have the shape of q")
        _same_device(q, o)
    _check_lse(lse, (B, H, T), dev)
    _check(load().mw_block_causal_attn_fwd_strided(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse),
                                                   _strides(q, k, v, o), B, H, T, D, int(chunk_len), scale,
                                                   _stream_handle(dev)))
    return o, lse


def mw_block_causal_attn_bwd_workspace_size(B: int, H: int, T: int, D: int) -> int:
    return int(load().mw_block_causal_attn_bwd_workspace_size(B, H, T, D))


def mw_block_causal_attn_bwd(q, k, v, o, d_o, lse, chunk_len: int, scale=None, workspace=None,
                             dq=None, dk=None, dv=None):
    """Backward of mw_block_causal_attn_fwd.  Returns (dq, dk, dv), bf16 [B,H,T,D]
    (views with a contiguous head dimension are accepted for every tensor)."""
    torch = _torch()
    plain = _plain_views([t for t in (q, k, v, o, d_o, dq, dk, dv) if t is not None], q.shape, q)
    if not plain:
        for n, t in (("q", q), ("k", k), ("v", v), ("o", o), ("d_o", d_o)):
            _bf16_4d(n, t, view=True)
            if t.shape != q.shape:
                raise ValueError(f"{n} must have the shape of q")
    B, H, T, D = q.shape
    if lse.shape != (B, H, T) or lse.dtype != torch.float32 or not lse.is_contiguous():
        raise ValueError("lse must be fp32 [B,H,T] contiguous")
    dev = _same_device(q, lse) if plain else _same_device(q, k, v, o, d_o, lse)
    scale = 1.0 / math.sqrt(D) if scale is None else float(scale)
    need = mw_block_causal_attn_bwd_workspace_size(B, H, T, D)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(q) if dk is None else dk
    dv = torch.empty_like(q) if dv is None else dv
    if not plain:
        for n, t in (("dq", dq), ("dk", dk), ("dv", dv)):
            _bf16_4d(n, t, view=True)
            if t.shape != q.shape:
                raise ValueError(f"{n} must have the shape of q")
    _same_device(q, workspace, dq, dk, dv)
    nbytes = workspace.numel() * workspace.element_size()
    _check(load().mw_block_causal_attn_bwd_strided(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(d_o), _ptr(lse),
                                                   _ptr(dq), _ptr(dk), _ptr(dv), _ptr(workspace), nbytes,
                                                   _strides(q, k, v, o, d_o, dq, dk, dv), B, H, T, D,
                                                   int(chunk_len), scale, _stream_handle(dev)))
    return dq, dk, dv


def mw_block_causal_attn_bwd_noalloc(q, k, v, o, d_o, lse, chunk_len: int, dq, dk, dv, scale=None):
    """The backward without a workspace: its row terms live in the library's own per-GPU
    scratch array, and neither the library nor this wrapper allocates anything, so dq, dk, dv
    must be given.  Contiguous bf16 [B,H,T,D] tensors, lse fp32 [B,H,T]; B*H*T <= 4,194,304.
    Calls that overlap on one GPU share the array and race.  Returns (dq, dk, dv)."""
    torch = _torch()
    for n, t in (("q", q), ("k", k), ("v", v), ("o", o), ("d_o", d_o), ("dq", dq), ("dk", dk), ("dv", dv)):
        _bf16_4d(n, t)
        if t.shape != q.shape:
            raise ValueError(f"{n} must have the shape of q")
    B, H, T, D = q.shape
    dev = _same_device(q, k, v, o, d_o, lse, dq, dk, dv)
    if lse is None:
        raise ValueError("lse is required")
    _check_lse(lse, (B, H, T), dev)
    scale = 1.0 / math.sqrt(D) if scale is None else float(scale)
    with torch.cuda.device(dev):  # the library takes the current device's copy of its array
        _check(load().mw_block_causal_attn_bwd_noalloc(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(d_o), _ptr(lse),
                                                       _ptr(dq), _ptr(dk), _ptr(dv), B, H, T, D, int(chunk_len),
                                                       scale, _stream_handle(dev)))
    return dq, dk, dv


class KVCache:
    """Ring-buffered rolling KV cache over torch-owned slot tensors: bf16
    [S,B,H,L,D], or with fp8=True e4m3 codes (uint8 [S,B,H,L,D]) with the
    per-tensor scales k_scale, v_scale (value = code * scale).

    Wraps the mw_kvcache descriptor; `head`/`tail` count commits/evictions.
    """

    def __init__(self, S: int, B: int, H: int, L: int, D: int, device="cuda", k_slots=None, v_slots=None,
                 fp8: bool = False, k_scale: float = 1.0, v_scale: float = 1.0):
        torch = _torch()
        shape = (S, B, H, L, D)
        dt = torch.uint8 if fp8 else torch.bfloat16
        self.fp8 = bool(fp8)
        self.k_slots = torch.empty(shape, dtype=dt, device=device) if k_slots is None else k_slots
        self.v_slots = torch.empty(shape, dtype=dt, device=device) if v_slots is None else v_slots
        for n, t in (("k_slots", self.k_slots), ("v_slots", self.v_slots)):
            if t.shape != shape or t.dtype != dt or not t.is_contiguous():
                raise ValueError(f"{n} must be {dt} contiguous {shape}")
        self.desc = mw_kvcache()
        if fp8:
            _check(load().mw_kvcache_init_fp8(ctypes.byref(self.desc), _ptr(self.k_slots), _ptr(self.v_slots),
                                              S, B, H, L, D, float(k_scale), float(v_scale)))
        else:
            _check(load().mw_kvcache_init(ctypes.byref(self.desc), _ptr(self.k_slots), _ptr(self.v_slots),
                                          S, B, H, L, D))

    @property
    def head(self) -> int:
        return int(self.desc.head)

    @property
    def tail(self) -> int:
        return int(self.desc.tail)

    @property
    def live(self) -> int:
        return _check(load().mw_kvcache_live(ctypes.byref(self.desc)))

    def slot_of(self, chunk: int) -> int:
        return int(load().mw_kvcache_slot_of(ctypes.byref(self.desc), int(chunk)))

    def set_sink(self, k_sink, v_sink) -> None:
        """Keep k_sink/v_sink (bf16 [B,H,sink_len,D]) as the sink anchor; None removes it."""
        d = self.desc
        if k_sink is None:
            _check(load().mw_kvcache_set_sink(ctypes.byref(d), None, None, 0))
            self._sink = None
            return
        for n, t in (("k_sink", k_sink), ("v_sink", v_sink)):
            if self.fp8:
                _u8_4d(n, t)
            else:
                _bf16_4d(n, t)
            if tuple(t.shape[:2]) != (d.B, d.H) or t.shape[3] != d.D or t.shape != k_sink.shape:
                raise ValueError(f"{n} must be [B,H,sink_len,D] with B,H,D of the cache")
        _check(load().mw_kvcache_set_sink(ctypes.byref(d), _ptr(k_sink), _ptr(v_sink), int(k_sink.shape[2])))
        self._sink = (k_sink, v_sink)  # keep the tensors alive while the cache points at them

    def snapshot(self) -> bytes:
        """A copy of the whole descriptor (ring counters, sink, e4m3 re-shift record); the slot
        buffers' contents are the caller's to save alongside."""
        return bytes(self.desc)

    def restore(self, snap: bytes) -> None:
        ctypes.memmove(ctypes.byref(self.desc), snap, ctypes.sizeof(mw_kvcache))


def mw_kvcache_append(cache: KVCache, k_chunk, v_chunk) -> int:
    """Commit one chunk (bf16 [B,H,L,D], or a view of one with a contiguous head
    dimension); returns the slot it was written to."""
    d = cache.desc
    if not _plain_views((k_chunk, v_chunk), (d.B, d.H, d.L, d.D), cache.k_slots):
        for n, t in (("k_chunk", k_chunk), ("v_chunk", v_chunk)):
            _bf16_4d(n, t, view=True)
            if tuple(t.shape) != (d.B, d.H, d.L, d.D):
                raise ValueError(f"{n} must be [B,H,L,D] = {(d.B, d.H, d.L, d.D)}")
        _same_device(cache.k_slots, k_chunk, v_chunk)
    dev = cache.k_slots.device
    _check(load().mw_kvcache_append_strided(ctypes.byref(d), _ptr(k_chunk), _ptr(v_chunk),
                                            _strides(k_chunk, v_chunk), _stream_handle(dev)))
    # the slot the library wrote: the newest committed chunk's, by the library's own rule
    return _check(load().mw_kvcache_slot_of(ctypes.byref(d), int(d.head) - 1))


def mw_kvcache_evict(cache: KVCache, n_chunks: int) -> None:
    _check(load().mw_kvcache_evict(ctypes.byref(cache.desc), int(n_chunks)))


def mw_kvcache_set_sink(cache: KVCache, k_sink, v_sink) -> None:
    cache.set_sink(k_sink, v_sink)


def mw_kvcache_rope_shift(cache: KVCache, shift: int, dim_offset: int, dim_count: int, theta: float = 10000.0) -> None:
    """Rotate the keys of all live chunks by -shift positions on the rope band: in place for a
    bf16 cache; recorded, and applied when a call loads the window, for an e4m3 cache."""
    rope = mw_rope(int(dim_offset), int(dim_count), float(theta))
    _check(load().mw_kvcache_rope_shift(ctypes.byref(cache.desc), int(shift), ctypes.byref(rope),
                                        _stream_handle(cache.k_slots.device)))


def mw_kvcache_slot_of(cache: KVCache, chunk: int) -> int:
    return cache.slot_of(chunk)


def mw_chunk_attn_cached_workspace_size(cache: KVCache, n_queued: int, q_len: int, window: int = -1) -> int:
    return int(load().mw_chunk_attn_cached_workspace_size(ctypes.byref(cache.desc), int(n_queued), int(q_len),
                                                          int(window)))


def mw_chunk_attn_cached_plan(cache: KVCache, n_queued: int, q_len: int, window: int = -1,
                              flags: int = MW_QUEUED_CAUSAL, workspace_bytes: int = -1):
    """(n_splits, n_whole) the cached call uses with `workspace_bytes` of workspace
    (-1: the size mw_chunk_attn_cached_workspace_size gives)."""
    if workspace_bytes < 0:
        workspace_bytes = mw_chunk_attn_cached_workspace_size(cache, n_queued, q_len, window)
    ns, nw = ctypes.c_int(0), ctypes.c_int(0)
    _check(load().mw_chunk_attn_cached_plan(ctypes.byref(cache.desc), int(n_queued), int(q_len), int(window),
                                            int(flags), int(workspace_bytes), ctypes.byref(ns), ctypes.byref(nw)))
    return ns.value, nw.value


def mw_chunk_attn_cached(q, k_new, v_new, n_queued: int, q_len: int, cache: KVCache, window: int = -1,
                         flags: int = MW_QUEUED_CAUSAL, scale=None, out=None, lse=None, want_lse: bool = False,
                         workspace=None, split: bool = True):
    """Cached chunk attention of n_queued in-flight chunks.  Returns (o, lse or None).

    With split=True and no workspace given, a workspace of the size the library
    asks for is allocated here (torch); split=False runs the single-pass kernel.
    """
    torch = _torch()
    d = cache.desc
    plain = _plain_views((q, k_new, v_new) if out is None else (q, k_new, v_new, out),
                         (d.B, d.H, n_queued * q_len, d.D), cache.k_slots)
    if not plain:
        for n, t in (("q", q), ("k_new", k_new), ("v_new", v_new)):
            _bf16_4d(n, t, view=True)
            if tuple(t.shape) != (d.B, d.H, n_queued * q_len, d.D):
                raise ValueError(f"{n} must be [B,H,n_queued*q_len,D] = {(d.B, d.H, n_queued * q_len, d.D)}")
        _same_device(cache.k_slots, q, k_new, v_new)
    dev = cache.k_slots.device
    scale = 1.0 / math.sqrt(d.D) if scale is None else float(scale)
    o = torch.empty_like(q) if out is None else out
    if not plain:
        _bf16_4d("out", o, view=True)
        if o.shape != q.shape:
            raise ValueError("out must have the shape of q")
    if want_lse and lse is None:
        lse = torch.empty((d.B, d.H, n_queued * q_len), dtype=torch.float32, device=dev)
    _check_lse(lse, (d.B, d.H, n_queued * q_len), dev)
    if split and workspace is None:
        need = mw_chunk_attn_cached_workspace_size(cache, n_queued, q_len, window)
        workspace = torch.empty(need, dtype=torch.uint8, device=dev) if need > 0 else None
    if not split:
        workspace = None
    _same_device(q, o, workspace)
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(load().mw_chunk_attn_cached_strided(_ptr(q), _ptr(k_new), _ptr(v_new), int(n_queued), int(q_len),
                                               ctypes.byref(d), int(window), int(flags), _ptr(o), _ptr(lse), scale,
                                               _ptr(workspace), nbytes, _strides(q, k_new, v_new, o),
                                               _stream_handle(dev)))
    return o, lse


# ----------------------------------------------------------------------------- fp8 inference variant

def mw_quantize_fp8(x, scale: float, out=None):
    """bf16 [B,H,T,D] view -> contiguous e4m3 codes (uint8 [B,H,T,D]), code = RNE(clamp(x / scale))."""
    torch = _torch()
    _bf16_4d("x", x, view=True)
    B, H, T, D = x.shape
    y = torch.empty((B, H, T, D), dtype=torch.uint8, device=x.device) if out is None else out
    _u8_4d("out", y)
    if tuple(y.shape) != (B, H, T, D):
        raise ValueError("out must have the shape of x")
    _same_device(x, y)
    _check(load().mw_quantize_fp8(_ptr(x), _strides(x), _ptr(y), B, H, T, D, float(scale), _stream_handle(x.device)))
    return y


def mw_chunk_attn_cached_fp8(q8, k8_new, v8_new, n_queued: int, q_len: int, cache: KVCache, q_scale: float,
                             window: int = -1, flags: int = MW_QUEUED_CAUSAL, scale=None, out=None, lse=None,
                             want_lse: bool = False, workspace=None, split: bool = True):
    """Cached chunk attention over an e4m3 cache.  q8, k8_new, v8_new: e4m3 codes
    (uint8 [B,H,n_queued*q_len,D]; q8 with q_scale, k8/v8 with the cache's
    scales).  Returns (o bf16, lse or None)."""
    torch = _torch()
    d = cache.desc
    for n, t in (("q8", q8), ("k8_new", k8_new), ("v8_new", v8_new)):
        _u8_4d(n, t)
        if tuple(t.shape) != (d.B, d.H, n_queued * q_len, d.D):
            raise ValueError(f"{n} must be [B,H,n_queued*q_len,D] = {(d.B, d.H, n_queued * q_len, d.D)}")
    dev = _same_device(cache.k_slots, q8, k8_new, v8_new)
    scale = 1.0 / math.sqrt(d.D) if scale is None else float(scale)
    o = torch.empty(tuple(q8.shape), dtype=torch.bfloat16, device=dev) if out is None else out
    _bf16_4d("out", o, view=True)
    if o.shape != q8.shape:
        raise ValueError("out must have the shape of q8")
    if want_lse and lse is None:
        lse = torch.empty((d.B, d.H, n_queued * q_len), dtype=torch.float32, device=dev)
    _check_lse(lse, (d.B, d.H, n_queued * q_len), dev)
    if split and workspace is None:
        need = mw_chunk_attn_cached_workspace_size(cache, n_queued, q_len, window)
        workspace = torch.empty(need, dtype=torch.uint8, device=dev) if need > 0 else None
    if not split:
        workspace = None
    _same_device(q8, o, workspace)
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(load().mw_chunk_attn_cached_fp8(_ptr(q8), _ptr(k8_new), _ptr(v8_new), int(n_queued), int(q_len),
                                           ctypes.byref(d), int(window), int(flags), _ptr(o), _ptr(lse), scale,
                                           float(q_scale), _ptr(workspace), nbytes, _strides(o), _stream_handle(dev)))
    return o, lse


# ----------------------------------------------------------------------------- cross attention

_HERE = contextlib.nullcontext()


def _on_device(dev):
    """The calls below launch on the current device: make `dev` current for one that is not."""
    torch = _torch()
    if not torch.cuda.is_initialized() or torch._C._cuda_getDevice() == dev.index:
        return _HERE
    return torch.cuda.device(dev)


def _check_like(name, t, shape, dev):
    """A bf16 view of the given shape on `dev` (its strides are the library's to check)."""
    _bf16_4d(name, t, view=True)
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.device != dev:
        raise ValueError("all tensors must be on the same device")


def _check_workspace(workspace, dev):
    if workspace is None:
        return 0
    if workspace.device != dev or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on the device of the inputs")
    return workspace.nbytes


def _cross_args(q, k, v, kv_len, rows, keys, named):
    """Sizes of a cross attention call.  `rows` are its [B,H,T,D] tensors, `keys` its [B,Hkv,M,D] ones; named() gives
    what of them is neither q, k nor v by name (or None), for the errors."""
    torch = _torch()
    if not (_plain_views(rows, q.shape, q) and _plain_views(keys, k.shape, q)):
        for n, t in (("q", q), ("k", k), ("v", v)):
            _bf16_4d(n, t, view=True)
        like_q, like_k = named()
        for n, t in like_q.items():
            if t is not None:
                _check_like(n, t, q.shape, q.device)
        for n, t in (("k", k), ("v", v), *like_k.items()):
            if t is not None:
                _check_like(n, t, k.shape, q.device)
    B, H, T, D = q.shape
    Bk, Hkv, M, Dk = k.shape
    if Bk != B or Dk != D:
        raise ValueError(f"k and v must be [B,Hkv,M,D] with B, D = {B}, {D}, got {tuple(k.shape)}")
    dev = q.device
    if kv_len is not None and (kv_len.dtype is not torch.int32 or kv_len.shape != (B,) or kv_len.device != dev
                               or not kv_len.is_contiguous()):
        raise ValueError(f"kv_len must be a contiguous int32 tensor of shape {(B,)} on the device of the inputs")
    return B, H, Hkv, T, M, D, dev


def _aligned(kv_len):
    """kv_len, or a copy of one whose first entry is not on 16 bytes, as the library wants it: a slice of a longer
    list of lengths.  (A sum, not a clone: a kernel, which a captured graph repeats over the list's new values.)"""
    return kv_len if kv_len is None or kv_len.data_ptr() % 16 == 0 else kv_len + 0


def mw_cross_attn_workspace_size(B: int, H: int, Hkv: int, T: int, M: int, D: int) -> int:
    return int(load().mw_cross_attn_workspace_size(B, H, Hkv, T, M, D))


def mw_cross_attn_fwd(q, k, v, kv_len=None, scale=None, out=None, lse=None, workspace=None):
    """Cross attention forward.  q: bf16 [B,H,T,D]; k, v: bf16 [B,Hkv,M,D] with Hkv dividing H (views with a
    contiguous head dimension are read in place); kv_len: int32 [B] on the GPU (a slice of a
    longer list too), the valid states of each batch member (None: all M).  Returns (o, lse).

    With no workspace given, one of the size the library asks for is allocated here (torch)."""
    torch = _torch()
    B, H, Hkv, T, M, D, dev = _cross_args(q, k, v, kv_len, (q,) if out is None else (q, out), (k, v),
                                             lambda: ({"out": out}, {}))
    scale = 1.0 / math.sqrt(D) if scale is None else float(scale)
    o = torch.empty_like(q) if out is None else out
    lse = torch.empty((B, H, T), dtype=torch.float32, device=dev) if lse is None else lse
    _check_lse(lse, (B, H, T), dev)
    if workspace is None:
        need = mw_cross_attn_workspace_size(B, H, Hkv, T, M, D)
        workspace = torch.empty(need, dtype=torch.uint8, device=dev) if need > 0 else None
    nbytes = _check_workspace(workspace, dev)
    kv_len = _aligned(kv_len)
    with _on_device(dev):
        _check(load().mw_cross_attn_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(kv_len), _ptr(o), _ptr(lse),
                                        _strides(q, k, v, o), B, H, Hkv, T, M, D, scale, _ptr(workspace), nbytes,
                                        _stream_handle(dev)))
    return o, lse


def mw_cross_attn_bwd_workspace_size(B: int, H: int, Hkv: int, T: int, M: int, D: int) -> int:
    return int(load().mw_cross_attn_bwd_workspace_size(B, H, Hkv, T, M, D))


def mw_cross_attn_bwd(q, k, v, o, d_o, lse, kv_len=None, scale=None, workspace=None, dq=None, dk=None, dv=None):
    """Backward of mw_cross_attn_fwd.  Returns (dq, dk, dv): bf16 [B,H,T,D] and twice [B,Hkv,M,D], the latter
    summed over the query heads that share a key head and 0 behind kv_len."""
    torch = _torch()
    B, H, Hkv, T, M, D, dev = _cross_args(q, k, v, kv_len, (q, o, d_o) if dq is None else (q, o, d_o, dq),
                                          (k, v, *(t for t in (dk, dv) if t is not None)),
                                          lambda: ({"o": o, "d_o": d_o, "dq": dq}, {"dk": dk, "dv": dv}))
    if lse is None:
        raise ValueError("lse is required")
    _check_lse(lse, (B, H, T), dev)
    scale = 1.0 / math.sqrt(D) if scale is None else float(scale)
    if workspace is None:
        workspace = torch.empty(mw_cross_attn_bwd_workspace_size(B, H, Hkv, T, M, D), dtype=torch.uint8, device=dev)
    nbytes = _check_workspace(workspace, dev)
    # (a gradient of states shared between batch members or heads does not share their strides)
    dq = torch.empty((B, H, T, D), dtype=q.dtype, device=dev) if dq is None else dq
    dk = torch.empty((B, Hkv, M, D), dtype=q.dtype, device=dev) if dk is None else dk
    dv = torch.empty((B, Hkv, M, D), dtype=q.dtype, device=dev) if dv is None else dv
    kv_len = _aligned(kv_len)
    with _on_device(dev):
        _check(load().mw_cross_attn_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(kv_len), _ptr(o), _ptr(d_o), _ptr(lse), _ptr(dq),
                                        _ptr(dk), _ptr(dv), _ptr(workspace), nbytes,
                                        _strides(q, k, v, o, d_o, dq, dk, dv), B, H, Hkv, T, M, D, scale,
                                        _stream_handle(dev)))
    return dq, dk, dv


# ----------------------------------------------------------------------------- packed sequences

class Packed:
    """Plan of a batch of sequences that lie one behind the other: cu_q int32 [N+1] on the GPU, the places where their
    queries begin (and the last one ends) among total_q tokens; cu_k and total_k those of their keys (default: the
    same).  H query heads share Hkv key heads of width D; chunk_len as in mw_block_causal_attn_fwd (1: token-causal).
    backward=True plans the backward too.

    update() plans again, over new contents of cu_q and cu_k; it may be captured into a graph.
    Wraps the mw_packed descriptor.
    """

    def __init__(self, cu_q, total_q: int, H: int, Hkv: int, D: int, chunk_len: int = 1, cu_k=None, total_k=None,
                 backward: bool = False):
        torch = _torch()
        self.cu_q, self.cu_k = cu_q, cu_q if cu_k is None else cu_k
        total_k = total_q if total_k is None else total_k
        for n, t in (("cu_q", self.cu_q), ("cu_k", self.cu_k)):
            if t.dtype is not torch.int32 or t.dim() != 1 or t.shape[0] < 2 or not t.is_contiguous() or t.device.type != "cuda":
                raise ValueError(f"{n} must be a contiguous int32 tensor of N + 1 entries on a GPU")
        if self.cu_k.shape != cu_q.shape or self.cu_k.device != cu_q.device:
            raise ValueError("cu_q and cu_k must have the same length and device")
        self.device = cu_q.device
        self._sizes = (cu_q.shape[0] - 1, *map(_int32, (total_q, total_k, H, Hkv, D, chunk_len)), int(bool(backward)))
        self.q_shape, self.k_shape = (self._sizes[1], H, D), (self._sizes[2], Hkv, D)
        self.lse_shape = (H, self._sizes[1])
        need = int(load().mw_packed_plan_bytes(*self._sizes))
        self.plan = torch.empty(need // 4, dtype=torch.int32, device=self.device)
        self.desc = mw_packed()
        self._ref = ctypes.byref(self.desc)
        self.scale = 1.0 / math.sqrt(max(1, self._sizes[5]))
        if need == 0:  # sizes out of range: the library says which
            _check(load().mw_packed_init(self._ref, _ptr(self.cu_q), _ptr(self.cu_k), 16, 0, *self._sizes, None))
        self.update()

    def update(self) -> None:
        with _on_device(self.device):
            _check(load().mw_packed_init(self._ref, _ptr(self.cu_q), _ptr(self.cu_k), _ptr(self.plan),
                                         self.plan.nbytes, *self._sizes, _stream_handle(self.device)))


def _packed_views(pack: Packed, queries, keys):
    """Strides of bf16 views [total_q,H,D] (`queries`: tensors by name, or None) and [total_k,Hkv,D] on the batch's
    device, as the library wants them, in the order given."""
    bf16, index = _torch().bfloat16, pack.device.index
    strides = []
    for shape, named in ((pack.q_shape, queries), (pack.k_shape, keys)):
        for n, t in named.items():
            s = t.stride()
            if t.dtype is bf16 and t.shape == shape and s[2] == 1 and t.get_device() == index:
                strides.append(s)
                continue
            if t.dtype is not bf16:
                raise TypeError(f"{n} must be bfloat16, got {t.dtype}")
            if t.shape != shape:
                raise ValueError(f"{n} must have shape {shape}, got {tuple(t.shape)}")
            if t.get_device() != index:
                raise ValueError("all tensors must be on the GPU of the batch")
            raise ValueError(f"{n} must have a contiguous last (head) dimension")
    return strides


@functools.lru_cache(maxsize=512)
def _packed_strides(*strides):
    """mw_strides array of [T,H,D] views (kept by its values, as _strides_array's)."""
    return _strides_array(*[(0, s[1], s[0]) for s in strides])


def mw_packed_attn_workspace_size(pack: Packed) -> int:
    return int(load().mw_packed_attn_workspace_size(pack._ref))


def mw_packed_attn_fwd(q, k, v, pack: Packed, scale=None, out=None, lse=None, workspace=None):
    """Attention of packed sequences.  q: bf16 [total_q,H,D]; k, v: bf16 [total_k,Hkv,D] (views with a contiguous head
    dimension are read in place).  Returns (o, lse): bf16 like q and fp32 [H,total_q]; rows behind the last
    sequence are not written.

    With no workspace given, one of the size the library asks for is allocated here (torch)."""
    torch = _torch()
    o = torch.empty_like(q) if out is None else out
    sq, so, sk, sv = _packed_views(pack, {"q": q, "out": o}, {"k": k, "v": v})
    dev = pack.device
    scale = pack.scale if scale is None else float(scale)
    lse = torch.empty(pack.lse_shape, dtype=torch.float32, device=dev) if lse is None else lse
    _check_lse(lse, pack.lse_shape, dev)
    if workspace is None:
        need = mw_packed_attn_workspace_size(pack)
        workspace = torch.empty(need, dtype=torch.uint8, device=dev) if need > 0 else None
    nbytes = _check_workspace(workspace, dev)
    with _on_device(dev):
        _check(load().mw_packed_attn_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), pack._ref, o.data_ptr(), lse.data_ptr(), scale,
                                         _ptr(workspace), nbytes, _packed_strides(sq, sk, sv, so), _stream_handle(dev)))
    return o, lse


def mw_packed_attn_bwd_workspace_size(pack: Packed) -> int:
    need = int(load().mw_packed_attn_bwd_workspace_size(pack._ref))
    if need == 0:
        _check(MW_EINVAL)  # (planned without the backward)
    return need


def mw_packed_attn_bwd(q, k, v, o, d_o, lse, pack: Packed, scale=None, workspace=None, dq=None, dk=None, dv=None):
    """Backward of mw_packed_attn_fwd, for a batch planned with backward=True.  Returns (dq, dk, dv): bf16 [total_q,H,D]
    and twice [total_k,Hkv,D], the latter summed over the query heads that share a key head."""
    torch = _torch()
    dev = pack.device
    # (a gradient of keys shared between heads does not share their strides)
    dq = torch.empty(pack.q_shape, dtype=q.dtype, device=dev) if dq is None else dq
    dk = torch.empty(pack.k_shape, dtype=q.dtype, device=dev) if dk is None else dk
    dv = torch.empty(pack.k_shape, dtype=q.dtype, device=dev) if dv is None else dv
    sq, so, sdo, sdq, sk, sv, sdk, sdv = _packed_views(pack, {"q": q, "o": o, "d_o": d_o, "dq": dq},
                                                       {"k": k, "v": v, "dk": dk, "dv": dv})
    if lse is None:
        raise ValueError("lse is required")
    _check_lse(lse, pack.lse_shape, dev)
    scale = pack.scale if scale is None else float(scale)
    if workspace is None:
        workspace = torch.empty(mw_packed_attn_bwd_workspace_size(pack), dtype=torch.uint8, device=dev)
    nbytes = _check_workspace(workspace, dev)
    with _on_device(dev):
        _check(load().mw_packed_attn_bwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), d_o.data_ptr(), lse.data_ptr(),
                                         pack._ref, dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), scale, _ptr(workspace), nbytes,
                                         _packed_strides(sq, sk, sv, so, sdo, sdq, sdk, sdv), _stream_handle(dev)))
    return dq, dk, dv


# ----------------------------------------------------------------------------- rotary positions

def rope_bands(bands, halves: bool = False, gain: float = 1.0) -> mw_rope_bands:
    """Bands of the head for mw_rope_apply (see include/mw.h): dicts of dim_offset and dim_count, and optionally theta
    (10000), axis (0), factor (1), trained_len, turns_lo and turns_hi.  halves: pairs (i, i + dim_count/2), else
    (2i, 2i+1)."""
    arr = (mw_rope_band * max(1, len(bands)))()
    for x, b in zip(arr, bands):
        b = {"theta": 1e4, "axis": 0, "factor": 1.0, "trained_len": 0.0, "turns_lo": 0.0, "turns_hi": 0.0, **b}
        for n, v in b.items():
            if n not in dict(mw_rope_band._fields_):
                raise ValueError(f"a band has no {n}")
            setattr(x, n, _int32(v) if n in ("dim_offset", "dim_count", "axis") else float(v))
    out = mw_rope_bands()
    _check(load().mw_rope_bands_init(ctypes.byref(out), arr, len(bands), int(bool(halves)), float(gain)))
    return out


def mw_rope_apply(q, k, bands: mw_rope_bands, positions=None, first: int = 0, inverse: bool = False, q_out=None, k_out=None):
    """Rotary positions applied to q (bf16 [B,H,T,D]) and k (bf16 [B,Hkv,T,D], or None), or with inverse=True taken
    back, which gives the gradients of q and k from those of the outputs.  positions: int32 or int64 on the GPU, [T] or
    [B,T], for bands of several axes [axes,T] or [axes,B,T]; None: first, first + 1, ...  Views with a contiguous
    head dimension are read and written in place; an output may be its input.  Returns (q_out, k_out)."""
    shape = q.shape
    if not _plain_views((q,) if q_out is None else (q, q_out), shape, q):
        _bf16_4d("q", q, view=True)
        if q_out is not None:
            _check_like("q_out", q_out, shape, q.device)
    B, H, T, D = shape
    dev, Hkv = q.device, 0
    if k is not None:
        k_shape = (B, k.shape[1] if k.dim() == 4 else 0, T, D)
        Hkv = k_shape[1]
        if not _plain_views((k,) if k_out is None else (k, k_out), k_shape, q):
            _check_like("k", k, k_shape, dev)
            if k_out is not None:
                _check_like("k_out", k_out, k_shape, dev)
    elif k_out is not None:
        raise ValueError("k_out without k")
    pos_strides, pos_bytes, pos = None, 0, 0
    if positions is not None:
        pos, pos_bytes, pos_strides = _positions(positions, bands.n_axes, B, T, dev)
    elif not -2**62 <= operator.index(first) < 2**62:
        raise ValueError(f"{first} is out of range")
    q_out = _torch().empty_like(q) if q_out is None else q_out
    if k is None:
        strides = _strides(q, q, q_out, q_out)
    else:
        k_out = _torch().empty_like(k) if k_out is None else k_out
        strides = _strides(q, k, q_out, k_out)
    with _on_device(dev):
        _check(load().mw_rope_apply(q.data_ptr(), _ptr(k), q_out.data_ptr(), _ptr(k_out), ctypes.byref(bands), pos, pos_bytes,
                                    pos_strides, first, 1 if inverse else 0, strides, B, H, Hkv, T, D, _stream_handle(dev)))
    return q_out, k_out


def _positions(p, axes, B, T, dev):
    """Address, bytes and strides (member, axis, token) of a tensor of positions."""
    torch = _torch()
    if p.dtype not in (torch.int32, torch.int64) or p.device != dev:
        raise ValueError("positions must be int32 or int64 on the device of q")
    s, shape = p.stride(), p.shape
    if axes > 1:
        if shape != (axes, T) and shape != (axes, B, T):
            raise ValueError(f"positions must be [axes,T] or [axes,B,T] = {(axes, B, T)}, got {tuple(shape)}")
        strides = (s[1] if len(s) == 3 else 0, s[0], s[-1])
    else:
        if shape != (T,) and shape != (B, T):
            raise ValueError(f"positions must be [T] or [B,T] = {(B, T)}, got {tuple(shape)}")
        strides = (s[0] if len(s) == 2 else 0, 0, s[-1])
    return p.data_ptr(), p.element_size(), _strides_array(strides)


# ----------------------------------------------------------------------------- paged 8-bit cache

class KVPages:
    """Paged cache of e4m3 keys and values with a power-of-two scale for each 64 tokens and head, over
    torch-owned tensors: k_pages, v_pages uint8 [P,H,L,D], k_scales, v_scales fp32 [P,H,L/64], table int32
    [N,W] and lens int32 [N].  N sequences of at most W pages of L tokens; the page bookkeeping is the library's.

    Wraps the mw_kvpages descriptor.
    """

    def __init__(self, P: int, H: int, L: int, D: int, N: int, W: int, device="cuda"):
        torch = _torch()
        device = torch.device(device)
        if device.type == "cuda" and device.index is None:
            device = torch.device("cuda", torch.cuda.current_device())
        need = int(load().mw_kvpages_host_bytes(P, N, W))
        if need == 0 or min(H, L, D) < 1:
            raise MWError(MW_EINVAL, f"KVPages: sizes out of range (P={P}, H={H}, L={L}, D={D}, N={N}, W={W})")
        self.k_pages, self.v_pages = (torch.empty((P, H, L, D), dtype=torch.uint8, device=device) for _ in range(2))
        self.k_scales, self.v_scales = (torch.empty((P, H, max(1, L // MW_PAGE_BLOCK)), dtype=torch.float32,
                                                    device=device) for _ in range(2))
        self.table = torch.empty((N, W), dtype=torch.int32, device=device)
        self.lens = torch.zeros((N,), dtype=torch.int32, device=device)
        self.device = device
        self._host = (ctypes.c_int32 * (need // 4))()
        self.desc = mw_kvpages()
        _check(load().mw_kvpages_init(ctypes.byref(self.desc), _ptr(self.k_pages), _ptr(self.v_pages),
                                      _ptr(self.k_scales), _ptr(self.v_scales), _ptr(self.table), _ptr(self.lens),
                                      ctypes.addressof(self._host), need, P, H, L, D, N, W))

    @property
    def n_free(self) -> int:
        return _check(load().mw_kvpages_n_free(ctypes.byref(self.desc)))

    def len(self, seq: int) -> int:
        return _check(load().mw_kvpages_len(ctypes.byref(self.desc), _int32(seq)))

    def page_of(self, seq: int, index: int) -> int:
        return _check(load().mw_kvpages_page_of(ctypes.byref(self.desc), _int32(seq), _int32(index)))


def _int32(x) -> int:
    """An integer that a C int holds (ctypes takes any and keeps its low bits)."""
    x = operator.index(x)
    if not -2**31 <= x < 2**31:
        raise ValueError(f"{x} is out of range")
    return x


@functools.lru_cache(maxsize=512)
def _seq_array(seqs):
    return (ctypes.c_int32 * len(seqs))(*seqs)


def _seqs(seqs):
    """Host array of sequence numbers (the library only reads it)."""
    if isinstance(seqs, ctypes.Array):
        return seqs
    return _seq_array(tuple(map(_int32, seqs)))


def mw_kvpages_append(cache: KVPages, seqs, k, v) -> None:
    """Commit k, v (bf16 [len(seqs),H,n_tokens,D] views) to the ends of the listed sequences."""
    d, dev = cache.desc, cache.device
    seqs = _seqs(seqs)
    if not _plain_views((k, v), k.shape, cache.k_pages) or (k.shape[0], k.shape[1], k.shape[3]) != (len(seqs), d.H, d.D):
        for n, t in (("k", k), ("v", v)):
            _bf16_4d(n, t, view=True)
            _check_like(n, t, (len(seqs), d.H, k.shape[2], d.D), dev)
    with _on_device(dev):
        _check(load().mw_kvpages_append(ctypes.byref(d), seqs, len(seqs), _ptr(k), _ptr(v), _strides(k, v), k.shape[2],
                                        _stream_handle(dev)))


def mw_kvpages_fork(cache: KVPages, src: int, dst: int) -> None:
    """Make the empty sequence dst a branch of src that shares its pages."""
    with _on_device(cache.device):
        _check(load().mw_kvpages_fork(ctypes.byref(cache.desc), _int32(src), _int32(dst), _stream_handle(cache.device)))


def mw_kvpages_copy(cache: KVPages, src: int, dst: int) -> None:
    """Make the empty sequence dst a copy of src in pages of its own."""
    with _on_device(cache.device):
        _check(load().mw_kvpages_copy(ctypes.byref(cache.desc), _int32(src), _int32(dst), _stream_handle(cache.device)))


def mw_kvpages_free(cache: KVPages, seqs) -> None:
    """Empty the listed sequences; pages that no other sequence shares become free."""
    seqs = _seqs(seqs)
    with _on_device(cache.device):
        _check(load().mw_kvpages_free(ctypes.byref(cache.desc), seqs, len(seqs), _stream_handle(cache.device)))


def mw_kvpages_evict(cache: KVPages, seq: int, first_page: int, n_pages: int) -> None:
    """Drop the full pages [first_page, first_page + n_pages) of a sequence."""
    with _on_device(cache.device):
        _check(load().mw_kvpages_evict(ctypes.byref(cache.desc), _int32(seq), _int32(first_page), _int32(n_pages),
                                       _stream_handle(cache.device)))


def mw_kvpages_compact(cache: KVPages) -> int:
    """Move live pages to the front of the pool; returns how many moved."""
    with _on_device(cache.device):
        return _check(load().mw_kvpages_compact(ctypes.byref(cache.desc), _stream_handle(cache.device)))


def mw_kvpages_weigh_workspace_size(cache: KVPages, seqs, H: int, T: int) -> int:
    seqs = _seqs(seqs)
    return int(load().mw_kvpages_weigh_workspace_size(ctypes.byref(cache.desc), seqs, len(seqs), _int32(H), _int32(T)))


def _check_weights(cache: KVPages, weights):
    d = cache.desc
    if weights.dtype is not _torch().float32 or weights.shape != (d.N, d.W * d.L) or not weights.is_contiguous():
        raise ValueError(f"weights must be a contiguous fp32 tensor of shape {(d.N, d.W * d.L)}, got {weights.dtype} "
                         f"{tuple(weights.shape)}")
    if weights.device != cache.device:
        raise ValueError("weights must be on the device of the cache")


def mw_kvpages_weigh(cache: KVPages, seqs, q, lse, weights, add: bool = True, scale=None, workspace=None) -> None:
    """Sum, over the rows and heads of a mw_chunk_attn_paged call, of the attention weight that each cached token of the
    listed sequences got, into weights (fp32 [N, W*L], a row for each sequence): added, or (add=False) written.
    q: bf16 [len(seqs),H,T,D] and lse: fp32 [len(seqs),H,T], as given to and left by that call.

    With no workspace given, one of the size the library asks for is allocated here (torch)."""
    torch = _torch()
    d, dev = cache.desc, cache.device
    seqs = _seqs(seqs)
    if not _plain_views((q,), q.shape, cache.k_pages) or (q.shape[0], q.shape[3]) != (len(seqs), d.D):
        _bf16_4d("q", q, view=True)
        _check_like("q", q, (len(seqs), *q.shape[1:3], d.D), dev)
    B, H, T, _ = q.shape
    if lse is None:
        raise ValueError("lse is required")
    _check_lse(lse, (B, H, T), dev)
    _check_weights(cache, weights)
    if workspace is None:
        need = mw_kvpages_weigh_workspace_size(cache, seqs, H, T)
        workspace = torch.empty(need, dtype=torch.uint8, device=dev) if need > 0 else None
    nbytes = _check_workspace(workspace, dev)
    scale = 1.0 / math.sqrt(d.D) if scale is None else float(scale)
    with _on_device(dev):
        _check(load().mw_kvpages_weigh(ctypes.byref(d), seqs, B, _ptr(q), _ptr(lse), H, T, _ptr(weights), int(bool(add)), scale,
                                       _ptr(workspace), nbytes, _strides(q), _stream_handle(dev)))


def mw_kvpages_evict_weighted_workspace_size(cache: KVPages, seqs, n_keep: int, first: int = 0) -> int:
    seqs = _seqs(seqs)
    return int(load().mw_kvpages_evict_weighted_workspace_size(ctypes.byref(cache.desc), seqs, len(seqs), _int32(n_keep),
                                                               _int32(first)))


def mw_kvpages_evict_weighted(cache: KVPages, seqs, weights, n_keep: int, first: int = 0, recent: int = 0,
                              workspace=None) -> None:
    """Drop the lightest tokens of the listed sequences by their rows of weights (fp32 [N, W*L], moved alike), so that
    n_keep stay: the first `first`, the last `recent` and the heaviest of the others, in their order."""
    dev = cache.device
    seqs = _seqs(seqs)
    _check_weights(cache, weights)
    if workspace is None:
        need = mw_kvpages_evict_weighted_workspace_size(cache, seqs, n_keep, first)
        workspace = _torch().empty(max(16, need), dtype=_torch().uint8, device=dev)
    nbytes = _check_workspace(workspace, dev)
    with _on_device(dev):
        _check(load().mw_kvpages_evict_weighted(ctypes.byref(cache.desc), seqs, len(seqs), _ptr(weights), _int32(n_keep),
                                                _int32(first), _int32(recent), _ptr(workspace), nbytes, _stream_handle(dev)))


def mw_chunk_attn_paged_workspace_size(cache: KVPages, seqs, H: int, n_queued: int, q_len: int) -> int:
    seqs = _seqs(seqs)
    return int(load().mw_chunk_attn_paged_workspace_size(ctypes.byref(cache.desc), seqs, len(seqs), int(H),
                                                         int(n_queued), int(q_len)))


def mw_chunk_attn_paged(q, k_new, v_new, n_queued: int, q_len: int, cache: KVPages, seqs,
                        flags: int = MW_QUEUED_CAUSAL, scale=None, out=None, lse=None, want_lse: bool = False,
                        workspace=None, split: bool = True):
    """Cached chunk attention of n_queued in-flight chunks over the pages of the listed sequences.  q: bf16
    [len(seqs),H,n_queued*q_len,D]; k_new, v_new: the queued tokens' keys and values with the cache's heads, or
    None, None.  Returns (o, lse or None); workspace and split as in mw_chunk_attn_cached."""
    torch = _torch()
    d, dev = cache.desc, cache.device
    seqs = _seqs(seqs)
    B, T = len(seqs), n_queued * q_len
    if (k_new is None) != (v_new is None):
        raise ValueError("k_new and v_new are given together or not at all")
    H = q.shape[1] if len(q.shape) == 4 else 0
    if not (_plain_views((q,) if out is None else (q, out), (B, H, T, d.D), cache.k_pages)
            and (k_new is None or _plain_views((k_new, v_new), (B, d.H, T, d.D), cache.k_pages))):
        for n, t, heads in (("q", q, H), ("out", out, H), ("k_new", k_new, d.H), ("v_new", v_new, d.H)):
            if t is not None:
                _check_like(n, t, (B, heads, T, d.D), dev)
    scale = 1.0 / math.sqrt(d.D) if scale is None else float(scale)
    o = torch.empty_like(q) if out is None else out
    if want_lse and lse is None:
        lse = torch.empty((B, H, T), dtype=torch.float32, device=dev)
    _check_lse(lse, (B, H, T), dev)
    if not split:
        workspace = None
    elif workspace is None:
        need = mw_chunk_attn_paged_workspace_size(cache, seqs, H, n_queued, q_len)
        workspace = torch.empty(need, dtype=torch.uint8, device=dev) if need > 0 else None
    nbytes = _check_workspace(workspace, dev)
    ks, vs = (q, q) if k_new is None else (k_new, v_new)
    with _on_device(dev):
        _check(load().mw_chunk_attn_paged(_ptr(q), _ptr(k_new), _ptr(v_new), int(n_queued), int(q_len), ctypes.byref(d),
                                          seqs, B, H, int(flags), _ptr(o), _ptr(lse), scale, _ptr(workspace), nbytes,
                                          _strides(q, ks, vs, o), _stream_handle(dev)))
    return o, lse


# ----------------------------------------------------------------------------- pipelined denoising schedule

def sched_config(window: int, stride: int, n_chunks: int, cache_chunks: int, frames_per_chunk: int,
                 sink_frames: int = 0, shift: float = 1.0, n_bins: int = 0) -> mw_sched_config:
    return mw_sched_config(int(window), int(stride), int(n_chunks), int(cache_chunks), int(frames_per_chunk),
                           int(sink_frames), float(shift), int(n_bins))


def mw_sched_num_ticks(cfg: mw_sched_config) -> int:
    return int(_check(load().mw_sched_num_ticks(ctypes.byref(cfg))))


def mw_sched_plan(cfg: mw_sched_config, tick: int) -> dict:
    """Plan of one tick of the pipelined denoiser (see include/mw.h) as a dict."""
    out = mw_sched_tick()
    _check(load().mw_sched_plan(ctypes.byref(cfg), int(tick), ctypes.byref(out)))
    n = out.n_active
    return {"tick": int(out.tick), "first": out.first, "n_active": n, "updates_per_chunk": out.updates_per_chunk,
            "ids": list(range(out.first, out.first + n)), "tau": list(out.tau[:n]), "dtau": list(out.dtau[:n]),
            "n_commit": out.n_commit, "committed": list(range(out.first, out.first + out.n_commit)),
            "n_evict": out.n_evict, "rope_shift": out.rope_shift, "cache_live": out.cache_live,
            "pos_first": out.pos_first}
