"""Python binding of the LUVC C-ABI library (``include/luvc.h``).

Argument marshalling only: every step of OIM (Section 3.2 of arXiv 2512.09010), of
SPU (Section 3.3, Algorithm 2) and of the paged key-value cache that takes their tokens
runs inside ``libluvc.so``'s CUDA kernels.  PyTorch is used for device memory and streams.  There is no CPU fallback: if the shared
library cannot be built or loaded, importing this package fails.
"""
from __future__ import annotations

import ctypes
import os

import torch

from . import _build

BF16, F32, E4M3 = 0, 1, 2
DEFAULT_CUTOFF = 0.125

STATUS_NAMES = {
    0: "LUVC_OK", 1: "LUVC_ERR_NULL", 2: "LUVC_ERR_SHAPE", 3: "LUVC_ERR_TARGET", 4: "LUVC_ERR_KEEP",
    5: "LUVC_ERR_CUTOFF", 6: "LUVC_ERR_ALIGN", 7: "LUVC_ERR_DTYPE", 8: "LUVC_ERR_WORKSPACE",
    9: "LUVC_ERR_CUDA", 10: "LUVC_ERR_TIMEOUT", 11: "LUVC_ERR_INTERNAL",
    12: "LUVC_ERR_PAGES",
}

# every symbol include/luvc.h declares
EXPORTS = (
    "luvc_version", "luvc_status_string", "luvc_set_stream", "luvc_shutdown", "luvc_kernel_launches",
    "luvc_profile_enable", "luvc_profile_read", "luvc_check_status", "luvc_read_status", "luvc_debug_wait_probes",
    "luvc_oim_plan", "luvc_oim_plan_anyres", "luvc_oim_workspace_bytes", "luvc_oim_workspace_bytes_ex", "luvc_oim_merge", "luvc_oim_merge_f32", "luvc_oim_merge_ex",
    "luvc_oim_merge_host", "luvc_oim_value_enhance", "luvc_spu_sigma", "luvc_spu_workspace_bytes", "luvc_spu_prune",
    "luvc_spu_prune_f32", "luvc_spu_prune_ex", "luvc_spu_prune_host", "luvc_spu_prune_static", "luvc_spu_static_status",
    "luvc_spu_cascade", "luvc_kv_workspace_bytes", "luvc_kv_reserve", "luvc_kv_write", "luvc_kv_fork", "luvc_kv_free",
    "luvc_kv_compact", "luvc_attn_workspace_bytes", "luvc_attn_decode",
)


class LuvcError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib.luvc_status_string(status).decode()
        super().__init__("%s: %s (%s)" % (where, STATUS_NAMES.get(status, status), msg))


class OimOpts(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int), ("stream", ctypes.c_void_p), ("workspace", ctypes.c_void_p),
        ("workspace_bytes", ctypes.c_size_t), ("out_h", ctypes.c_int), ("out_w", ctypes.c_int),
        ("merge_per_step", ctypes.c_int), ("height_first", ctypes.c_int), ("trace", ctypes.c_void_p),
        ("trace_bytes", ctypes.c_size_t), ("out_log_sizes", ctypes.c_void_p), ("matching", ctypes.c_int),
        ("device_status", ctypes.c_void_p), ("merge_per_step_h", ctypes.c_int), ("merge_per_step_w", ctypes.c_int),
    ]


class SpuOpts(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int), ("stream", ctypes.c_void_p), ("workspace", ctypes.c_void_p),
        ("workspace_bytes", ctypes.c_size_t), ("no_window", ctypes.c_int), ("out_scores", ctypes.c_void_p),
        ("device_status", ctypes.c_void_p),
    ]


class KvCacheStruct(ctypes.Structure):
    _fields_ = [
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("lengths", ctypes.c_void_p), ("refs", ctypes.c_void_p),
        ("table", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p), ("layers", ctypes.c_int),
        ("pages", ctypes.c_int), ("heads", ctypes.c_int), ("page_size", ctypes.c_int), ("D", ctypes.c_int),
        ("slots", ctypes.c_int), ("max_pages", ctypes.c_int), ("dtype", ctypes.c_int),
    ]


class KvOpts(ctypes.Structure):
    _fields_ = [
        ("stream", ctypes.c_void_p), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
        ("device_status", ctypes.c_void_p),
    ]


class AttnOpts(ctypes.Structure):
    _fields_ = [
        ("stream", ctypes.c_void_p), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
        ("device_status", ctypes.c_void_p), ("scale", ctypes.c_float), ("key_bias", ctypes.c_void_p),
        ("bias_width", ctypes.c_int), ("bias_stride", ctypes.c_longlong), ("lse", ctypes.c_void_p),
    ]


def _load() -> ctypes.CDLL:
    path = _build.LIB
    if _build.is_stale():
        try:
            _build.build()
        except Exception as exc:  # no compiler: a stale or missing library is an error, not a fallback
            if not os.path.exists(path):
                raise ImportError("libluvc.so is missing and could not be built: %s" % exc) from exc
    L = ctypes.CDLL(path)
    i, p, f, sz = ctypes.c_int, ctypes.c_void_p, ctypes.c_float, ctypes.c_size_t
    L.luvc_version.restype = i
    L.luvc_status_string.restype = ctypes.c_char_p
    L.luvc_status_string.argtypes = [i]
    L.luvc_set_stream.argtypes = [p]
    L.luvc_kernel_launches.restype = ctypes.c_longlong
    L.luvc_check_status.argtypes = [p]
    L.luvc_read_status.argtypes = [p, p]
    L.luvc_debug_wait_probes.argtypes = [i, i, p, p]
    L.luvc_spu_static_status.argtypes = [p]
    L.luvc_oim_plan_anyres.argtypes = [i, i, i, i] + [ctypes.POINTER(i)] * 5
    L.luvc_profile_enable.argtypes = [i]
    L.luvc_profile_read.argtypes = [ctypes.POINTER(ctypes.c_float), i]
    L.luvc_oim_plan.argtypes = [i, i, i, i, ctypes.POINTER(i), ctypes.POINTER(i), ctypes.POINTER(i)]
    L.luvc_oim_workspace_bytes.restype = sz
    L.luvc_oim_workspace_bytes.argtypes = [i, i, i, i, i]
    L.luvc_oim_workspace_bytes_ex.restype = sz
    L.luvc_oim_workspace_bytes_ex.argtypes = [i, i, i, i, i, i]
    L.luvc_oim_merge.argtypes = [p, i, i, i, i, i, p, p, p]
    L.luvc_oim_merge_f32.argtypes = [p, i, i, i, i, i, p, p, p]
    L.luvc_oim_merge_ex.argtypes = [p, i, i, i, i, i, p, p, p, ctypes.POINTER(OimOpts)]
    L.luvc_oim_merge_host.argtypes = [p, i, i, i, i, i, i, p, p, p]
    L.luvc_oim_value_enhance.argtypes = [p, p, i, i, i, i, p, p]
    L.luvc_spu_sigma.argtypes = [i, f]
    L.luvc_spu_workspace_bytes.restype = sz
    L.luvc_spu_workspace_bytes.argtypes = [i, i, i, f, i]
    L.luvc_spu_prune.argtypes = [p, i, i, i, f, i, p, p]
    L.luvc_spu_prune_f32.argtypes = [p, i, i, i, f, i, p, p]
    L.luvc_spu_prune_ex.argtypes = [p, i, i, i, f, i, p, p, ctypes.POINTER(SpuOpts)]
    L.luvc_spu_prune_host.argtypes = [p, i, i, i, f, i, i, p, p]
    L.luvc_spu_prune_static.argtypes = [p, i, i, i, f, i, i, p, p, p]
    L.luvc_spu_cascade.argtypes = [p, i, i, i, i, ctypes.POINTER(i), ctypes.POINTER(f), i, p, p, p]
    cache, kv, ll = ctypes.POINTER(KvCacheStruct), ctypes.POINTER(KvOpts), ctypes.c_longlong
    L.luvc_kv_workspace_bytes.restype = sz
    L.luvc_kv_workspace_bytes.argtypes = [cache, i]
    L.luvc_kv_reserve.argtypes = [cache, p, i, p, kv]
    L.luvc_kv_write.argtypes = [cache, i, p, i, p, p, ll, ll, i, p, p, i, kv]
    L.luvc_kv_fork.argtypes = [cache, p, p, i, kv]
    L.luvc_kv_free.argtypes = [cache, p, i, kv]
    L.luvc_kv_compact.argtypes = [cache, p, i, p, p, p, i, p, kv]
    L.luvc_attn_workspace_bytes.restype = sz
    L.luvc_attn_workspace_bytes.argtypes = []
    L.luvc_attn_decode.argtypes = [p, ll, cache, i, p, i, i, i, p, ctypes.POINTER(AttnOpts)]
    return L


lib = _load()


def _check(status: int, where: str) -> None:
    if status != 0:
        raise LuvcError(status, where)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise TypeError("luvc supports bfloat16 and float32 tensors, got %s" % t.dtype)


def _stream_ptr(device) -> int:
    return torch.cuda.current_stream(device).cuda_stream


def version() -> int:
    return lib.luvc_version()


def kernel_launches() -> int:
    return int(lib.luvc_kernel_launches())


def shutdown() -> None:
    _check(lib.luvc_shutdown(), "luvc_shutdown")


def check_status(device=None) -> int:
    """Synchronises the current torch stream and returns (and clears) the device status word."""
    return int(lib.luvc_check_status(_stream_ptr(device)))


PHASES = ("oim_steps", "oim_total", "spu_transform", "spu_select", "spu_gather")


def profile_enable(on: bool) -> None:
    _check(lib.luvc_profile_enable(int(bool(on))), "luvc_profile_enable")


def profile_read() -> dict:
    """Elapsed milliseconds of the phases of the most recent calls (synchronises their events)."""
    buf = (ctypes.c_float * len(PHASES))()
    _check(lib.luvc_profile_read(buf, len(PHASES)), "luvc_profile_read")
    return {name: float(buf[k]) for k, name in enumerate(PHASES)}


def oim_plan(H: int, W: int, target_count: int, merge_per_step: int = 0):
    """(out_h, out_w, n_steps) for a target token count (host only)."""
    h, w, n = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
    _check(lib.luvc_oim_plan(H, W, target_count, merge_per_step, ctypes.byref(h), ctypes.byref(w), ctypes.byref(n)),
           "luvc_oim_plan")
    return h.value, w.value, n.value


def oim_plan_anyres(H: int, W: int, n_ops: int, merge_per_step: int = 0):
    """((merge_h, merge_w), (out_h, out_w), n_steps) for a grid whose sides differ (host only)."""
    v = [ctypes.c_int() for _ in range(5)]
    _check(lib.luvc_oim_plan_anyres(H, W, n_ops, merge_per_step, *[ctypes.byref(c) for c in v]), "luvc_oim_plan_anyres")
    return (v[0].value, v[1].value), (v[2].value, v[3].value), v[4].value


def read_status(block: torch.Tensor) -> int:
    """luvc_read_status on a caller-owned status block (int32 tensor of >= 4 words on the device)."""
    return int(lib.luvc_read_status(block.data_ptr(), _stream_ptr(block.device)))


def spu_sigma(N: int, cutoff: float = 0.0) -> int:
    return lib.luvc_spu_sigma(N, float(cutoff))


def oim_merge(tokens: torch.Tensor, target_count: int, *, out_hw=None, merge_per_step: int = 0,
              height_first: bool = False, want_trace: bool = False, workspace: torch.Tensor | None = None,
              want_log_sizes: bool = False, matching: str = "adjacent", merge_per_step_hw=None,
              device_status: torch.Tensor | None = None):
    """luvc_oim_merge_ex on a CUDA tensor [B,H,W,D]; returns (out_tokens [B,T,D], out_sizes [B,T] int32,
    out_map [B,H*W] int32) and, with want_trace, the per-merge decision log [B,H*W-T] int32.
    matching: "adjacent" or "bipartite" (luvc_oim_matching); merge_per_step_hw: (per column in a height
    step, per row in a width step); device_status: a caller-owned status block (see read_status)."""
    if not tokens.is_cuda:
        raise ValueError("tokens must live on a CUDA device; host buffers go through oim_merge_host")
    tokens = tokens.contiguous()
    B, H, W, D = tokens.shape
    T = int(target_count)
    dev = tokens.device
    with torch.cuda.device(dev):
        out_tokens = torch.empty((B, max(T, 0), D), dtype=tokens.dtype, device=dev)
        out_sizes = torch.empty((B, max(T, 0)), dtype=torch.int32, device=dev)
        out_map = torch.empty((B, H * W), dtype=torch.int32, device=dev)
        trace = torch.zeros((B, max(H * W - T, 0)), dtype=torch.int32, device=dev) if want_trace else None
        o = OimOpts()
        o.dtype = _dtype_code(tokens)
        o.stream = _stream_ptr(dev)
        if workspace is not None:
            o.workspace, o.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
        if out_hw is not None:
            o.out_h, o.out_w = int(out_hw[0]), int(out_hw[1])
        o.merge_per_step = int(merge_per_step)
        o.height_first = int(bool(height_first))
        o.matching = {"adjacent": 0, "bipartite": 1}[matching]
        o.trace = trace.data_ptr() if (trace is not None and trace.numel()) else None
        o.trace_bytes = trace.numel() * 4 if trace is not None else 0
        if merge_per_step_hw is not None:
            o.merge_per_step_h, o.merge_per_step_w = int(merge_per_step_hw[0]), int(merge_per_step_hw[1])
        o.device_status = device_status.data_ptr() if device_status is not None else None
        log_sizes = torch.empty((B, max(T, 0)), dtype=torch.float32, device=dev) if want_log_sizes else None
        o.out_log_sizes = log_sizes.data_ptr() if log_sizes is not None else None
        _check(lib.luvc_oim_merge_ex(tokens.data_ptr(), B, H, W, D, T, out_tokens.data_ptr(), out_sizes.data_ptr(),
                                     out_map.data_ptr(), ctypes.byref(o)), "luvc_oim_merge_ex")
    res = (out_tokens, out_sizes, out_map)
    if want_trace:
        res = res + (trace,)
    if want_log_sizes:
        res = res + (log_sizes,)
    return res


def oim_value_enhance(values: torch.Tensor, sizes: torch.Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
    """luvc_oim_value_enhance: values [B,T,D] + log(sizes [B,T]) per row (Eq. 2); `out` may be `values`."""
    values = values.contiguous()
    sizes = sizes.contiguous()
    B, T, D = values.shape
    dev = values.device
    if out is None:
        out = torch.empty_like(values)
    with torch.cuda.device(dev):
        _check(lib.luvc_oim_value_enhance(values.data_ptr(), sizes.data_ptr(), B, T, D, _dtype_code(values),
                                          out.data_ptr(), _stream_ptr(dev)), "luvc_oim_value_enhance")
    return out


def oim_merge_plain(tokens: torch.Tensor, target_count: int):
    """The spec entry points luvc_oim_merge / luvc_oim_merge_f32 on the current torch stream."""
    tokens = tokens.contiguous()
    B, H, W, D = tokens.shape
    T = int(target_count)
    dev = tokens.device
    with torch.cuda.device(dev):
        out_tokens = torch.empty((B, T, D), dtype=tokens.dtype, device=dev)
        out_sizes = torch.empty((B, T), dtype=torch.int32, device=dev)
        out_map = torch.empty((B, H * W), dtype=torch.int32, device=dev)
        _check(lib.luvc_set_stream(_stream_ptr(dev)), "luvc_set_stream")
        fn = lib.luvc_oim_merge if _dtype_code(tokens) == BF16 else lib.luvc_oim_merge_f32
        _check(fn(tokens.data_ptr(), B, H, W, D, T, out_tokens.data_ptr(), out_sizes.data_ptr(), out_map.data_ptr()),
               "luvc_oim_merge")
    return out_tokens, out_sizes, out_map


def spu_prune(hidden: torch.Tensor, keep: int, cutoff: float = 0.0, *, no_window: bool = False,
              want_scores: bool = False, workspace: torch.Tensor | None = None,
              device_status: torch.Tensor | None = None):
    """luvc_spu_prune_ex on a CUDA tensor [B,N,D]; returns (out_idx [B,keep] int32, out_hidden [B,keep,D])
    and, with want_scores, the energies E [B,N] float32."""
    if not hidden.is_cuda:
        raise ValueError("hidden must live on a CUDA device; host buffers go through spu_prune_host")
    hidden = hidden.contiguous()
    B, N, D = hidden.shape
    dev = hidden.device
    k = int(keep)
    with torch.cuda.device(dev):
        out_idx = torch.empty((B, max(k, 0)), dtype=torch.int32, device=dev)
        out_hidden = torch.empty((B, max(k, 0), D), dtype=hidden.dtype, device=dev)
        scores = torch.empty((B, N), dtype=torch.float32, device=dev) if want_scores else None
        o = SpuOpts()
        o.dtype = _dtype_code(hidden)
        o.stream = _stream_ptr(dev)
        if workspace is not None:
            o.workspace, o.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
        o.no_window = int(bool(no_window))
        o.out_scores = scores.data_ptr() if scores is not None else None
        o.device_status = device_status.data_ptr() if device_status is not None else None
        _check(lib.luvc_spu_prune_ex(hidden.data_ptr(), B, N, D, float(cutoff), k, out_idx.data_ptr(),
                                     out_hidden.data_ptr(), ctypes.byref(o)), "luvc_spu_prune_ex")
    if want_scores:
        return out_idx, out_hidden, scores
    return out_idx, out_hidden


def spu_prune_plain(hidden: torch.Tensor, keep: int, cutoff: float = 0.0):
    """The spec entry points luvc_spu_prune / luvc_spu_prune_f32 on the current torch stream."""
    hidden = hidden.contiguous()
    B, N, D = hidden.shape
    dev = hidden.device
    with torch.cuda.device(dev):
        out_idx = torch.empty((B, keep), dtype=torch.int32, device=dev)
        out_hidden = torch.empty((B, keep, D), dtype=hidden.dtype, device=dev)
        _check(lib.luvc_set_stream(_stream_ptr(dev)), "luvc_set_stream")
        fn = lib.luvc_spu_prune if _dtype_code(hidden) == BF16 else lib.luvc_spu_prune_f32
        _check(fn(hidden.data_ptr(), B, N, D, float(cutoff), int(keep), out_idx.data_ptr(), out_hidden.data_ptr()),
               "luvc_spu_prune")
    return out_idx, out_hidden


def spu_cascade(hidden: torch.Tensor, keeps, cutoffs=None):
    """luvc_spu_cascade: prunes back to back, stage t on the survivors of stage t-1.  Returns
    (out_idx [B, keeps[-1]] int32 into the original sequence, out_hidden [B, keeps[-1], D])."""
    hidden = hidden.contiguous()
    B, N, D = hidden.shape
    dev = hidden.device
    n = len(keeps)
    k_arr = (ctypes.c_int * n)(*[int(k) for k in keeps])
    c_arr = (ctypes.c_float * n)(*[float(c) for c in cutoffs]) if cutoffs is not None else None
    with torch.cuda.device(dev):
        out_idx = torch.empty((B, int(keeps[-1])), dtype=torch.int32, device=dev)
        out_hidden = torch.empty((B, int(keeps[-1]), D), dtype=hidden.dtype, device=dev)
        _check(lib.luvc_spu_cascade(hidden.data_ptr(), B, N, D, n, k_arr, c_arr, _dtype_code(hidden), _stream_ptr(dev),
                                    out_idx.data_ptr(), out_hidden.data_ptr()), "luvc_spu_cascade")
    return out_idx, out_hidden


SPU_STATIC_MAX_BYTES = 32 * 1024 * 1024


def spu_prune_static(hidden: torch.Tensor, keep: int, cutoff: float = 0.0):
    """luvc_spu_prune_static: the prune for callers that cannot allocate device memory.  The library
    call allocates nothing (its workspace is a fixed array inside the library, at most
    SPU_STATIC_MAX_BYTES); this wrapper still creates the two output tensors, which a caller with
    such a constraint would own beforehand.  Returns (out_idx [B,keep] int32, out_hidden [B,keep,D])."""
    if not hidden.is_cuda:
        raise ValueError("hidden must live on a CUDA device")
    hidden = hidden.contiguous()
    B, N, D = hidden.shape
    dev = hidden.device
    with torch.cuda.device(dev):
        out_idx = torch.empty((B, max(int(keep), 0)), dtype=torch.int32, device=dev)
        out_hidden = torch.empty((B, max(int(keep), 0), D), dtype=hidden.dtype, device=dev)
        _check(lib.luvc_spu_prune_static(hidden.data_ptr(), B, N, D, float(cutoff), int(keep), _dtype_code(hidden),
                                         _stream_ptr(dev), out_idx.data_ptr(), out_hidden.data_ptr()),
               "luvc_spu_prune_static")
    return out_idx, out_hidden


def oim_merge_host(tokens: torch.Tensor, target_count: int, out_tokens: torch.Tensor, out_sizes: torch.Tensor,
                   out_map: torch.Tensor) -> None:
    """luvc_oim_merge_host: all four tensors are HOST tensors (pinned recommended); synchronous."""
    B, H, W, D = tokens.shape
    _check(lib.luvc_set_stream(_stream_ptr(None)), "luvc_set_stream")
    _check(lib.luvc_oim_merge_host(tokens.data_ptr(), B, H, W, D, int(target_count), _dtype_code(tokens),
                                   out_tokens.data_ptr(), out_sizes.data_ptr(), out_map.data_ptr()),
           "luvc_oim_merge_host")


def spu_prune_host(hidden: torch.Tensor, keep: int, cutoff: float, out_idx: torch.Tensor,
                   out_hidden: torch.Tensor) -> None:
    """luvc_spu_prune_host: all tensors are HOST tensors (pinned recommended); synchronous."""
    B, N, D = hidden.shape
    _check(lib.luvc_set_stream(_stream_ptr(None)), "luvc_set_stream")
    _check(lib.luvc_spu_prune_host(hidden.data_ptr(), B, N, D, float(cutoff), int(keep), _dtype_code(hidden),
                                   out_idx.data_ptr(), out_hidden.data_ptr()), "luvc_spu_prune_host")


# ---- paged key-value cache and the attention over it ---------------------------------------------


class KvCache:
    """A paged key-value cache of a group of decoder layers that hold the same tokens (luvc_kv_cache).

    k, v: the caller's pools, CUDA tensors [layers, pages, heads, page_size, D] in bfloat16, float32 or
    float8_e4m3fn (then with k_scale / v_scale, float32 [layers, heads]: a stored x stands for x * scale).
    slots: sequences; max_pages: pages a sequence may have.  meta: optional int32 tensor of
    slots + pages + slots * max_pages entries that holds the books (made empty if not given); `lengths`, `refs`
    and `table` are views of it, so that one copy of `meta` is a snapshot of all three."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, slots: int, max_pages: int, *, meta: torch.Tensor | None = None,
                 k_scale: torch.Tensor | None = None, v_scale: torch.Tensor | None = None):
        if not (k.is_cuda and v.is_cuda and k.device == v.device):
            raise ValueError("the pools must live on one CUDA device")
        if k.dim() != 5 or k.shape != v.shape or k.dtype != v.dtype or not (k.is_contiguous() and v.is_contiguous()):
            raise ValueError("k and v must be contiguous [layers, pages, heads, page_size, D] tensors of one shape and type")
        if k.dtype not in _CACHE_DTYPES:
            raise TypeError("a key-value cache holds bfloat16, float32 or float8_e4m3fn, got %s" % k.dtype)
        layers, pages, heads, page_size, D = k.shape
        size = slots + pages + slots * max_pages
        if meta is None:
            meta = torch.zeros(size, dtype=torch.int32, device=k.device)
            meta[slots + pages:] = -1
        if meta.dtype != torch.int32 or meta.shape != (size,) or not meta.is_contiguous() or meta.device != k.device:
            raise ValueError("meta must be a contiguous int32 tensor of %d entries on the pools' device" % size)
        for s in (k_scale, v_scale):
            if (s is not None) != (k.dtype == torch.float8_e4m3fn):
                raise ValueError("k_scale and v_scale go with float8_e4m3fn pools, and only with them")
            if s is not None and (s.dtype != torch.float32 or s.shape != (layers, heads) or not s.is_contiguous()
                                  or s.device != k.device):
                raise ValueError("scales must be contiguous float32 [layers, heads] tensors on the pools' device")
        self.k, self.v, self.meta, self.k_scale, self.v_scale = k, v, meta, k_scale, v_scale
        self.lengths = meta[:slots]
        self.refs = meta[slots:slots + pages]
        self.table = meta[slots + pages:].view(slots, max_pages)
        self.device, self.index, self.dtype = k.device, k.get_device(), k.dtype
        self.layers, self.pages, self.heads, self.page_size, self.head_dim = layers, pages, heads, page_size, D
        self.slots, self.max_pages = slots, max_pages
        # of queries, new rows and outputs
        self.io_dtype, self.io_code = (torch.float32, F32) if k.dtype == torch.float32 else (torch.bfloat16, BF16)
        self.struct = KvCacheStruct(
            k.data_ptr(), v.data_ptr(), self.lengths.data_ptr(), self.refs.data_ptr(), self.table.data_ptr(),
            k_scale.data_ptr() if k_scale is not None else None, v_scale.data_ptr() if v_scale is not None else None,
            layers, pages, heads, page_size, D, slots, max_pages, _CACHE_DTYPES[k.dtype])


_CACHE_DTYPES = {torch.bfloat16: BF16, torch.float32: F32, torch.float8_e4m3fn: E4M3}


# A decode step makes many small calls, so what these bindings do per call is kept short: the stream's handle without a
# torch.cuda.Stream object, no device context where the cache's device is current already, one comparison per rule.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_INT32 = torch.int32


def _ints(t: torch.Tensor | None, cache: KvCache, count: int, name: str):
    """Address of a contiguous int32 tensor [count] on the cache's device (None: NULL)."""
    if t is None:
        return None
    if t.dtype is not _INT32 or t.dim() != 1 or t.numel() != count or t.get_device() != cache.index or not t.is_contiguous():
        raise ValueError("%s must be a contiguous int32 tensor of %d entries on %s" % (name, count, cache.device))
    return t.data_ptr()


def _buffers(o, cache: KvCache, workspace, device_status) -> None:
    """Enters a caller's workspace and status block (None: the library's) into the options."""
    if workspace is not None:
        if workspace.get_device() != cache.index or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous tensor on %s" % cache.device)
        o.workspace, o.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    if device_status is not None:
        if device_status.dtype is not _INT32 or device_status.numel() < 4 or device_status.get_device() != cache.index \
                or not device_status.is_contiguous():
            raise ValueError("device_status must be a contiguous int32 tensor of 4 entries at least on %s" % cache.device)
        o.device_status = device_status.data_ptr()


def _kv_opts(cache: KvCache, workspace, device_status) -> KvOpts:
    o = KvOpts(_raw_stream(cache.index))
    _buffers(o, cache, workspace, device_status)
    return o


def _kv_call(fn, cache: KvCache, *args) -> None:
    """fn(*args) with the cache's device current; an error status raises."""
    if _current_device() == cache.index:
        status = fn(*args)
    else:
        with torch.cuda.device(cache.index):
            status = fn(*args)
    if status != 0:
        raise LuvcError(status, fn.__name__)


def kv_workspace_bytes(cache: KvCache, n: int) -> int:
    """Bytes a caller's workspace for kv_fork or kv_compact of n sequences must have (256-byte aligned)."""
    return int(lib.luvc_kv_workspace_bytes(cache.struct, n))


def attn_workspace_bytes() -> int:
    """Bytes a caller's workspace for attn_decode must have (256-byte aligned, zeroed before its first use; one per stream)."""
    return int(lib.luvc_attn_workspace_bytes())


def kv_reserve(cache: KvCache, counts: torch.Tensor, *, seqs: torch.Tensor | None = None,
               device_status: torch.Tensor | None = None) -> None:
    """luvc_kv_reserve: room for counts[i] further tokens of each sequence (int32 [n]); seqs: slots (None: 0 .. n-1)."""
    n = counts.numel()
    _kv_call(lib.luvc_kv_reserve, cache, cache.struct, _ints(seqs, cache, n, "seqs"), n, _ints(counts, cache, n, "counts"),
             _kv_opts(cache, None, device_status))


def _token_stride(t: torch.Tensor, cache: KvCache, heads: int, name: str) -> int:
    """Elements from one token to the next of a [tokens, heads, D] tensor whose tokens are contiguous."""
    D = cache.head_dim
    shape = t.shape
    if len(shape) != 3 or shape[1] != heads or shape[2] != D or t.get_device() != cache.index:
        raise ValueError("%s must be [tokens, %d, %d] on %s" % (name, heads, D, cache.device))
    if t.dtype is not cache.io_dtype:
        raise TypeError("%s must be %s for a %s cache, got %s" % (name, cache.io_dtype, cache.dtype, t.dtype))
    s0, s1, s2 = t.stride()
    if s2 != 1 or (s1 != D and heads > 1):
        raise ValueError("%s: the heads * D elements of a token must be contiguous" % name)
    return s0 if shape[0] > 1 else heads * D            # the stride of a lone token is not used


def kv_write(cache: KvCache, k: torch.Tensor, v: torch.Tensor, *, layer: int = 0, starts: torch.Tensor | None = None,
             seqs: torch.Tensor | None = None, sizes: torch.Tensor | None = None,
             device_status: torch.Tensor | None = None) -> None:
    """luvc_kv_write: the rows k, v [tokens, heads, D] become the last tokens of the sequences in `layer`.
    starts: int32 [n+1], rows starts[i] .. starts[i+1]-1 belong to sequence i (None: one row each); sizes: int32
    [tokens], the values are written as v + log(size) (Eq. 2).  k and v may be parts of a wider tensor."""
    tokens = k.shape[0]
    n = tokens if starts is None else starts.numel() - 1
    ks, vs = _token_stride(k, cache, cache.heads, "k"), _token_stride(v, cache, cache.heads, "v")
    if v.shape[0] != tokens:
        raise ValueError("k and v must have one shape")
    _kv_call(lib.luvc_kv_write, cache, cache.struct, layer, _ints(seqs, cache, n, "seqs"), n, k.data_ptr(), v.data_ptr(), ks, vs,
             tokens, _ints(starts, cache, n + 1, "starts"), _ints(sizes, cache, tokens, "sizes"), cache.io_code,
             _kv_opts(cache, None, device_status))


def kv_fork(cache: KvCache, src: torch.Tensor, dst: torch.Tensor, *, workspace: torch.Tensor | None = None,
            device_status: torch.Tensor | None = None) -> None:
    """luvc_kv_fork: the empty slots dst (int32 [n]) become copies of the sequences src (int32 [n]); full pages are shared."""
    n = dst.numel()
    _kv_call(lib.luvc_kv_fork, cache, cache.struct, _ints(src, cache, n, "src"), _ints(dst, cache, n, "dst"), n,
             _kv_opts(cache, workspace, device_status))


def kv_free(cache: KvCache, seqs: torch.Tensor, *, device_status: torch.Tensor | None = None) -> None:
    """luvc_kv_free: empties the slots seqs (int32 [n]); pages nobody holds any more are free again."""
    n = seqs.numel()
    _kv_call(lib.luvc_kv_free, cache, cache.struct, _ints(seqs, cache, n, "seqs"), n, _kv_opts(cache, None, device_status))


def kv_compact(cache: KvCache, first: torch.Tensor, span: torch.Tensor, idx: torch.Tensor, *,
               counts: torch.Tensor | None = None, seqs: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
               device_status: torch.Tensor | None = None) -> None:
    """luvc_kv_compact: of the block of span[i] tokens from first[i] on, sequence i keeps the tokens idx[i] (int32
    [n, keep], relative to the block, ascending: the out_idx of spu_prune) and everything outside the block."""
    n, keep = idx.shape
    _kv_call(lib.luvc_kv_compact, cache, cache.struct, _ints(seqs, cache, n, "seqs"), n, _ints(first, cache, n, "first"),
             _ints(span, cache, n, "span"), _ints(idx.view(-1), cache, n * keep, "idx") if keep else None, keep,
             _ints(counts, cache, n, "counts"), _kv_opts(cache, workspace, device_status))


def attn_decode(q: torch.Tensor, cache: KvCache, *, layer: int = 0, seqs: torch.Tensor | None = None, scale: float = 0.0,
                key_bias: torch.Tensor | None = None, want_lse: bool = False, out: torch.Tensor | None = None,
                workspace: torch.Tensor | None = None, device_status: torch.Tensor | None = None):
    """luvc_attn_decode: attention of the queries q [n, q_heads, D], one new token per sequence, over the cached tokens of
    `layer`.  key_bias: float32 [n, width], added to the scores of the first `width` tokens; scale 0: 1/sqrt(D).
    workspace: None, the library's own, which calls on other streams must not use at the same time, or attn_workspace_bytes()
    zeroed bytes.  Returns out [n, q_heads, D] and, with want_lse, the log-sum-exp of the scores [n, q_heads] float32."""
    n, q_heads = q.shape[0], q.shape[1]
    stride = _token_stride(q, cache, q_heads, "q")
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    elif out.shape != q.shape or out.dtype is not q.dtype or not out.is_contiguous() or out.device != q.device:
        raise ValueError("out must be a contiguous tensor of q's shape and type")
    o = AttnOpts(_raw_stream(cache.index))
    if scale:
        o.scale = scale
    _buffers(o, cache, workspace, device_status)
    if key_bias is not None:
        if key_bias.dtype is not torch.float32 or key_bias.dim() != 2 or key_bias.shape[0] != n \
                or key_bias.get_device() != cache.index or (key_bias.shape[1] > 1 and key_bias.stride(1) != 1):
            raise ValueError("key_bias must be a float32 [n, width] tensor on the cache's device, its rows contiguous")
        o.key_bias, o.bias_width = key_bias.data_ptr(), key_bias.shape[1]
        o.bias_stride = key_bias.stride(0) if n > 1 else max(key_bias.stride(0), key_bias.shape[1])
    lse = None
    if want_lse:
        lse = torch.empty((n, q_heads), dtype=torch.float32, device=q.device)
        o.lse = lse.data_ptr()
    _kv_call(lib.luvc_attn_decode, cache, q.data_ptr(), stride, cache.struct, layer, _ints(seqs, cache, n, "seqs"), n, q_heads,
             cache.io_code, out.data_ptr(), o)
    return (out, lse) if want_lse else out
