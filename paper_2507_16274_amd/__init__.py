"""Thin binding of libstalloc.so (include/stalloc.h): argument marshalling only.

Every step of the planning path, and every operator of a training step (attention,
norm, log probabilities, clipping), runs inside the HIP library; PyTorch is used for
device memory and streams.  There is no CPU fallback: if the library has not been
built (`python paper_2507_16274_amd/build.py`) importing the entry points fails.

Tensors are CUDA/HIP tensors on the current device.  Byte quantities are int64
tensors holding the library's uint64 bit patterns (all values stay below 2^63);
timestamps, orders and indices are int32 tensors holding uint32 values below 2^31.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, Optional

import torch  # loaded first so that the HIP runtime already in the process is shared

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libstalloc.so")

STATUS = {0: "STALLOC_OK", 1: "STALLOC_ERR_INVALID_ARG", 2: "STALLOC_ERR_BAD_TRACE", 3: "STALLOC_ERR_OVERFLOW",
          4: "STALLOC_ERR_NOMEM", 5: "STALLOC_ERR_DEVICE", 6: "STALLOC_ERR_BAD_ORDER", 7: "STALLOC_ERR_BAD_WINDOW",
          8: "STALLOC_ERR_BAD_LAYER", 9: "STALLOC_ERR_TOO_LARGE", 10: "STALLOC_ERR_BAD_BOUNDS", 11: "STALLOC_ERR_BAD_TOKEN"}
INVALID_ARG = 1                  # decided on the host, before anything is enqueued
STATIC_MAX_T_END = 524288        # STALLOC_STATIC_MAX_T_END of include/stalloc.h
EXPORTS = ("stalloc_plan", "stalloc_validate", "stalloc_lower_bound", "stalloc_lower_bound_static",
           "stalloc_reusable_space",
           "stalloc_memory_layers", "stalloc_expand_layers", "stalloc_tmp", "stalloc_make_orders",
           "stalloc_status_string", "stalloc_plan_lds_capacity", "stalloc_plan_report", "stalloc_probe",
           "stalloc_fuse_groups", "stalloc_plan_sized",
           "stalloc_attention", "stalloc_attention_backward", "stalloc_rms_norm", "stalloc_rms_norm_backward",
           "stalloc_token_logprobs", "stalloc_token_logprobs_backward", "stalloc_clip_gradients")
KERNELS = {0: "none", 1: "bitmap", 2: "list_lds", 3: "list_memory", 4: "long_list"}


DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}          # stalloc_dtype
MOST_TOP = 64                    # alternatives that stalloc_token_logprobs lists at most


class StallocError(RuntimeError):
    def __init__(self, code: int, where: str):
        super().__init__(f"{where}: {STATUS.get(code, code)}")
        self.code = code


class _Trace(ctypes.Structure):
    _fields_ = [("n", ctypes.c_uint32), ("t_end", ctypes.c_uint32), ("size", ctypes.c_void_p),
                ("t_alloc", ctypes.c_void_p), ("t_free", ctypes.c_void_p)]


class _PlanInfo(ctypes.Structure):
    _fields_ = [("kernel", ctypes.c_uint32), ("granule_log2", ctypes.c_uint32), ("granules", ctypes.c_uint64),
                ("plans_64bit", ctypes.c_uint32), ("lifetime_threshold", ctypes.c_uint32),
                ("long_requests", ctypes.c_uint32), ("address_bits", ctypes.c_uint32),
                ("large_size", ctypes.c_uint64), ("large_requests", ctypes.c_uint32), ("list_entry_bytes", ctypes.c_uint32)]


class _Heads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_uint64), ("head_stride", ctypes.c_uint64)]


class _AttentionShape(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_uint32), ("tokens", ctypes.c_uint32), ("sequences", ctypes.c_uint32), ("heads", ctypes.c_uint32),
                ("kv_heads", ctypes.c_uint32), ("head_dim", ctypes.c_uint32), ("scale", ctypes.c_float)]


class _Tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("out", ctypes.c_void_p), ("count", ctypes.c_uint64), ("dtype", ctypes.c_uint64)]


def _load() -> ctypes.CDLL:
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is missing: build it with `python paper_2507_16274_amd/build.py` "
                          "(hipcc, gfx950); there is no fallback path")
    lib = ctypes.CDLL(_LIB_PATH)
    vp, u32 = ctypes.c_void_p, ctypes.c_uint32
    szp = ctypes.POINTER(ctypes.c_size_t)
    tp = ctypes.POINTER(_Trace)
    lib.stalloc_plan.argtypes = [tp, vp, u32, vp, vp, vp, vp, vp, vp, szp, vp]
    lib.stalloc_plan_sized.argtypes = [tp, vp, u32, vp, vp, vp, vp, vp, ctypes.c_uint64, ctypes.c_uint64, vp, szp, vp]
    lib.stalloc_validate.argtypes = [tp, vp, u32, vp, vp, vp, vp, szp, vp]
    lib.stalloc_lower_bound.argtypes = [tp, vp, vp, vp, vp, szp, vp]
    lib.stalloc_lower_bound_static.argtypes = [tp, vp, vp, vp, vp]
    lib.stalloc_reusable_space.argtypes = [tp, vp, vp, u32, u32, vp, vp, vp, vp, vp, szp, vp]
    lib.stalloc_memory_layers.argtypes = [tp, vp, vp, vp, vp, vp, vp, vp, szp, vp]
    lib.stalloc_expand_layers.argtypes = [u32, u32, vp, vp, u32, vp, vp, vp]
    lib.stalloc_tmp.argtypes = [tp, vp, u32, vp, vp, vp, szp, vp]
    lib.stalloc_make_orders.argtypes = [tp, u32, u32, ctypes.c_uint64, vp, vp, vp, szp, vp]
    lib.stalloc_fuse_groups.argtypes = [tp, vp, vp, vp, u32, u32, u32, vp, vp, vp, vp, vp, vp, szp, vp]
    hp, sp, u64, f32 = ctypes.POINTER(_Heads), ctypes.POINTER(_AttentionShape), ctypes.c_uint64, ctypes.c_float
    lib.stalloc_attention.argtypes = [sp, hp, hp, hp, vp, hp, vp, vp, vp, szp, vp]
    lib.stalloc_attention_backward.argtypes = [sp, hp, hp, hp, hp, hp, vp, vp, hp, hp, hp, vp, vp, szp, vp]
    lib.stalloc_rms_norm.argtypes = [u32, u32, u32, vp, u64, vp, u64, vp, f32, vp, vp, vp, vp, vp, vp]
    lib.stalloc_rms_norm_backward.argtypes = [u32, u32, u32, vp, u64, vp, vp, vp, vp, vp, vp, vp, szp, vp]
    lib.stalloc_token_logprobs.argtypes = [u32, u32, u32, vp, u64, vp, u32, vp, vp, vp, vp, vp, vp, vp, szp, vp]
    lib.stalloc_token_logprobs_backward.argtypes = [u32, u32, u32, vp, u64, vp, vp, vp, vp, vp, vp, u64, vp, vp]
    lib.stalloc_clip_gradients.argtypes = [ctypes.POINTER(_Tensor), u32, f32, vp, vp, vp, szp, vp]
    for name in ("stalloc_plan", "stalloc_validate", "stalloc_lower_bound", "stalloc_lower_bound_static",
                 "stalloc_reusable_space", "stalloc_memory_layers", "stalloc_expand_layers", "stalloc_tmp",
                 "stalloc_make_orders", "stalloc_fuse_groups", "stalloc_plan_sized",
                 "stalloc_attention", "stalloc_attention_backward", "stalloc_rms_norm", "stalloc_rms_norm_backward",
                 "stalloc_token_logprobs", "stalloc_token_logprobs_backward", "stalloc_clip_gradients"):
        getattr(lib, name).restype = ctypes.c_int
    lib.stalloc_plan_report.argtypes = [vp, ctypes.POINTER(_PlanInfo), vp]
    lib.stalloc_plan_report.restype = ctypes.c_int
    lib.stalloc_probe.argtypes = [u32, vp, ctypes.c_size_t, u32, ctypes.POINTER(ctypes.c_uint64), vp]
    lib.stalloc_probe.restype = ctypes.c_int
    lib.stalloc_status_string.argtypes = [ctypes.c_int]
    lib.stalloc_status_string.restype = ctypes.c_char_p
    lib.stalloc_plan_lds_capacity.argtypes = []
    lib.stalloc_plan_lds_capacity.restype = ctypes.c_uint32
    return lib


lib = _load()


def _dev(t: Optional[torch.Tensor], dtype: torch.dtype, name: str) -> Optional[int]:
    if t is None:
        return None
    if not (t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise TypeError(f"{name}: expected a contiguous {dtype} tensor on the GPU")
    return t.data_ptr()


def _trace(size: torch.Tensor, t_alloc: torch.Tensor, t_free: torch.Tensor, t_end: int) -> _Trace:
    n = size.numel()
    if t_alloc.numel() != n or t_free.numel() != n:
        raise ValueError("size, t_alloc and t_free must have the same length")
    return _Trace(n, int(t_end), _dev(size, torch.int64, "size"), _dev(t_alloc, torch.int32, "t_alloc"),
                  _dev(t_free, torch.int32, "t_free"))


def _stream(stream: Optional[torch.cuda.Stream]) -> int:
    if stream is not None:
        return stream.cuda_stream
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)       # not part of torch's interface; current_stream() makes an object first: 2.7 us
    return torch.cuda.current_stream().cuda_stream if raw is None else raw(torch.cuda.current_device())


def _workspace(nbytes: int, device, cache: Optional[Dict]) -> torch.Tensor:
    if cache is not None:
        ws = cache.get("ws")
        if ws is None or ws.numel() < nbytes:
            ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
            cache["ws"] = ws
        return ws
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


def _check(rc: int, where: str) -> None:
    if rc != 0:
        raise StallocError(rc, where)


def stalloc_plan(size, t_alloc, t_free, t_end: int, orders, *, want_offsets: bool = True,
                 want_best_offsets: bool = True, stream=None, workspace_cache: Optional[Dict] = None,
                 out: Optional[Dict] = None) -> Dict[str, torch.Tensor]:
    """Enqueue stalloc_plan; returns the (asynchronously filled) output tensors.

    orders: int32 [P][n].  Outputs: offsets int64 [P][n] (None unless want_offsets),
    peaks int64 [P], best_offsets int64 [n] (None unless want_best_offsets),
    best_plan int32 [1], status int32 [1].  `out` may carry preallocated outputs.
    """
    return _plan(lib.stalloc_plan, "stalloc_plan", (), size, t_alloc, t_free, t_end, orders, want_offsets, want_best_offsets,
                 stream, workspace_cache, out)


def stalloc_plan_sized(size, t_alloc, t_free, t_end: int, orders, largest_size: int, granule: int, *,
                       want_offsets: bool = True, want_best_offsets: bool = True, stream=None,
                       workspace_cache: Optional[Dict] = None, out: Optional[Dict] = None) -> Dict[str, torch.Tensor]:
    """stalloc_plan for a caller that knows an upper bound of its sizes and a power of two dividing them all."""
    return _plan(lib.stalloc_plan_sized, "stalloc_plan_sized", (int(largest_size), int(granule)), size, t_alloc, t_free, t_end,
                 orders, want_offsets, want_best_offsets, stream, workspace_cache, out)


def _plan(fn, name, extra, size, t_alloc, t_free, t_end, orders, want_offsets, want_best_offsets, stream, workspace_cache, out):
    tr = _trace(size, t_alloc, t_free, t_end)
    if orders.dim() != 2 or orders.shape[1] != tr.n:
        raise ValueError("orders must be [P][n]")
    P, n, dev = orders.shape[0], tr.n, size.device
    out = dict(out) if out else {}
    if want_offsets and out.get("offsets") is None:
        out["offsets"] = torch.empty((P, n), dtype=torch.int64, device=dev)
    if not want_offsets:
        out["offsets"] = None
    if out.get("peaks") is None:
        out["peaks"] = torch.empty(P, dtype=torch.int64, device=dev)
    if want_best_offsets and out.get("best_offsets") is None:
        out["best_offsets"] = torch.empty(n, dtype=torch.int64, device=dev)
    if not want_best_offsets:
        out["best_offsets"] = None
    if out.get("best_plan") is None:
        out["best_plan"] = torch.empty(1, dtype=torch.int32, device=dev)
    if out.get("status") is None:
        out["status"] = torch.empty(1, dtype=torch.int32, device=dev)
    args = (ctypes.byref(tr), _dev(orders, torch.int32, "orders"), P,
            _dev(out["offsets"], torch.int64, "offsets"), _dev(out["peaks"], torch.int64, "peaks"),
            _dev(out["best_offsets"], torch.int64, "best_offsets"),
            _dev(out["best_plan"], torch.int32, "best_plan"), _dev(out["status"], torch.int32, "status")) + tuple(extra)
    need = ctypes.c_size_t(0)
    _check(fn(*args, None, ctypes.byref(need), None), name + "(workspace query)")
    ws = _workspace(need.value, dev, workspace_cache)
    have = ctypes.c_size_t(ws.numel())
    _check(fn(*args, ws.data_ptr(), ctypes.byref(have), _stream(stream)), name)
    out["workspace"] = ws
    out["workspace_bytes"] = need.value
    return out


def stalloc_plan_report(plan: Dict[str, torch.Tensor], *, stream=None) -> Dict[str, int]:
    """What the stalloc_plan call that produced `plan` did (synchronises): kernel name, address granule, ..."""
    info = _PlanInfo()
    _check(lib.stalloc_plan_report(plan["workspace"].data_ptr(), ctypes.byref(info), _stream(stream)), "stalloc_plan_report")
    return {"kernel": KERNELS.get(info.kernel, str(info.kernel)), "granule_log2": info.granule_log2,
            "granules": info.granules, "plans_64bit": info.plans_64bit,
            "lifetime_threshold": info.lifetime_threshold, "long_requests": info.long_requests,
            "address_bits": info.address_bits, "large_size": info.large_size, "large_requests": info.large_requests,
            "list_entry_bytes": info.list_entry_bytes}


def stalloc_probe(what: int, buffer: torch.Tensor, iters: int = 0, *, stream=None) -> int:
    """Enqueue one probe kernel (0 copy, 1 LDS read, 2 integer ALU) on `buffer` (uint8); returns its work."""
    done = ctypes.c_uint64(0)
    _check(lib.stalloc_probe(int(what), _dev(buffer, torch.uint8, "buffer"), buffer.numel(), int(iters),
                             ctypes.byref(done), _stream(stream)), "stalloc_probe")
    return int(done.value)


def stalloc_validate(size, t_alloc, t_free, t_end: int, offsets, *, stream=None,
                     workspace_cache: Optional[Dict] = None) -> Dict[str, torch.Tensor]:
    """offsets int64 [P][n] -> conflicts int64 [P], first_pair int32 [P][2] (-1, -1 when valid)."""
    tr = _trace(size, t_alloc, t_free, t_end)
    if offsets.dim() != 2 or offsets.shape[1] != tr.n:
        raise ValueError("offsets must be [P][n]")
    P, dev = offsets.shape[0], size.device
    out = {"conflicts": torch.empty(P, dtype=torch.int64, device=dev),
           "first_pair": torch.empty((P, 2), dtype=torch.int32, device=dev),
           "status": torch.empty(1, dtype=torch.int32, device=dev)}
    args = (ctypes.byref(tr), _dev(offsets, torch.int64, "offsets"), P, out["conflicts"].data_ptr(),
            out["first_pair"].data_ptr(), out["status"].data_ptr())
    need = ctypes.c_size_t(0)
    _check(lib.stalloc_validate(*args, None, ctypes.byref(need), None), "stalloc_validate(workspace query)")
    ws = _workspace(need.value, dev, workspace_cache)
    have = ctypes.c_size_t(ws.numel())
    _check(lib.stalloc_validate(*args, ws.data_ptr(), ctypes.byref(have), _stream(stream)), "stalloc_validate")
    out["workspace"] = ws
    return out


def stalloc_lower_bound(size, t_alloc, t_free, t_end: int, *, stream=None,
                        workspace_cache: Optional[Dict] = None) -> Dict[str, torch.Tensor]:
    """-> lower_bound int64 [1], t_at_max int32 [1], status int32 [1]."""
    tr = _trace(size, t_alloc, t_free, t_end)
    dev = size.device
    out = {"lower_bound": torch.empty(1, dtype=torch.int64, device=dev),
           "t_at_max": torch.empty(1, dtype=torch.int32, device=dev),
           "status": torch.empty(1, dtype=torch.int32, device=dev)}
    args = (ctypes.byref(tr), out["lower_bound"].data_ptr(), out["t_at_max"].data_ptr(), out["status"].data_ptr())
    need = ctypes.c_size_t(0)
    _check(lib.stalloc_lower_bound(*args, None, ctypes.byref(need), None), "stalloc_lower_bound(workspace query)")
    ws = _workspace(need.value, dev, workspace_cache)
    have = ctypes.c_size_t(ws.numel())
    _check(lib.stalloc_lower_bound(*args, ws.data_ptr(), ctypes.byref(have), _stream(stream)), "stalloc_lower_bound")
    out["workspace"] = ws
    return out


def stalloc_lower_bound_static(size, t_alloc, t_free, t_end: int, *, out: Dict[str, torch.Tensor],
                               stream=None) -> Dict[str, torch.Tensor]:
    """stalloc_lower_bound without a workspace; `out` carries the preallocated outputs
    (lower_bound int64 [1], t_at_max int32 [1], status int32 [1]), so nothing is allocated here either."""
    tr = _trace(size, t_alloc, t_free, t_end)
    _check(lib.stalloc_lower_bound_static(ctypes.byref(tr), _dev(out["lower_bound"], torch.int64, "lower_bound"),
                                          _dev(out["t_at_max"], torch.int32, "t_at_max"),
                                          _dev(out["status"], torch.int32, "status"), _stream(stream)),
           "stalloc_lower_bound_static")
    return out


def stalloc_reusable_space(size, t_alloc, t_free, t_end: int, offsets, windows, max_ranges: int, *, stream=None,
                           workspace_cache: Optional[Dict] = None) -> Dict[str, torch.Tensor]:
    """offsets int64 [n], windows int32 [k][2] -> ranges int64 [k][max_ranges][2], counts int32 [k],
    idle_bytes int64 [k], status int32 [1]."""
    tr = _trace(size, t_alloc, t_free, t_end)
    if offsets.dim() != 1 or offsets.numel() != tr.n:
        raise ValueError("offsets must be [n]")
    if windows.dim() != 2 or windows.shape[1] != 2:
        raise ValueError("windows must be [k][2]")
    k, dev = windows.shape[0], size.device
    out = {"ranges": torch.empty((k, max_ranges, 2), dtype=torch.int64, device=dev) if max_ranges else None,
           "counts": torch.empty(k, dtype=torch.int32, device=dev),
           "idle_bytes": torch.empty(k, dtype=torch.int64, device=dev),
           "status": torch.empty(1, dtype=torch.int32, device=dev)}
    args = (ctypes.byref(tr), _dev(offsets, torch.int64, "offsets"), _dev(windows, torch.int32, "windows"), k,
            int(max_ranges), out["ranges"].data_ptr() if max_ranges else None, out["counts"].data_ptr(),
            out["idle_bytes"].data_ptr(), out["status"].data_ptr())
    need = ctypes.c_size_t(0)
    _check(lib.stalloc_reusable_space(*args, None, ctypes.byref(need), None), "stalloc_reusable_space(workspace query)")
    ws = _workspace(need.value, dev, workspace_cache)
    have = ctypes.c_size_t(ws.numel())
    _check(lib.stalloc_reusable_space(*args, ws.data_ptr(), ctypes.byref(have), _stream(stream)), "stalloc_reusable_space")
    out["workspace"] = ws
    return out


def check_status(out: Dict[str, torch.Tensor], where: str = "stalloc") -> None:
    """Synchronising read of the device status word; raises StallocError when non-zero."""
    code = int(out["status"].item())
    if code != 0:
        raise StallocError(code, where)


def trace_to_device(trace, device="cuda"):
    """numpy trace (size uint64, t_alloc/t_free uint32) -> (size, t_alloc, t_free) device tensors."""
    import numpy as np
    size = torch.from_numpy(np.ascontiguousarray(trace.size).view(np.int64)).to(device)
    ta = torch.from_numpy(np.ascontiguousarray(trace.t_alloc).view(np.int32)).to(device)
    tf = torch.from_numpy(np.ascontiguousarray(trace.t_free).view(np.int32)).to(device)
    return size, ta, tf


def stalloc_memory_layers(size, t_alloc, t_free, t_end: int, *, stream=None,
                          workspace_cache: Optional[Dict] = None) -> Dict[str, torch.Tensor]:
    """-> layer_of int32 [n], n_layers int32 [1], layer_size int64 [n], layer_t_alloc / layer_t_free int32 [n]
    (the first n_layers entries are written), status int32 [1]."""
    tr = _trace(size, t_alloc, t_free, t_end)
    dev, n = size.device, tr.n
    out = {"layer_of": torch.empty(n, dtype=torch.int32, device=dev),
           "n_layers": torch.empty(1, dtype=torch.int32, device=dev),
           "layer_size": torch.empty(n, dtype=torch.int64, device=dev),
           "layer_t_alloc": torch.empty(n, dtype=torch.int32, device=dev),
           "layer_t_free": torch.empty(n, dtype=torch.int32, device=dev),
           "status": torch.empty(1, dtype=torch.int32, device=dev)}
    args = (ctypes.byref(tr), out["layer_of"].data_ptr(), out["n_layers"].data_ptr(), out["layer_size"].data_ptr(),
            out["layer_t_alloc"].data_ptr(), out["layer_t_free"].data_ptr(), out["status"].data_ptr())
    need = ctypes.c_size_t(0)
    _check(lib.stalloc_memory_layers(*args, None, ctypes.byref(need), None), "stalloc_memory_layers(workspace query)")
    ws = _workspace(need.value, dev, workspace_cache)
    have = ctypes.c_size_t(ws.numel())
    _check(lib.stalloc_memory_layers(*args, ws.data_ptr(), ctypes.byref(have), _stream(stream)), "stalloc_memory_layers")
    out["workspace"] = ws
    return out


def stalloc_expand_layers(layer_of, layer_offsets, *, stream=None) -> Dict[str, torch.Tensor]:
    """layer_of int32 [n], layer_offsets int64 [P][n_layers] -> offsets int64 [P][n], status int32 [1]."""
    if layer_of.dim() != 1 or layer_offsets.dim() != 2:
        raise ValueError("layer_of must be [n] and layer_offsets [P][n_layers]")
    n, (P, n_layers), dev = layer_of.numel(), layer_offsets.shape, layer_of.device
    out = {"offsets": torch.empty((P, n), dtype=torch.int64, device=dev),
           "status": torch.empty(1, dtype=torch.int32, device=dev)}
    _check(lib.stalloc_expand_layers(n, P, _dev(layer_of, torch.int32, "layer_of"),
                                     _dev(layer_offsets, torch.int64, "layer_offsets"), n_layers,
                                     out["offsets"].data_ptr(), out["status"].data_ptr(), _stream(stream)),
           "stalloc_expand_layers")
    return out


def stalloc_tmp(size, t_alloc, t_free, t_end: int, extents, *, stream=None,
                workspace_cache: Optional[Dict] = None) -> Dict[str, torch.Tensor]:
    """extents int64 [P] (`peaks` of stalloc_plan) -> tmp float64 [P], status int32 [1]."""
    tr = _trace(size, t_alloc, t_free, t_end)
    if extents.dim() != 1:
        raise ValueError("extents must be [P]")
    P, dev = extents.numel(), size.device
    out = {"tmp": torch.empty(P, dtype=torch.float64, device=dev),
           "status": torch.empty(1, dtype=torch.int32, device=dev)}
    args = (ctypes.byref(tr), _dev(extents, torch.int64, "extents"), P, out["tmp"].data_ptr(), out["status"].data_ptr())
    need = ctypes.c_size_t(0)
    _check(lib.stalloc_tmp(*args, None, ctypes.byref(need), None), "stalloc_tmp(workspace query)")
    ws = _workspace(need.value, dev, workspace_cache)
    have = ctypes.c_size_t(ws.numel())
    _check(lib.stalloc_tmp(*args, ws.data_ptr(), ctypes.byref(have), _stream(stream)), "stalloc_tmp")
    out["workspace"] = ws
    return out


def stalloc_fuse_groups(size, t_alloc, t_free, t_end: int, members, pair_begin, count1, largest_pair: int, *,
                        stream=None, workspace_cache: Optional[Dict] = None) -> Dict[str, torch.Tensor]:
    """members int32 [m], pair_begin int32 [k+1], count1 int32 [k], largest_pair = the largest pair's size ->
    order int32 [m], addr int64 [m], extents int64 [k][3], accepted int32 [k], status int32 [1]."""
    tr = _trace(size, t_alloc, t_free, t_end)
    k, m, dev = count1.numel(), members.numel(), size.device
    if pair_begin.numel() != k + 1:
        raise ValueError("pair_begin must hold k + 1 entries")
    out = {"order": torch.empty(m, dtype=torch.int32, device=dev), "addr": torch.empty(m, dtype=torch.int64, device=dev),
           "extents": torch.empty((k, 3), dtype=torch.int64, device=dev),
           "accepted": torch.empty(k, dtype=torch.int32, device=dev),
           "status": torch.empty(1, dtype=torch.int32, device=dev)}
    args = (ctypes.byref(tr), _dev(members, torch.int32, "members"), _dev(pair_begin, torch.int32, "pair_begin"),
            _dev(count1, torch.int32, "count1"), k, m, int(largest_pair), out["order"].data_ptr(), out["addr"].data_ptr(),
            out["extents"].data_ptr(), out["accepted"].data_ptr(), out["status"].data_ptr())
    need = ctypes.c_size_t(0)
    _check(lib.stalloc_fuse_groups(*args, None, ctypes.byref(need), None), "stalloc_fuse_groups(workspace query)")
    ws = _workspace(need.value, dev, workspace_cache)
    have = ctypes.c_size_t(ws.numel())
    _check(lib.stalloc_fuse_groups(*args, ws.data_ptr(), ctypes.byref(have), _stream(stream)), "stalloc_fuse_groups")
    out["workspace"] = ws
    return out


def stalloc_make_orders(size, t_alloc, t_free, t_end: int, P: int, *, seed: int = 1000, first_plan: int = 0,
                        stream=None, workspace_cache: Optional[Dict] = None) -> Dict[str, torch.Tensor]:
    """-> orders int32 [P][n] (rows first_plan .. first_plan + P - 1), status int32 [1]."""
    tr = _trace(size, t_alloc, t_free, t_end)
    dev = size.device
    out = {"orders": torch.empty((P, tr.n), dtype=torch.int32, device=dev),
           "status": torch.empty(1, dtype=torch.int32, device=dev)}
    args = (ctypes.byref(tr), int(first_plan), int(P), int(seed), out["orders"].data_ptr(), out["status"].data_ptr())
    need = ctypes.c_size_t(0)
    _check(lib.stalloc_make_orders(*args, None, ctypes.byref(need), None), "stalloc_make_orders(workspace query)")
    ws = _workspace(need.value, dev, workspace_cache)
    have = ctypes.c_size_t(ws.numel())
    _check(lib.stalloc_make_orders(*args, ws.data_ptr(), ctypes.byref(have), _stream(stream)), "stalloc_make_orders")
    out["workspace"] = ws
    return out


# ---------------------------------------------------------------------------------------------
# Operators of a training step.  `out` may carry preallocated outputs (all of a call's or some), for
# instance views of a pool at the addresses of a plan; what it lacks is allocated on the stream of the
# call.  Inputs must not be freed or overwritten on other streams before the call is through.

def _new(out, name: str, shape, dtype, like, stream):
    """The output `name` of `out`, checked, or a new tensor that belongs to the call's stream."""
    t = out.get(name)
    if t is None:
        if stream is None:
            t = torch.empty(shape, dtype=dtype, device=like.device)
        else:
            with torch.cuda.stream(stream):
                t = torch.empty(shape, dtype=dtype, device=like.device)
        out[name] = t
    elif t.shape != shape or t.dtype != dtype or not t.is_cuda:
        raise ValueError(f"{name}: expected a {dtype} tensor {tuple(shape)} on the GPU")
    return t


def _flat(t: Optional[torch.Tensor], name: str) -> Optional[int]:
    """Address of a contiguous tensor."""
    if t is None:
        return None
    if not (t.is_cuda and t.is_contiguous()):
        raise TypeError(f"{name}: expected a contiguous tensor on the GPU")
    return t.data_ptr()


def _call(fn, name, args, like, stream, workspace_cache, out):
    """Query, workspace, call.  With a workspace at hand the call comes first: it takes one that is large enough.  Only a refusal, which comes before any
    work, leads to the query, and only a workspace that is too small to another call."""
    ws = workspace_cache.get("ws") if workspace_cache is not None else None
    rc = 0
    if ws is not None:
        rc = fn(*args, ws.data_ptr(), ctypes.byref(ctypes.c_size_t(ws.numel())), _stream(stream))
        if rc == 0:
            out["workspace"] = ws
            return out
        if rc != INVALID_ARG:
            _check(rc, name)
    need = ctypes.c_size_t(0)
    _check(fn(*args, None, ctypes.byref(need), None), name + "(workspace query)")
    if ws is not None and ws.numel() >= need.value:
        _check(rc, name)
    if stream is None:
        ws = _workspace(need.value, like.device, workspace_cache)
    else:
        with torch.cuda.stream(stream):
            ws = _workspace(need.value, like.device, workspace_cache)
    have = ctypes.c_size_t(ws.numel())
    _check(fn(*args, ws.data_ptr(), ctypes.byref(have), _stream(stream)), name)
    out["workspace"] = ws
    return out


def _dtype_of(t: torch.Tensor, name: str) -> int:
    code = DTYPES.get(t.dtype)
    if code is None or not t.is_cuda:
        raise TypeError(f"{name}: expected a float32, bfloat16 or float16 tensor on the GPU")
    return code


def _sizes(*counts: int) -> None:
    """What the library takes in 32 bits (ctypes would cut it short)."""
    if max(counts) >> 31:
        raise ValueError("fewer than 2^31 rows, columns, tokens or sequences are expected")


def _by_heads(t: torch.Tensor, shape, dtype, name: str) -> _Heads:
    if not t.is_cuda or t.dtype != dtype or t.shape != shape:
        raise ValueError(f"{name}: expected a {dtype} tensor {tuple(shape)} on the GPU")
    stride = t.stride()
    if stride[2] != 1:
        raise ValueError(f"{name}: the numbers of a head must be neighbours in memory")
    return _Heads(t.data_ptr(), stride[0] if shape[0] > 1 else 0, stride[1] if shape[1] > 1 else 0)


def _attention_shape(q, k, bounds, scale) -> _AttentionShape:
    if q.dim() != 3 or k.dim() != 3 or bounds.dim() != 1 or bounds.numel() < 2:
        raise ValueError("q must be [tokens][heads][head_dim], k and v [tokens][kv_heads][head_dim], bounds [sequences + 1]")
    tokens, heads, head_dim = q.shape
    _sizes(tokens, bounds.numel() - 1, heads, k.shape[1], head_dim)
    return _AttentionShape(_dtype_of(q, "q"), tokens, bounds.numel() - 1, heads, k.shape[1], head_dim, head_dim ** -0.5 if scale is None else scale)


def stalloc_attention(q, k, v, bounds, *, scale: Optional[float] = None, out: Optional[Dict] = None, stream=None,
                      workspace_cache: Optional[Dict] = None) -> Dict[str, torch.Tensor]:
    """Causal attention over packed sequences: q [tokens][heads][head_dim], k, v [tokens][kv_heads][head_dim] (bfloat16 or
    float16, views with neighbouring last elements are fine), bounds int32 [sequences + 1] from 0 to at most tokens ->
    o like q, lse float32 [heads][tokens], status int32 [1].  scale: of the scores, head_dim ** -0.5 unless given."""
    shape = _attention_shape(q, k, bounds, scale)
    tokens, heads, head_dim = q.shape
    of_keys = (tokens, shape.kv_heads, head_dim)
    out = dict(out) if out else {}
    o = _by_heads(_new(out, "o", q.shape, q.dtype, q, stream), q.shape, q.dtype, "o")
    lse = _new(out, "lse", (heads, tokens), torch.float32, q, stream)
    status = _new(out, "status", (1,), torch.int32, q, stream)
    args = (shape, _by_heads(q, q.shape, q.dtype, "q"), _by_heads(k, of_keys, q.dtype, "k"), _by_heads(v, of_keys, q.dtype, "v"),
            _dev(bounds, torch.int32, "bounds"), o, _flat(lse, "lse"), status.data_ptr())
    return _call(lib.stalloc_attention, "stalloc_attention", args, q, stream, workspace_cache, out)


def stalloc_attention_backward(d_o, q, k, v, o, lse, bounds, *, scale: Optional[float] = None, out: Optional[Dict] = None, stream=None,
                               workspace_cache: Optional[Dict] = None) -> Dict[str, torch.Tensor]:
    """Gradients of stalloc_attention for the gradient d_o of its output o (with the lse it gave) -> dq, dk, dv, status."""
    shape = _attention_shape(q, k, bounds, scale)
    tokens, heads, head_dim = q.shape
    of_keys = torch.Size((tokens, shape.kv_heads, head_dim))
    if lse.shape != (heads, tokens):
        raise ValueError("lse must be [heads][tokens]")
    out = dict(out) if out else {}
    grads = [_by_heads(_new(out, name, size, q.dtype, q, stream), size, q.dtype, name)
             for name, size in (("dq", q.shape), ("dk", of_keys), ("dv", of_keys))]
    status = _new(out, "status", (1,), torch.int32, q, stream)
    args = (shape, _by_heads(d_o, q.shape, q.dtype, "d_o"), _by_heads(q, q.shape, q.dtype, "q"), _by_heads(k, of_keys, q.dtype, "k"),
            _by_heads(v, of_keys, q.dtype, "v"), _by_heads(o, q.shape, q.dtype, "o"), _dev(lse, torch.float32, "lse"),
            _dev(bounds, torch.int32, "bounds"), *grads, status.data_ptr())
    return _call(lib.stalloc_attention_backward, "stalloc_attention_backward", args, q, stream, workspace_cache, out)


def _rows(t: torch.Tensor, shape, dtype, name: str):
    """Address and row stride of a matrix whose rows are contiguous."""
    if not t.is_cuda or t.dtype != dtype or t.shape != shape or (t.stride(1) != 1 and shape[1] > 1):
        raise ValueError(f"{name}: expected a {dtype} matrix {tuple(shape)} with contiguous rows on the GPU")
    return t.data_ptr(), t.stride(0) if shape[0] > 1 else shape[1]


def stalloc_rms_norm(x, weight, *, residual=None, eps: float = 1e-6, eight_bits: bool = False, out: Optional[Dict] = None,
                     stream=None) -> Dict[str, torch.Tensor]:
    """x, residual [rows][width], weight [width] -> sum = x + residual (x itself without one), rstd float32 [rows], and y, or with
    eight_bits q float8_e4m3fn [rows][width] and scales float32 [rows][ceil(width / 128)]; both where `out` carries both.
    `sum` may be x or residual itself (out={"sum": residual})."""
    if x.dim() != 2:
        raise ValueError("x must be [rows][width]")
    _sizes(*x.shape)
    code, (rows, width) = _dtype_of(x, "x"), x.shape
    out = dict(out) if out else {}
    y = _new(out, "y", x.shape, x.dtype, x, stream) if not eight_bits or out.get("y") is not None else None
    q = scales = None
    if eight_bits or out.get("q") is not None:
        q = _new(out, "q", x.shape, torch.float8_e4m3fn, x, stream)
        scales = _new(out, "scales", (rows, -(-width // 128)), torch.float32, x, stream)
    if weight.shape != (width,) or weight.dtype != x.dtype:
        raise ValueError("weight must be [width], of the type of x")
    rstd = _new(out, "rstd", (rows,), torch.float32, x, stream)
    r, kept = (None, 0), None
    if residual is not None:
        r = _rows(residual, x.shape, x.dtype, "residual")
        kept = _new(out, "sum", x.shape, x.dtype, x, stream)
    else:
        out["sum"] = x
    _check(lib.stalloc_rms_norm(code, rows, width, *_rows(x, x.shape, x.dtype, "x"), *r, _flat(weight, "weight"), eps, _flat(kept, "sum"),
                                _flat(y, "y"), _flat(q, "q"), _flat(scales, "scales"), _flat(rstd, "rstd"), _stream(stream)), "stalloc_rms_norm")
    return out


def stalloc_rms_norm_backward(d_y, sum, weight, rstd, *, d_sum=None, out: Optional[Dict] = None, stream=None,
                              workspace_cache: Optional[Dict] = None) -> Dict[str, torch.Tensor]:
    """d_y, sum, d_sum [rows][width] -> dx (the gradient of x and of the residual), dweight float32 [width].  d_sum: the gradient that
    reaches `sum` by other ways.  dx may be d_sum or d_y itself."""
    if sum.dim() != 2:
        raise ValueError("sum must be [rows][width]")
    _sizes(*sum.shape)
    code, (rows, width) = _dtype_of(sum, "sum"), sum.shape
    if weight.shape != (width,) or weight.dtype != sum.dtype or rstd.shape != (rows,):
        raise ValueError("weight must be [width], of the type of sum, and rstd [rows]")
    if d_sum is not None and (d_sum.shape != sum.shape or d_sum.dtype != sum.dtype):
        raise ValueError("d_sum must be like sum")
    out = dict(out) if out else {}
    dx = _new(out, "dx", sum.shape, sum.dtype, sum, stream)
    dweight = _new(out, "dweight", (width,), torch.float32, sum, stream)
    args = (code, rows, width, *_rows(d_y, sum.shape, sum.dtype, "d_y"), _flat(sum, "sum"), _flat(weight, "weight"),
            _dev(rstd, torch.float32, "rstd"), _flat(d_sum, "d_sum"), _flat(dx, "dx"), _flat(dweight, "dweight"))
    return _call(lib.stalloc_rms_norm_backward, "stalloc_rms_norm_backward", args, sum, stream, workspace_cache, out)


def stalloc_token_logprobs(logits, tokens, *, top: int = 0, out: Optional[Dict] = None, stream=None,
                           workspace_cache: Optional[Dict] = None) -> Dict[str, torch.Tensor]:
    """logits [rows][vocabulary], tokens int32 [rows] (negative: none) -> logprob, entropy, lse float32 [rows], with `top` the most likely
    tokens top_tokens int32 [rows][top] (lower number first among equals) and top_logprobs float32 [rows][top]; status int32 [1]."""
    if logits.dim() != 2 or tokens.shape != (logits.shape[0],):
        raise ValueError("logits must be [rows][vocabulary] and tokens [rows]")
    _sizes(*logits.shape)
    if not 0 <= top <= min(MOST_TOP, logits.shape[1]):
        raise ValueError(f"top must be 0 .. min({MOST_TOP}, vocabulary)")
    code, (rows, vocabulary) = _dtype_of(logits, "logits"), logits.shape
    out = dict(out) if out else {}
    one = [_flat(_new(out, name, (rows,), torch.float32, logits, stream), name) for name in ("logprob", "entropy", "lse")]
    best = [None, None]
    if top:
        best = [_flat(_new(out, "top_tokens", (rows, top), torch.int32, logits, stream), "top_tokens"),
                _flat(_new(out, "top_logprobs", (rows, top), torch.float32, logits, stream), "top_logprobs")]
    status = _new(out, "status", (1,), torch.int32, logits, stream)
    args = (code, rows, vocabulary, *_rows(logits, logits.shape, logits.dtype, "logits"), _dev(tokens, torch.int32, "tokens"), top, *one, *best,
            status.data_ptr())
    return _call(lib.stalloc_token_logprobs, "stalloc_token_logprobs", args, logits, stream, workspace_cache, out)


def stalloc_token_logprobs_backward(logits, tokens, lse, entropy, d_logprob, d_entropy=None, *, out: Optional[Dict] = None,
                                    stream=None) -> Dict[str, torch.Tensor]:
    """Gradient of stalloc_token_logprobs' logprob and entropy for d_logprob, d_entropy float32 [rows] -> d_logits like logits, status.
    d_logits may be logits itself (out={"d_logits": logits})."""
    if logits.dim() != 2 or any(t is not None and t.shape != (logits.shape[0],) for t in (tokens, lse, entropy, d_logprob, d_entropy)):
        raise ValueError("logits must be [rows][vocabulary], everything else [rows]")
    _sizes(*logits.shape)
    code, (rows, vocabulary) = _dtype_of(logits, "logits"), logits.shape
    out = dict(out) if out else {}
    d_logits = _new(out, "d_logits", logits.shape, logits.dtype, logits, stream)
    status = _new(out, "status", (1,), torch.int32, logits, stream)
    _check(lib.stalloc_token_logprobs_backward(code, rows, vocabulary, *_rows(logits, logits.shape, logits.dtype, "logits"),
                                               _dev(tokens, torch.int32, "tokens"), _dev(lse, torch.float32, "lse"),
                                               _dev(entropy, torch.float32, "entropy"), _dev(d_logprob, torch.float32, "d_logprob"),
                                               _dev(d_entropy, torch.float32, "d_entropy"), *_rows(d_logits, logits.shape, logits.dtype, "d_logits"),
                                               status.data_ptr(), _stream(stream)), "stalloc_token_logprobs_backward")
    return out


class TensorList:
    """Addresses, sizes and types of tensors that stay where they are, as stalloc_clip_gradients takes them."""

    def __init__(self, tensors, outs=None):
        tensors = list(tensors)
        outs = [None] * len(tensors) if outs is None else list(outs)
        if not tensors or len(outs) != len(tensors):
            raise ValueError("expected at least one tensor, and an output for each or none")
        self.entries = (_Tensor * len(tensors))()
        for e, t, o in zip(self.entries, tensors, outs):
            e.dtype = _dtype_of(t, "tensors")
            e.data, e.count = _flat(t, "tensors"), t.numel()
            if o is not None:
                if o.shape != t.shape or o.dtype != t.dtype:
                    raise ValueError("an output must be like its tensor")
                e.out = _flat(o, "outs")
        self.keep = (tensors, outs)


def stalloc_tensor_list(tensors, outs=None) -> TensorList:
    """The tensors (contiguous, float32, bfloat16 or float16) whose norm is wanted, and where their clipped values go: `outs` like
    them, which may be the tensors themselves; None: the norm only."""
    return TensorList(tensors, outs)


def stalloc_clip_gradients(tensors: TensorList, max_norm: float, *, out: Optional[Dict] = None, stream=None,
                           workspace_cache: Optional[Dict] = None) -> Dict[str, torch.Tensor]:
    """-> norm float32 [1] over all tensors of the list, factor = min(1, max_norm / norm) float32 [1] (1 where the norm is not
    finite); the list's outputs receive tensor * factor."""
    like = tensors.keep[0][0]
    out = dict(out) if out else {}
    norm, factor = _new(out, "norm", (1,), torch.float32, like, stream), _new(out, "factor", (1,), torch.float32, like, stream)
    args = (tensors.entries, len(tensors.entries), max_norm, norm.data_ptr(), factor.data_ptr())
    return _call(lib.stalloc_clip_gradients, "stalloc_clip_gradients", args, like, stream, workspace_cache, out)
