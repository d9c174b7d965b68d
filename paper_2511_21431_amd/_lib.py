"""ctypes binding of libmemfine.so, the MI355X chunked MoE expert layer.

Argument marshalling only: every function here turns torch tensors into raw
pointers and sizes, checks on the host that they match the shape the kernels
will assume (so that no kernel is launched on a mismatched buffer), and calls
the C entry point of the same name declared in include/memfine.h.  There is
no fallback: if the library is not built, loading it raises.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Dict, Optional, Sequence

import numpy as np

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libmemfine.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_BUDGET, ERR_OOM, ERR_HIP = 0, -1, -2, -3, -4, -5
ERR_SCRATCH = -6
NOALLOC_SCRATCH_BYTES = 64 << 20
BF16, F32 = 0, 1
PASS_FWD, PASS_BWD = 0, 1

KERNELS = ["count", "dispatch", "fc1", "fc2", "combine", "fc1_recompute", "fc2_dgrad",
           "fc2_wgrad", "fc1_wgrad", "fc1_dgrad", "unpermute", "fc1_dgrad_wgrad",
           "router_fwd", "router_bwd_dx", "router_wgrad", "router_reduce", "norm_fwd", "norm_bwd",
           "route_fwd", "route_bwd", "mx_linear", "mx_fc1", "mx_fc2", "mx_combine"]


class MemfineError(RuntimeError):
    def __init__(self, code: int, where: str):
        super().__init__(f"{where}: {status_str(code)} ({code})")
        self.code = code


class Shape(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int64), ("h", ctypes.c_int32), ("F", ctypes.c_int32),
                ("E", ctypes.c_int32), ("k", ctypes.c_int32), ("dtype", ctypes.c_int32)]


ALLOC_FN = ctypes.CFUNCTYPE(ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_void_p)
RELEASE_FN = ctypes.CFUNCTYPE(None, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p,
                              ctypes.c_void_p)


class Allocator(ctypes.Structure):
    _fields_ = [("alloc", ALLOC_FN), ("release", RELEASE_FN), ("ctx", ctypes.c_void_p)]


class PlanInfo(ctypes.Structure):
    _fields_ = [("s_recv", ctypes.c_int64), ("beta", ctypes.c_int64), ("avail", ctypes.c_int64),
                ("s_max", ctypes.c_double), ("c_theory", ctypes.c_int64),
                ("chunks", ctypes.c_int32), ("fits", ctypes.c_int32),
                ("paper_peak_bytes", ctypes.c_int64), ("beta_paper", ctypes.c_int64),
                ("beta_impl", ctypes.c_int64), ("workspace_bytes", ctypes.c_int64),
                ("paper_chunks", ctypes.c_int32), ("reserved", ctypes.c_int32)]


TILE_AUTO, TILE_128, TILE_256, TILE_256_REG = 0, 1, 2, 3
CHUNK_TOKENS, CHUNK_EXPERTS = 0, 1


class LaunchOptions(ctypes.Structure):
    """memfine_launch_options: GEMM tile shape, tile order, split tail, paired
    FC1 backward launch, side streams (all bit-identical), chunk order."""
    _fields_ = [("tile", ctypes.c_int32), ("raster", ctypes.c_int32),
                ("split_tail", ctypes.c_int32), ("pair", ctypes.c_int32),
                ("streams", ctypes.c_int32), ("chunk_order", ctypes.c_int32)]


class Model(ctypes.Structure):
    """memfine_model: the memory model's configuration (notation-table symbols)."""
    _fields_ = [("b", ctypes.c_int64), ("s", ctypes.c_int64), ("h", ctypes.c_int64),
                ("a", ctypes.c_int64), ("h_d", ctypes.c_int64), ("k_a", ctypes.c_int64),
                ("e_n", ctypes.c_int64), ("g_e", ctypes.c_int64), ("t", ctypes.c_int32),
                ("c", ctypes.c_int32), ("v", ctypes.c_int32), ("p", ctypes.c_int32),
                ("D_t", ctypes.c_int32), ("full_recompute", ctypes.c_int32)]


SCORE_SOFTMAX, SCORE_SIGMOID = 0, 1
SCORES = {"softmax": SCORE_SOFTMAX, "sigmoid": SCORE_SIGMOID}


class Gating(ctypes.Structure):
    """memfine_gating: how memfine_route_fwd selects experts and forms gates."""
    _fields_ = [("E", ctypes.c_int32), ("k", ctypes.c_int32), ("score", ctypes.c_int32),
                ("groups", ctypes.c_int32), ("top_groups", ctypes.c_int32),
                ("renorm", ctypes.c_int32), ("scale", ctypes.c_float)]


class KernelStat(ctypes.Structure):
    _fields_ = [("launches", ctypes.c_int64), ("total_ms", ctypes.c_double),
                ("flops", ctypes.c_double), ("bytes", ctypes.c_double)]


_LIB = None
P = ctypes.c_void_p
I32P = ctypes.POINTER(ctypes.c_int32)
I64P = ctypes.POINTER(ctypes.c_int64)
SHP = ctypes.POINTER(Shape)
ALP = ctypes.POINTER(Allocator)
GTP = ctypes.POINTER(Gating)

_SIGS = {
    "memfine_count": (ctypes.c_int, [SHP, P, P, I64P, P]),
    "memfine_dispatch": (ctypes.c_int, [SHP, P, ctypes.c_int64, ctypes.c_int64, P, P, P, P, ALP, P]),
    "memfine_plan": (ctypes.c_int, [SHP, I64P, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64,
                                    I32P, ctypes.c_int32, I32P, ctypes.POINTER(PlanInfo)]),
    "memfine_workspace_bytes": (ctypes.c_int64, [SHP, ctypes.c_int32, ctypes.c_int32]),
    "memfine_workspace_held": (ctypes.c_int, [P, I64P]),
    "memfine_workspace_trim": (ctypes.c_int, [P, ctypes.c_int64]),
    "memfine_pool_high_water": (ctypes.c_int, [I64P, ctypes.c_int32]),
    "memfine_set_launch_options": (ctypes.c_int, [ctypes.POINTER(LaunchOptions)]),
    "memfine_get_launch_options": (ctypes.c_int, [ctypes.POINTER(LaunchOptions)]),
    "memfine_moe_fwd": (ctypes.c_int, [SHP, ctypes.c_int32, P, P, P, P, P, P, ALP, P]),
    "memfine_moe_fwd_noalloc": (ctypes.c_int, [SHP, ctypes.c_int32, P, P, P, P, P, P, P]),
    "memfine_moe_bwd": (ctypes.c_int, [SHP, ctypes.c_int32, P, P, P, P, P, P, P, P, P, P,
                                       ctypes.c_int32, ALP, P]),
    "memfine_static_memory": (ctypes.c_int, [I64P, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                             ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, I64P]),
    "memfine_activation_memory": (ctypes.c_int, [ctypes.POINTER(Model), ctypes.c_int32,
                                                 ctypes.c_int64, I64P]),
    "memfine_mact_thresholds": (ctypes.c_int, [ctypes.POINTER(Model), ctypes.c_int32, ctypes.c_int64,
                                               ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, I32P,
                                               ctypes.c_int32, I64P]),
    "memfine_mact_select": (ctypes.c_int, [I32P, I64P, ctypes.c_int32, ctypes.c_int64, I32P]),
    "memfine_router_fwd": (ctypes.c_int, [SHP, P, P, P, P, P, P]),
    "memfine_router_bwd": (ctypes.c_int, [SHP, P, P, P, P, P, P, P, ctypes.c_int32,
                                          ctypes.c_int32, ALP, P]),
    "memfine_norm_fwd": (ctypes.c_int, [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32,
                                        ctypes.c_float, P, P, P, P, P, P, P, P]),
    "memfine_norm_bwd": (ctypes.c_int, [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32,
                                        ctypes.c_float, P, P, P, P, P, P, ctypes.c_int32, ALP, P]),
    "memfine_mx_values": (ctypes.c_int, [ctypes.c_int64, ctypes.c_int32, P, P, ctypes.c_int32, P,
                                         P]),
    "memfine_route_fwd": (ctypes.c_int, [ctypes.c_int64, GTP, P, P, P, P, P]),
    "memfine_route_bwd": (ctypes.c_int, [ctypes.c_int64, GTP, P, P, P, P, P]),
    "memfine_router_logits": (ctypes.c_int, [SHP, P, P, P, P]),
    "memfine_router_logits_bwd": (ctypes.c_int, [SHP, P, P, P, P, P, ctypes.c_int32,
                                                 ctypes.c_int32, ALP, P]),
    "memfine_mxw_code_bytes": (ctypes.c_int64, [ctypes.c_int32, ctypes.c_int32]),
    "memfine_mxw_scale_bytes": (ctypes.c_int64, [ctypes.c_int32, ctypes.c_int32]),
    "memfine_mxw_pack": (ctypes.c_int, [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, P, P, P, P,
                                        P]),
    "memfine_mxw_quantize": (ctypes.c_int, [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                            ctypes.c_int32, P, P, P, P]),
    "memfine_mxw_unpack": (ctypes.c_int, [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, P, P,
                                          ctypes.c_int32, P, P]),
    "memfine_linear_mxw": (ctypes.c_int, [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, P, P, P,
                                          P, ctypes.c_int32, P, P]),
    "memfine_linear_mxw_alloc": (ctypes.c_int, [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, P,
                                                P, P, P, ctypes.c_int32, P, ALP, P]),
    "memfine_linear_mxw_workspace_bytes": (ctypes.c_int64, [ctypes.c_int64, ctypes.c_int32,
                                                            ctypes.c_int32, ctypes.c_int32]),
    "memfine_moe_fwd_mxw": (ctypes.c_int, [SHP, ctypes.c_int32, P, P, P, P, P, P, P, P, P, ALP, P]),
    "memfine_moe_mxw_workspace_bytes": (ctypes.c_int64, [SHP, ctypes.c_int32, ctypes.c_int32]),
    "memfine_status_str": (ctypes.c_char_p, [ctypes.c_int]),
    "memfine_profile_begin": (ctypes.c_int, [ctypes.c_uint32]),
    "memfine_profile_end": (ctypes.c_int, [ctypes.POINTER(KernelStat)]),
}


def lib() -> ctypes.CDLL:
    """The loaded library; raises if it has not been built."""
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with "
                              "`python -m paper_2511_21431_amd.build` (there is no fallback)")
        # torch first, when it is installed: the library then binds to the HIP
        # runtime torch has loaded.  Loaded before torch, it would bring in the
        # system's runtime, and torch would load its own beside it; two runtimes
        # in one process share neither device memory nor streams, and the
        # library's first launch on torch's tensors fails.
        try:
            import torch  # noqa: F401
        except ImportError:
            pass
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGS.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _LIB = L
    return _LIB


def status_str(code: int) -> str:
    return lib().memfine_status_str(int(code)).decode()


def _check(code: int, where: str, allow=(OK,)) -> int:
    if code not in allow:
        raise MemfineError(code, where)
    return code


def make_shape(T: int, h: int, F: int, E: int, k: int, dtype: int) -> Shape:
    return Shape(int(T), int(h), int(F), int(E), int(k), int(dtype))


# ----------------------------------------------------------- tensor checks
_TORCH = None


def _torch():
    global _TORCH
    if _TORCH is None:
        import torch
        _TORCH = torch
    return _TORCH


def _dt(shape: Shape):
    torch = _torch()
    return torch.bfloat16 if shape.dtype == BF16 else torch.float32


def _ptr(t, shape_tuple, dtype, name) -> int:
    """Address of a contiguous device tensor of that shape and dtype.  (One
    condition for the tensor that passes: a call of a few microseconds on the
    GPU has half a dozen of these.)"""
    if t is not None and t.shape == shape_tuple and t.dtype == dtype and t.is_contiguous():
        if t.is_cuda:
            return t.data_ptr()
        if t.numel() == 0:
            return 0
        raise ValueError(f"{name} must be a device tensor")
    if t is None:
        raise ValueError(f"{name} is required")
    if tuple(t.shape) != tuple(shape_tuple):
        raise ValueError(f"{name}: shape {tuple(t.shape)} != expected {tuple(shape_tuple)}")
    if t.dtype != dtype:
        raise ValueError(f"{name}: dtype {t.dtype} != expected {dtype}")
    raise ValueError(f"{name} must be contiguous")


def _stream(stream):
    """Handle of the stream (None: torch's current stream on the current device)."""
    if stream is None:
        torch = _torch()
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    if hasattr(stream, "cuda_stream"):
        return stream.cuda_stream
    return int(stream)


def _torch_stream(handle, device):
    """The torch stream object for a stream handle."""
    torch = _torch()
    ptr = int(handle or 0)
    for cand in (torch.cuda.current_stream(device), torch.cuda.default_stream(device)):
        if cand.cuda_stream == ptr:
            return cand
    return torch.cuda.ExternalStream(ptr, device=device)


class TorchAllocator:
    """Serves the layer's per-chunk buffers from torch's caching allocator,
    so that torch.cuda.max_memory_allocated sees the layer's true peak.

    The library asks for and hands back each buffer in order on the stream of
    its call: a buffer is allocated on that stream (torch then reuses it only
    in that stream's order), and released with record_stream on it, so torch
    never hands the memory to other work before the library's kernels that
    use it have run."""

    def __init__(self, device=None):
        torch = _torch()
        self.device = torch.device("cuda", torch.cuda.current_device()) if device is None else device
        self.live: Dict[int, object] = {}
        self.live_bytes = 0
        self.high_water = 0                    # most bytes held at once
        self.calls = 0
        self.fail_at: Optional[int] = None     # for tests: fail the n-th allocation
        self._alloc = ALLOC_FN(self._do_alloc)
        self._release = RELEASE_FN(self._do_release)
        self.struct = Allocator(self._alloc, self._release, None)

    def _stream(self, stream):
        return _torch_stream(stream, self.device)

    def _do_alloc(self, nbytes, stream, ctx):
        torch = _torch()
        self.calls += 1
        if self.fail_at is not None and self.calls >= self.fail_at:
            return None
        with torch.cuda.stream(self._stream(stream)):
            t = torch.empty(int(nbytes), dtype=torch.uint8, device=self.device)
        p = t.data_ptr()
        self.live[p] = t
        self.live_bytes += int(nbytes)
        self.high_water = max(self.high_water, self.live_bytes)
        return p

    def _do_release(self, ptr, nbytes, stream, ctx):
        t = self.live.pop(int(ptr), None)
        if t is not None:
            t.record_stream(self._stream(stream))
            self.live_bytes -= int(nbytes)


def _alloc_arg(allocator):
    if allocator is None:
        return None
    if isinstance(allocator, TorchAllocator):
        return ctypes.byref(allocator.struct)
    return ctypes.byref(allocator)


# --------------------------------------------------------------- entry points
def memfine_count(shape: Shape, idx, work, stream=None) -> np.ndarray:
    torch = _torch()
    out = np.zeros(shape.E, dtype=np.int64)
    rc = lib().memfine_count(ctypes.byref(shape), _ptr(idx, (shape.T, shape.k), torch.int32, "idx"),
                             _ptr(work, (shape.E + 1,), torch.int32, "work"),
                             out.ctypes.data_as(I64P), _stream(stream))
    _check(rc, "memfine_count")
    return out


def memfine_dispatch(shape: Shape, idx, t0: int, t1: int, counts, offsets, sorted_slot,
                     row_of_slot, allocator=None, stream=None) -> None:
    torch = _torch()
    n = (t1 - t0) * shape.k
    rc = lib().memfine_dispatch(
        ctypes.byref(shape), _ptr(idx, (shape.T, shape.k), torch.int32, "idx"), int(t0), int(t1),
        _ptr(counts, (shape.E,), torch.int32, "counts"),
        _ptr(offsets, (shape.E + 1,), torch.int32, "offsets"),
        _ptr(sorted_slot, (n,), torch.int32, "sorted_slot"),
        _ptr(row_of_slot, (n,), torch.int32, "row_of_slot"), _alloc_arg(allocator),
        _stream(stream))
    _check(rc, "memfine_dispatch")


def memfine_plan(shape: Shape, counts: Sequence[int], budget_bytes: int, bins=(1, 2, 4, 8),
                 fixed_bytes: int = 0, beta_bytes: int = 0):
    """Returns (status, chunks, info dict); status is OK or ERR_BUDGET."""
    c = np.ascontiguousarray(np.asarray(counts, dtype=np.int64))
    b = np.ascontiguousarray(np.asarray(bins, dtype=np.int32))
    if c.size != shape.E:
        raise ValueError("counts must have E entries")
    out = ctypes.c_int32(0)
    info = PlanInfo()
    rc = lib().memfine_plan(ctypes.byref(shape), c.ctypes.data_as(I64P), int(budget_bytes),
                            int(fixed_bytes), int(beta_bytes), b.ctypes.data_as(I32P), int(b.size),
                            ctypes.byref(out), ctypes.byref(info))
    _check(rc, "memfine_plan", allow=(OK, ERR_BUDGET))
    return rc, int(out.value), {f: getattr(info, f) for f, _ in PlanInfo._fields_}


def make_model(**kw) -> Model:
    """memfine_model from keyword fields (b, s, h, a, h_d, k_a, e_n, g_e, t, c, v, p,
    D_t, full_recompute); unspecified fields default to 0 except the parallel
    sizes and b (1), D_t (2) and full_recompute (1)."""
    d = dict(b=1, t=1, c=1, v=1, p=1, D_t=2, full_recompute=1)
    d.update(kw)
    m = Model()
    for f, _ in Model._fields_:
        setattr(m, f, int(d.get(f, 0)))
    return m


def memfine_static_memory(S_para: Sequence[int], v: int, l: int, D_para: int = 2,
                          D_grad: int = 2, D_opt: int = 4) -> int:
    a = np.ascontiguousarray(np.asarray(list(S_para), dtype=np.int64))
    out = ctypes.c_int64(0)
    rc = lib().memfine_static_memory(a.ctypes.data_as(I64P), int(a.size), int(v), int(l),
                                     int(D_para), int(D_grad), int(D_opt), ctypes.byref(out))
    _check(rc, "memfine_static_memory")
    return int(out.value)


def memfine_activation_memory(model: Model, r_pp: int, s_recv: int) -> int:
    out = ctypes.c_int64(0)
    rc = lib().memfine_activation_memory(ctypes.byref(model), int(r_pp), int(s_recv),
                                         ctypes.byref(out))
    _check(rc, "memfine_activation_memory")
    return int(out.value)


def memfine_mact_thresholds(model: Model, r_pp: int, M_gpu: int, alpha_num: int, alpha_den: int,
                            M_sta: int, bins=(1, 2, 4, 8)) -> list:
    b = np.ascontiguousarray(np.asarray(bins, dtype=np.int32))
    out = np.zeros(b.size, dtype=np.int64)
    rc = lib().memfine_mact_thresholds(ctypes.byref(model), int(r_pp), int(M_gpu), int(alpha_num),
                                       int(alpha_den), int(M_sta), b.ctypes.data_as(I32P),
                                       int(b.size), out.ctypes.data_as(I64P))
    _check(rc, "memfine_mact_thresholds")
    return [int(x) for x in out]


def memfine_mact_select(bins: Sequence[int], thresholds: Sequence[int], s_recv: int):
    """Returns (status, chunks); status is OK or ERR_BUDGET."""
    b = np.ascontiguousarray(np.asarray(bins, dtype=np.int32))
    th = np.ascontiguousarray(np.asarray(thresholds, dtype=np.int64))
    if b.size != th.size:
        raise ValueError("one threshold per bin")
    out = ctypes.c_int32(0)
    rc = lib().memfine_mact_select(b.ctypes.data_as(I32P), th.ctypes.data_as(I64P), int(b.size),
                                   int(s_recv), ctypes.byref(out))
    _check(rc, "memfine_mact_select", allow=(OK, ERR_BUDGET))
    return rc, int(out.value)


def memfine_workspace_bytes(shape: Shape, chunks: int, pass_: int) -> int:
    v = lib().memfine_workspace_bytes(ctypes.byref(shape), int(chunks), int(pass_))
    if v < 0:
        raise MemfineError(int(v), "memfine_workspace_bytes")
    return int(v)


def memfine_workspace_held(stream=None) -> int:
    """Bytes of the library's cached workspace block for the stream."""
    out = ctypes.c_int64(0)
    _check(lib().memfine_workspace_held(_stream(stream), ctypes.byref(out)),
           "memfine_workspace_held")
    return int(out.value)


def memfine_workspace_trim(keep_bytes: int = 0, stream=None) -> None:
    _check(lib().memfine_workspace_trim(_stream(stream), int(keep_bytes)), "memfine_workspace_trim")


def memfine_pool_high_water(reset: bool = False) -> int:
    out = ctypes.c_int64(0)
    _check(lib().memfine_pool_high_water(ctypes.byref(out), 1 if reset else 0),
           "memfine_pool_high_water")
    return int(out.value)


def memfine_set_launch_options(tile: int = TILE_AUTO, raster: int = -1, split_tail: bool = True,
                               pair: bool = False, streams: bool = False,
                               chunk_order: int = CHUNK_TOKENS) -> None:
    o = LaunchOptions(int(tile), int(raster), int(bool(split_tail)), int(bool(pair)),
                      int(bool(streams)), int(chunk_order))
    _check(lib().memfine_set_launch_options(ctypes.byref(o)), "memfine_set_launch_options")


def memfine_get_launch_options() -> Dict[str, int]:
    o = LaunchOptions()
    _check(lib().memfine_get_launch_options(ctypes.byref(o)), "memfine_get_launch_options")
    return {f: getattr(o, f) for f, _ in LaunchOptions._fields_}


def memfine_moe_fwd(shape: Shape, chunks: int, X, idx, gates, W1, W2, Y, allocator=None,
                    stream=None) -> None:
    torch = _torch()
    dt = _dt(shape)
    T, h, F, E, k = shape.T, shape.h, shape.F, shape.E, shape.k
    rc = lib().memfine_moe_fwd(
        ctypes.byref(shape), int(chunks), _ptr(X, (T, h), dt, "X"),
        _ptr(idx, (T, k), torch.int32, "idx"), _ptr(gates, (T, k), torch.float32, "gates"),
        _ptr(W1, (E, 2 * F, h), dt, "W1"), _ptr(W2, (E, h, F), dt, "W2"),
        _ptr(Y, (T, h), dt, "Y"), _alloc_arg(allocator), _stream(stream))
    _check(rc, "memfine_moe_fwd")


def memfine_moe_fwd_noalloc(shape: Shape, chunks: int, X, idx, gates, W1, W2, Y,
                            stream=None) -> None:
    """memfine_moe_fwd with the chunk buffers in the library's static device
    scratch (no allocation); MemfineError(ERR_SCRATCH) when the largest chunk
    needs more than NOALLOC_SCRATCH_BYTES."""
    torch = _torch()
    dt = _dt(shape)
    T, h, F, E, k = shape.T, shape.h, shape.F, shape.E, shape.k
    rc = lib().memfine_moe_fwd_noalloc(
        ctypes.byref(shape), int(chunks), _ptr(X, (T, h), dt, "X"),
        _ptr(idx, (T, k), torch.int32, "idx"), _ptr(gates, (T, k), torch.float32, "gates"),
        _ptr(W1, (E, 2 * F, h), dt, "W1"), _ptr(W2, (E, h, F), dt, "W2"),
        _ptr(Y, (T, h), dt, "Y"), _stream(stream))
    _check(rc, "memfine_moe_fwd_noalloc")


def memfine_moe_bwd(shape: Shape, chunks: int, X, idx, gates, W1, W2, dY, dX, dW1, dW2, dgates,
                    accumulate_dW: bool = False, allocator=None, stream=None) -> None:
    torch = _torch()
    dt = _dt(shape)
    T, h, F, E, k = shape.T, shape.h, shape.F, shape.E, shape.k
    rc = lib().memfine_moe_bwd(
        ctypes.byref(shape), int(chunks), _ptr(X, (T, h), dt, "X"),
        _ptr(idx, (T, k), torch.int32, "idx"), _ptr(gates, (T, k), torch.float32, "gates"),
        _ptr(W1, (E, 2 * F, h), dt, "W1"), _ptr(W2, (E, h, F), dt, "W2"),
        _ptr(dY, (T, h), dt, "dY"), _ptr(dX, (T, h), dt, "dX"),
        _ptr(dW1, (E, 2 * F, h), torch.float32, "dW1"),
        _ptr(dW2, (E, h, F), torch.float32, "dW2"),
        _ptr(dgates, (T, k), torch.float32, "dgates"), 1 if accumulate_dW else 0,
        _alloc_arg(allocator), _stream(stream))
    _check(rc, "memfine_moe_bwd")


def memfine_status_str(code: int) -> str:
    return status_str(code)


def memfine_router_fwd(shape: Shape, X, Wr, idx, gates, logits=None, stream=None) -> None:
    """Router forward into caller-owned idx [T, k] int32, gates [T, k] fp32 and
    optionally logits [T, E] fp32."""
    torch = _torch()
    dt = _dt(shape)
    T, h, E, k = shape.T, shape.h, shape.E, shape.k
    rc = lib().memfine_router_fwd(
        ctypes.byref(shape), _ptr(X, (T, h), dt, "X"), _ptr(Wr, (E, h), dt, "Wr"),
        _ptr(idx, (T, k), torch.int32, "idx"), _ptr(gates, (T, k), torch.float32, "gates"),
        None if logits is None else _ptr(logits, (T, E), torch.float32, "logits"), _stream(stream))
    _check(rc, "memfine_router_fwd")


def memfine_router_bwd(shape: Shape, X, Wr, idx, gates, dgates, dX, dWr, accumulate_dX=False,
                       accumulate_dWr=False, allocator=None, stream=None) -> None:
    torch = _torch()
    dt = _dt(shape)
    T, h, E, k = shape.T, shape.h, shape.E, shape.k
    rc = lib().memfine_router_bwd(
        ctypes.byref(shape), _ptr(X, (T, h), dt, "X"), _ptr(Wr, (E, h), dt, "Wr"),
        _ptr(idx, (T, k), torch.int32, "idx"), _ptr(gates, (T, k), torch.float32, "gates"),
        _ptr(dgates, (T, k), torch.float32, "dgates"), _ptr(dX, (T, h), dt, "dX"),
        _ptr(dWr, (E, h), torch.float32, "dWr"), int(bool(accumulate_dX)),
        int(bool(accumulate_dWr)), _alloc_arg(allocator), _stream(stream))
    _check(rc, "memfine_router_bwd")


# ------------------------------------------------------- around the layer
def _dtype_of(t, name) -> int:
    torch = _torch()
    if t is None:
        raise ValueError(f"{name} is required")
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise ValueError(f"{name}: dtype {t.dtype} is neither bfloat16 nor float32")


def _rows(t, name):
    """(rows, columns) of a matrix argument."""
    if t is None:
        raise ValueError(f"{name} is required")
    if t.dim() != 2:
        raise ValueError(f"{name}: expected a matrix, got shape {tuple(t.shape)}")
    return t.shape[0], t.shape[1]


def _opt(t, shape_tuple, dtype, name):
    return None if t is None else _ptr(t, shape_tuple, dtype, name)


def memfine_norm_fwd(eps: float, X, w, R=None, S=None, Y=None, Q=None, QS=None,
                     stream=None) -> None:
    """S = X + R and its RMS norm Y, both [T, h] in X's dtype, and Y's MX8 form
    in Q uint8 [T, h], QS uint8 [T, h/32]; outputs are the caller's, None: not
    asked for."""
    torch = _torch()
    T, h = _rows(X, "X")
    rc = lib().memfine_norm_fwd(
        T, h, _dtype_of(X, "X"), float(eps), _ptr(X, (T, h), X.dtype, "X"),
        _opt(R, (T, h), X.dtype, "R"), _ptr(w, (h,), X.dtype, "w"), _opt(S, (T, h), X.dtype, "S"),
        _opt(Y, (T, h), X.dtype, "Y"), _opt(Q, (T, h), torch.uint8, "Q"),
        _opt(QS, (T, h // 32), torch.uint8, "QS"), _stream(stream))
    _check(rc, "memfine_norm_fwd")


def memfine_norm_bwd(eps: float, X, w, dY, dX, dw, dS=None, accumulate_dw: bool = False,
                     allocator=None, stream=None) -> None:
    """Gradient of the norm: X is the norm's input (the forward's S), dX [T, h],
    dw float [h]."""
    torch = _torch()
    T, h = _rows(X, "X")
    rc = lib().memfine_norm_bwd(
        T, h, _dtype_of(X, "X"), float(eps), _ptr(X, (T, h), X.dtype, "X"),
        _ptr(w, (h,), X.dtype, "w"), _ptr(dY, (T, h), X.dtype, "dY"),
        _opt(dS, (T, h), X.dtype, "dS"), _ptr(dX, (T, h), X.dtype, "dX"),
        _ptr(dw, (h,), torch.float32, "dw"), int(bool(accumulate_dw)), _alloc_arg(allocator),
        _stream(stream))
    _check(rc, "memfine_norm_bwd")


def memfine_mx_values(Q, QS, out, stream=None) -> None:
    """The values of an MX8 tensor, into out [T, h], bfloat16 or float32."""
    torch = _torch()
    T, h = _rows(Q, "Q")
    rc = lib().memfine_mx_values(T, h, _ptr(Q, (T, h), torch.uint8, "Q"),
                                 _ptr(QS, (T, h // 32), torch.uint8, "QS"), _dtype_of(out, "out"),
                                 _ptr(out, (T, h), out.dtype, "out"), _stream(stream))
    _check(rc, "memfine_mx_values")


def make_gating(E: int, k: int, score: str = "softmax", groups: int = 1, top_groups: int = 1,
                renorm: bool = True, scale: float = 1.0) -> Gating:
    """memfine_gating; score is "softmax" or "sigmoid"."""
    if score not in SCORES:
        raise ValueError(f"score: {score!r} is neither 'softmax' nor 'sigmoid'")
    return Gating(E, k, SCORES[score], groups, top_groups, bool(renorm), scale)


def memfine_route_fwd(gating: Gating, logits, idx, gates, bias=None, stream=None) -> None:
    """Routing from logits float [T, E] into idx int32 [T, k], gates float [T, k]."""
    torch = _torch()
    T, _ = _rows(logits, "logits")
    E, k = gating.E, gating.k
    rc = lib().memfine_route_fwd(
        T, ctypes.byref(gating), _ptr(logits, (T, E), torch.float32, "logits"),
        _opt(bias, (E,), torch.float32, "bias"), _ptr(idx, (T, k), torch.int32, "idx"),
        _ptr(gates, (T, k), torch.float32, "gates"), _stream(stream))
    _check(rc, "memfine_route_fwd")


def memfine_route_bwd(gating: Gating, logits, idx, dgates, dlogits, stream=None) -> None:
    """Gradient of the gates with respect to the logits, into dlogits float [T, E]."""
    torch = _torch()
    T, _ = _rows(logits, "logits")
    E, k = gating.E, gating.k
    rc = lib().memfine_route_bwd(
        T, ctypes.byref(gating), _ptr(logits, (T, E), torch.float32, "logits"),
        _ptr(idx, (T, k), torch.int32, "idx"), _ptr(dgates, (T, k), torch.float32, "dgates"),
        _ptr(dlogits, (T, E), torch.float32, "dlogits"), _stream(stream))
    _check(rc, "memfine_route_bwd")


def memfine_router_logits(shape: Shape, X, Wr, logits, stream=None) -> None:
    """logits float [T, E] = X Wr^T."""
    torch = _torch()
    dt = _dt(shape)
    T, h, E = shape.T, shape.h, shape.E
    rc = lib().memfine_router_logits(
        ctypes.byref(shape), _ptr(X, (T, h), dt, "X"), _ptr(Wr, (E, h), dt, "Wr"),
        _ptr(logits, (T, E), torch.float32, "logits"), _stream(stream))
    _check(rc, "memfine_router_logits")


def memfine_router_logits_bwd(shape: Shape, X, Wr, dlogits, dX, dWr, accumulate_dX=False,
                              accumulate_dWr=False, allocator=None, stream=None) -> None:
    torch = _torch()
    dt = _dt(shape)
    T, h, E = shape.T, shape.h, shape.E
    rc = lib().memfine_router_logits_bwd(
        ctypes.byref(shape), _ptr(X, (T, h), dt, "X"), _ptr(Wr, (E, h), dt, "Wr"),
        _ptr(dlogits, (T, E), torch.float32, "dlogits"), _ptr(dX, (T, h), dt, "dX"),
        _ptr(dWr, (E, h), torch.float32, "dWr"), int(bool(accumulate_dX)),
        int(bool(accumulate_dWr)), _alloc_arg(allocator), _stream(stream))
    _check(rc, "memfine_router_logits_bwd")


def memfine_mxw_code_bytes(N: int, K: int) -> int:
    v = lib().memfine_mxw_code_bytes(int(N), int(K))
    if v < 0:
        raise MemfineError(int(v), "memfine_mxw_code_bytes")
    return int(v)


def memfine_mxw_scale_bytes(N: int, K: int) -> int:
    v = lib().memfine_mxw_scale_bytes(int(N), int(K))
    if v < 0:
        raise MemfineError(int(v), "memfine_mxw_scale_bytes")
    return int(v)


@functools.lru_cache(maxsize=256)
def _mxw_bytes(N: int, K: int):
    return memfine_mxw_code_bytes(N, K), memfine_mxw_scale_bytes(N, K)


def _mxw_weights(E, N, K, codes, scales, names=("codes", "scales")):
    """Pointers of E laid-out MX4 matrices."""
    torch = _torch()
    cb, sb = _mxw_bytes(N, K)
    return (_ptr(codes, (E, cb), torch.uint8, names[0]),
            _ptr(scales, (E, sb), torch.uint8, names[1]))


def _mxw_outputs(E, N, K, codes, scales, device, stream):
    """(codes, scales, their pointers), allocated where None is given: in the order
    of the call's stream, which writes them (memory of the current stream's order
    could still be in use there), and kept for the current stream's uses."""
    torch = _torch()
    cb, sb = _mxw_bytes(N, K)

    def made(t, nbytes):
        if t is not None:
            return t
        if stream is None or device.type != "cuda":
            return torch.empty((E, nbytes), dtype=torch.uint8, device=device)
        with torch.cuda.stream(_torch_stream(_stream(stream), device)):
            t = torch.empty((E, nbytes), dtype=torch.uint8, device=device)
        t.record_stream(torch.cuda.current_stream(device))
        return t
    codes, scales = made(codes, cb), made(scales, sb)
    return (codes, scales) + _mxw_weights(E, N, K, codes, scales)


def memfine_mxw_pack(E: int, N: int, K: int, row_codes, row_scales, codes=None, scales=None,
                     stream=None):
    """Lays row-major MX4 matrices out, codes uint8 [E, N, K/2] and scales uint8
    [E, N, K/32]; returns (codes, scales), allocated where None is given."""
    torch = _torch()
    codes, scales, pc, ps = _mxw_outputs(E, N, K, codes, scales, row_codes.device,
                                         stream)
    rc = lib().memfine_mxw_pack(
        int(E), int(N), int(K), _ptr(row_codes, (E, N, K // 2), torch.uint8, "row_codes"),
        _ptr(row_scales, (E, N, K // 32), torch.uint8, "row_scales"), pc, ps, _stream(stream))
    _check(rc, "memfine_mxw_pack")
    return codes, scales


def memfine_mxw_quantize(W, codes=None, scales=None, stream=None):
    """Rounds matrices [E, N, K] (bfloat16 or float32) to MX4, laid out; returns
    (codes, scales), allocated where None is given."""
    E, N, K = W.shape
    codes, scales, pc, ps = _mxw_outputs(E, N, K, codes, scales, W.device, stream)
    rc = lib().memfine_mxw_quantize(int(E), int(N), int(K), _dtype_of(W, "W"),
                                    _ptr(W, (E, N, K), W.dtype, "W"), pc, ps, _stream(stream))
    _check(rc, "memfine_mxw_quantize")
    return codes, scales


def memfine_mxw_unpack(codes, scales, W, stream=None) -> None:
    """The values of laid-out MX4 matrices, into W [E, N, K], bfloat16 or float32."""
    E, N, K = W.shape
    pc, ps = _mxw_weights(E, N, K, codes, scales)
    rc = lib().memfine_mxw_unpack(int(E), int(N), int(K), pc, ps, _dtype_of(W, "W"),
                                  _ptr(W, (E, N, K), W.dtype, "W"), _stream(stream))
    _check(rc, "memfine_mxw_unpack")


def _act(X, XS, T, K):
    """Pointers of activations [T, K]: bfloat16, or e4m3 bytes with scales (MX8)."""
    torch = _torch()
    dt = torch.bfloat16 if XS is None else torch.uint8
    return _ptr(X, (T, K), dt, "X"), _opt(XS, (T, K // 32), torch.uint8, "XS")


def memfine_linear_mxw(N: int, K: int, X, codes, scales, Y, XS=None, stream=None,
                       allocator=None) -> None:
    """Y [T, N] (bfloat16 or float32) = X [T, K] W^T, W one laid-out MX4 matrix
    (codes, scales: [1, bytes]); X bfloat16, or e4m3 bytes with scales XS.  The
    allocator serves the partial results of a split reduction."""
    T, _ = _rows(X, "X")
    pc, ps = _mxw_weights(1, N, K, codes, scales)
    px, pxs = _act(X, XS, T, K)
    rc = lib().memfine_linear_mxw_alloc(T, int(N), int(K), px, pxs, pc, ps, _dtype_of(Y, "Y"),
                                        _ptr(Y, (T, N), Y.dtype, "Y"), _alloc_arg(allocator),
                                        _stream(stream))
    _check(rc, "memfine_linear_mxw")


def memfine_linear_mxw_workspace_bytes(T: int, N: int, K: int, mx8: bool = False) -> int:
    v = lib().memfine_linear_mxw_workspace_bytes(int(T), int(N), int(K), int(bool(mx8)))
    if v < 0:
        raise MemfineError(int(v), "memfine_linear_mxw_workspace_bytes")
    return int(v)


def memfine_moe_fwd_mxw(shape: Shape, chunks: int, X, idx, gates, W1_codes, W1_scales, W2_codes,
                        W2_scales, Y, XS=None, allocator=None, stream=None) -> None:
    """memfine_moe_fwd with laid-out MX4 weights; X bfloat16 [T, h], or e4m3
    bytes with scales XS uint8 [T, h/32]."""
    torch = _torch()
    T, h, F, E, k = shape.T, shape.h, shape.F, shape.E, shape.k
    p1, q1 = _mxw_weights(E, 2 * F, h, W1_codes, W1_scales, ("W1_codes", "W1_scales"))
    p2, q2 = _mxw_weights(E, h, F, W2_codes, W2_scales, ("W2_codes", "W2_scales"))
    px, pxs = _act(X, XS, T, h)
    rc = lib().memfine_moe_fwd_mxw(
        ctypes.byref(shape), int(chunks), px, pxs, _ptr(idx, (T, k), torch.int32, "idx"),
        _ptr(gates, (T, k), torch.float32, "gates"), p1, q1, p2, q2,
        _ptr(Y, (T, h), torch.bfloat16, "Y"), _alloc_arg(allocator), _stream(stream))
    _check(rc, "memfine_moe_fwd_mxw")


def memfine_moe_mxw_workspace_bytes(shape: Shape, chunks: int, mx8: bool = False) -> int:
    v = lib().memfine_moe_mxw_workspace_bytes(ctypes.byref(shape), int(chunks), int(bool(mx8)))
    if v < 0:
        raise MemfineError(int(v), "memfine_moe_mxw_workspace_bytes")
    return int(v)


def memfine_profile_begin(kernels: Sequence[str] = tuple(KERNELS)) -> None:
    mask = 0
    for name in kernels:
        mask |= 1 << KERNELS.index(name)
    _check(lib().memfine_profile_begin(mask), "memfine_profile_begin")


def memfine_profile_end() -> Dict[str, Dict[str, float]]:
    arr = (KernelStat * len(KERNELS))()
    _check(lib().memfine_profile_end(arr), "memfine_profile_end")
    return {name: {"launches": arr[i].launches, "total_ms": arr[i].total_ms,
                   "flops": arr[i].flops, "bytes": arr[i].bytes}
            for i, name in enumerate(KERNELS) if arr[i].launches > 0}
