"""Python binding of the C ABI in include/roomie.h (argument marshalling only).

Every function has the name of its C entry point, takes torch tensors that
live on the GPU, enqueues work on torch's current stream and returns torch
tensors.  All computation happens in librm.so's HIP kernels; if the library
is not built, or a tensor is not on the GPU, the call raises.
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "librm.so")

RM_OK, RM_EINVAL, RM_EWORKSPACE, RM_EUNSUPPORTED, RM_ELAUNCH, RM_ETOOLARGE = 0, 1, 2, 3, 4, 5
RM_STATIC_SCRATCH_BYTES = 64 << 20
ALIGN_FIRST, ALIGN_CONFLICT_STARTS, ALIGN_OFFSETS, ALIGN_SAMPLED_STARTS = 0, 1, 2, 3
REDUCE_MEDIAN, REDUCE_MAX = 0, 1
SWEEP_TEMPORAL, SWEEP_LOCKSTEP, SWEEP_ADJUSTED = 0, 1, 2
DROP_ISO, DROP_ADJUSTED = 0, 1

ST_INFEASIBLE_KERNEL = 1
ST_BAD_DURATION = 2
ST_BAD_OFFSETS = 4
ST_EMPTY_MODEL = 8
ST_PAIR_TOO_LONG = 16
ST_BAD_MODEL_ID = 32
ST_BAD_EVENT = 64
ST_INVALID_CONFIG = 128
ST_BAD_DELAY = 256
ST_WAIT_TIMEOUT = 512
ST_BAD_LENGTH = 1024
ST_BAD_PAGE = 2048

ALIGN_NAMES = {"first": ALIGN_FIRST, "conflict_starts": ALIGN_CONFLICT_STARTS,
               "offsets": ALIGN_OFFSETS, "sampled_starts": ALIGN_SAMPLED_STARTS}
REDUCE_NAMES = {"median": REDUCE_MEDIAN, "max": REDUCE_MAX}
SWEEP_NAMES = {"temporal": SWEEP_TEMPORAL, "lockstep": SWEEP_LOCKSTEP,
               "adjusted": SWEEP_ADJUSTED}
POLICY_EQUAL, POLICY_PRIORITY, POLICY_FCFS = 0, 1, 2
POLICY_NAMES = {"equal": POLICY_EQUAL, "priority": POLICY_PRIORITY, "fcfs": POLICY_FCFS}

TYPES = {torch.bfloat16: 0, torch.float16: 1}
CODES = {torch.int8: 0, torch.float8_e4m3fn: 1}
ACT_NAMES = {"none": 0, "swiglu": 1}
NORM_NAMES = {"rms": 0, "layer": 1}
ROTARY_NAMES = {"half": 0, "interleaved": 1}


class DeviceDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "num_sm", "max_threads_per_sm", "max_blocks_per_sm",
        "regs_per_sm", "smem_per_sm", "warp_size")]

    @classmethod
    def of(cls, d):
        if isinstance(d, cls):
            return d
        return cls(**{k: int(d[k]) for k, _ in cls._fields_})


class PairOpts(ctypes.Structure):
    _fields_ = [("align_mode", ctypes.c_int32), ("reduce_mode", ctypes.c_int32),
                ("num_offsets", ctypes.c_int32), ("max_kernels_per_model", ctypes.c_int32),
                ("sweep_event_begin", ctypes.c_void_p), ("sweep_event_end", ctypes.c_void_p),
                ("sweep_mode", ctypes.c_int32), ("start_draws", ctypes.c_void_p),
                ("policy", ctypes.c_int32)]


class Cache(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("k", "v", "k_scale", "v_scale")] +
                [(n, ctypes.c_int32) for n in ("n_pages", "kv_heads", "page_tokens", "head_dim",
                                               "codes")])


class Sequences(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("table", "lengths", "token_offsets")] +
                [(n, ctypes.c_int32) for n in ("n_seqs", "table_stride", "n_tokens",
                                               "max_tokens")])


class Launch(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("grid", "threads", "regs", "smem")]


_lib = None


def library():
    """The loaded librm.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("librm.so is not built: run `python -m paper_2607_16784_amd.build`")
        lib = ctypes.CDLL(LIB_PATH)
        P, i32, i64, f64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_double
        D = ctypes.POINTER(DeviceDesc)
        O = ctypes.POINTER(PairOpts)
        lib.rm_occupancy.argtypes = [D, i64, P, P, P, P, P, P, P, P, P, P, P]
        lib.rm_occupancy.restype = ctypes.c_int
        lib.rm_pair_workspace_bytes.argtypes = [i32, i64, O]
        lib.rm_pair_workspace_bytes.restype = ctypes.c_size_t
        lib.rm_pair_slowdown_matrix.argtypes = [D, i32, P, i64, P, P, P, P, P, O, P, P, P, P, P,
                                                P, ctypes.c_size_t, P, P]
        lib.rm_pair_slowdown_matrix.restype = ctypes.c_int
        lib.rm_pair_slowdown_matrix_static.argtypes = [D, i32, P, i64, P, P, P, P, P, O, P, P, P,
                                                       P, P, P, P]
        lib.rm_pair_slowdown_matrix_static.restype = ctypes.c_int
        lib.rm_aggregate_greedy.argtypes = [i32, P, P, P, i32, P, P, i32, P, P, P, P]
        lib.rm_aggregate_greedy.restype = ctypes.c_int
        lib.rm_place.argtypes = [i32, P, P, P, i32, i32, P, P, i32, P, f64, i32, P, P, P, P]
        lib.rm_place.restype = ctypes.c_int
        lib.rm_place_optimal_workspace_bytes.argtypes = [i32, i32, i32]
        lib.rm_place_optimal_workspace_bytes.restype = ctypes.c_size_t
        lib.rm_place_optimal.argtypes = [i32, P, P, P, i32, P, i32, i32, i32, P, P, P,
                                         ctypes.c_size_t, P, P]
        lib.rm_place_optimal.restype = ctypes.c_int
        f32, sz = ctypes.c_float, ctypes.c_size_t
        C, S = ctypes.POINTER(Cache), ctypes.POINTER(Sequences)
        lib.rm_w4_linear_workspace_bytes.argtypes = [i32, i32, i32, i32]
        lib.rm_w4_linear_workspace_bytes.restype = sz
        lib.rm_w4_linear.argtypes = [i32, i32, i32, i32, P, i64, P, i64, i32, P, P, P, i32, P,
                                     i64, P, sz, P]
        lib.rm_rotary_append.argtypes = [i32, C, S, i32, P, i64, i64, P, i64, i64, P, i64, i64, P,
                                         P, i32, i32, f32, P, P, P]
        lib.rm_cache_read.argtypes = [i32, C, i32, P, P, P, P, P]
        lib.rm_cache_attention_workspace_bytes.argtypes = [C, S, i32]
        lib.rm_cache_attention_workspace_bytes.restype = sz
        lib.rm_cache_attention.argtypes = [i32, C, S, i32, P, i64, i64, f32, i32, P, P, sz, P, P]
        lib.rm_norm_residual.argtypes = [i32, i32, i32, i32, P, i64, P, i64, P, i64, i32, P, P, P,
                                         f32, f32, P, P, P]
        lib.rm_trace_begin.argtypes = [ctypes.POINTER(Launch), i32]
        lib.rm_trace_begin_timed.argtypes = [ctypes.POINTER(Launch), ctypes.POINTER(f32), i32]
        lib.rm_trace_end.argtypes = [ctypes.POINTER(i32)]
        for f in (lib.rm_w4_linear, lib.rm_rotary_append, lib.rm_cache_read,
                  lib.rm_cache_attention, lib.rm_norm_residual, lib.rm_trace_begin,
                  lib.rm_trace_begin_timed, lib.rm_trace_end):
            f.restype = ctypes.c_int
        lib.rm_status_string.argtypes = [ctypes.c_int]
        lib.rm_status_string.restype = ctypes.c_char_p
        _lib = lib
    return _lib


def rm_status_string(code: int) -> str:
    return library().rm_status_string(int(code)).decode()


def _check(code: int, what: str):
    if code != RM_OK:
        raise RuntimeError(f"{what}: {rm_status_string(code)} (code {code})")


def _ptr(t):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError("expected a GPU tensor")
    if not t.is_contiguous():
        raise ValueError("expected a contiguous tensor")
    return ctypes.c_void_p(t.data_ptr())


def _want(t, dtype, n=None, name="tensor"):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name}: expected a GPU tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name}: expected {dtype}, got {t.dtype}")
    if n is not None and t.numel() != n:
        raise ValueError(f"{name}: expected {n} elements, got {t.numel()}")
    return t


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _empty(n, dtype, device):
    return torch.empty(n, dtype=dtype, device=device)


def new_status(device="cuda"):
    return torch.zeros(1, dtype=torch.int32, device=device)


def library_to_device(lib_np, device="cuda"):
    """Copy a numpy kernel-trace library (see workloads.py) to GPU tensors."""
    dt = {"offsets": torch.int64, "grid": torch.int32, "threads": torch.int32,
          "regs": torch.int32, "smem": torch.int32, "duration": torch.float64}
    return {k: torch.as_tensor(lib_np[k]).to(device=device, dtype=dt[k]).contiguous()
            for k in dt}


def rm_occupancy(dev, grid, threads, regs, smem, status=None, out=None):
    """Per-kernel b, beta, a, limiter and o (Sec. 3.1, Eq. 1)."""
    n = grid.numel()
    for name, t in (("grid", grid), ("threads", threads), ("regs", regs), ("smem", smem)):
        _want(t, torch.int32, n, name)
    d = grid.device
    if out is None:
        out = {k: _empty(n, torch.int32, d) for k in
               ("blocks_per_sm", "resident_blocks", "active_warps", "limiter")}
        out["occupancy"] = _empty(n, torch.float64, d)
    code = library().rm_occupancy(
        ctypes.byref(DeviceDesc.of(dev)), n, _ptr(grid), _ptr(threads), _ptr(regs), _ptr(smem),
        _ptr(out["blocks_per_sm"]), _ptr(out["resident_blocks"]), _ptr(out["active_warps"]),
        _ptr(out["limiter"]), _ptr(out["occupancy"]), _ptr(status), _stream())
    _check(code, "rm_occupancy")
    return out


def pair_opts(align_mode=ALIGN_FIRST, reduce_mode=REDUCE_MEDIAN, num_offsets=1,
              max_kernels_per_model=0, events=None, sweep_mode=SWEEP_TEMPORAL,
              start_draws=None, policy=POLICY_EQUAL):
    o = PairOpts()
    o.policy = POLICY_NAMES.get(policy, policy)
    o.align_mode = ALIGN_NAMES.get(align_mode, align_mode)
    o.reduce_mode = REDUCE_NAMES.get(reduce_mode, reduce_mode)
    o.sweep_mode = SWEEP_NAMES.get(sweep_mode, sweep_mode)
    o.num_offsets = int(num_offsets)
    o.max_kernels_per_model = int(max_kernels_per_model)
    if events is not None:
        if not events[0].cuda_event or not events[1].cuda_event:
            raise ValueError("timing events must have been recorded once (torch creates the "
                             "HIP event lazily)")
        o.sweep_event_begin = ctypes.c_void_p(events[0].cuda_event)
        o.sweep_event_end = ctypes.c_void_p(events[1].cuda_event)
    if start_draws is not None:
        _want(start_draws, torch.uint64, None, "start_draws")
        o.start_draws = _ptr(start_draws)
    return o


def rm_pair_workspace_bytes(n_models, n_kernels, opts) -> int:
    return int(library().rm_pair_workspace_bytes(int(n_models), int(n_kernels),
                                                 ctypes.byref(opts)))


def rm_pair_slowdown_matrix(dev, kernel_offsets, grid, threads, regs, smem, duration,
                            align_mode=ALIGN_FIRST, reduce_mode=REDUCE_MEDIAN, num_offsets=1,
                            max_kernels_per_model=0, per_alignment=False, workspace=None,
                            out=None, status=None, events=None, sweep_mode=SWEEP_TEMPORAL,
                            start_draws=None, policy=POLICY_EQUAL):
    """Ordered N x N delay and slowdown matrices (Alg. 1 on every pair).

    `sweep_mode` selects Alg. 1's temporal sweep or the Sec. 3.2
    adjusted-occupancy simulation.  `start_draws` (SAMPLED_STARTS): a uint64
    GPU tensor of num_offsets draws per unordered pair, row-major pairs.  `events` = (begin, end) torch.cuda.Event
    pair recorded around the sweep kernel.  `out` may hold preallocated
    "delay", "slowdown", "iso_time", "kernel_count" (and "per_alignment")
    tensors.
    """
    N = kernel_offsets.numel() - 1
    nk = grid.numel()
    _want(kernel_offsets, torch.int64, N + 1, "kernel_offsets")
    for name, t in (("grid", grid), ("threads", threads), ("regs", regs), ("smem", smem)):
        _want(t, torch.int32, nk, name)
    _want(duration, torch.float64, nk, "duration")
    o = pair_opts(align_mode, reduce_mode, num_offsets, max_kernels_per_model, events,
                  sweep_mode, start_draws, policy)
    if o.align_mode == ALIGN_SAMPLED_STARTS:
        if start_draws is None:
            raise ValueError("rm_pair_slowdown_matrix: SAMPLED_STARTS needs start_draws")
        _want(start_draws, torch.uint64, N * (N + 1) // 2 * o.num_offsets, "start_draws")
    d = grid.device
    need = rm_pair_workspace_bytes(N, nk, o)
    if need == 0:
        raise ValueError("rm_pair_slowdown_matrix: invalid sizes or options")
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(need, dtype=torch.uint8, device=d)
    if out is None:
        out = _pair_outputs(N, nk, o, per_alignment, d)
    code = library().rm_pair_slowdown_matrix(
        ctypes.byref(DeviceDesc.of(dev)), N, _ptr(kernel_offsets), nk, _ptr(grid), _ptr(threads),
        _ptr(regs), _ptr(smem), _ptr(duration), ctypes.byref(o), _ptr(out["delay"]),
        _ptr(out.get("slowdown")), _ptr(out.get("per_alignment")), _ptr(out["iso_time"]),
        _ptr(out["kernel_count"]), _ptr(workspace), workspace.numel(), _ptr(status), _stream())
    _check(code, "rm_pair_slowdown_matrix")
    out["workspace"] = workspace
    return out


def rm_pair_slowdown_matrix_static(dev, kernel_offsets, grid, threads, regs, smem, duration,
                                   align_mode=ALIGN_FIRST, reduce_mode=REDUCE_MEDIAN,
                                   num_offsets=1, max_kernels_per_model=0, per_alignment=False,
                                   out=None, status=None, events=None,
                                   sweep_mode=SWEEP_TEMPORAL, start_draws=None,
                                   policy=POLICY_EQUAL):
    """rm_pair_slowdown_matrix with the library's static scratch instead of a
    workspace (for callers that cannot allocate device memory).  `out` may
    hold preallocated outputs as for rm_pair_slowdown_matrix; otherwise they
    are allocated here, before the call."""
    N = kernel_offsets.numel() - 1
    nk = grid.numel()
    _want(kernel_offsets, torch.int64, N + 1, "kernel_offsets")
    for name, t in (("grid", grid), ("threads", threads), ("regs", regs), ("smem", smem)):
        _want(t, torch.int32, nk, name)
    _want(duration, torch.float64, nk, "duration")
    o = pair_opts(align_mode, reduce_mode, num_offsets, max_kernels_per_model, events,
                  sweep_mode, start_draws, policy)
    if o.align_mode == ALIGN_SAMPLED_STARTS:
        if start_draws is None:
            raise ValueError("rm_pair_slowdown_matrix_static: SAMPLED_STARTS needs start_draws")
        _want(start_draws, torch.uint64, N * (N + 1) // 2 * o.num_offsets, "start_draws")
    d = grid.device
    if out is None:
        out = _pair_outputs(N, nk, o, per_alignment, d)
    code = library().rm_pair_slowdown_matrix_static(
        ctypes.byref(DeviceDesc.of(dev)), N, _ptr(kernel_offsets), nk, _ptr(grid), _ptr(threads),
        _ptr(regs), _ptr(smem), _ptr(duration), ctypes.byref(o), _ptr(out["delay"]),
        _ptr(out.get("slowdown")), _ptr(out.get("per_alignment")), _ptr(out["iso_time"]),
        _ptr(out["kernel_count"]), _ptr(status), _stream())
    _check(code, "rm_pair_slowdown_matrix_static")
    return out


def _pair_outputs(N, nk, o, per_alignment, d):
    out = {"delay": _empty(N * N, torch.float64, d), "slowdown": _empty(N * N, torch.float64, d),
           "iso_time": _empty(N, torch.float64, d), "kernel_count": _empty(N, torch.int32, d)}
    if per_alignment:
        if o.align_mode == ALIGN_CONFLICT_STARTS:
            size = nk * nk
        elif o.align_mode in (ALIGN_OFFSETS, ALIGN_SAMPLED_STARTS):
            size = N * N * o.num_offsets
        else:
            size = N * N
        out["per_alignment"] = _empty(size, torch.float64, d)
    return out


def rm_aggregate_greedy(delay, iso_time, kernel_count, set_offsets, set_members,
                        drop_mode=DROP_ISO, status=None, out=None):
    """Per-member drop and per-set mean drop (Alg. 1, Eq. 5)."""
    N = iso_time.numel()
    _want(delay, torch.float64, N * N, "delay")
    _want(kernel_count, torch.int32, N, "kernel_count")
    _want(set_offsets, torch.int32, None, "set_offsets")
    _want(set_members, torch.int32, None, "set_members")
    n_sets = set_offsets.numel() - 1
    d = delay.device
    if out is None:
        out = {"mu": _empty(max(set_members.numel(), 1), torch.float64, d),
               "mu_mean": _empty(max(n_sets, 1), torch.float64, d)}
    code = library().rm_aggregate_greedy(
        N, _ptr(delay), _ptr(iso_time), _ptr(kernel_count), n_sets, _ptr(set_offsets),
        _ptr(set_members), int(drop_mode), _ptr(out["mu"]), _ptr(out["mu_mean"]), _ptr(status),
        _stream())
    _check(code, "rm_aggregate_greedy")
    return out


def rm_place(delay, iso_time, kernel_count, n_devices, capacity, events, lam,
             drop_mode=DROP_ISO, resident=None, resident_count=None, status=None, out=None):
    """Alg. 2 over an event stream; `resident`/`resident_count` are updated in place."""
    N = iso_time.numel()
    _want(delay, torch.float64, N * N, "delay")
    _want(kernel_count, torch.int32, N, "kernel_count")
    _want(events, torch.int32, None, "events")
    d = delay.device
    if resident is None:
        resident = torch.full((n_devices * capacity,), -1, dtype=torch.int32, device=d)
    if resident_count is None:
        resident_count = torch.zeros(n_devices, dtype=torch.int32, device=d)
    _want(resident, torch.int32, n_devices * capacity, "resident")
    _want(resident_count, torch.int32, n_devices, "resident_count")
    E = events.numel()
    if out is None:
        out = {"placed_device": _empty(max(E, 1), torch.int32, d),
               "placed_mu_mean": _empty(max(E, 1), torch.float64, d)}
    code = library().rm_place(
        N, _ptr(delay), _ptr(iso_time), _ptr(kernel_count), int(n_devices), int(capacity),
        _ptr(resident), _ptr(resident_count), E, _ptr(events), float(lam), int(drop_mode),
        _ptr(out["placed_device"]), _ptr(out["placed_mu_mean"]), _ptr(status), _stream())
    _check(code, "rm_place")
    out["resident"] = resident
    out["resident_count"] = resident_count
    return out


def rm_place_optimal_workspace_bytes(n_place, n_devices, capacity) -> int:
    return int(library().rm_place_optimal_workspace_bytes(int(n_place), int(n_devices),
                                                          int(capacity)))


def rm_place_optimal(delay, iso_time, kernel_count, models, n_devices, capacity,
                     drop_mode=DROP_ISO, workspace=None, status=None, out=None):
    """Smallest mean drop over every placement of `models` (Sec. 6.4 accuracy
    baseline) and one placement attaining it."""
    N = iso_time.numel()
    _want(delay, torch.float64, N * N, "delay")
    _want(kernel_count, torch.int32, N, "kernel_count")
    _want(models, torch.int32, None, "models")
    n = models.numel()
    d = delay.device
    need = rm_place_optimal_workspace_bytes(n, n_devices, capacity)
    if need == 0:
        raise ValueError("rm_place_optimal: sizes outside the limits")
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(need, dtype=torch.uint8, device=d)
    if out is None:
        out = {"best_mean": _empty(1, torch.float64, d),
               "best_device": _empty(max(n, 1), torch.int32, d)}
    code = library().rm_place_optimal(
        N, _ptr(delay), _ptr(iso_time), _ptr(kernel_count), n, _ptr(models), int(n_devices),
        int(capacity), int(drop_mode), _ptr(out["best_mean"]), _ptr(out["best_device"]),
        _ptr(workspace), workspace.numel(), _ptr(status), _stream())
    _check(code, "rm_place_optimal")
    out["workspace"] = workspace
    return out


# ---- kernels of a decode layer ---------------------------------------------

# These run before every launch of a few microseconds, so they are written for
# the accepted case: one expression, the message only where it fails.

def _on_gpu(t, dtype, shape, gpu, name):
    """Address of a contiguous tensor of this type and shape on this GPU; None for None."""
    if t is None:
        return None
    if t.get_device() == gpu and t.dtype is dtype and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    raise ValueError(f"{name}: expected a contiguous tensor of {dtype} and shape {tuple(shape)} "
                     f"on cuda:{gpu}, got {t.dtype} {tuple(t.shape)} on {t.device}")


def _rows(t, dtype, shape, gpu, name):
    """Strides of a tensor on this GPU whose last axis is consecutive."""
    if t.get_device() == gpu and t.dtype is dtype and t.shape == shape:
        strides = t.stride()
        if strides[-1] == 1 or shape[-1] <= 1:
            return strides
        raise ValueError(f"{name}: the last axis must be consecutive")
    raise ValueError(f"{name}: expected a tensor of {dtype} and shape {tuple(shape)} on "
                     f"cuda:{gpu}, got {t.dtype} {tuple(t.shape)} on {t.device}")


def _scratch(t, gpu):
    """Address and bytes of a caller's workspace."""
    if t.get_device() == gpu and t.is_contiguous():
        return t.data_ptr(), t.numel() * t.element_size()
    raise ValueError(f"workspace: expected a contiguous tensor on cuda:{gpu}, got strides "
                     f"{t.stride()} on {t.device}")


def _pitch(stride, rows, width, name):
    """Elements between rows; rows may not overlap."""
    if rows <= 1:
        return width
    if stride < width:
        raise ValueError(f"{name}: rows overlap")
    return stride


def _type_of(t, name):
    """The type's code and the GPU that all tensors of the call have to be on."""
    code, gpu = TYPES.get(t.dtype), t.get_device()
    if code is None or gpu < 0:
        raise ValueError(f"{name}: expected a GPU tensor of bfloat16 or float16, got {t.dtype} "
                         f"on {t.device}")
    return code, gpu


def _named(names, value, what):
    code = names.get(value)
    if code is None:
        raise ValueError(f"{what}: expected one of {sorted(names)}, got {value!r}")
    return code


# ctypes takes the low 32 bits of a larger number without a word.

def _too_large(name, *values):
    raise ValueError(f"{name}: {values} beyond 31 bits")


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_gpu = getattr(torch._C, "_cuda_getDevice", None)


# A call runs on the current stream of its tensors' GPU, which has to be the current
# GPU for it: a default stream's handle is 0 on every GPU.


def new_cache(n_pages, kv_heads, page_tokens, head_dim, codes=torch.int8, device="cuda"):
    """An empty paged 8-bit cache: codes int8 or float8_e4m3fn, one float32
    scale for each page of tokens and head (include/roomie.h, rm_cache)."""
    if codes not in CODES:
        raise ValueError(f"codes: expected int8 or float8_e4m3fn, got {codes}")
    shape = (n_pages, kv_heads)
    return {"k": torch.zeros(shape + (page_tokens, head_dim), dtype=torch.uint8,
                             device=device).view(codes),
            "v": torch.zeros(shape + (head_dim, page_tokens), dtype=torch.uint8,
                             device=device).view(codes),
            "k_scale": torch.zeros(shape, dtype=torch.float32, device=device),
            "v_scale": torch.zeros(shape, dtype=torch.float32, device=device)}


def _cache_of(cache, gpu):
    k, v, ks, vs = cache["k"], cache["v"], cache["k_scale"], cache["v_scale"]
    codes = CODES.get(k.dtype)
    if k.dim() != 4 or codes is None:
        raise ValueError("cache: expected codes int8 or float8_e4m3fn [pages, kv_heads, "
                         f"page_tokens, head_dim], got {k.dtype} {tuple(k.shape)}")
    shape = pages, heads, tokens, dim = k.shape
    return Cache(_on_gpu(k, k.dtype, shape, gpu, "cache k"),
                 _on_gpu(v, k.dtype, (pages, heads, dim, tokens), gpu, "cache v"),
                 _on_gpu(ks, torch.float32, (pages, heads), gpu, "cache k_scale"),
                 _on_gpu(vs, torch.float32, (pages, heads), gpu, "cache v_scale"),
                 pages, heads, tokens, dim, codes)


def _sequences_of(table, lengths, token_offsets, n_tokens, max_tokens, gpu):
    if table.dim() != 2:
        raise ValueError("table: expected [sequences, pages]")
    n, pages = shape = table.shape
    if (n | pages | n_tokens) >> 31:
        _too_large("sizes", n, pages, n_tokens)
    if not -1 << 31 <= max_tokens < 1 << 31:
        _too_large("max_tokens", max_tokens)
    return Sequences(_on_gpu(table, torch.int32, shape, gpu, "table"),
                     _on_gpu(lengths, torch.int32, (n,), gpu, "lengths"),
                     _on_gpu(token_offsets, torch.int32, (n + 1,), gpu, "token_offsets"),
                     n, pages, n_tokens, max_tokens)


def rm_w4_linear(x, codes, scales, group, zeros=None, bias=None, act="none", out=None,
                 workspace=None):
    """x [rows, k] through 4-bit weights: codes uint8 [n, ceil(k / 2)] (rows may
    be strided), even elements in the low half; scales [n, ceil(k / group)] of
    x's type; zeros uint8 like scales (None: 8); bias [n].  act "swiglu" takes
    the first half of the outputs as gates of the second."""
    (kind, gpu), dtype = _type_of(x, "x"), x.dtype
    if gpu != _current_gpu():
        with torch.cuda.device(gpu):
            return rm_w4_linear(x, codes, scales, group, zeros, bias, act, out, workspace)
    if x.dim() != 2 or codes.dim() != 2:
        raise ValueError("rm_w4_linear: expected x [rows, k] and codes [n, ceil(k / 2)]")
    rows, k = shape = x.shape
    n = codes.shape[0]
    if group < 1 or group % 32:
        raise ValueError(f"group: expected a multiple of 32, got {group}")
    if (rows | n | k | group) >> 31:
        _too_large("sizes", rows, n, k, group)
    row_bytes = (k + 1) // 2
    groups = (n, -(-k // group))
    act = _named(ACT_NAMES, act, "act")
    width = n // 2 if act else n
    if out is None:
        out = x.new_empty((rows, width))
        out_pitch = width
    else:
        out_pitch = _pitch(_rows(out, dtype, (rows, width), gpu, "out")[0], rows, width, "out")
    x_pitch = _pitch(_rows(x, dtype, shape, gpu, "x")[0], rows, k, "x")
    code_pitch = _pitch(_rows(codes, torch.uint8, (n, row_bytes), gpu, "codes")[0], n, row_bytes,
                        "codes")
    args = (kind, rows, n, k, x.data_ptr(), x_pitch, codes.data_ptr(), code_pitch, group,
            _on_gpu(scales, dtype, groups, gpu, "scales"),
            _on_gpu(zeros, torch.uint8, groups, gpu, "zeros"),
            _on_gpu(bias, dtype, (n,), gpu, "bias"), act, out.data_ptr(), out_pitch)
    lib, stream = _lib or library(), _raw_stream(gpu)
    if workspace is None:
        code = lib.rm_w4_linear(*args, None, 0, stream)
        if code == RM_EWORKSPACE:     # most sizes need none, so it is asked for only then
            workspace = torch.empty(lib.rm_w4_linear_workspace_bytes(rows, n, k, act),
                                    dtype=torch.uint8, device=x.device)
    if workspace is not None:
        code = lib.rm_w4_linear(*args, *_scratch(workspace, gpu), stream)
    if code:
        _check(code, "rm_w4_linear")
    return out


def rm_rotary_append(q, k, v, inv_freq, cache, table, lengths, token_offsets=None, max_tokens=1,
                     positions=None, layout="half", rot_scale=1.0, q_out=None, status=None):
    """Turns q [tokens, heads, dim] and k [tokens, kv_heads, dim] by their
    positions (2 * len(inv_freq) channels of each head, times rot_scale) and
    appends k and v to the cache, whose `lengths` count the call's tokens
    already.  q, k and v may be views of one projection.  Returns the turned
    q (None for q None)."""
    (kind, gpu), dtype = _type_of(k, "k"), k.dtype
    if gpu != _current_gpu():
        with torch.cuda.device(gpu):
            return rm_rotary_append(q, k, v, inv_freq, cache, table, lengths, token_offsets,
                                    max_tokens, positions, layout, rot_scale, q_out, status)
    c = _cache_of(cache, gpu)
    if k.dim() != 3:
        raise ValueError("k: expected [tokens, kv_heads, head_dim]")
    tokens, dim = k.shape[0], c.head_dim
    shape = (tokens, c.kv_heads, dim)
    s = _sequences_of(table, lengths, token_offsets, tokens, max_tokens, gpu)
    ks, vs = _rows(k, dtype, shape, gpu, "k"), _rows(v, dtype, shape, gpu, "v")
    heads, qp, qs, op = 0, None, (0, 0), None
    if q is not None:
        if q.dim() != 3:
            raise ValueError("q: expected [tokens, heads, head_dim]")
        heads = q.shape[1]
        shape = (tokens, heads, dim)
        qs, qp = _rows(q, dtype, shape, gpu, "q"), q.data_ptr()
        if q_out is None:
            q_out = k.new_empty(shape)
            op = q_out.data_ptr()
        else:
            op = _on_gpu(q_out, dtype, shape, gpu, "q_out")
    half = inv_freq.numel()
    code = (_lib or library()).rm_rotary_append(
        kind, c, s, heads, qp, qs[0], qs[1], k.data_ptr(), ks[0], ks[1], v.data_ptr(), vs[0],
        vs[1], _on_gpu(positions, torch.int32, (tokens,), gpu, "positions"),
        _on_gpu(inv_freq, torch.float32, (half,), gpu, "inv_freq"), 2 * half,
        _named(ROTARY_NAMES, layout, "layout"), rot_scale, op,
        _on_gpu(status, torch.int32, (1,), gpu, "status"), _raw_stream(gpu))
    if code:
        _check(code, "rm_rotary_append")
    return q_out


def rm_cache_read(cache, pages, dtype=torch.bfloat16, status=None):
    """Keys and values that `pages` (int32) hold: two tensors [pages,
    page_tokens, kv_heads, head_dim]."""
    gpu = pages.get_device()
    if gpu < 0:
        raise ValueError(f"pages: expected a GPU tensor, got one on {pages.device}")
    if gpu != _current_gpu():
        with torch.cuda.device(gpu):
            return rm_cache_read(cache, pages, dtype, status)
    c = _cache_of(cache, gpu)
    n = pages.numel()
    if n >> 31:
        _too_large("sizes", n)
    kind = TYPES.get(dtype)
    if kind is None:
        raise ValueError(f"dtype: expected bfloat16 or float16, got {dtype}")
    both = torch.empty((2, n, c.page_tokens, c.kv_heads, c.head_dim), dtype=dtype,
                       device=pages.device)
    k, v = both.unbind()
    code = (_lib or library()).rm_cache_read(
        kind, c, n, _on_gpu(pages, torch.int32, (n,), gpu, "pages"), k.data_ptr(), v.data_ptr(),
        _on_gpu(status, torch.int32, (1,), gpu, "status"), _raw_stream(gpu))
    if code:
        _check(code, "rm_cache_read")
    return k, v


def rm_cache_attention(q, cache, table, lengths, token_offsets=None, max_tokens=1, scale=None,
                       window=0, workspace=None, out=None, status=None):
    """Attention of q [tokens, heads, dim] over the cache (causal; `window` > 0
    keeps each token's last `window`).  scale None: 1 / sqrt(dim)."""
    (kind, gpu), dtype = _type_of(q, "q"), q.dtype
    if gpu != _current_gpu():
        with torch.cuda.device(gpu):
            return rm_cache_attention(q, cache, table, lengths, token_offsets, max_tokens, scale,
                                      window, workspace, out, status)
    if not -1 << 31 <= window < 1 << 31:
        _too_large("window", window)
    c = _cache_of(cache, gpu)
    if q.dim() != 3:
        raise ValueError("q: expected [tokens, heads, head_dim]")
    tokens, heads, dim = shape = q.shape
    qs = _rows(q, dtype, (tokens, heads, c.head_dim), gpu, "q")
    s = _sequences_of(table, lengths, token_offsets, tokens, max_tokens, gpu)
    lib = _lib or library()
    if workspace is None:
        need = lib.rm_cache_attention_workspace_bytes(c, s, heads)
        if need == 0:
            raise ValueError("rm_cache_attention: invalid sizes or options")
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
        wp = workspace.data_ptr()
    else:
        wp, need = _scratch(workspace, gpu)
    if out is None:
        out = q.new_empty(shape)
        op = out.data_ptr()
    else:
        op = _on_gpu(out, dtype, shape, gpu, "out")
    code = lib.rm_cache_attention(
        kind, c, s, heads, q.data_ptr(), qs[0], qs[1], dim ** -0.5 if scale is None else scale,
        window, op, wp, need,
        _on_gpu(status, torch.int32, (1,), gpu, "status"), _raw_stream(gpu))
    if code:
        _check(code, "rm_cache_attention")
    return out


def rm_norm_residual(x, y=None, gate=None, post_weight=None, pre_weight=None, pre_bias=None,
                     kind="rms", alpha=1.0, eps=1e-6, x_out=None, n_out=None):
    """(x', n): x' = x + alpha * gate * y, y normalised and times post_weight
    where that is given; n = x' normalised times pre_weight plus pre_bias.
    x, y [rows, width]; gate [width], [rows, 1] or [rows, width].  Without y
    x' is x itself."""
    (code_type, gpu), dtype = _type_of(x, "x"), x.dtype
    if gpu != _current_gpu():
        with torch.cuda.device(gpu):
            return rm_norm_residual(x, y, gate, post_weight, pre_weight, pre_bias, kind, alpha,
                                    eps, x_out, n_out)
    if x.dim() != 2:
        raise ValueError("x: expected [rows, width]")
    rows, width = shape = x.shape
    if (rows | width) >> 31:
        _too_large("sizes", rows, width)
    x_pitch = _pitch(_rows(x, dtype, shape, gpu, "x")[0], rows, width, "x")
    yp, y_pitch = None, 0
    if y is not None:
        y_pitch = _pitch(_rows(y, dtype, shape, gpu, "y")[0], rows, width, "y")
        yp = y.data_ptr()
    gp, gs, gw = None, 0, 0
    if gate is not None:
        if gate.dim() == 1:
            gp, gw = _on_gpu(gate, dtype, (width,), gpu, "gate"), width
        else:
            gw = gate.shape[1]
            gs = _rows(gate, dtype, (rows, gw), gpu, "gate")[0] if rows > 1 else 0
            gp = gate.data_ptr() if rows > 1 else _on_gpu(gate, dtype, (rows, gw), gpu, "gate")
    whole = x.is_contiguous()        # empty_like takes two thirds of new_empty's time
    if x_out is None:
        if y is None:
            x_out, xo = x, None
        else:
            x_out = torch.empty_like(x) if whole else x.new_empty(shape)
            xo = x_out.data_ptr()
    else:
        xo = _on_gpu(x_out, dtype, shape, gpu, "x_out")
    if n_out is None:
        n_out = torch.empty_like(x) if whole else x.new_empty(shape)
        no = n_out.data_ptr()
    else:
        no = _on_gpu(n_out, dtype, shape, gpu, "n_out")
    wide = (width,)
    code = (_lib or library()).rm_norm_residual(
        code_type, _named(NORM_NAMES, kind, "kind"), rows, width, x.data_ptr(), x_pitch, yp,
        y_pitch, gp, gs, gw, _on_gpu(post_weight, dtype, wide, gpu, "post_weight"),
        _on_gpu(pre_weight, dtype, wide, gpu, "pre_weight"),
        _on_gpu(pre_bias, dtype, wide, gpu, "pre_bias"), alpha, eps, xo, no, _raw_stream(gpu))
    if code:
        _check(code, "rm_norm_residual")
    return x_out, n_out


class rm_trace:
    """Context manager: the launch shapes of the decode-layer calls inside it,
    as a list of dicts `launches` (grid, threads, regs, smem) after it; `timed`
    adds `duration`, the microseconds that each launch took on the GPU (the end
    of the block then waits for them; not for graphs in capture)."""

    def __init__(self, capacity=4096, timed=False):
        self._records = (Launch * capacity)()
        self._times = (ctypes.c_float * capacity)() if timed else None
        self.launches = []

    def __enter__(self):
        n = len(self._records)
        if self._times is None:
            _check(library().rm_trace_begin(self._records, n), "rm_trace_begin")
        else:
            _check(library().rm_trace_begin_timed(self._records, self._times, n),
                   "rm_trace_begin_timed")
        return self

    def __exit__(self, *exc):
        n = ctypes.c_int32()
        _check(library().rm_trace_end(ctypes.byref(n)), "rm_trace_end")
        if n.value > len(self._records) and exc[0] is None:
            raise RuntimeError(f"rm_trace: {n.value} launches, room for {len(self._records)}")
        self.launches = [{f: getattr(r, f) for f, _ in Launch._fields_}
                         for r in self._records[:min(n.value, len(self._records))]]
        for i, launch in enumerate(self.launches if self._times is not None else ()):
            launch["duration"] = self._times[i]
        return False
