"""ctypes binding of ``libkimad.so`` (C ABI in ``include/kimad.h``), same names as the C calls.

Argument marshalling only: every step of the compression pass runs in the CUDA library.  PyTorch
appears here for device memory and streams.  There is no CPU fallback: if the library is missing
the import of a symbol fails loudly.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

from . import build as _build

KIMAD_OK = 0
KIMAD_STATUS_INFEASIBLE = 1
KIMAD_STATUS_PLATEAU = 2
KIMAD_ERR_INVALID_ARG = -1
KIMAD_ERR_WORKSPACE = -2
KIMAD_ERR_CAPACITY = -3
KIMAD_ERR_NONFINITE = -4
KIMAD_ERR_TIMEOUT = -5
KIMAD_ERR_CUDA = -6
KIMAD_ERR_NOMEM = -7
KIMAD_ERR_TOO_LARGE = -8
KIMAD_BUILTIN_SCRATCH_BYTES = 32 << 20


class kimad_options(C.Structure):
    _fields_ = [("D", C.c_uint32), ("value_dtype", C.c_uint32), ("check_finite", C.c_uint32),
                ("infeasible_policy", C.c_uint32), ("max_packed_elems", C.c_uint64), ("worker_stride", C.c_uint64),
                ("curve_mode", C.c_uint32), ("policy", C.c_uint32), ("cost_model", C.c_uint32)]


class kimad_stats(C.Structure):
    _fields_ = [("budget_bytes", C.c_uint64), ("used_bytes", C.c_uint64), ("n_selected", C.c_uint64),
                ("total_err", C.c_float), ("status", C.c_int32)]


class kimad_packed(C.Structure):
    _fields_ = [("idx", C.c_void_p), ("val", C.c_void_p), ("offs", C.c_void_p), ("k", C.c_void_p),
                ("j", C.c_void_p), ("stats", C.c_void_p), ("dense", C.c_void_p)]


class kimad_mx4_message(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p), ("err", C.c_void_p), ("stats", C.c_void_p)]


KIMAD_F32, KIMAD_BF16, KIMAD_F16 = 0, 1, 2

STATS_DTYPE = np.dtype([("budget_bytes", "<u8"), ("used_bytes", "<u8"), ("n_selected", "<u8"),
                        ("total_err", "<f4"), ("status", "<i4")])

_lib = None


class KimadError(RuntimeError):
    def __init__(self, code, what):
        self.code = code
        super().__init__(f"{what}: {kimad_strerror(code)} ({code})")


def lib_path() -> str:
    """The ordinary build, or the checked build when the environment has KIMAD_CHECKED=1."""
    return _build.CHECKED_LIB_PATH if os.environ.get("KIMAD_CHECKED") == "1" else _build.LIB_PATH


def load():
    """Loads the compiled library; raises if it has not been built (no fallback path exists)."""
    global _lib
    if _lib is not None:
        return _lib
    path = lib_path()
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -m paper_2312_08053_b200.build` "
                           "(nvcc, sm_100a); there is no fallback implementation")
    L = C.CDLL(path)
    vp, u32, u64, dbl = C.c_void_p, C.c_uint32, C.c_uint64, C.c_double
    L.kimad_create.restype = C.c_int
    L.kimad_create.argtypes = [C.POINTER(vp), C.POINTER(u64), u32, u32, C.POINTER(dbl), u32,
                               C.POINTER(kimad_options)]
    L.kimad_destroy.restype = None
    L.kimad_destroy.argtypes = [vp]
    L.kimad_workspace_bytes.restype = C.c_size_t
    L.kimad_workspace_bytes.argtypes = [vp]
    L.kimad_set_workspace.restype = C.c_int
    L.kimad_set_workspace.argtypes = [vp, vp, C.c_size_t]
    step_args = [vp, vp, vp, C.POINTER(dbl), dbl, C.POINTER(kimad_packed), vp]
    L.kimad_step.restype = C.c_int
    L.kimad_step.argtypes = step_args
    L.kimad_step_builtin_scratch.restype = C.c_int
    L.kimad_step_builtin_scratch.argtypes = step_args
    L.kimad_debug_step_with_err.restype = C.c_int
    L.kimad_debug_step_with_err.argtypes = step_args + [vp]
    L.kimad_debug_step_with_j.restype = C.c_int
    L.kimad_debug_step_with_j.argtypes = step_args + [vp]
    L.kimad_apply_packed.restype = C.c_int
    L.kimad_apply_packed.argtypes = [vp, C.POINTER(kimad_packed), vp, vp]
    L.kimad_aggregate.restype = C.c_int
    L.kimad_aggregate.argtypes = [vp, vp, u64, u32, u64, C.POINTER(C.c_float), C.c_float, vp]
    L.kimad_get_k.restype = C.c_int
    L.kimad_get_k.argtypes = [vp, vp, vp]
    L.kimad_get_k_table.restype = C.c_int
    L.kimad_get_k_table.argtypes = [vp, vp]
    L.kimad_plan_budget.restype = C.c_int
    L.kimad_plan_budget.argtypes = [vp, dbl, dbl, C.POINTER(u64), vp]
    L.kimad_debug_get_curve.restype = C.c_int
    L.kimad_debug_get_curve.argtypes = [vp, vp, vp, vp, vp]
    L.kimad_debug_get_selection.restype = C.c_int
    L.kimad_debug_get_selection.argtypes = [vp, vp, vp]
    L.kimad_debug_enable_stage_timing.restype = C.c_int
    L.kimad_debug_enable_stage_timing.argtypes = [vp, C.c_int]
    L.kimad_debug_stage_times.restype = C.c_int
    L.kimad_debug_stage_times.argtypes = [vp, vp]
    L.kimad_debug_set_schedule.restype = C.c_int
    L.kimad_debug_set_schedule.argtypes = [vp, C.c_int]
    L.kimad_debug_set_search.restype = C.c_int
    L.kimad_debug_set_search.argtypes = [vp, C.c_int]
    L.kimad_debug_searches.restype = C.c_int
    L.kimad_debug_searches.argtypes = [vp, C.POINTER(u64)]
    L.kimad_debug_set_wait_limit.restype = C.c_int
    L.kimad_debug_set_wait_limit.argtypes = [vp, u64]
    L.kimad_debug_trace_step.restype = C.c_int
    L.kimad_debug_trace_step.argtypes = [vp, vp, vp, C.POINTER(dbl), dbl, vp, vp, C.c_char_p, C.c_size_t]
    L.kimad_debug_get_band_meta.restype = C.c_int
    L.kimad_debug_get_band_meta.argtypes = [vp, vp]
    L.kimad_debug_exact_path_layers.restype = C.c_int
    L.kimad_debug_exact_path_layers.argtypes = [vp, C.POINTER(u64)]
    L.kimad_debug_check.restype = C.c_int
    L.kimad_debug_check.argtypes = [vp, C.POINTER(u32), C.POINTER(u32)]
    L.kimad_launch_count.restype = u64
    L.kimad_launch_count.argtypes = [vp]
    L.kimad_mx4_message_bytes.restype = C.c_int
    L.kimad_mx4_message_bytes.argtypes = [vp, C.POINTER(u64), C.POINTER(u64)]
    L.kimad_mx4_step.restype = C.c_int
    L.kimad_mx4_step.argtypes = [vp, vp, u32, vp, C.POINTER(kimad_mx4_message), vp]
    L.kimad_mx4_apply.restype = C.c_int
    L.kimad_mx4_apply.argtypes = [vp, C.POINTER(kimad_mx4_message), vp, vp, C.POINTER(C.c_float), C.c_float, vp]
    L.kimad_mx4_read.restype = C.c_int
    L.kimad_mx4_read.argtypes = [vp, C.POINTER(kimad_mx4_message), vp, u32, vp]
    L.kimad_mx4_operand_bytes.restype = C.c_int
    L.kimad_mx4_operand_bytes.argtypes = [u64, u64, C.POINTER(u64), C.POINTER(u64)]
    L.kimad_mx4_quantize.restype = C.c_int
    L.kimad_mx4_quantize.argtypes = [vp, u32, u64, u64, u64, u64, u64, u32, vp, vp, vp]
    L.kimad_mx4_dequantize.restype = C.c_int
    L.kimad_mx4_dequantize.argtypes = [vp, vp, vp, u32, u64, u64, u64, u64, u64, u32, vp]
    L.kimad_debug_mx4_set_wait_limit.restype = C.c_int
    L.kimad_debug_mx4_set_wait_limit.argtypes = [u64, C.c_int]
    L.kimad_mx4_product.restype = C.c_int
    L.kimad_mx4_product.argtypes = [vp] + [u64] * 6 + [vp] * 4 + [C.c_float, C.c_float, vp, vp]
    L.kimad_mx4_product_status.restype = C.c_int
    L.kimad_mx4_product_status.argtypes = [C.c_int, vp]
    L.kimad_monitor_create.restype = C.c_int
    L.kimad_monitor_create.argtypes = [C.POINTER(vp), u32, dbl]
    L.kimad_monitor_destroy.restype = None
    L.kimad_monitor_destroy.argtypes = [vp]
    L.kimad_monitor_observe.restype = C.c_int
    L.kimad_monitor_observe.argtypes = [vp, u64, dbl]
    L.kimad_monitor_estimate.restype = dbl
    L.kimad_monitor_estimate.argtypes = [vp]
    L.kimad_strerror.restype = C.c_char_p
    L.kimad_strerror.argtypes = [C.c_int]
    _lib = L
    return L


def kimad_strerror(code: int) -> str:
    return load().kimad_strerror(int(code)).decode()


def _check(code, what):
    if code < 0:
        raise KimadError(code, what)
    return code


class Ctx:
    """Owning handle of a ``kimad_ctx*`` plus the shapes needed to size buffers."""

    def __init__(self, handle, L, W, K, N, opts: kimad_options):
        self.handle, self.L, self.W, self.K, self.N = handle, L, W, K, N
        self.D = opts.D or 1000
        self.value_dtype = opts.value_dtype
        self.cap = opts.max_packed_elems or N
        self.stride = opts.worker_stride or N
        self.layer_sizes = b""  # u64 [L], as bytes
        self._keep = []  # tensors the context points into (workspace)

    def __del__(self):
        h, self.handle = getattr(self, "handle", None), None
        if h and _lib is not None:
            _lib.kimad_destroy(h)


def kimad_create(layer_sizes, n_workers, ratio_grid, D=0, value_dtype=0, check_finite=0, max_packed_elems=0,
                 worker_stride=0, curve_mode=0, policy=0, cost_model=0) -> Ctx:
    ls = np.ascontiguousarray(layer_sizes, dtype=np.uint64)
    rg = np.ascontiguousarray(ratio_grid, dtype=np.float64)
    opts = kimad_options(D, value_dtype, check_finite, 0, max_packed_elems, worker_stride, curve_mode, policy, cost_model)
    h = C.c_void_p()
    _check(load().kimad_create(C.byref(h), ls.ctypes.data_as(C.POINTER(C.c_uint64)), ls.size, n_workers,
                               rg.ctypes.data_as(C.POINTER(C.c_double)), rg.size, C.byref(opts)), "kimad_create")
    ctx = Ctx(h, int(ls.size), int(n_workers), int(rg.size), int(ls.sum()), opts)
    ctx.layer_sizes = ls.tobytes()
    return ctx


def kimad_destroy(ctx: Ctx) -> None:
    h, ctx.handle = ctx.handle, None
    if h:
        load().kimad_destroy(h)


def kimad_workspace_bytes(ctx: Ctx) -> int:
    return int(load().kimad_workspace_bytes(ctx.handle))


def kimad_set_workspace(ctx: Ctx, workspace) -> None:
    """``workspace``: a CUDA uint8 tensor of at least kimad_workspace_bytes(ctx) bytes (kept alive by ctx)."""
    _check(load().kimad_set_workspace(ctx.handle, workspace.data_ptr(), workspace.numel() * workspace.element_size()),
           "kimad_set_workspace")
    ctx._keep = [workspace]


class Packed:
    """Device output buffers of one step (torch tensors) and the matching ``kimad_packed`` struct."""

    def __init__(self, ctx: Ctx, device="cuda"):
        import torch

        W, L, cap = ctx.W, ctx.L, ctx.cap
        self.idx = torch.zeros((W, cap), dtype=torch.int32, device=device)
        self.val = torch.zeros((W, cap), dtype=torch.float32 if ctx.value_dtype == 0 else torch.bfloat16, device=device)
        self.offs = torch.zeros((W, L + 1), dtype=torch.int64, device=device)
        self.k = torch.zeros((W, L), dtype=torch.int32, device=device)
        self.j = torch.zeros((W, L), dtype=torch.int32, device=device)
        self.stats = torch.zeros((W, STATS_DTYPE.itemsize), dtype=torch.uint8, device=device)
        self.dense = torch.zeros((W, L), dtype=torch.int32, device=device)
        self.c = kimad_packed(self.idx.data_ptr(), self.val.data_ptr(), self.offs.data_ptr(), self.k.data_ptr(),
                              self.j.data_ptr(), self.stats.data_ptr(), self.dense.data_ptr())

    def stats_host(self) -> np.ndarray:
        return self.stats.cpu().numpy().view(STATS_DTYPE).reshape(-1)


def _stream_ptr(stream):
    if stream is None:
        import torch

        return torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def kimad_apply_packed(ctx: Ctx, msg: "Packed", est, stream=None) -> int:
    """est: CUDA float32 tensor [W][ctx.stride], the receiver's copies of the senders' estimators (in place)."""
    return _check(load().kimad_apply_packed(ctx.handle, C.byref(msg.c), est.data_ptr(), _stream_ptr(stream)),
                  "kimad_apply_packed")


def kimad_aggregate(x, est, weights, gamma, stream=None) -> int:
    """x: CUDA float32 [n] (in place); est: CUDA float32 [W][stride]; weights: W host floats."""
    w = np.ascontiguousarray(weights, dtype=np.float32)
    return _check(load().kimad_aggregate(x.data_ptr(), est.data_ptr(), est.stride(0), w.size, x.numel(),
                                         w.ctypes.data_as(C.POINTER(C.c_float)), C.c_float(gamma),
                                         _stream_ptr(stream)), "kimad_aggregate")


def _bw(ctx, bandwidth):
    bw = np.ascontiguousarray(bandwidth, dtype=np.float64).reshape(-1)
    assert bw.size == ctx.W, "one bandwidth per worker"
    return bw


def kimad_step(ctx: Ctx, grads, state, bandwidth_bytes_per_s, t_target_s, out: Packed, stream=None) -> None:
    bw = _bw(ctx, bandwidth_bytes_per_s)
    _check(load().kimad_step(ctx.handle, grads.data_ptr(), state.data_ptr(), bw.ctypes.data_as(C.POINTER(C.c_double)),
                             float(t_target_s), C.byref(out.c), _stream_ptr(stream)), "kimad_step")


def kimad_step_builtin_scratch(ctx: Ctx, grads, state, bandwidth_bytes_per_s, t_target_s, out: Packed, stream=None) -> None:
    """kimad_step with the scratch in the library's built-in device array: for callers that cannot allocate
    device memory.  No workspace has to be attached to ``ctx``; raises KimadError(KIMAD_ERR_TOO_LARGE) when the
    context needs more than KIMAD_BUILTIN_SCRATCH_BYTES."""
    bw = _bw(ctx, bandwidth_bytes_per_s)
    _check(load().kimad_step_builtin_scratch(ctx.handle, grads.data_ptr(), state.data_ptr(),
                                             bw.ctypes.data_as(C.POINTER(C.c_double)), float(t_target_s),
                                             C.byref(out.c), _stream_ptr(stream)), "kimad_step_builtin_scratch")


def kimad_debug_step_with_err(ctx: Ctx, grads, state, bandwidth_bytes_per_s, t_target_s, out: Packed, err_dev,
                              stream=None) -> None:
    bw = _bw(ctx, bandwidth_bytes_per_s)
    _check(load().kimad_debug_step_with_err(ctx.handle, grads.data_ptr(), state.data_ptr(),
                                            bw.ctypes.data_as(C.POINTER(C.c_double)), float(t_target_s),
                                            C.byref(out.c), _stream_ptr(stream), err_dev.data_ptr()),
           "kimad_debug_step_with_err")


def kimad_debug_step_with_j(ctx: Ctx, grads, state, bandwidth_bytes_per_s, t_target_s, out: Packed, j_dev,
                            stream=None) -> None:
    bw = _bw(ctx, bandwidth_bytes_per_s)
    _check(load().kimad_debug_step_with_j(ctx.handle, grads.data_ptr(), state.data_ptr(),
                                          bw.ctypes.data_as(C.POINTER(C.c_double)), float(t_target_s),
                                          C.byref(out.c), _stream_ptr(stream), j_dev.data_ptr()),
           "kimad_debug_step_with_j")


def kimad_get_k(ctx: Ctx, stream=None):
    """Returns (status, k[W][L]) of the last step after synchronising the stream."""
    k = np.zeros((ctx.W, ctx.L), dtype=np.uint32)
    st = load().kimad_get_k(ctx.handle, k.ctypes.data, _stream_ptr(stream))
    return int(st), k


def kimad_get_k_table(ctx: Ctx) -> np.ndarray:
    kt = np.zeros((ctx.L, ctx.K), dtype=np.uint64)
    _check(load().kimad_get_k_table(ctx.handle, kt.ctypes.data), "kimad_get_k_table")
    return kt


def kimad_plan_budget(ctx: Ctx, bandwidth_bytes_per_s: float, t_target_s: float):
    """Returns (status, budget_bytes, cells[L][K] or None)."""
    c = C.c_uint64(0)
    cells = np.zeros((ctx.L, ctx.K), dtype=np.uint64)
    st = _check(load().kimad_plan_budget(ctx.handle, float(bandwidth_bytes_per_s), float(t_target_s), C.byref(c),
                                         cells.ctypes.data), "kimad_plan_budget")
    return st, int(c.value), (cells if st == 0 else None)


def kimad_debug_get_curve(ctx: Ctx):
    """Returns (err f32, tau u32, keep_eq u32, shift u32), each [W][L][K], of the last step."""
    shape = (ctx.W, ctx.L, ctx.K)
    err = np.zeros(shape, np.float32)
    tau = np.zeros(shape, np.uint32)
    keq = np.zeros(shape, np.uint32)
    shift = np.zeros(shape, np.uint32)
    _check(load().kimad_debug_get_curve(ctx.handle, err.ctypes.data, tau.ctypes.data, keq.ctypes.data,
                                        shift.ctypes.data), "kimad_debug_get_curve")
    return err, tau, keq, shift


def kimad_debug_get_selection(ctx: Ctx):
    """Returns (tau u32, keep_eq u32), each [W][L]: exact threshold of the chosen candidate of every layer."""
    tau = np.zeros((ctx.W, ctx.L), np.uint32)
    keq = np.zeros((ctx.W, ctx.L), np.uint32)
    _check(load().kimad_debug_get_selection(ctx.handle, tau.ctypes.data, keq.ctypes.data),
           "kimad_debug_get_selection")
    return tau, keq


STAGE_NAMES = ["sample", "sweep", "curve", "exact_fallback", "dp", "select_count", "select_scan", "select_write"]


def kimad_debug_enable_stage_timing(ctx: Ctx, enable: bool) -> None:
    _check(load().kimad_debug_enable_stage_timing(ctx.handle, int(bool(enable))), "kimad_debug_enable_stage_timing")


def kimad_debug_set_schedule(ctx: Ctx, mode: int) -> None:
    """0: two worker groups for large steps, 1: whenever W >= 2, 2: one group."""
    _check(load().kimad_debug_set_schedule(ctx.handle, int(mode)), "kimad_debug_set_schedule")


def kimad_debug_set_search(ctx: Ctx, mode: int) -> None:
    """0: windows of the knapsack's rows and whole rows at the same time, 1: one after the other, 2: whole rows (see kimad.h)."""
    _check(load().kimad_debug_set_search(ctx.handle, int(mode)), "kimad_debug_set_search")


def kimad_debug_set_wait_limit(ctx: Ctx, clocks: int) -> None:
    """Limit of the knapsack kernel's waits in SM clocks (see kimad.h); 2^31 by default."""
    _check(load().kimad_debug_set_wait_limit(ctx.handle, int(clocks)), "kimad_debug_set_wait_limit")


def kimad_debug_trace_step(ctx: Ctx, grads, state, bandwidth_bytes_per_s, t_target_s, out: "Packed", stream=None) -> str:
    """One step with CUDA events around every launch; returns the timeline, one line per launch."""
    bw = _bw(ctx, bandwidth_bytes_per_s)
    buf = C.create_string_buffer(1 << 16)
    _check(load().kimad_debug_trace_step(ctx.handle, grads.data_ptr(), state.data_ptr(),
                                         bw.ctypes.data_as(C.POINTER(C.c_double)), float(t_target_s), C.byref(out.c),
                                         _stream_ptr(stream), buf, len(buf)), "kimad_debug_trace_step")
    return buf.value.decode()


def kimad_debug_stage_times(ctx: Ctx) -> np.ndarray:
    """Stage durations (ms) of the last step, order as STAGE_NAMES."""
    ms = np.zeros(len(STAGE_NAMES), np.float32)
    _check(load().kimad_debug_stage_times(ctx.handle, ms.ctypes.data), "kimad_debug_stage_times")
    return ms


def kimad_debug_get_band_meta(ctx: Ctx, n_regular: int) -> np.ndarray:
    """u32 [W][n_regular][4]: bins, entries of the cell table in use, flag, detail (see kimad.h)."""
    out = np.zeros((ctx.W, n_regular, 4), np.uint32)
    _check(load().kimad_debug_get_band_meta(ctx.handle, out.ctypes.data), "kimad_debug_get_band_meta")
    return out


def kimad_debug_exact_path_layers(ctx: Ctx, detail: bool = False):
    """Layers handed to the exact radix path so far; with detail also the count per reason
    (forced, bands too wide, threshold outside band, bound too loose even after refinement), the number of
    layers refined, and per candidate how often its first bound was loose."""
    n = (C.c_uint64 * (6 + ctx.K))()
    _check(load().kimad_debug_exact_path_layers(ctx.handle, n), "kimad_debug_exact_path_layers")
    return [int(x) for x in n] if detail else int(n[0])


def kimad_debug_searches(ctx: Ctx) -> list:
    """Searches over windows of the knapsack's rows so far: undecided, decided by their first windows, by their second ones."""
    n = (C.c_uint64 * 3)()
    _check(load().kimad_debug_searches(ctx.handle, n), "kimad_debug_searches")
    return [int(x) for x in n]


def kimad_debug_check(ctx: Ctx):
    """Returns (checked build?, failed-check bits, damaged canaries) -- see kimad.h."""
    w, b = C.c_uint32(0), C.c_uint32(0)
    rc = _check(load().kimad_debug_check(ctx.handle, C.byref(w), C.byref(b)), "kimad_debug_check")
    return bool(rc), int(w.value), int(b.value)


def kimad_launch_count(ctx: Ctx) -> int:
    return int(load().kimad_launch_count(ctx.handle))


def new_context(layer_sizes, n_workers, ratio_grid, device="cuda", **opts):
    """Convenience: create a context, allocate its workspace with torch and attach it."""
    import torch

    ctx = kimad_create(layer_sizes, n_workers, ratio_grid, **opts)
    ws = torch.empty(kimad_workspace_bytes(ctx) + 256, dtype=torch.uint8, device=device)
    off = (-ws.data_ptr()) % 256
    kimad_set_workspace(ctx, ws[off:])
    ctx._keep.append(ws)
    return ctx


# The 4-bit calls are short (a few microseconds on the GPU for a small model), so what surrounds the C call is kept short too: types are looked up
# by object, shapes compared as tuples, and the current stream asked for without making a Stream object of it.
_MX4_DTYPES = {}
_mx4_device = _mx4_raw_stream = None


def _mx4_setup():
    global _mx4_device, _mx4_raw_stream
    import torch

    _MX4_DTYPES.update({torch.float32: KIMAD_F32, torch.bfloat16: KIMAD_BF16, torch.float16: KIMAD_F16})
    c = torch._C
    _mx4_device = getattr(c, "_cuda_getDevice", torch.cuda.current_device)
    _mx4_raw_stream = getattr(c, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)


def _mx4_dtype(t, what, most=KIMAD_F16):
    """The code of a tensor's type, one of float32, bfloat16, float16 up to `most`."""
    if not _MX4_DTYPES:
        _mx4_setup()
    code = _MX4_DTYPES.get(t.dtype, 99)
    if code > most:
        raise TypeError(f"{what}: {t.dtype}, not one of {list(_MX4_DTYPES)[:most + 1]}")
    return code


def _mx4_stream(what, stream, here, *others):
    """The stream's handle.  The library takes memory of the current device: a tensor of another one is refused, as is one in host memory (device -1)."""
    for d in others:
        if d != here:
            raise ValueError(f"{what}: tensors on different devices")
    if here < 0:
        raise ValueError(f"{what}: a tensor in host memory")
    if here != _mx4_device():
        raise ValueError(f"{what}: a tensor on cuda:{here}, the current device is cuda:{_mx4_device()}")
    return _mx4_raw_stream(here) if stream is None else _stream_ptr(stream)


def _mx4_home(ctx, here):
    """The device of the context's workspace, which the kernels read (`here` where none is attached: the library refuses that)."""
    return ctx._keep[0].get_device() if ctx._keep else here


def _mx4_workers(ctx, t, what):
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or shape[0] != ctx.W or shape[1] < ctx.N or (shape[1] > 1 and stride[1] != 1) or (ctx.W > 1 and stride[0] != ctx.stride):
        raise ValueError(f"{what}: [{ctx.W}][{ctx.stride}] with rows of consecutive elements, not {tuple(shape)} with strides {stride}")


def kimad_mx4_message_bytes(ctx: Ctx):
    """(bytes of codes, bytes of scales) of one worker's 4-bit message."""
    c, s = C.c_uint64(0), C.c_uint64(0)
    _check(load().kimad_mx4_message_bytes(ctx.handle, C.byref(c), C.byref(s)), "kimad_mx4_message_bytes")
    return int(c.value), int(s.value)


def _mx4_shape(ctx):
    """What two contexts share that can read each other's messages: the workers and the layers' sizes, which decide where blocks begin."""
    shape = getattr(ctx, "_mx4_shape", None)
    if shape is None:
        shape = ctx._mx4_shape = (ctx.W, ctx.L, *kimad_mx4_message_bytes(ctx), ctx.layer_sizes)
    return shape


class Mx4Message:
    """Device buffers of all workers' 4-bit messages (tensors that stay where they are) and the matching ``kimad_mx4_message`` struct."""

    def __init__(self, ctx: Ctx, device="cuda"):
        import torch

        self.shape = _mx4_shape(ctx)
        W, L, code_bytes, scale_bytes, _ = self.shape
        self.codes = torch.zeros((W, code_bytes), dtype=torch.uint8, device=device)
        self.scales = torch.zeros((W, scale_bytes), dtype=torch.uint8, device=device)
        self.err = torch.zeros((W, L), dtype=torch.float32, device=device)
        self.stats = torch.zeros((W, STATS_DTYPE.itemsize), dtype=torch.uint8, device=device)
        self.c = kimad_mx4_message(self.codes.data_ptr(), self.scales.data_ptr(), self.err.data_ptr(), self.stats.data_ptr())
        self.ref = C.byref(self.c)
        self.device = self.codes.get_device()

    def stats_host(self) -> np.ndarray:
        return self.stats.cpu().numpy().view(STATS_DTYPE).reshape(-1)


def _mx4_message(ctx, msg, what):
    shape = _mx4_shape(ctx)
    if msg.shape is not shape and msg.shape != shape:
        raise ValueError(f"{what}: a message of another context's shape")
    return msg.ref


def kimad_mx4_step(ctx: Ctx, grads, state, msg: Mx4Message, stream=None) -> None:
    """grads: CUDA float32, bfloat16 or float16 [W][ctx.stride]; state: CUDA float32 of that shape, updated in place."""
    dtype = _mx4_dtype(grads, "grads")
    _mx4_dtype(state, "state", KIMAD_F32)
    _mx4_workers(ctx, grads, "grads")
    _mx4_workers(ctx, state, "state")
    m = _mx4_message(ctx, msg, "kimad_mx4_step")
    s = _mx4_stream("kimad_mx4_step", stream, here := grads.get_device(), state.get_device(), msg.device, _mx4_home(ctx, here))
    _check((_lib or load()).kimad_mx4_step(ctx.handle, grads.data_ptr(), dtype, state.data_ptr(), m, s), "kimad_mx4_step")


def kimad_mx4_apply(ctx: Ctx, msg: Mx4Message, est, x=None, weights=None, gamma=0.0, stream=None) -> None:
    """est: CUDA float32 [W][ctx.stride], in place.  With x (CUDA float32 [N], in place) also the model step: weights, W host floats, and gamma."""
    _mx4_dtype(est, "est", KIMAD_F32)
    _mx4_workers(ctx, est, "est")
    m = _mx4_message(ctx, msg, "kimad_mx4_apply")
    if x is None:
        s = _mx4_stream("kimad_mx4_apply", stream, here := est.get_device(), msg.device, _mx4_home(ctx, here))
        _check((_lib or load()).kimad_mx4_apply(ctx.handle, m, est.data_ptr(), None, None, 0.0, s), "kimad_mx4_apply")
        return
    _mx4_dtype(x, "x", KIMAD_F32)
    w = np.ascontiguousarray([] if weights is None else weights, dtype=np.float32).reshape(-1)
    if w.size != ctx.W or x.dim() != 1 or x.numel() != ctx.N or (ctx.N > 1 and x.stride(0) != 1):
        raise ValueError(f"kimad_mx4_apply: x of {ctx.N} consecutive elements and {ctx.W} weights")
    s = _mx4_stream("kimad_mx4_apply", stream, here := est.get_device(), x.get_device(), msg.device, _mx4_home(ctx, here))
    _check((_lib or load()).kimad_mx4_apply(ctx.handle, m, est.data_ptr(), x.data_ptr(), w.ctypes.data_as(C.POINTER(C.c_float)), gamma, s), "kimad_mx4_apply")


def kimad_mx4_read(ctx: Ctx, msg: Mx4Message, out, stream=None) -> None:
    """out: CUDA float32 or bfloat16 [W][ctx.stride], the values that the messages stand for."""
    dtype = _mx4_dtype(out, "out", KIMAD_BF16)
    _mx4_workers(ctx, out, "out")
    m = _mx4_message(ctx, msg, "kimad_mx4_read")
    s = _mx4_stream("kimad_mx4_read", stream, here := out.get_device(), msg.device, _mx4_home(ctx, here))
    _check((_lib or load()).kimad_mx4_read(ctx.handle, m, out.data_ptr(), dtype, s), "kimad_mx4_read")


def kimad_mx4_operand_bytes(lines: int, length: int):
    """(bytes of codes, bytes of scales) of one quantised matrix of ``lines`` lines of ``length`` values."""
    c, s = C.c_uint64(0), C.c_uint64(0)
    _check(load().kimad_mx4_operand_bytes(lines, length, C.byref(c), C.byref(s)), "kimad_mx4_operand_bytes")
    return int(c.value), int(s.value)


class Mx4Operand:
    """``batch`` matrices of ``lines`` lines of ``length`` values, quantised along their lines (see kimad.h for the layout): new device buffers, or
    those of a message that has arrived (tensors that stay where they are)."""

    def __init__(self, lines: int, length: int, batch: int = 1, codes=None, scales=None, device="cuda"):
        import torch

        self.lines, self.length, self.batch = int(lines), int(length), int(batch)
        code_bytes, scale_bytes = kimad_mx4_operand_bytes(self.lines, self.length)
        self.codes = torch.empty((batch, code_bytes), dtype=torch.uint8, device=device) if codes is None else codes
        self.scales = torch.empty((batch, scale_bytes), dtype=torch.uint8, device=device) if scales is None else scales
        for t, n in ((self.codes, code_bytes), (self.scales, scale_bytes)):
            if t.dtype != torch.uint8 or not t.is_contiguous() or t.numel() != batch * n:
                raise ValueError(f"an operand of {batch} x {lines} x {length} has {batch * n} contiguous bytes, not {tuple(t.shape)} of {t.dtype}")
        if self.codes.get_device() != self.scales.get_device():
            raise ValueError("an operand's codes and scales are on one device")
        self.device = self.codes.get_device()
        self.shapes = ((self.batch, self.length, self.lines), (self.batch, self.lines, self.length))  # of the matrix, by `along`
        self.codes_ptr, self.scales_ptr = self.codes.data_ptr(), self.scales.data_ptr()


def _mx4_matrix(t, shape, what):
    """(row stride, matrix stride) of a [rows][cols] or [batch][rows][cols] tensor of this shape."""
    batch, rows, cols = shape
    stride = t.stride()
    if (t.shape if len(stride) == 3 else (1, *t.shape)) != shape:
        raise ValueError(f"{what}: {tuple(t.shape)} does not go with an operand, {batch} x {rows} x {cols} does")
    ld = stride[-2] if rows > 1 else cols
    if (cols > 1 and stride[-1] != 1) or ld < cols:
        raise ValueError(f"{what}: rows of consecutive elements that do not overlap, not strides {stride}")
    return ld, stride[0] if batch > 1 else 0


def _mx4_along(op, along):
    if along not in (0, 1):
        raise ValueError("along: 0, blocks over the rows, or 1, over the columns")
    return op.shapes[along]


def kimad_mx4_quantize(x, op: Mx4Operand, along: int, stream=None) -> None:
    """x: CUDA float32, bfloat16 or float16, [rows][cols] or [batch][rows][cols].  along 0: blocks over the rows (the operand is x transposed), 1: over
    the columns."""
    dtype = _mx4_dtype(x, "x")
    shape = _mx4_along(op, along)
    ld, bs = _mx4_matrix(x, shape, "x")
    s = _mx4_stream("kimad_mx4_quantize", stream, x.get_device(), op.device)
    _check((_lib or load()).kimad_mx4_quantize(x.data_ptr(), dtype, shape[1], shape[2], ld, shape[0], bs, along, op.codes_ptr, op.scales_ptr, s),
           "kimad_mx4_quantize")


def kimad_mx4_dequantize(op: Mx4Operand, out, along: int, stream=None) -> None:
    """out: CUDA float32 or bfloat16, shaped as kimad_mx4_quantize's x."""
    dtype = _mx4_dtype(out, "out", KIMAD_BF16)
    shape = _mx4_along(op, along)
    ld, bs = _mx4_matrix(out, shape, "out")
    s = _mx4_stream("kimad_mx4_dequantize", stream, out.get_device(), op.device)
    _check((_lib or load()).kimad_mx4_dequantize(op.codes_ptr, op.scales_ptr, out.data_ptr(), dtype, shape[1], shape[2], ld, shape[0], bs, along, s),
           "kimad_mx4_dequantize")


def kimad_mx4_product(a: Mx4Operand, b: Mx4Operand, out, alpha=1.0, beta=0.0, status=None, stream=None) -> None:
    """out <- beta out + alpha a b^T.  out: CUDA float32 [a.lines][b.lines] or [batch][a.lines][b.lines], rows of consecutive elements at any stride
    and place; status: CUDA int32 tensor of one element or None (kimad_mx4_product_status tells of all products of the device)."""
    _mx4_dtype(out, "out", KIMAD_F32)
    if a.length != b.length or a.batch != b.batch:
        raise ValueError(f"kimad_mx4_product: operands of {a.batch} x {a.length} and of {b.batch} x {b.length}")
    ld, bs = _mx4_matrix(out, (a.batch, a.lines, b.lines), "out")
    s = _mx4_stream("kimad_mx4_product", stream, out.get_device(), a.device, b.device)
    if status is not None:
        if str(status.dtype) != "torch.int32" or status.numel() < 1:
            raise TypeError("kimad_mx4_product: status is an int32 tensor")
        _mx4_stream("kimad_mx4_product", stream, status.get_device())
    _check((_lib or load()).kimad_mx4_product(out.data_ptr(), ld, bs, a.lines, b.lines, a.length, a.batch, a.codes_ptr, a.scales_ptr,
                                    b.codes_ptr, b.scales_ptr, alpha, beta, None if status is None else status.data_ptr(), s), "kimad_mx4_product")


def kimad_mx4_product_status(reset: bool = False, stream=None) -> int:
    """KIMAD_ERR_TIMEOUT if a bounded wait ran out in a product on the current device since the last reset, else KIMAD_OK.  Waits for the stream; to be asked
    before the results of products are relied on."""
    st = load().kimad_mx4_product_status(int(bool(reset)), _stream_ptr(stream))
    return st if st == KIMAD_ERR_TIMEOUT else _check(st, "kimad_mx4_product_status")


def kimad_debug_mx4_set_wait_limit(clocks: int, withhold: bool = False) -> None:
    """Limit of the waits inside the product's kernels in SM clocks, 2^31 by default; withhold: let them run out (see kimad.h)."""
    _check(load().kimad_debug_mx4_set_wait_limit(int(clocks), int(bool(withhold))), "kimad_debug_mx4_set_wait_limit")


class Monitor:
    """Owning handle of a ``kimad_monitor*`` (bandwidth estimate from the history of finished transfers)."""

    def __init__(self, window: int = 8, alpha: float = 1.0):
        h = C.c_void_p()
        _check(load().kimad_monitor_create(C.byref(h), int(window), float(alpha)), "kimad_monitor_create")
        self.handle = h

    def __del__(self):
        h, self.handle = getattr(self, "handle", None), None
        if h and _lib is not None:
            _lib.kimad_monitor_destroy(h)


def kimad_monitor_create(window: int = 8, alpha: float = 1.0) -> Monitor:
    return Monitor(window, alpha)


def kimad_monitor_observe(m: Monitor, n_bytes: int, seconds: float) -> None:
    _check(load().kimad_monitor_observe(m.handle, int(n_bytes), float(seconds)), "kimad_monitor_observe")


def kimad_monitor_estimate(m: Monitor) -> float:
    return float(load().kimad_monitor_estimate(m.handle))


def kimad_monitor_destroy(m: Monitor) -> None:
    h, m.handle = m.handle, None
    if h:
        load().kimad_monitor_destroy(h)
