"""Thin ctypes binding of libguide.so (include/guide.h): argument marshalling
only.  Every step of the evaluated path runs in the HIP kernels; there is no
CPU fallback, and a missing library is an error.  Device buffers are torch
tensors (torch is used for device memory and streams only).
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libguide.so")

OK, E_ARG, E_RANGE, E_NOMEM, E_DEVICE = 0, -1, -2, -3, -4
TIME_ROOFLINE, TIME_ADDITIVE = 0, 1
AXIS_GEOM2, AXIS_TABLE = 0, 1
SELECT_TOPK, SELECT_PARETO = 0, 1
SIM_OK, SIM_INFEASIBLE, SIM_BAD_INPUT, SIM_INTERNAL = 0, 1, 2, 3
SCHED_SPLIT_FUSE, SCHED_PREFILL_FIRST = 0, 1
SIM_CLOSED_FORM_RUNS = 256       # may be OR-ed into simulate()'s scheduler; no effect
NO_INDEX = 2 ** 64 - 1
MAX_CONSTRAINTS = 4
STATIC_SELECT_MAX_ROWS = 1 << 21

EXPORTS = ("guide_create", "guide_destroy", "guide_last_error", "guide_set_models", "guide_set_hardware",
           "guide_eval_grid", "guide_eval_extras", "guide_eval_sampled", "guide_simulate_workspace_bytes", "guide_simulate",
           "guide_select_workspace_bytes", "guide_select", "guide_select_static",
           "guide_eval_select_workspace_bytes", "guide_eval_select",
           "guide_profile_enable", "guide_profile_read",
           "guide_quantise", "guide_rms_norm", "guide_product", "guide_prompt_attention",
           "guide_cache_append", "guide_cache_read", "guide_cache_attention_workspace_bytes", "guide_cache_attention")


class GuideError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"libguide error {code}: {msg}")
        self.code = code


class CModel(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("L", "d", "n_h", "n_kv", "d_ff", "V", "E", "k")]


class CHw(C.Structure):
    _fields_ = [(n, C.c_double) for n in ("peak_flops", "hbm_bw", "cap_bytes", "link_bw", "link_lat")]


class CAxis(C.Structure):
    _fields_ = [("count", C.c_uint32), ("kind", C.c_uint32), ("start", C.c_uint64), ("values", C.POINTER(C.c_uint64))]


class CGrid(C.Structure):
    _fields_ = [(n, CAxis) for n in ("model", "hw", "batch", "s_in", "s_out", "tp", "wbits", "kv_block", "mbt")]


class CEff(C.Structure):
    _fields_ = [("n", C.c_uint32), ("e_c", C.c_void_p), ("e_b", C.c_void_p)]


METRIC_COLUMNS = ("t_prefill", "t_decode", "t_batch", "decode_tok_s", "cost", "b_max", "feasible")
STATS_COLUMNS = ("ttft_mean", "ttft_p10", "ttft_p90", "t_batch_mean", "t_batch_p10", "t_batch_p90", "cost", "b_max",
                 "feasible")
EXTRAS_COLUMNS = ("s_max", "dp_max", "max_parallelism", "cluster_tok_s", "paper_tok_s", "b_adj", "n_sub_batches",
                  "n_segments", "s_adj", "b_max_kept", "s_max_kept", "feasible_kept")
SAMPLED_COLUMNS = ("feasible_count", "win_val", "win_idx", "hist", "t_prefill", "t_batch", "cost", "b_max",
                   "feasible", "bucket")
SIM_COLUMNS = ("ttft_p50", "ttft_p99", "mean_tpot", "tokens_s", "status", "n_steps", "n_request_steps")


class CMetrics(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in METRIC_COLUMNS]


class CStats(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in STATS_COLUMNS]


class CExtras(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in EXTRAS_COLUMNS[:9]] + [("kv_keep", C.c_double)] + \
               [(n, C.c_void_p) for n in EXTRAS_COLUMNS[9:]]


class CSpace(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("heads", "peak", "bw", "cap", "batch", "s_in", "s_out", "tp", "wbits",
                                          "kv_block", "mbt", "kv_choices")] + \
               [(n, C.c_uint32) for n in ("layers_lo", "layers_n", "ffn_lo_x2", "ffn_span_x2", "vocab")] + \
               [("link_div", C.c_double)]


class CSampledOut(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in SAMPLED_COLUMNS]


class CTrace(C.Structure):
    _fields_ = [("n", C.c_uint32), ("arrival_unit", C.c_void_p), ("n_in", C.c_void_p), ("n_out", C.c_void_p)]


class CSimOut(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in SIM_COLUMNS]


class CConstraint(C.Structure):
    _fields_ = [("column", C.c_void_p), ("cap", C.c_double)]


class CSelectSpec(C.Structure):
    _fields_ = [("mode", C.c_uint32), ("objective", C.c_void_p), ("objective_y", C.c_void_p),
                ("feasible", C.c_void_p), ("n_constraints", C.c_uint32),
                ("constraints", CConstraint * MAX_CONSTRAINTS), ("group", C.c_void_p),
                ("n_groups", C.c_uint32), ("k", C.c_uint32)]


class CSelectOut(C.Structure):
    _fields_ = [("idx", C.c_void_p), ("val", C.c_void_p), ("count", C.c_void_p), ("capacity", C.c_uint64)]


COLUMN_IDS = {"t_prefill": 0, "t_decode": 1, "t_batch": 2, "decode_tok_s": 3, "cost": 4}


class CColumnConstraint(C.Structure):
    _fields_ = [("column", C.c_uint32), ("reserved", C.c_uint32), ("cap", C.c_double)]


class CColumnSelect(C.Structure):
    _fields_ = [("mode", C.c_uint32), ("objective", C.c_uint32), ("objective_y", C.c_uint32),
                ("use_feasible", C.c_uint32), ("n_constraints", C.c_uint32), ("k", C.c_uint32),
                ("constraints", CColumnConstraint * MAX_CONSTRAINTS), ("out", CSelectOut)]


# guide_layer.h

BF16, F16, F32 = 0, 1, 2
MX_GROUP = 32            # values per scale
NORM_MAX_WIDTH = 32768
PRODUCT_MAX = 1_000_000


class CQuantiseSpec(C.Structure):
    _fields_ = [("type", C.c_uint32), ("bits", C.c_uint32), ("rows", C.c_uint32), ("cols", C.c_uint32),
                ("x", C.c_void_p), ("x_stride", C.c_int64), ("codes", C.c_void_p), ("scales", C.c_void_p),
                ("codes_stride", C.c_int64), ("scales_stride", C.c_int64)]


class CNormSpec(C.Structure):
    _fields_ = [("type", C.c_uint32), ("bits", C.c_uint32), ("rows", C.c_uint32), ("d", C.c_uint32), ("eps", C.c_float),
                ("x", C.c_void_p), ("residual", C.c_void_p), ("weight", C.c_void_p),
                ("x_stride", C.c_int64), ("residual_stride", C.c_int64), ("total", C.c_void_p), ("total_stride", C.c_int64),
                ("codes", C.c_void_p), ("scales", C.c_void_p), ("codes_stride", C.c_int64), ("scales_stride", C.c_int64)]


class CProductSpec(C.Structure):
    _fields_ = [("type", C.c_uint32), ("a_bits", C.c_uint32), ("m", C.c_uint32), ("n", C.c_uint32), ("k", C.c_uint32)] + \
               [(n, C.c_void_p) for n in ("a_codes", "a_scales", "w_codes", "w_scales")] + \
               [(n, C.c_int64) for n in ("a_codes_stride", "a_scales_stride", "w_codes_stride", "w_scales_stride")] + \
               [("out", C.c_void_p), ("out_stride", C.c_int64)]


class CPromptSpec(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("type", "n_seq", "n_h", "n_kv", "d", "total_q", "total_k")] + \
               [("scale", C.c_float)] + [(n, C.c_void_p) for n in ("q", "k", "v", "out")] + \
               [(n, C.c_int64) for n in ("q_stride", "q_head_stride", "k_stride", "k_head_stride", "v_stride",
                                         "v_head_stride", "out_stride", "out_head_stride")] + \
               [("q_starts", C.c_void_p), ("k_starts", C.c_void_p)]


class CCache(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("n_pages", "n_kv", "kv_block", "d")] + [("codes", C.c_void_p), ("scales", C.c_void_p)]


class CCacheTokens(C.Structure):
    _fields_ = [("type", C.c_uint32), ("tokens", C.c_uint32), ("k", C.c_void_p), ("v", C.c_void_p)] + \
               [(n, C.c_int64) for n in ("k_stride", "k_head_stride", "v_stride", "v_head_stride")] + [("slots", C.c_void_p)]


class CCacheQueries(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("type", "n_seq", "n_h", "max_pages")] + [("scale", C.c_float)] + \
               [("q", C.c_void_p), ("out", C.c_void_p)] + \
               [(n, C.c_int64) for n in ("q_stride", "q_head_stride", "out_stride", "out_head_stride")] + \
               [("pages", C.c_void_p), ("pages_stride", C.c_int64), ("lengths", C.c_void_p)]


_lib = None


def load() -> C.CDLL:
    """Loads libguide.so; raises if it has not been built (python -m paper_2412_04788_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} is missing: build it with paper_2412_04788_amd/build.py")
        # torch ships its own HIP runtime; it must be in the process before libguide's
        # dependency on libamdhip64 is resolved, or two runtimes would be loaded
        import torch  # noqa: F401
        lib = C.CDLL(LIB_PATH)
        lib.guide_create.argtypes = [C.POINTER(C.c_void_p), C.c_int]
        lib.guide_destroy.argtypes = [C.c_void_p]
        lib.guide_destroy.restype = None
        lib.guide_last_error.argtypes = [C.c_void_p]
        lib.guide_last_error.restype = C.c_char_p
        lib.guide_set_models.argtypes = [C.c_void_p, C.c_void_p, C.c_uint32]
        lib.guide_set_hardware.argtypes = [C.c_void_p, C.c_void_p, C.c_uint32]
        lib.guide_eval_grid.argtypes = [C.c_void_p, C.POINTER(CGrid), C.c_uint64, C.c_uint64, C.POINTER(CEff),
                                        C.c_uint32, C.POINTER(CMetrics), C.POINTER(CStats), C.c_void_p]
        lib.guide_eval_extras.argtypes = [C.c_void_p, C.POINTER(CGrid), C.c_uint64, C.c_uint64, C.c_uint32,
                                          C.c_uint32, C.POINTER(CExtras), C.c_void_p]
        lib.guide_eval_sampled.argtypes = [C.c_void_p, C.POINTER(CSpace), C.c_uint64, C.c_uint64, C.c_uint64,
                                           C.c_void_p, C.c_uint32, C.c_double, C.c_uint32, C.POINTER(CSampledOut),
                                           C.c_void_p]
        lib.guide_simulate_workspace_bytes.argtypes = [C.c_uint32, C.c_uint32]
        lib.guide_simulate_workspace_bytes.restype = C.c_size_t
        lib.guide_simulate.argtypes = [C.c_void_p, C.POINTER(CGrid), C.c_void_p, C.c_void_p, C.c_uint32,
                                       C.POINTER(CTrace), C.c_uint32, C.c_uint32, C.POINTER(CSimOut), C.c_void_p,
                                       C.c_size_t, C.c_void_p]
        lib.guide_select_workspace_bytes.argtypes = [C.POINTER(CSelectSpec), C.c_uint64]
        lib.guide_select_workspace_bytes.restype = C.c_size_t
        lib.guide_select.argtypes = [C.c_void_p, C.POINTER(CSelectSpec), C.c_uint64, C.POINTER(CSelectOut),
                                     C.c_void_p, C.c_size_t, C.c_void_p]
        lib.guide_select_static.argtypes = [C.c_void_p, C.POINTER(CSelectSpec), C.c_uint64, C.POINTER(CSelectOut),
                                            C.c_void_p]
        lib.guide_eval_select_workspace_bytes.argtypes = [C.c_void_p, C.c_uint32, C.c_uint64]
        lib.guide_eval_select_workspace_bytes.restype = C.c_size_t
        lib.guide_eval_select.argtypes = [C.c_void_p, C.POINTER(CGrid), C.c_uint64, C.c_uint64, C.POINTER(CEff),
                                          C.c_uint32, C.POINTER(CMetrics), C.c_void_p, C.c_uint32, C.c_void_p,
                                          C.c_size_t, C.c_void_p]
        lib.guide_profile_enable.argtypes = [C.c_void_p, C.c_uint32, C.c_uint32]
        lib.guide_profile_read.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(C.c_uint32)]
        for name, spec in (("guide_quantise", CQuantiseSpec), ("guide_rms_norm", CNormSpec), ("guide_product", CProductSpec),
                           ("guide_prompt_attention", CPromptSpec)):
            getattr(lib, name).argtypes = [C.c_void_p, C.POINTER(spec), C.c_void_p]
        for name in ("guide_cache_append", "guide_cache_read"):
            getattr(lib, name).argtypes = [C.c_void_p, C.POINTER(CCache), C.POINTER(CCacheTokens), C.c_void_p]
        lib.guide_cache_attention_workspace_bytes.argtypes = [C.c_uint32] * 4 + [C.c_uint64]
        lib.guide_cache_attention_workspace_bytes.restype = C.c_size_t
        lib.guide_cache_attention.argtypes = [C.c_void_p, C.POINTER(CCache), C.POINTER(CCacheQueries), C.c_void_p, C.c_size_t,
                                              C.c_void_p]
        _lib = lib
    return _lib


class _Ref:
    """byref() of a ctypes struct that also keeps the struct (and what it points to) alive."""

    def __init__(self, struct, keep=None):
        self.struct, self.keep = struct, keep
        self._as_parameter_ = C.byref(struct)


class _Arr:
    """Address of a ctypes array, kept alive together with what its elements point to."""

    def __init__(self, arr, keep=None):
        self.arr, self.keep = arr, keep
        self._as_parameter_ = C.cast(arr, C.c_void_p)


class _Ptr:
    """Address of a host numpy array, kept alive."""

    def __init__(self, array):
        self.array = array
        self._as_parameter_ = C.c_void_p(array.ctypes.data)


def _dev_ptr(t) -> Optional[int]:
    """data_ptr() of a contiguous CUDA tensor (None passes NULL)."""
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("device buffers must be contiguous CUDA tensors")
    return t.data_ptr()


_TYPES = {"torch.bfloat16": BF16, "torch.float16": F16, "torch.float32": F32}
_type_of = {}                    # torch dtype -> GUIDE_* (filled as dtypes are met: torch is imported late)


def _elem(t) -> int:
    """GUIDE_* of a tensor's dtype."""
    e = _type_of.get(t.dtype)
    if e is None:
        e = _TYPES.get(str(t.dtype))
        if e is None:
            raise ValueError(f"tensors of {t.dtype} are not supported: bfloat16, float16 or float32")
        _type_of[t.dtype] = e
    return e


def _strided(t, dims: int, dtype=None):
    """data_ptr() and strides of a CUDA tensor of `dims` dimensions whose last one is contiguous."""
    st = t.stride()
    if len(st) != dims or (st[-1] != 1 and t.shape[-1] > 1) or not t.is_cuda:
        raise ValueError(f"a CUDA tensor of {dims} dimensions with a contiguous last one is needed")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"dtypes differ: {t.dtype} and {dtype}")
    return t.data_ptr(), st


def _shaped(what: str, t, shape):
    if t.shape != shape:
        raise ValueError(f"{what}: shape {tuple(t.shape)}, {tuple(shape)} is needed")


def _too_many():
    """Counts go to the library in 32 bits."""
    return ValueError("2^32 or more rows, columns or tokens")


def _codes(what: str, t, shape):
    """Pointer and row stride of a matrix of bytes."""
    _shaped(what, t, shape)
    if t.element_size() != 1:
        raise ValueError("codes and scales are tensors of bytes")
    p, st = _strided(t, 2)
    return p, st[0]


def _ints(t, size: int) -> int:
    """data_ptr() of a contiguous CUDA tensor of integers of `size` bytes."""
    if t.element_size() != size or t.is_floating_point():
        raise ValueError(f"integers of {8 * size} bits are needed")
    return _dev_ptr(t)


_raw_stream = None


def _stream_ptr(stream) -> Optional[int]:
    if stream is not None:
        return stream.cuda_stream or None
    global _raw_stream
    if _raw_stream is None:
        import torch
        try:                     # the current stream's handle without a Stream object around it: 3 us less in every call
            raw, device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
            _raw_stream = lambda: raw(device())
        except AttributeError:
            _raw_stream = lambda: torch.cuda.current_stream().cuda_stream
    return _raw_stream() or None


def make_axis(values: Sequence[int], geom2_start: int = 0):
    """Returns (CAxis, keep-alive array)."""
    ax = CAxis()
    ax.count = len(values)
    if geom2_start:
        ax.kind, ax.start, keep = AXIS_GEOM2, geom2_start, None
    else:
        keep = np.ascontiguousarray(values, dtype=np.uint64)
        ax.kind, ax.start = AXIS_TABLE, 0
        ax.values = keep.ctypes.data_as(C.POINTER(C.c_uint64))
    return ax, keep


class GridArg:
    """C grid descriptor from nine (values, geom2_start) pairs, slow -> fast."""

    def __init__(self, axes):
        assert len(axes) == 9
        self.c = CGrid()
        self._keep = []
        self.size = 1
        for (name, _), (values, start) in zip(CGrid._fields_, axes):
            ax, keep = make_axis(values, start)
            setattr(self.c, name, ax)
            self._keep.append(keep)
            self.size *= len(values)


class Context:
    """guide_ctx handle.  Methods mirror the C entry points one to one."""

    def __init__(self, device: int = 0):
        self._lib = load()
        h = C.c_void_p()
        rc = self._lib.guide_create(C.byref(h), device)
        if rc:
            raise GuideError(rc, "guide_create failed")
        self._h = h
        self.device = device

    def close(self):
        if getattr(self, "_h", None):
            self._lib.guide_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def last_error(self) -> str:
        return self._lib.guide_last_error(self._h).decode()

    def _check(self, rc):
        if rc:
            raise GuideError(rc, self.last_error())

    def set_models(self, rows):
        a = np.ascontiguousarray(rows, dtype=np.uint32).reshape(-1, 8)
        self._check(self._lib.guide_set_models(self._h, a.ctypes.data, len(a)))

    def set_hardware(self, rows):
        a = np.ascontiguousarray(rows, dtype=np.float64).reshape(-1, 5)
        self._check(self._lib.guide_set_hardware(self._h, a.ctypes.data, len(a)))

    def prepared(self, method: str, *args, **kw):
        """Marshals the arguments of `method` once and returns a zero-argument callable that
        repeats the same C call (for loops that re-issue one call many times; the stream is
        the one current at preparation time)."""
        calls = []
        real = self._invoke
        self._invoke = lambda fn, *a: calls.append((fn, a))
        try:
            getattr(self, method)(*args, **kw)
        finally:
            self._invoke = real
        (fn, a), = calls
        keep = (args, kw)

        def run(_fn=fn, _a=a, _keep=keep, _check=self._check):
            _check(_fn(*_a))
        return run

    def _invoke(self, fn, *a):
        self._check(fn(*a))

    def eval_grid(self, grid: GridArg, first: int, count: int, out: dict = None, stats: dict = None,
                  e_c=None, e_b=None, time_model: int = TIME_ROOFLINE, stream=None):
        """out / stats: dicts column name -> CUDA tensor (missing = not written)."""
        eff = None
        if e_c is not None:
            e_c = np.ascontiguousarray(e_c, dtype=np.float64)
            e_b = np.ascontiguousarray(e_b, dtype=np.float64)
            eff = CEff(len(e_c), e_c.ctypes.data, e_b.ctypes.data)
        cm = cs = None
        if out is not None:
            cm = CMetrics(*[_dev_ptr(out.get(k)) for k in METRIC_COLUMNS])
        if stats is not None:
            cs = CStats(*[_dev_ptr(stats.get(k)) for k in STATS_COLUMNS])
        self._invoke(self._lib.guide_eval_grid, self._h, _Ref(grid.c, grid), first, count,
                     _Ref(eff, (e_c, e_b)) if eff else None, time_model,
                     _Ref(cm) if cm else None, _Ref(cs) if cs else None, _stream_ptr(stream))

    @staticmethod
    def column_select(mode: int, objective: str, out_idx, out_val, out_count, objective_y: str = None,
                      use_feasible: bool = True, constraints=(), k: int = 1, capacity: int = 0) -> CColumnSelect:
        """guide_column_select from column names; constraints = [(column name, cap), ...]."""
        c = CColumnSelect()
        c.mode = mode
        c.objective = COLUMN_IDS[objective]
        c.objective_y = COLUMN_IDS[objective_y] if objective_y is not None else 0
        c.use_feasible = 1 if use_feasible else 0
        c.n_constraints = len(constraints)
        for i, (col, cap) in enumerate(list(constraints)[:MAX_CONSTRAINTS]):
            c.constraints[i].column = COLUMN_IDS[col]
            c.constraints[i].cap = float(cap)
        c.k = k
        c.out = CSelectOut(_dev_ptr(out_idx), _dev_ptr(out_val), _dev_ptr(out_count), capacity)
        c._keep = (out_idx, out_val, out_count)
        return c

    def eval_select_workspace_bytes(self, selections: Sequence[CColumnSelect], count: int) -> int:
        arr = (CColumnSelect * max(len(selections), 1))(*selections)
        return self._lib.guide_eval_select_workspace_bytes(C.cast(arr, C.c_void_p), len(selections), count)

    def eval_select(self, grid: GridArg, first: int, count: int, out: dict, selections: Sequence[CColumnSelect],
                    workspace, e_c=None, e_b=None, time_model: int = TIME_ROOFLINE, stream=None):
        """guide_eval_select: evaluate [first, first + count) into `out` and run the selections on it."""
        eff = None
        if e_c is not None:
            e_c = np.ascontiguousarray([e_c], dtype=np.float64).reshape(-1)
            e_b = np.ascontiguousarray([e_b], dtype=np.float64).reshape(-1)
            eff = CEff(len(e_c), e_c.ctypes.data, e_b.ctypes.data)
        cm = CMetrics(*[_dev_ptr(out.get(k)) for k in METRIC_COLUMNS])
        arr = (CColumnSelect * max(len(selections), 1))(*selections)
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
        self._invoke(self._lib.guide_eval_select, self._h, _Ref(grid.c, grid), first, count,
                     _Ref(eff, (e_c, e_b)) if eff else None, time_model, _Ref(cm, out),
                     _Arr(arr, selections), len(selections),
                     _dev_ptr(workspace), ws_bytes, _stream_ptr(stream))

    def profile_enable(self, capacity: int, every: int = 1):
        self._check(self._lib.guide_profile_enable(self._h, capacity, every))

    def profile_read(self, capacity: int) -> np.ndarray:
        """Elapsed milliseconds of the evaluation kernels timed since the last read."""
        ms = np.zeros(max(capacity, 1), dtype=np.float32)
        n = C.c_uint32(0)
        self._check(self._lib.guide_profile_read(self._h, ms.ctypes.data, C.byref(n)))
        return ms[:n.value].copy()

    def eval_extras(self, grid: GridArg, first: int, count: int, n_gpus: int, out: dict,
                    time_model: int = TIME_ROOFLINE, stream=None, kv_keep: float = 0.0):
        ce = CExtras(**{k: _dev_ptr(out.get(k)) for k in EXTRAS_COLUMNS}, kv_keep=float(kv_keep))
        self._invoke(self._lib.guide_eval_extras, self._h, _Ref(grid.c, grid), first, count, n_gpus, time_model,
                     _Ref(ce), _stream_ptr(stream))

    def eval_sampled(self, space: dict, seed: int, first: int, count: int, edges, ttft_cap: float, out: dict,
                     time_model: int = TIME_ROOFLINE, stream=None):
        """space: dict of host numpy tables and scalars named as guide_space's fields."""
        keep = {}
        cs = CSpace()
        for name in ("heads", "batch", "s_in", "s_out", "tp", "wbits", "kv_block", "mbt", "kv_choices"):
            keep[name] = np.ascontiguousarray(space[name], dtype=np.uint32)
            setattr(cs, name, keep[name].ctypes.data)
        for name in ("peak", "bw", "cap"):
            keep[name] = np.ascontiguousarray(space[name], dtype=np.float64)
            setattr(cs, name, keep[name].ctypes.data)
        for name in ("layers_lo", "layers_n", "ffn_lo_x2", "ffn_span_x2", "vocab"):
            setattr(cs, name, int(space[name]))
        cs.link_div = float(space["link_div"])
        edges = np.ascontiguousarray(edges, dtype=np.float64)
        co = CSampledOut(*[_dev_ptr(out.get(k)) for k in SAMPLED_COLUMNS])
        self._invoke(self._lib.guide_eval_sampled, self._h, _Ref(cs, keep), seed, first, count,
                     _Ptr(edges), len(edges), ttft_cap, time_model, _Ref(co), _stream_ptr(stream))

    def simulate_workspace_bytes(self, n_cfg: int, n_requests: int) -> int:
        return self._lib.guide_simulate_workspace_bytes(n_cfg, n_requests)

    def simulate(self, grid: GridArg, cfg_idx, rate, trace, out: dict, workspace, time_model: int = TIME_ROOFLINE,
                 scheduler: int = SCHED_SPLIT_FUSE, stream=None):
        """cfg_idx (u32) / rate (f64): CUDA tensors; trace: (arrival_unit, n_in, n_out) host arrays."""
        arr = np.ascontiguousarray(trace[0], dtype=np.float64)
        n_in = np.ascontiguousarray(trace[1], dtype=np.uint32)
        n_out = np.ascontiguousarray(trace[2], dtype=np.uint32)
        ct = CTrace(len(arr), arr.ctypes.data, n_in.ctypes.data, n_out.ctypes.data)
        co = CSimOut(*[_dev_ptr(out.get(k)) for k in SIM_COLUMNS])
        self._invoke(self._lib.guide_simulate, self._h, _Ref(grid.c, grid), _dev_ptr(cfg_idx), _dev_ptr(rate),
                     cfg_idx.numel(), _Ref(ct, (arr, n_in, n_out)), time_model, scheduler, _Ref(co),
                     _dev_ptr(workspace), workspace.numel() * workspace.element_size(), _stream_ptr(stream))

    def _select_spec(self, mode, objective, objective_y, feasible, constraints, group, n_groups, k):
        s = CSelectSpec()
        s.mode = mode
        s.objective = _dev_ptr(objective)
        s.objective_y = _dev_ptr(objective_y)
        s.feasible = _dev_ptr(feasible)
        s.n_constraints = len(constraints)
        for i, (col, cap) in enumerate(constraints[:MAX_CONSTRAINTS]):
            s.constraints[i].column = _dev_ptr(col)
            s.constraints[i].cap = float(cap)
        s.group = _dev_ptr(group)
        s.n_groups = n_groups
        s.k = k
        return s

    def select_workspace_bytes(self, mode: int, n: int, n_groups: int = 1) -> int:
        s = CSelectSpec()
        s.mode, s.n_groups, s.k = mode, n_groups, 1
        return self._lib.guide_select_workspace_bytes(C.byref(s), n)

    def select(self, mode: int, n: int, objective, out_idx, out_val, out_count, workspace, objective_y=None,
               feasible=None, constraints=(), group=None, n_groups: int = 1, k: int = 1, capacity: int = 0,
               stream=None):
        s = self._select_spec(mode, objective, objective_y, feasible, list(constraints), group, n_groups, k)
        o = CSelectOut(_dev_ptr(out_idx), _dev_ptr(out_val), _dev_ptr(out_count), capacity)
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
        self._invoke(self._lib.guide_select, self._h, _Ref(s), n, _Ref(o), _dev_ptr(workspace), ws_bytes,
                     _stream_ptr(stream))

    def select_static(self, mode: int, n: int, objective, out_idx, out_val, out_count, objective_y=None,
                      feasible=None, constraints=(), group=None, n_groups: int = 1, k: int = 1, capacity: int = 0,
                      stream=None):
        """guide_select_static: guide_select on the library's static device scratch (no workspace, no allocation)."""
        s = self._select_spec(mode, objective, objective_y, feasible, list(constraints), group, n_groups, k)
        o = CSelectOut(_dev_ptr(out_idx), _dev_ptr(out_val), _dev_ptr(out_count), capacity)
        self._invoke(self._lib.guide_select_static, self._h, _Ref(s), n, _Ref(o), _stream_ptr(stream))

    # ---- guide_layer.h: the tasks of a decoder layer on the card (last dimensions contiguous, other strides free)

    @staticmethod
    def _code_rows(codes, scales, rows: int, cols: int, bits: int):
        """Pointers and strides of code and scale buffers of `rows` rows of `cols` values."""
        if bits != 4 and bits != 8:
            raise ValueError(f"codes of {bits} bits: 4 or 8")
        if (rows | cols) >> 32:
            raise _too_many()
        groups = -(-cols // MX_GROUP)
        return (*_codes("codes", codes, (rows, groups * 4 * bits)), *_codes("scales", scales, (rows, groups)))

    def quantise(self, x, codes, scales, bits: int = 4, stream=None):
        """x [rows, cols] into codes [rows, ceil(cols / 32) * 32 * bits / 8] and scales [rows, ceil(cols / 32)] (bytes)."""
        rows, cols = x.shape
        c, cs, s, ss = self._code_rows(codes, scales, rows, cols, bits)
        p, st = _strided(x, 2)
        self._invoke(self._lib.guide_quantise, self._h, CQuantiseSpec(_elem(x), bits, rows, cols, p, st[0], c, s, cs, ss),
                     _stream_ptr(stream))

    def rms_norm(self, x, weight, codes, scales, residual=None, total=None, eps: float = 1e-5, bits: int = 8, stream=None):
        """Norm of x (+ residual) [rows, d], times weight [d], as codes; total receives x + residual."""
        shape, dtype = x.shape, x.dtype
        rows, d = shape
        c, cs, s, ss = self._code_rows(codes, scales, rows, d, bits)
        _shaped("weight", weight, (d,))
        r = o = None
        rs = os_ = (0,)
        if residual is not None:
            _shaped("residual", residual, shape)
            r, rs = _strided(residual, 2, dtype)
        if total is not None:
            _shaped("total", total, shape)
            o, os_ = _strided(total, 2, dtype)
        p, st = _strided(x, 2)
        spec = CNormSpec(_elem(x), bits, rows, d, eps, p, r, _strided(weight, 1, dtype)[0], st[0], rs[0], o, os_[0], c, s, cs, ss)
        self._invoke(self._lib.guide_rms_norm, self._h, spec, _stream_ptr(stream))

    def product(self, a_codes, a_scales, w_codes, w_scales, out, bits: int = 8, stream=None):
        """out [m, n] = A W' for A [m, k] in codes of `bits` bits and W [n, k] in 4-bit codes."""
        (m, n), k = out.shape, w_scales.shape[1] * MX_GROUP
        a, astr, sa, sastr = self._code_rows(a_codes, a_scales, m, k, bits)
        w, wstr, sw, swstr = self._code_rows(w_codes, w_scales, n, k, 4)
        o, st = _strided(out, 2)
        self._invoke(self._lib.guide_product, self._h,
                     CProductSpec(_elem(out), bits, m, n, k, a, sa, w, sw, astr, sastr, wstr, swstr, o, st[0]), _stream_ptr(stream))

    def prompt_attention(self, q, k, v, q_starts, k_starts, out, scale: float = None, stream=None):
        """Causal attention of packed sequences: q, out [total_q, n_h, d], k, v [total_k, n_kv, d], starts int32 [n_seq + 1]."""
        shape, dtype = q.shape, q.dtype
        (tq, n_h, d), (tk, n_kv, dk), n = shape, k.shape, q_starts.numel()
        if (tq | tk | n) >> 32:
            raise _too_many()
        _shaped("out", out, shape)
        _shaped("v", v, k.shape)
        _shaped("q_starts", q_starts, (n,))
        _shaped("k_starts", k_starts, (n,))
        if dk != d or n < 1:
            raise ValueError(f"head dimensions {d} and {dk}, {n} starts")
        (pq, qs), (pk, ks), (pv, vs), (po, os_) = _strided(q, 3), _strided(k, 3, dtype), _strided(v, 3, dtype), _strided(out, 3, dtype)
        spec = CPromptSpec(_elem(q), n - 1, n_h, n_kv, d, tq, tk, d ** -0.5 if scale is None else scale, pq, pk, pv, po,
                           qs[0], qs[1], ks[0], ks[1], vs[0], vs[1], os_[0], os_[1], _ints(q_starts, 4), _ints(k_starts, 4))
        self._invoke(self._lib.guide_prompt_attention, self._h, spec, _stream_ptr(stream))

    @staticmethod
    def _cache(codes, scales) -> CCache:
        """codes [n_pages, n_kv, 2, kv_block, d / 2] and scales [n_pages, n_kv, 2, d / 32, kv_block], bytes."""
        n_pages, n_kv, two, block, half = codes.shape
        _shaped("scales", scales, (n_pages, n_kv, 2, half // 16, block))
        if two != 2 or codes.element_size() != 1 or scales.element_size() != 1:
            raise ValueError("the cache holds keys and values in bytes")
        return CCache(n_pages, n_kv, block, 2 * half, _dev_ptr(codes), _dev_ptr(scales))

    def _cache_tokens(self, fn, k, v, slots, codes, scales, stream):
        cache = self._cache(codes, scales)
        shape = (slots.numel(), cache.n_kv, cache.d)
        if shape[0] >> 32:
            raise _too_many()
        _shaped("k", k, shape)
        _shaped("v", v, shape)
        (pk, ks), (pv, vs) = _strided(k, 3), _strided(v, 3, k.dtype)
        spec = CCacheTokens(_elem(k), shape[0], pk, pv, ks[0], ks[1], vs[0], vs[1], _ints(slots, 8))
        self._invoke(fn, self._h, cache, spec, _stream_ptr(stream))

    def cache_append(self, k, v, slots, codes, scales, stream=None):
        """Writes k, v [tokens, n_kv, d] to the slots (int64, page * kv_block + offset) of the cache, each a slot of its own or one outside
        the cache (-1), which is skipped."""
        self._cache_tokens(self._lib.guide_cache_append, k, v, slots, codes, scales, stream)

    def cache_read(self, slots, codes, scales, k, v, stream=None):
        """Reads k, v [tokens, n_kv, d] back from the slots of the cache."""
        self._cache_tokens(self._lib.guide_cache_read, k, v, slots, codes, scales, stream)

    def cache_attention_workspace_bytes(self, n_seq: int, n_h: int, n_kv: int, d: int, max_len: int) -> int:
        return self._lib.guide_cache_attention_workspace_bytes(n_seq, n_h, n_kv, d, max_len)

    def cache_attention(self, q, codes, scales, pages, lengths, out, workspace=None, scale: float = None, stream=None):
        """One token per sequence: q, out [n_seq, n_h, d]; pages int32 [n_seq, max_pages], lengths int32 [n_seq]."""
        cache = self._cache(codes, scales)
        shape = q.shape
        n_seq, n_h, d = shape
        if n_seq >> 32:
            raise _too_many()
        if d != cache.d:
            raise ValueError(f"head dimensions {d} and {cache.d}")
        _shaped("out", out, shape)
        _shaped("lengths", lengths, (n_seq,))
        _shaped("pages", pages, (n_seq, pages.shape[-1]))
        if pages.element_size() != 4 or pages.is_floating_point():
            raise ValueError("integers of 32 bits are needed")
        (pq, qs), (po, os_), (pp, ps) = _strided(q, 3), _strided(out, 3, q.dtype), _strided(pages, 2)
        spec = CCacheQueries(_elem(q), n_seq, n_h, pages.shape[1], d ** -0.5 if scale is None else scale, pq, po,
                             qs[0], qs[1], os_[0], os_[1], pp, ps[0], _ints(lengths, 4))
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
        self._invoke(self._lib.guide_cache_attention, self._h, cache, spec, _dev_ptr(workspace), ws_bytes, _stream_ptr(stream))
