"""ctypes binding of ``libmebptt.so`` -- argument marshalling only.

Every function here has the name of the C entry point it calls (see ``include/mebptt.h``); all
planning and all arithmetic run inside the library.  PyTorch appears only as the owner of
device memory and of the HIP stream.  There is no fallback: if the library has not been built
the first call raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

import numpy as np

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libmebptt.so")
_lib = None

OK, EINVAL, ENOMEM_SLOTS, EWORKSPACE, ESHAPE, EINFEASIBLE, EHIP, ENOMEM_HOST = 0, -1, -2, -3, -4, -5, -6, -7
HSM, ISM, MSM = 0, 1, 2
OP_FWD_RUN, OP_BWD = 1, 2
LOC_NONE, LOC_T0, LOC_T1, LOC_CORE, LOC_INIT = -1, -2, -3, -4, -5
COST_INF = 1 << 60


class MebpttError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"mebptt error {code}: {message}")
        self.code = code


class mebptt_op(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("op", "step", "count", "src", "dst", "keep", "prev")]


class mebptt_decision(C.Structure):
    _fields_ = [("store", C.c_int32), ("y", C.c_int32)]


STORE_HIDDEN, STORE_INTERNAL = 1, 2


class mebptt_layer(C.Structure):
    _fields_ = [("cost", C.c_int64), ("state_units", C.c_int32), ("work_units", C.c_int32)]


class mebptt_chain_op(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("op", "layer", "count", "src", "dst")]


class mebptt_chain_desc(C.Structure):
    _fields_ = [("n", C.c_int32), ("B", C.c_int32), ("widths", C.POINTER(C.c_int32)), ("unit_bytes", C.c_size_t)]


class mebptt_chain_stats(C.Structure):
    _fields_ = [("forward_cost", C.c_int64), ("backward_ops", C.c_int64), ("peak_units", C.c_int32),
                ("reserved", C.c_int32)]


CHAIN_FORWARD, CHAIN_BACKWARD = 1, 2
CHAIN_INPUT, CHAIN_WORKING = -1, -2


class mebptt_lstm_desc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("B", "I", "H", "t", "gemm_dtype", "loss", "dy_first_step", "cell")]


CELL_LSTM, CELL_GRU = 0, 1


class mebptt_stats(C.Structure):
    _fields_ = [("forward_ops", C.c_int64), ("backward_ops", C.c_int64), ("peak", C.c_int32),
                ("reserved", C.c_int32), ("peak_slot_bytes", C.c_size_t)]


K_FORWARD, K_BACKWARD, K_WGRAD, K_DGRAD, K_SETUP, K_PAIR, K_CHAIN, K_SWEEP, K_FWD_BATCH, K_CLASSES = 0, 1, 2, 3, 4, 5, 6, 7, 8, 9
K_NAMES = ("forward", "backward", "wgrad", "dgrad", "setup", "backward+forward", "forward chain", "sweep",
           "forward batch")


class mebptt_profile(C.Structure):
    _fields_ = [("launches", C.c_int64 * K_CLASSES), ("sampled", C.c_int64 * K_CLASSES),
                ("sampled_ms", C.c_double * K_CLASSES), ("forward_run_launches", C.c_int64),
                ("forward_run_ms", C.c_double), ("chain_steps", C.c_int64), ("chain_ms", C.c_double),
                ("sweep_steps", C.c_int64), ("sweep_ms", C.c_double), ("sampled_groups", C.c_int64 * K_CLASSES),
                ("sweep_forward_steps", C.c_int64), ("batch_steps", C.c_int64), ("batch_ms", C.c_double)]


FP32, BF16, INT8 = 0, 1, 2


class mebptt_seq(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride_t", C.c_int64), ("stride_b", C.c_int64)]


class mebptt_norm_desc(C.Structure):
    _fields_ = [("rows", C.c_int64), ("width", C.c_int32), ("x_dtype", C.c_int32), ("residual_dtype", C.c_int32),
                ("y_dtype", C.c_int32), ("eps", C.c_float)]


class mebptt_int8_desc(C.Structure):
    _fields_ = [("M", C.c_int64), ("N", C.c_int32), ("K", C.c_int32), ("out_dtype", C.c_int32)]


class mebptt_conv_desc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("t", "B", "C", "taps", "dtype", "silu")]


class mebptt_scan_desc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("t", "B", "D", "N", "G", "dtype", "softplus", "stretch")]


class mebptt_scan_inputs(C.Structure):
    _fields_ = ([(n, mebptt_seq) for n in ("u", "delta", "z", "Bm", "Cm")]
                + [(n, C.c_void_p) for n in ("A", "skip", "delta_bias", "lengths", "h0")])


class mebptt_scan_grads(C.Structure):
    _fields_ = ([(n, mebptt_seq) for n in ("du", "ddelta", "dz", "dBm", "dCm")]
                + [(n, C.c_void_p) for n in ("dA", "dskip", "ddelta_bias", "dh0")])


class mebptt_delta_desc(C.Structure):
    _fields_ = ([(n, C.c_int32) for n in ("t", "B", "Hk", "H", "dk", "dv", "dtype", "activate", "normalise", "stretch")]
                + [("scale", C.c_float), ("eps", C.c_float)])


class mebptt_delta_inputs(C.Structure):
    _fields_ = [(n, mebptt_seq) for n in ("q", "k", "v", "a", "b")] + [(n, C.c_void_p) for n in ("A", "a_bias", "lengths", "h0")]


class mebptt_delta_grads(C.Structure):
    _fields_ = [(n, mebptt_seq) for n in ("dq", "dk", "dv", "db", "da")] + [(n, C.c_void_p) for n in ("dA", "da_bias", "dh0")]


class mebptt_join_desc(C.Structure):
    _fields_ = [("rows", C.c_int64), ("width", C.c_int32), ("group", C.c_int32), ("x_dtype", C.c_int32), ("residual_dtype", C.c_int32),
                ("scale", C.c_float), ("eps", C.c_float), ("again", C.c_int32), ("reserved", C.c_int32)]


ADAMW_NO_DECAY = 1


class mebptt_adamw_tensor(C.Structure):
    _fields_ = ([(n, C.c_void_p) for n in ("param", "grad", "m", "v", "m_scale", "v_scale", "copy")] + [("n", C.c_int64)]
                + [(n, C.c_int32) for n in ("grad_dtype", "state_dtype", "flags", "reserved")])


class mebptt_adamw_desc(C.Structure):
    _fields_ = ([(n, C.c_double) for n in ("rate", "beta1", "beta2", "eps", "decay")]
                + [("step", C.c_int64), ("seed", C.c_uint32), ("reserved", C.c_int32)])


# name -> (restype, argtypes): every symbol the header declares
_P = C.c_void_p
_DESC = C.POINTER(mebptt_lstm_desc)
SIGNATURES = {
    "mebptt_plan": (C.c_int, [C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.POINTER(_P)]),
    "mebptt_plan_from_policy": (C.c_int, [C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.POINTER(mebptt_decision),
                                          C.c_size_t, C.POINTER(_P)]),
    "mebptt_plan_chen_sqrt": (C.c_int, [C.c_int32, C.c_int32, C.c_int32, C.POINTER(_P)]),
    "mebptt_plan_chen_recursive": (C.c_int, [C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.POINTER(_P)]),
    "mebptt_plan_free": (None, [_P]),
    "mebptt_chain_plan": (C.c_int, [C.POINTER(mebptt_layer), C.c_int32, C.c_int32, C.POINTER(_P)]),
    "mebptt_chain_plan_free": (None, [_P]),
    "mebptt_chain_cost": (C.c_int64, [_P, C.c_int32, C.c_int32, C.c_int32]),
    "mebptt_chain_split": (C.c_int32, [_P, C.c_int32, C.c_int32, C.c_int32]),
    "mebptt_chain_plan_forward_cost": (C.c_int64, [_P]),
    "mebptt_chain_plan_peak": (C.c_int32, [_P]),
    "mebptt_chain_plan_schedule": (C.POINTER(mebptt_chain_op), [_P, C.POINTER(C.c_size_t)]),
    "mebptt_chain_plan_layers": (C.POINTER(mebptt_layer), [_P, C.POINTER(C.c_int32)]),
    "mebptt_chain_layers": (C.c_int, [C.POINTER(mebptt_chain_desc), C.POINTER(mebptt_layer)]),
    "mebptt_chain_workspace_bytes": (C.c_size_t, [C.POINTER(mebptt_chain_desc)]),
    "mebptt_chain_run": (C.c_int, [C.POINTER(mebptt_chain_desc), _P, C.POINTER(_P), C.POINTER(_P), _P, _P, _P, C.c_size_t,
                                   _P, C.c_size_t, C.POINTER(_P), C.POINTER(_P), _P, _P, C.POINTER(mebptt_chain_stats), _P]),
    "mebptt_plan_cost": (C.POINTER(C.c_int64), [_P, C.c_int32]),
    "mebptt_plan_split": (C.POINTER(C.c_int32), [_P, C.c_int32]),
    "mebptt_plan_choice": (C.POINTER(C.c_uint8), [_P]),
    "mebptt_plan_length": (C.c_int32, [_P]),
    "mebptt_plan_budget": (C.c_int32, [_P]),
    "mebptt_plan_kind": (C.c_int32, [_P]),
    "mebptt_plan_forward_ops": (C.c_int64, [_P]),
    "mebptt_plan_peak": (C.c_int32, [_P]),
    "mebptt_plan_schedule": (C.POINTER(mebptt_op), [_P, C.POINTER(C.c_size_t)]),
    "mebptt_unit_bytes": (C.c_size_t, [_DESC]),
    "mebptt_slot_pool_bytes": (C.c_size_t, [_DESC, _P]),
    "mebptt_workspace_bytes": (C.c_size_t, [_DESC]),
    "mebptt_units_for_bytes": (C.c_int32, [_DESC, C.c_int32, C.c_size_t]),
    "mebptt_run": (C.c_int, [_DESC, _P] + [_P] * 7 + [_P, C.c_size_t, _P, C.c_size_t] + [_P] * 7
                   + [C.POINTER(mebptt_stats), _P]),
    "mebptt_prepare": (C.c_int, [_DESC] + [_P] * 3 + [_P, C.c_size_t, _P]),
    "mebptt_run_prepared": (C.c_int, [_DESC, _P] + [_P] * 4 + [_P, C.c_size_t, _P, C.c_size_t] + [_P] * 7
                            + [C.POINTER(mebptt_stats), _P]),
    "mebptt_run_static": (C.c_int, [_DESC, _P] + [_P] * 7 + [_P, C.c_size_t] + [_P] * 7
                          + [C.POINTER(mebptt_stats), _P]),
    "mebptt_static_workspace_bytes": (C.c_size_t, []),
    "mebptt_run_status": (C.c_int, [_DESC, _P, C.c_size_t, _P, C.POINTER(C.c_int32)]),
    "mebptt_forward_chain_enable": (C.c_int, [C.c_int32]),
    "mebptt_resident_wait_limit": (C.c_int, [C.c_int64]),
    "mebptt_resident_patience": (C.c_int, [C.c_int64]),
    "mebptt_shutdown": (C.c_int, []),
    "mebptt_norm_forward": (C.c_int, [C.POINTER(mebptt_norm_desc), _P, C.c_int64, _P, C.c_int64, _P, _P, C.c_int64, _P, _P,
                                      C.c_int64, _P, _P]),
    "mebptt_norm_workspace_bytes": (C.c_size_t, [C.POINTER(mebptt_norm_desc)]),
    "mebptt_norm_backward": (C.c_int, [C.POINTER(mebptt_norm_desc), _P, C.c_int64, _P, _P, _P, C.c_int64, _P, C.c_int64, _P,
                                       C.c_int64, _P, C.c_int64, _P, _P, C.c_size_t, _P]),
    "mebptt_int8_workspace_bytes": (C.c_size_t, [C.POINTER(mebptt_int8_desc)]),
    "mebptt_int8_product": (C.c_int, [C.POINTER(mebptt_int8_desc), _P, C.c_int64, _P, _P, C.c_int64, _P, _P, _P, C.c_int64, _P,
                                      C.c_size_t, _P]),
    "mebptt_conv_forward": (C.c_int, [C.POINTER(mebptt_conv_desc), mebptt_seq, _P, _P, _P, _P, mebptt_seq, _P, _P]),
    "mebptt_conv_workspace_bytes": (C.c_size_t, [C.POINTER(mebptt_conv_desc)]),
    "mebptt_conv_backward": (C.c_int, [C.POINTER(mebptt_conv_desc), mebptt_seq, _P, _P, _P, _P, mebptt_seq, _P, mebptt_seq, _P,
                                       _P, _P, _P, C.c_size_t, _P]),
    "mebptt_conv_step": (C.c_int, [C.POINTER(mebptt_conv_desc), _P, C.c_int64, _P, _P, _P, C.c_int64, _P, _P, C.c_int64, _P,
                                   _P]),
    "mebptt_scan_state_bytes": (C.c_size_t, [C.POINTER(mebptt_scan_desc)]),
    "mebptt_scan_workspace_bytes": (C.c_size_t, [C.POINTER(mebptt_scan_desc), C.c_int32]),
    "mebptt_scan_forward": (C.c_int, [C.POINTER(mebptt_scan_desc), C.POINTER(mebptt_scan_inputs), mebptt_seq, _P, _P, C.c_size_t,
                                      _P, C.c_size_t, _P]),
    "mebptt_scan_backward": (C.c_int, [C.POINTER(mebptt_scan_desc), C.POINTER(mebptt_scan_inputs), mebptt_seq, _P, _P, C.c_size_t,
                                       C.POINTER(mebptt_scan_grads), _P, C.c_size_t, _P]),
    "mebptt_scan_step": (C.c_int, [C.POINTER(mebptt_scan_desc), C.POINTER(mebptt_scan_inputs), _P, C.c_int64, _P, mebptt_seq, _P,
                                   _P]),
    "mebptt_delta_state_bytes": (C.c_size_t, [C.POINTER(mebptt_delta_desc)]),
    "mebptt_delta_workspace_bytes": (C.c_size_t, [C.POINTER(mebptt_delta_desc), C.c_int32]),
    "mebptt_delta_forward": (C.c_int, [C.POINTER(mebptt_delta_desc), C.POINTER(mebptt_delta_inputs), mebptt_seq, _P, _P, C.c_size_t,
                                       _P, C.c_size_t, _P]),
    "mebptt_delta_backward": (C.c_int, [C.POINTER(mebptt_delta_desc), C.POINTER(mebptt_delta_inputs), mebptt_seq, _P, _P, C.c_size_t,
                                        C.POINTER(mebptt_delta_grads), _P, C.c_size_t, _P]),
    "mebptt_delta_step": (C.c_int, [C.POINTER(mebptt_delta_desc), C.POINTER(mebptt_delta_inputs), _P, C.c_int64, _P, mebptt_seq, _P,
                                    _P]),
    "mebptt_join_forward": (C.c_int, [C.POINTER(mebptt_join_desc), _P, C.c_int64, _P, C.c_int64, _P, _P, C.c_int64, _P, _P, C.c_int64, _P,
                                      C.c_int64, _P, _P, _P]),
    "mebptt_join_workspace_bytes": (C.c_size_t, [C.POINTER(mebptt_join_desc)]),
    "mebptt_join_backward": (C.c_int, [C.POINTER(mebptt_join_desc), _P, C.c_int64, _P, C.c_int64, _P, _P, C.c_int64, _P, _P, _P, _P, C.c_int64,
                                       _P, C.c_int64, _P, C.c_int64, _P, C.c_int64, _P, _P, C.c_int64, _P, _P, C.c_size_t, _P]),
    "mebptt_adamw_table_bytes": (C.c_size_t, [C.POINTER(mebptt_adamw_tensor), C.c_int32]),
    "mebptt_adamw_prepare": (C.c_int, [C.POINTER(mebptt_adamw_tensor), C.c_int32, _P, C.c_size_t, _P]),
    "mebptt_adamw_workspace_bytes": (C.c_size_t, [C.POINTER(mebptt_adamw_tensor), C.c_int32]),
    "mebptt_adamw_norm": (C.c_int, [C.POINTER(mebptt_adamw_tensor), C.c_int32, _P, C.c_size_t, C.c_float, _P, _P, C.c_size_t, _P]),
    "mebptt_adamw_step": (C.c_int, [C.POINTER(mebptt_adamw_desc), C.POINTER(mebptt_adamw_tensor), C.c_int32, _P, C.c_size_t, _P, _P, _P, _P]),
    "mebptt_adamw_unpack": (C.c_int, [_P, _P, C.c_int64, C.c_int32, _P, C.c_int32, _P]),
    "mebptt_null_launch_us": (C.c_int, [C.c_int32, _P, C.POINTER(C.c_double)]),
    "mebptt_measure_sync": (C.c_int, [C.c_int32, C.c_int32, _P, C.POINTER(C.c_double), C.POINTER(C.c_int32)]),
    "mebptt_chunk_steps": (C.c_int32, [_DESC]),
    "mebptt_stage_steps": (C.c_int32, [_DESC]),
    "mebptt_measure_forward_stream": (C.c_int, [_DESC, _P, C.c_size_t, C.c_int32, _P, C.POINTER(C.c_double), C.POINTER(C.c_double)]),
    "mebptt_bracket_overhead_us": (C.c_int, [C.c_double, C.c_int32, _P, C.POINTER(C.c_double), C.POINTER(C.c_double)]),
    "mebptt_measure_gemms": (C.c_int, [_DESC, _P, C.c_size_t, C.c_int32, _P, C.POINTER(C.c_double), C.POINTER(C.c_double)]),
    "mebptt_profile_enable": (C.c_int, [C.c_int32]),
    "mebptt_profile_collect": (C.c_int, [C.POINTER(mebptt_profile)]),
    "mebptt_last_error": (C.c_char_p, []),
    "mebptt_version": (C.c_char_p, []),
}


def lib() -> C.CDLL:
    """Loads the library on first use.  Raises if it is missing: there is no other code path."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} is missing: build it with `python -m paper_1606_03401_amd.build`")
        l = C.CDLL(_LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(l, name)
            fn.restype = res
            fn.argtypes = args
        _lib = l
    return _lib


def mebptt_last_error() -> str:
    return lib().mebptt_last_error().decode()


def mebptt_version() -> str:
    return lib().mebptt_version().decode()


def _check(rc: int) -> None:
    if rc != OK:
        raise MebpttError(rc, mebptt_last_error())


class Plan:
    """Owner of a ``mebptt_plan_t*``; the table properties are read-only numpy views of the
    library's memory (valid while this object lives)."""

    def __init__(self, handle: int):
        self.handle = handle

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.mebptt_plan_free(self.handle)
            self.handle = None

    @property
    def t(self) -> int:
        return lib().mebptt_plan_length(self.handle)

    @property
    def m(self) -> int:
        return lib().mebptt_plan_budget(self.handle)

    @property
    def kind(self) -> int:
        return lib().mebptt_plan_kind(self.handle)

    @property
    def forward_ops(self) -> int:
        return lib().mebptt_plan_forward_ops(self.handle)

    @property
    def peak(self) -> int:
        return lib().mebptt_plan_peak(self.handle)

    def _table(self, ptr, dtype):
        if not ptr:
            return None
        shape = (self.t + 1, self.m + 1)
        a = np.ctypeslib.as_array(ptr, shape=shape)
        a = a.view(dtype)
        a.flags.writeable = False
        return a

    def cost(self, which: int = 0):
        return self._table(lib().mebptt_plan_cost(self.handle, which), np.int64)

    def split(self, which: int = 0):
        return self._table(lib().mebptt_plan_split(self.handle, which), np.int32)

    def choice(self):
        return self._table(lib().mebptt_plan_choice(self.handle), np.uint8)

    def schedule(self) -> np.ndarray:
        """Structured array with fields op, step, count, src, dst, keep, prev (a copy)."""
        n = C.c_size_t(0)
        ptr = lib().mebptt_plan_schedule(self.handle, C.byref(n))
        dt = np.dtype([(f, np.int32) for f, _ in mebptt_op._fields_])
        if n.value == 0:
            return np.zeros(0, dt)
        raw = np.ctypeslib.as_array(C.cast(ptr, C.POINTER(C.c_int32)), shape=(n.value, 7))
        return raw.copy().view(dt).reshape(n.value)


def mebptt_plan(t: int, m: int, kind: int, alpha: int = 4, beta: int = 3) -> Plan:
    out = _P()
    _check(lib().mebptt_plan(t, m, kind, alpha, beta, C.byref(out)))
    return Plan(out.value)


class ChainPlan:
    """Owner of a ``mebptt_chain_plan_t*`` (non-homogeneous chain; planning only)."""

    def __init__(self, handle: int, n: int, m: int):
        self.handle, self.n, self.m = handle, n, m

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.mebptt_chain_plan_free(self.handle)
            self.handle = None

    def cost(self, t: int, m: int, x: int) -> int:
        return lib().mebptt_chain_cost(self.handle, t, m, x)

    def split(self, t: int, m: int, x: int) -> int:
        return lib().mebptt_chain_split(self.handle, t, m, x)

    @property
    def forward_cost(self) -> int:
        return lib().mebptt_chain_plan_forward_cost(self.handle)

    @property
    def peak(self) -> int:
        return lib().mebptt_chain_plan_peak(self.handle)

    def schedule(self) -> np.ndarray:
        n = C.c_size_t(0)
        ptr = lib().mebptt_chain_plan_schedule(self.handle, C.byref(n))
        dt = np.dtype([(f, np.int32) for f, _ in mebptt_chain_op._fields_])
        if n.value == 0:
            return np.zeros(0, dt)
        raw = np.ctypeslib.as_array(C.cast(ptr, C.POINTER(C.c_int32)), shape=(n.value, 5))
        return raw.copy().view(dt).reshape(n.value)


def mebptt_chain_plan(layers, m: int) -> ChainPlan:
    """`layers`: sequence of (cost, state_units, work_units)."""
    arr = (mebptt_layer * max(len(layers), 1))(*[mebptt_layer(int(u), int(s), int(p)) for u, s, p in layers])
    out = _P()
    _check(lib().mebptt_chain_plan(arr, len(layers), m, C.byref(out)))
    return ChainPlan(out.value, len(layers), m)


def mebptt_plan_from_policy(t: int, m: int, decisions, alpha: int = 4, beta: int = 3) -> Plan:
    """`decisions`: sequence of (store, y) pairs, store = STORE_HIDDEN or STORE_INTERNAL."""
    arr = (mebptt_decision * max(len(decisions), 1))(*[mebptt_decision(int(s), int(y)) for s, y in decisions])
    out = _P()
    _check(lib().mebptt_plan_from_policy(t, m, alpha, beta, arr, len(decisions), C.byref(out)))
    return Plan(out.value)


def mebptt_plan_chen_sqrt(t: int, alpha: int = 4, beta: int = 3) -> Plan:
    out = _P()
    _check(lib().mebptt_plan_chen_sqrt(t, alpha, beta, C.byref(out)))
    return Plan(out.value)


def mebptt_plan_chen_recursive(t: int, k: int, alpha: int = 4, beta: int = 3) -> Plan:
    out = _P()
    _check(lib().mebptt_plan_chen_recursive(t, k, alpha, beta, C.byref(out)))
    return Plan(out.value)


def make_desc(B: int, I: int, H: int, t: int, gemm_dtype: int, loss: int, dy_first_step: int = 1,
              cell: int = CELL_LSTM) -> mebptt_lstm_desc:
    return mebptt_lstm_desc(B, I, H, t, gemm_dtype, loss, dy_first_step, cell)


def mebptt_unit_bytes(desc: mebptt_lstm_desc) -> int:
    return lib().mebptt_unit_bytes(C.byref(desc))


def mebptt_slot_pool_bytes(desc: mebptt_lstm_desc, plan: Plan) -> int:
    return lib().mebptt_slot_pool_bytes(C.byref(desc), plan.handle)


def mebptt_workspace_bytes(desc: mebptt_lstm_desc) -> int:
    return lib().mebptt_workspace_bytes(C.byref(desc))


def mebptt_units_for_bytes(desc: mebptt_lstm_desc, kind: int, budget_bytes: int) -> int:
    return lib().mebptt_units_for_bytes(C.byref(desc), kind, budget_bytes)


def mebptt_profile_enable(every_n: int) -> None:
    _check(lib().mebptt_profile_enable(every_n))


def mebptt_profile_collect() -> mebptt_profile:
    out = mebptt_profile()
    _check(lib().mebptt_profile_collect(C.byref(out)))
    return out


def _ptr(t) -> Optional[int]:
    """Device pointer of a torch tensor (or None)."""
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors handed to mebptt_run must be contiguous")
    return t.data_ptr()


def mebptt_run(desc: mebptt_lstm_desc, plan: Plan, W_ih, W_hh, b, x, dy, h0, c0, slots, workspace,
               dW_ih, dW_hh, db, dh0, dc0, dx=None, y_out=None, stream: Optional[int] = None) -> mebptt_stats:
    """Enqueues one gradient step.  Tensor arguments are torch CUDA tensors (float32; `slots` and
    `workspace` are uint8 buffers); `stream` is a raw hipStream_t (default: torch's current stream).
    Returns the host-side statistics.  The caller synchronises."""
    if stream is None:
        import torch
        stream = torch.cuda.current_stream().cuda_stream
    stats = mebptt_stats()
    rc = lib().mebptt_run(C.byref(desc), plan.handle, _ptr(W_ih), _ptr(W_hh), _ptr(b), _ptr(x), _ptr(dy), _ptr(h0),
                          _ptr(c0), _ptr(slots), slots.numel() * slots.element_size(), _ptr(workspace),
                          workspace.numel() * workspace.element_size(), _ptr(dW_ih), _ptr(dW_hh), _ptr(db), _ptr(dh0),
                          _ptr(dc0), _ptr(dx), _ptr(y_out), C.byref(stats), stream)
    _check(rc)
    return stats


def _stream(stream: Optional[int]) -> int:
    if stream is None:
        import torch
        stream = torch.cuda.current_stream().cuda_stream
    return stream


def _nbytes(t) -> int:
    return t.numel() * t.element_size()


def mebptt_prepare(desc: mebptt_lstm_desc, W_ih, W_hh, b, workspace, stream: Optional[int] = None) -> None:
    """Builds the operand copies of the weights inside `workspace` (see mebptt_run_prepared)."""
    _check(lib().mebptt_prepare(C.byref(desc), _ptr(W_ih), _ptr(W_hh), _ptr(b), _ptr(workspace), _nbytes(workspace),
                                _stream(stream)))


def mebptt_run_prepared(desc: mebptt_lstm_desc, plan: Plan, x, dy, h0, c0, slots, workspace, dW_ih, dW_hh, db, dh0,
                        dc0, dx=None, y_out=None, stream: Optional[int] = None) -> mebptt_stats:
    """mebptt_run on a workspace that mebptt_prepare has filled for these weights."""
    stats = mebptt_stats()
    _check(lib().mebptt_run_prepared(C.byref(desc), plan.handle, _ptr(x), _ptr(dy), _ptr(h0), _ptr(c0), _ptr(slots),
                                     _nbytes(slots), _ptr(workspace), _nbytes(workspace), _ptr(dW_ih), _ptr(dW_hh),
                                     _ptr(db), _ptr(dh0), _ptr(dc0), _ptr(dx), _ptr(y_out), C.byref(stats),
                                     _stream(stream)))
    return stats


def mebptt_run_static(desc: mebptt_lstm_desc, plan: Plan, W_ih, W_hh, b, x, dy, h0, c0, slots, dW_ih, dW_hh, db, dh0,
                      dc0, dx=None, y_out=None, stream: Optional[int] = None) -> mebptt_stats:
    """mebptt_run with the workspace in the library's static device array: allocates nothing."""
    stats = mebptt_stats()
    _check(lib().mebptt_run_static(C.byref(desc), plan.handle, _ptr(W_ih), _ptr(W_hh), _ptr(b), _ptr(x), _ptr(dy),
                                   _ptr(h0), _ptr(c0), _ptr(slots), _nbytes(slots), _ptr(dW_ih), _ptr(dW_hh), _ptr(db),
                                   _ptr(dh0), _ptr(dc0), _ptr(dx), _ptr(y_out), C.byref(stats), _stream(stream)))
    return stats


def mebptt_static_workspace_bytes() -> int:
    return lib().mebptt_static_workspace_bytes()


def mebptt_run_status(desc: mebptt_lstm_desc, workspace, stream: Optional[int] = None) -> int:
    """Waits for the stream and returns the status word of the last run on `workspace` (0 = fine)."""
    out = C.c_int32(0)
    _check(lib().mebptt_run_status(C.byref(desc), _ptr(workspace), _nbytes(workspace), _stream(stream), C.byref(out)))
    return out.value


def mebptt_forward_chain_enable(on: bool) -> None:
    _check(lib().mebptt_forward_chain_enable(1 if on else 0))


def mebptt_resident_wait_limit(ticks: int) -> None:
    _check(lib().mebptt_resident_wait_limit(int(ticks)))


def mebptt_resident_patience(ticks: int) -> None:
    _check(lib().mebptt_resident_patience(int(ticks)))


def mebptt_shutdown() -> None:
    _check(lib().mebptt_shutdown())


def mebptt_null_launch_us(launches: int = 2000, stream: Optional[int] = None) -> float:
    out = C.c_double(0.0)
    _check(lib().mebptt_null_launch_us(launches, _stream(stream), C.byref(out)))
    return out.value


def mebptt_measure_sync(variant: int, iters: int = 3000, stream: Optional[int] = None):
    """(microseconds per synchronisation, status) of the stand-alone synchronisation kernel."""
    out, status = C.c_double(0.0), C.c_int32(0)
    _check(lib().mebptt_measure_sync(variant, iters, _stream(stream), C.byref(out), C.byref(status)))
    return out.value, status.value


def mebptt_bracket_overhead_us(kernel_us: float, reps: int = 200, stream: Optional[int] = None):
    """(time per launch back to back, mean time of the same launch inside its own event pair), in us."""
    a, b = C.c_double(0.0), C.c_double(0.0)
    _check(lib().mebptt_bracket_overhead_us(float(kernel_us), reps, _stream(stream), C.byref(a), C.byref(b)))
    return a.value, b.value


def make_chain_desc(widths, B: int, unit_bytes: int) -> mebptt_chain_desc:
    """Descriptor of a chain of dense tanh layers; keeps the widths array alive on the object."""
    arr = (C.c_int32 * len(widths))(*[int(v) for v in widths])
    d = mebptt_chain_desc(len(widths) - 1, B, arr, unit_bytes)
    d._widths_keepalive = arr
    return d


def mebptt_chain_layers(desc: mebptt_chain_desc):
    """The (cost, state_units, work_units) table of the chain, as mebptt_chain_plan takes it."""
    out = (mebptt_layer * desc.n)()
    _check(lib().mebptt_chain_layers(C.byref(desc), out))
    return [(l.cost, l.state_units, l.work_units) for l in out]


def mebptt_chain_workspace_bytes(desc: mebptt_chain_desc) -> int:
    return lib().mebptt_chain_workspace_bytes(C.byref(desc))


def mebptt_chain_run(desc: mebptt_chain_desc, plan: ChainPlan, W, b, x0, dy, pool, workspace, dW, db, dx0=None,
                     y_out=None, stream: Optional[int] = None) -> mebptt_chain_stats:
    """Enqueues one gradient step of the chain.  W, b, dW, db: lists of n torch tensors (b entries
    may be None); the others torch tensors; `pool` may be None when the plan memorises nothing."""
    n = desc.n
    arr = lambda ts: (_P * n)(*[_ptr(t) for t in ts])
    stats = mebptt_chain_stats()
    rc = lib().mebptt_chain_run(C.byref(desc), plan.handle, arr(W), arr(b), _ptr(x0), _ptr(dy), _ptr(pool),
                                0 if pool is None else _nbytes(pool), _ptr(workspace), _nbytes(workspace), arr(dW),
                                arr(db), _ptr(dx0), _ptr(y_out), C.byref(stats), _stream(stream))
    _check(rc)
    return stats


def mebptt_measure_forward_stream(desc: mebptt_lstm_desc, workspace, reps: int = 50, stream: Optional[int] = None):
    """(us per launch, bytes read per launch) of the kernel that only streams a forward launch's operand panels."""
    a, b = C.c_double(0.0), C.c_double(0.0)
    _check(lib().mebptt_measure_forward_stream(C.byref(desc), _ptr(workspace), _nbytes(workspace), reps, _stream(stream),
                                               C.byref(a), C.byref(b)))
    return a.value, b.value


def mebptt_chunk_steps(desc: mebptt_lstm_desc) -> int:
    n = lib().mebptt_chunk_steps(C.byref(desc))
    if n < 0:
        _check(n)
    return n


def mebptt_stage_steps(desc: mebptt_lstm_desc) -> int:
    n = lib().mebptt_stage_steps(C.byref(desc))
    if n < 0:
        _check(n)
    return n


def mebptt_measure_gemms(desc: mebptt_lstm_desc, workspace, reps: int = 20, stream: Optional[int] = None):
    """(wgrad_us, dgrad_us): the two time-batched GEMMs of one full chunk, alone on the device."""
    a, b = C.c_double(0.0), C.c_double(0.0)
    _check(lib().mebptt_measure_gemms(C.byref(desc), _ptr(workspace), _nbytes(workspace), reps, _stream(stream),
                                      C.byref(a), C.byref(b)))
    return a.value, b.value


# ---- operators of a selective state space block ------------------------------------------------------
#
# Tensors are checked here for type, shape and device, which the library cannot see; it checks everything else.  Sequences
# are [t, B, channels], of any strides over t and B; states, parameters and their gradients are contiguous.  Single tokens come
# in calls of a few microseconds, so the checks are one comparison each and say what was wrong only when something was.

_torch = None
_DTYPES = ()
_current_device = _current_stream = None


def _load_torch():
    global _torch, _DTYPES, _current_device, _current_stream
    import torch
    torch.cuda.init()
    _DTYPES = (torch.float32, torch.bfloat16, torch.int8)
    _current_device = torch._C._cuda_getDevice
    # the raw handle without a Stream object around it
    _current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)
    _torch = torch      # last: whoever finds it goes on with all the others


def _dtype(code: int):
    if not 0 <= code < 3:
        raise ValueError(f"unknown dtype {code}")
    return _DTYPES[code]


def _gpu(t) -> int:
    """Index of the GPU that holds `t`, the first tensor of a call."""
    dev = -1 if t is None else t.get_device()
    if dev < 0:
        raise ValueError("tensors in a GPU's memory are needed")
    if _torch is None:
        _load_torch()
    return dev


def _wrong(t, name: str, shape, dtype, dev: int):
    if t is None:
        raise ValueError(f"{name} is required")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, {tuple(shape)} is needed")
    if t.dtype is not dtype:
        raise ValueError(f"{name} has type {t.dtype}, {dtype} is needed")
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, the call's other tensors on GPU {dev}")
    raise ValueError(f"{name} must be contiguous" if not t.is_contiguous() else f"{name} is not usable")


def _whole(t, name: str, shape, dtype, dev: int) -> int:
    """Pointer of a contiguous tensor."""
    if t is None or t.shape != shape or t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous():
        _wrong(t, name, shape, dtype, dev)
    return t.data_ptr()


def _maybe(t, name: str, shape, dtype, dev: int) -> Optional[int]:
    return None if t is None else _whole(t, name, shape, dtype, dev)


def _rows(t, name: str, rows: int, width: int, dtype, dev: int):
    """(pointer, row stride) of a [rows, width] tensor whose rows are contiguous."""
    if t is None or t.shape != (rows, width) or t.dtype is not dtype or t.get_device() != dev:
        _wrong(t, name, (rows, width), dtype, dev)
    ld, one = t.stride()
    if one != 1 and width > 1 and rows:
        raise ValueError(f"rows of {name} must be contiguous")
    return t.data_ptr(), ld if rows > 1 else width


def _maybe_rows(t, name: str, rows: int, width: int, dtype, dev: int):
    return (None, 0) if t is None else _rows(t, name, rows, width, dtype, dev)


def _seq(t, name: str, steps: int, B: int, channels: int, dtype, dev: int) -> mebptt_seq:
    """A [t, B, channels] tensor whose channels are contiguous."""
    if t is None or t.shape != (steps, B, channels) or t.dtype is not dtype or t.get_device() != dev:
        _wrong(t, name, (steps, B, channels), dtype, dev)
    st, sb, one = t.stride()
    if one != 1 and channels > 1 and steps and B:
        raise ValueError(f"the channels of {name} must be contiguous")
    # the stride of an axis of one is whatever it is: never used, and not to be looked at
    return mebptt_seq(t.data_ptr() or None, st if steps > 1 else B * channels, sb if B > 1 else channels)


def _maybe_seq(t, name: str, steps: int, B: int, channels: int, dtype, dev: int) -> mebptt_seq:
    return mebptt_seq(None, 0, 0) if t is None else _seq(t, name, steps, B, channels, dtype, dev)


def _room(t, name: str, dev: int):
    """(pointer, bytes) of a workspace; None where the call needs none."""
    if t is None:
        return None, 0
    if t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous and on the GPU of the call's other tensors")
    return t.data_ptr(), t.numel() * t.element_size()


def _call(dev: int, stream: Optional[int], fn, *args) -> None:
    """The library's call on the tensors' GPU and `stream` (default: that GPU's current one)."""
    if dev != _current_device():
        with _torch.cuda.device(dev):
            return _call(dev, stream, fn, *args)
    rc = fn(*args, _current_stream(dev) if stream is None else stream)
    if rc != OK:
        _check(rc)


def make_norm_desc(rows: int, width: int, x_dtype: int, residual_dtype: int, y_dtype: int, eps: float = 1e-5) -> mebptt_norm_desc:
    return mebptt_norm_desc(rows, width, x_dtype, residual_dtype, y_dtype, eps)


def mebptt_norm_workspace_bytes(desc: mebptt_norm_desc) -> int:
    return lib().mebptt_norm_workspace_bytes(C.byref(desc))


def mebptt_norm_forward(desc: mebptt_norm_desc, x, residual, weight, y, y_scale=None, residual_out=None, rstd=None,
                        stream: Optional[int] = None) -> None:
    """r = x + residual, y = RMS norm of r times `weight`; residual_out receives r, rstd the rows' 1 / rms (for the backward call),
    y_scale the rows' scales of an 8-bit y."""
    dev, M, W = _gpu(x), desc.rows, desc.width
    f32, rt = _DTYPES[0], _dtype(desc.residual_dtype)
    _call(dev, stream, lib().mebptt_norm_forward, C.byref(desc), *_rows(x, "x", M, W, _dtype(desc.x_dtype), dev),
          *_maybe_rows(residual, "residual", M, W, rt, dev), _maybe(weight, "weight", (W,), f32, dev),
          *_rows(y, "y", M, W, _dtype(desc.y_dtype), dev), _maybe(y_scale, "y_scale", (M,), f32, dev),
          *_maybe_rows(residual_out, "residual_out", M, W, rt, dev), _maybe(rstd, "rstd", (M,), f32, dev))


def mebptt_norm_backward(desc: mebptt_norm_desc, r, weight, rstd, dy, dresidual_out, dx, dresidual, dweight, workspace,
                         stream: Optional[int] = None) -> None:
    """Gradients of mebptt_norm_forward from r (its residual_out, or x without a residual) and rstd."""
    dev, M, W = _gpu(r), desc.rows, desc.width
    f32, xt, rt = _DTYPES[0], _dtype(desc.x_dtype), _dtype(desc.residual_dtype)
    _call(dev, stream, lib().mebptt_norm_backward, C.byref(desc), *_rows(r, "r", M, W, rt, dev), _maybe(weight, "weight", (W,), f32, dev),
          _whole(rstd, "rstd", (M,), f32, dev), *_rows(dy, "dy", M, W, xt, dev),
          *_maybe_rows(dresidual_out, "dresidual_out", M, W, rt, dev), *_maybe_rows(dx, "dx", M, W, xt, dev),
          *_maybe_rows(dresidual, "dresidual", M, W, rt, dev), _maybe(dweight, "dweight", (W,), f32, dev),
          *_room(workspace, "workspace", dev))


def make_int8_desc(M: int, N: int, K: int, out_dtype: int) -> mebptt_int8_desc:
    return mebptt_int8_desc(M, N, K, out_dtype)


def mebptt_int8_workspace_bytes(desc: mebptt_int8_desc) -> int:
    return lib().mebptt_int8_workspace_bytes(C.byref(desc))


def mebptt_int8_product(desc: mebptt_int8_desc, a, a_scale, b, b_scale, bias, out, workspace=None, stream: Optional[int] = None) -> None:
    """out = a_scale[:, None] * b_scale * (a @ b.T) + bias: a [M, K] and b [N, K] int8, scales and bias float32."""
    dev, M, N, K = _gpu(a), desc.M, desc.N, desc.K
    f32, i8 = _DTYPES[0], _DTYPES[2]
    _call(dev, stream, lib().mebptt_int8_product, C.byref(desc), *_rows(a, "a", M, K, i8, dev), _whole(a_scale, "a_scale", (M,), f32, dev),
          *_rows(b, "b", N, K, i8, dev), _whole(b_scale, "b_scale", (N,), f32, dev), _maybe(bias, "bias", (N,), f32, dev),
          *_rows(out, "out", M, N, _dtype(desc.out_dtype), dev), *_room(workspace, "workspace", dev))


def make_conv_desc(t: int, B: int, C_: int, taps: int, dtype: int, silu: int = 1) -> mebptt_conv_desc:
    return mebptt_conv_desc(t, B, C_, taps, dtype, silu)


def mebptt_conv_workspace_bytes(desc: mebptt_conv_desc) -> int:
    return lib().mebptt_conv_workspace_bytes(C.byref(desc))


def _conv_params(desc, weight, bias, dev: int):
    return _whole(weight, "weight", (desc.C, desc.taps), _DTYPES[0], dev), _maybe(bias, "bias", (desc.C,), _DTYPES[0], dev)


def mebptt_conv_forward(desc: mebptt_conv_desc, x, weight, bias, lengths, state_in, y, state_out=None,
                        stream: Optional[int] = None) -> None:
    """Depthwise causal convolution of [t, B, C]; states are the last taps - 1 inputs, [B, taps - 1, C]."""
    dev, T = _gpu(x), _dtype(desc.dtype)
    shape, state = (desc.t, desc.B, desc.C), (desc.B, desc.taps - 1, desc.C)
    _call(dev, stream, lib().mebptt_conv_forward, C.byref(desc), _seq(x, "x", *shape, T, dev), *_conv_params(desc, weight, bias, dev),
          _maybe(lengths, "lengths", (desc.B,), _torch.int32, dev), _maybe(state_in, "state_in", state, T, dev),
          _seq(y, "y", *shape, T, dev), _maybe(state_out, "state_out", state, T, dev))


def mebptt_conv_backward(desc: mebptt_conv_desc, x, weight, bias, lengths, state_in, dy, dstate_out, dx, dweight, dbias, dstate_in,
                         workspace, stream: Optional[int] = None) -> None:
    dev, T = _gpu(x), _dtype(desc.dtype)
    shape, state = (desc.t, desc.B, desc.C), (desc.B, desc.taps - 1, desc.C)
    _call(dev, stream, lib().mebptt_conv_backward, C.byref(desc), _seq(x, "x", *shape, T, dev), *_conv_params(desc, weight, bias, dev),
          _maybe(lengths, "lengths", (desc.B,), _torch.int32, dev), _maybe(state_in, "state_in", state, T, dev),
          _seq(dy, "dy", *shape, T, dev), _maybe(dstate_out, "dstate_out", state, T, dev), _seq(dx, "dx", *shape, T, dev),
          _whole(dweight, "dweight", (desc.C, desc.taps), _DTYPES[0], dev), _maybe(dbias, "dbias", (desc.C,), _DTYPES[0], dev),
          _maybe(dstate_in, "dstate_in", state, T, dev), *_room(workspace, "workspace", dev))


def _pool(state_in, state_out, row, dtype, dev: int, needed: bool):
    """(pointer, slots, pointer) of a pool of states and of the pool that receives them."""
    if state_in is None and not needed:
        return None, 1 << 31, None
    shape = (state_in.shape[0] if state_in is not None and state_in.dim() else 0, *row)
    return _whole(state_in, "state_in", shape, dtype, dev), shape[0], _whole(state_out, "state_out", shape, dtype, dev)


def mebptt_conv_step(desc: mebptt_conv_desc, x, weight, bias, state_in, index, y, state_out, stream: Optional[int] = None) -> None:
    """One token: x, y [B, C]; state_in, state_out [slots, taps - 1, C] (one tensor or two); index [B] int32 names every sequence's
    slot, None: its own number."""
    dev, T = _gpu(x), _dtype(desc.dtype)
    B, Ch = desc.B, desc.C
    pin, slots, pout = _pool(state_in, state_out, (desc.taps - 1, Ch), T, dev, desc.taps > 1)
    _call(dev, stream, lib().mebptt_conv_step, C.byref(desc), *_rows(x, "x", B, Ch, T, dev), *_conv_params(desc, weight, bias, dev), pin,
          slots, _maybe(index, "index", (B,), _torch.int32, dev), *_rows(y, "y", B, Ch, T, dev), pout)


def make_scan_desc(t: int, B: int, D: int, N: int, G: int, dtype: int, softplus: int = 1, stretch: int = 64) -> mebptt_scan_desc:
    return mebptt_scan_desc(t, B, D, N, G, dtype, softplus, stretch)


def mebptt_scan_state_bytes(desc: mebptt_scan_desc) -> int:
    return lib().mebptt_scan_state_bytes(C.byref(desc))


def mebptt_scan_workspace_bytes(desc: mebptt_scan_desc, backward: bool) -> int:
    return lib().mebptt_scan_workspace_bytes(C.byref(desc), 1 if backward else 0)


def _scan_inputs(desc, u, delta, A, Bm, Cm, skip, z, delta_bias, lengths, h0, T, dev: int) -> mebptt_scan_inputs:
    f32, t, B, D, N, GN = _DTYPES[0], desc.t, desc.B, desc.D, desc.N, desc.G * desc.N
    return mebptt_scan_inputs(_seq(u, "u", t, B, D, T, dev), _seq(delta, "delta", t, B, D, T, dev), _maybe_seq(z, "z", t, B, D, T, dev),
                              _seq(Bm, "Bm", t, B, GN, T, dev), _seq(Cm, "Cm", t, B, GN, T, dev), _whole(A, "A", (D, N), f32, dev),
                              _maybe(skip, "skip", (D,), f32, dev), _maybe(delta_bias, "delta_bias", (D,), f32, dev),
                              _maybe(lengths, "lengths", (B,), _torch.int32, dev), _maybe(h0, "h0", (B, D, N), f32, dev))


def mebptt_scan_forward(desc: mebptt_scan_desc, u, delta, A, Bm, Cm, skip, z, delta_bias, lengths, h0, y, h_out=None, states=None,
                        workspace=None, stream: Optional[int] = None) -> None:
    """Selective scan.  u, delta, z, y [t, B, D]; Bm, Cm [t, B, G N]; A [D, N]; h0, h_out [B, D, N]; `states` (uint8) keeps what a
    backward call needs."""
    dev, T = _gpu(u), _dtype(desc.dtype)
    given = _scan_inputs(desc, u, delta, A, Bm, Cm, skip, z, delta_bias, lengths, h0, T, dev)
    _call(dev, stream, lib().mebptt_scan_forward, C.byref(desc), C.byref(given), _seq(y, "y", desc.t, desc.B, desc.D, T, dev),
          _maybe(h_out, "h_out", (desc.B, desc.D, desc.N), _DTYPES[0], dev), *_room(states, "states", dev),
          *_room(workspace, "workspace", dev))


def mebptt_scan_backward(desc: mebptt_scan_desc, u, delta, A, Bm, Cm, skip, z, delta_bias, lengths, h0, dy, dh_out, states, du, ddelta,
                         dA, dB, dC, dskip, dz, ddelta_bias, dh0, workspace, stream: Optional[int] = None) -> None:
    dev, T = _gpu(u), _dtype(desc.dtype)
    f32, t, B, D, N, GN = _DTYPES[0], desc.t, desc.B, desc.D, desc.N, desc.G * desc.N
    given = _scan_inputs(desc, u, delta, A, Bm, Cm, skip, z, delta_bias, lengths, h0, T, dev)
    grads = mebptt_scan_grads(_seq(du, "du", t, B, D, T, dev), _seq(ddelta, "ddelta", t, B, D, T, dev),
                              (_maybe_seq if z is None else _seq)(dz, "dz", t, B, D, T, dev), _seq(dB, "dB", t, B, GN, T, dev),
                              _seq(dC, "dC", t, B, GN, T, dev), _whole(dA, "dA", (D, N), f32, dev),
                              _maybe(dskip, "dskip", (D,), f32, dev), _maybe(ddelta_bias, "ddelta_bias", (D,), f32, dev),
                              _maybe(dh0, "dh0", (B, D, N), f32, dev))
    _call(dev, stream, lib().mebptt_scan_backward, C.byref(desc), C.byref(given), _seq(dy, "dy", t, B, D, T, dev),
          _maybe(dh_out, "dh_out", (B, D, N), f32, dev), *_room(states, "states", dev), C.byref(grads), *_room(workspace, "workspace", dev))


def _token(t, name: str, B: int, channels: int, dtype, dev: int) -> mebptt_seq:
    p, ld = _rows(t, name, B, channels, dtype, dev)
    return mebptt_seq(p, 0, ld)


def mebptt_scan_step(desc: mebptt_scan_desc, u, delta, A, Bm, Cm, skip, z, delta_bias, state_in, index, y, state_out,
                     stream: Optional[int] = None) -> None:
    """One token: u, delta, z, y [B, D]; Bm, Cm [B, G N]; state_in, state_out [slots, D, N] float32 (one tensor or two); index as
    in mebptt_conv_step."""
    dev, T = _gpu(u), _dtype(desc.dtype)
    f32, B, D, N, GN = _DTYPES[0], desc.B, desc.D, desc.N, desc.G * desc.N
    given = mebptt_scan_inputs(_token(u, "u", B, D, T, dev), _token(delta, "delta", B, D, T, dev),
                               mebptt_seq(None, 0, 0) if z is None else _token(z, "z", B, D, T, dev), _token(Bm, "Bm", B, GN, T, dev),
                               _token(Cm, "Cm", B, GN, T, dev), _whole(A, "A", (D, N), f32, dev), _maybe(skip, "skip", (D,), f32, dev),
                               _maybe(delta_bias, "delta_bias", (D,), f32, dev), None, None)
    pin, slots, pout = _pool(state_in, state_out, (D, N), f32, dev, True)
    _call(dev, stream, lib().mebptt_scan_step, C.byref(desc), C.byref(given), pin, slots, _maybe(index, "index", (B,), _torch.int32, dev),
          _token(y, "y", B, D, T, dev), pout)


# ---- a block with a matrix for a state, and the step that trains it ----------------------------------


def make_delta_desc(t: int, B: int, Hk: int, H: int, dk: int, dv: int, dtype: int, activate: int = 1, normalise: int = 1, stretch: int = 256,
                    scale: float = 1.0, eps: float = 1e-6) -> mebptt_delta_desc:
    return mebptt_delta_desc(t, B, Hk, H, dk, dv, dtype, activate, normalise, stretch, scale, eps)


def mebptt_delta_state_bytes(desc: mebptt_delta_desc) -> int:
    return lib().mebptt_delta_state_bytes(C.byref(desc))


def mebptt_delta_workspace_bytes(desc: mebptt_delta_desc, backward: bool) -> int:
    return lib().mebptt_delta_workspace_bytes(C.byref(desc), 1 if backward else 0)


def _delta_inputs(desc, q, k, v, a, b, A, a_bias, lengths, h0, T, dev: int) -> mebptt_delta_inputs:
    f32, t, B, H = _DTYPES[0], desc.t, desc.B, desc.H
    return mebptt_delta_inputs(_seq(q, "q", t, B, desc.Hk * desc.dk, T, dev), _seq(k, "k", t, B, desc.Hk * desc.dk, T, dev),
                               _seq(v, "v", t, B, H * desc.dv, T, dev), _maybe_seq(a, "a", t, B, H, T, dev), _seq(b, "b", t, B, H, T, dev),
                               _maybe(A, "A", (H,), f32, dev), _maybe(a_bias, "a_bias", (H,), f32, dev),
                               _maybe(lengths, "lengths", (B,), _torch.int32, dev), _maybe(h0, "h0", (B, H, desc.dk, desc.dv), f32, dev))


def mebptt_delta_forward(desc: mebptt_delta_desc, q, k, v, a, b, A, a_bias, lengths, h0, y, h_out=None, states=None, workspace=None,
                         stream: Optional[int] = None) -> None:
    """Gated delta rule.  q, k [t, B, Hk dk]; v, y [t, B, H dv]; a (None: no decay), b [t, B, H]; A, a_bias [H]; h0, h_out [B, H, dk, dv];
    `states` (uint8) keeps what a backward call needs."""
    dev, T = _gpu(q), _dtype(desc.dtype)
    given = _delta_inputs(desc, q, k, v, a, b, A, a_bias, lengths, h0, T, dev)
    _call(dev, stream, lib().mebptt_delta_forward, C.byref(desc), C.byref(given), _seq(y, "y", desc.t, desc.B, desc.H * desc.dv, T, dev),
          _maybe(h_out, "h_out", (desc.B, desc.H, desc.dk, desc.dv), _DTYPES[0], dev), *_room(states, "states", dev),
          *_room(workspace, "workspace", dev))


def mebptt_delta_backward(desc: mebptt_delta_desc, q, k, v, a, b, A, a_bias, lengths, h0, dy, dh_out, states, dq, dk, dv, da, db, dA, da_bias,
                          dh0, workspace, stream: Optional[int] = None) -> None:
    """Gradients of mebptt_delta_forward from the states that it kept; da where there is an a."""
    dev, T = _gpu(q), _dtype(desc.dtype)
    f32, t, B, H, state = _DTYPES[0], desc.t, desc.B, desc.H, (desc.B, desc.H, desc.dk, desc.dv)
    given = _delta_inputs(desc, q, k, v, a, b, A, a_bias, lengths, h0, T, dev)
    grads = mebptt_delta_grads(_seq(dq, "dq", t, B, desc.Hk * desc.dk, T, dev), _seq(dk, "dk", t, B, desc.Hk * desc.dk, T, dev),
                               _seq(dv, "dv", t, B, H * desc.dv, T, dev), _seq(db, "db", t, B, H, T, dev),
                               (_maybe_seq if a is None else _seq)(da, "da", t, B, H, T, dev), _maybe(dA, "dA", (H,), f32, dev),
                               _maybe(da_bias, "da_bias", (H,), f32, dev), _maybe(dh0, "dh0", state, f32, dev))
    _call(dev, stream, lib().mebptt_delta_backward, C.byref(desc), C.byref(given), _seq(dy, "dy", t, B, H * desc.dv, T, dev),
          _maybe(dh_out, "dh_out", state, f32, dev), *_room(states, "states", dev), C.byref(grads), *_room(workspace, "workspace", dev))


def mebptt_delta_step(desc: mebptt_delta_desc, q, k, v, a, b, A, a_bias, state_in, index, y, state_out, stream: Optional[int] = None) -> None:
    """One token: q, k [B, Hk dk]; v, y [B, H dv]; a, b [B, H]; state_in, state_out [slots, H, dk, dv] float32 (one tensor or two); index as
    in mebptt_conv_step."""
    dev, T = _gpu(q), _dtype(desc.dtype)
    f32, B, H, dk, dv = _DTYPES[0], desc.B, desc.H, desc.dk, desc.dv
    given = mebptt_delta_inputs(_token(q, "q", B, desc.Hk * dk, T, dev), _token(k, "k", B, desc.Hk * dk, T, dev), _token(v, "v", B, H * dv, T, dev),
                                mebptt_seq(None, 0, 0) if a is None else _token(a, "a", B, H, T, dev), _token(b, "b", B, H, T, dev),
                                _maybe(A, "A", (H,), f32, dev), _maybe(a_bias, "a_bias", (H,), f32, dev), None, None)
    pin, slots, pout = _pool(state_in, state_out, (H, dk, dv), f32, dev, True)
    _call(dev, stream, lib().mebptt_delta_step, C.byref(desc), C.byref(given), pin, slots, _maybe(index, "index", (B,), _torch.int32, dev),
          _token(y, "y", B, H * dv, T, dev), pout)


def make_join_desc(rows: int, width: int, group: int, x_dtype: int, residual_dtype: int = FP32, scale: float = 1.0,
                   eps: float = 1e-5, again: bool = False) -> mebptt_join_desc:
    return mebptt_join_desc(rows, width, group, x_dtype, residual_dtype, scale, eps, int(again), 0)


def mebptt_join_workspace_bytes(desc: mebptt_join_desc) -> int:
    return lib().mebptt_join_workspace_bytes(C.byref(desc))


def mebptt_join_forward(desc: mebptt_join_desc, x, z, weight, residual, weight_next, y, residual_out=None, rstd=None, rstd_next=None,
                        stream: Optional[int] = None) -> None:
    """branch = norm of x per group times `weight` times silu(z); without a residual y = branch, with one r = scale residual + branch goes to
    residual_out and y = norm(r) times weight_next.  rstd [rows, width / group] and rstd_next [rows] are for the backward call."""
    dev, M, W = _gpu(x), desc.rows, desc.width
    f32, xt, rt = _DTYPES[0], _dtype(desc.x_dtype), _dtype(desc.residual_dtype)
    _call(dev, stream, lib().mebptt_join_forward, C.byref(desc), *_rows(x, "x", M, W, xt, dev), *_maybe_rows(z, "z", M, W, xt, dev),
          _maybe(weight, "weight", (W,), f32, dev), *_maybe_rows(residual, "residual", M, W, rt, dev),
          _maybe(weight_next, "weight_next", (W,), f32, dev), *_rows(y, "y", M, W, xt, dev), *_maybe_rows(residual_out, "residual_out", M, W, rt, dev),
          _maybe(rstd, "rstd", (M, W // max(desc.group, 1)), f32, dev), _maybe(rstd_next, "rstd_next", (M,), f32, dev))


def mebptt_join_backward(desc: mebptt_join_desc, x, z, weight, r, weight_next, rstd, rstd_next, dy, dresidual_out, dx, dz, dweight, dresidual,
                         dweight_next, workspace, stream: Optional[int] = None) -> None:
    """Gradients of mebptt_join_forward; r is its residual_out, or where the description says `again` its residual, from which the sum is computed once more
    without its rounding to the stream's type (None: there was no residual)."""
    dev, M, W = _gpu(x), desc.rows, desc.width
    f32, xt, rt = _DTYPES[0], _dtype(desc.x_dtype), _dtype(desc.residual_dtype)
    _call(dev, stream, lib().mebptt_join_backward, C.byref(desc), *_rows(x, "x", M, W, xt, dev), *_maybe_rows(z, "z", M, W, xt, dev),
          _maybe(weight, "weight", (W,), f32, dev), *_maybe_rows(r, "r", M, W, rt, dev), _maybe(weight_next, "weight_next", (W,), f32, dev),
          _whole(rstd, "rstd", (M, W // max(desc.group, 1)), f32, dev), _maybe(rstd_next, "rstd_next", (M,), f32, dev),
          *_rows(dy, "dy", M, W, xt, dev), *_maybe_rows(dresidual_out, "dresidual_out", M, W, rt, dev), *_rows(dx, "dx", M, W, xt, dev),
          *_maybe_rows(dz, "dz", M, W, xt, dev), _maybe(dweight, "dweight", (W,), f32, dev), *_maybe_rows(dresidual, "dresidual", M, W, rt, dev),
          _maybe(dweight_next, "dweight_next", (W,), f32, dev), *_room(workspace, "workspace", dev))


class AdamwTensors:
    """What mebptt_adamw_* take of a list of tensors; keeps them alive."""

    def __init__(self, array, device: int, kept):
        self.array, self.count, self.device, self.kept = array, len(kept), device, kept


def make_adamw_tensors(params, grads, m, v, m_scale=None, v_scale=None, copies=None, no_decay=None) -> AdamwTensors:
    """Lists of one length: params float32; grads float32 or bfloat16; m and v float32, or uint8 with scales of ceil(n / 256) float32 each; copies
    (entries may be None) bfloat16; no_decay: truth values.  All contiguous and on one GPU."""
    params = list(params)
    if not params:
        raise ValueError("at least one tensor is needed")
    dev, n = _gpu(params[0]), len(params)
    f32, bf16, byte = _DTYPES[0], _DTYPES[1], _torch.uint8
    lists = {"grads": grads, "m": m, "v": v, "m_scale": m_scale, "v_scale": v_scale, "copies": copies, "no_decay": no_decay}
    lists = {k: [None] * n if x is None else list(x) for k, x in lists.items()}
    for k, x in lists.items():
        if len(x) != n:
            raise ValueError(f"{k} has {len(x)} entries, {n} are needed")
    array, kept = (mebptt_adamw_tensor * n)(), []
    for i, p in enumerate(params):
        g, mi, vi, ms, vs, c, flag = (lists[k][i] for k in ("grads", "m", "v", "m_scale", "v_scale", "copies", "no_decay"))
        shape, blocks = None if p is None else p.shape, 0 if p is None else (-(-p.numel() // 256),)
        small = mi is not None and mi.dtype is byte
        st = byte if small else f32
        wide = g is None or g.dtype is not bf16
        array[i] = mebptt_adamw_tensor(
            _whole(p, f"params[{i}]", shape, f32, dev), _whole(g, f"grads[{i}]", shape, f32 if wide else bf16, dev),
            _whole(mi, f"m[{i}]", shape, st, dev), _whole(vi, f"v[{i}]", shape, st, dev), _whole(ms, f"m_scale[{i}]", blocks, f32, dev) if small else None,
            _whole(vs, f"v_scale[{i}]", blocks, f32, dev) if small else None, _maybe(c, f"copies[{i}]", shape, bf16, dev), p.numel(),
            FP32 if wide else BF16, INT8 if small else FP32, ADAMW_NO_DECAY if flag else 0, 0)
        kept.append((p, g, mi, vi, ms, vs, c))
    return AdamwTensors(array, dev, kept)


def make_adamw_desc(rate: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, decay: float = 0.01, step: int = 1,
                    seed: int = 0) -> mebptt_adamw_desc:
    return mebptt_adamw_desc(rate, beta1, beta2, eps, decay, step, seed & 0xFFFFFFFF, 0)


def mebptt_adamw_table_bytes(tensors: AdamwTensors) -> int:
    return lib().mebptt_adamw_table_bytes(tensors.array, tensors.count)


def mebptt_adamw_workspace_bytes(tensors: AdamwTensors) -> int:
    return lib().mebptt_adamw_workspace_bytes(tensors.array, tensors.count)


def mebptt_adamw_prepare(tensors: AdamwTensors, table, stream: Optional[int] = None) -> None:
    """Writes what the other calls need to know of the tensors into `table` (uint8)."""
    _call(tensors.device, stream, lib().mebptt_adamw_prepare, tensors.array, tensors.count, *_room(table, "table", tensors.device))


def mebptt_adamw_norm(tensors: AdamwTensors, table, max_norm: float, out, workspace, stream: Optional[int] = None) -> None:
    """out [2] float32: the norm of all gradients, and the factor that limits it to max_norm."""
    dev = tensors.device
    _call(dev, stream, lib().mebptt_adamw_norm, tensors.array, tensors.count, *_room(table, "table", dev), max_norm,
          _whole(out, "out", (2,), _DTYPES[0], dev), *_room(workspace, "workspace", dev))


def mebptt_adamw_step(desc: mebptt_adamw_desc, tensors: AdamwTensors, table, factor=None, rate=None, step=None,
                      stream: Optional[int] = None) -> None:
    """One step over all tensors.  factor, rate ([1] float32) and step ([1] int64) are read on the GPU when the step runs."""
    dev = tensors.device
    _call(dev, stream, lib().mebptt_adamw_step, C.byref(desc), tensors.array, tensors.count, *_room(table, "table", dev),
          _maybe(factor, "factor", (1,), _DTYPES[0], dev), _maybe(rate, "rate", (1,), _DTYPES[0], dev),
          _maybe(step, "step", (1,), _torch.int64, dev))


def mebptt_adamw_unpack(codes, scale, is_signed: bool, out, stream: Optional[int] = None) -> None:
    """The values that one tensor's 8-bit states stand for (`is_signed`: those of m), to float32 or bfloat16."""
    dev = _gpu(codes)
    n = codes.numel()
    wide = out is None or out.dtype is not _DTYPES[1]
    _call(dev, stream, lib().mebptt_adamw_unpack, _whole(codes, "codes", codes.shape, _torch.uint8, dev),
          _whole(scale, "scale", (-(-n // 256),), _DTYPES[0], dev), n, 1 if is_signed else 0,
          _whole(out, "out", codes.shape, _DTYPES[0] if wide else _DTYPES[1], dev), FP32 if wide else BF16)
