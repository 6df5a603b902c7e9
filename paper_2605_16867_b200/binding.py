"""ctypes binding with the same names as the C ABI (see include/goodserve.h).

Argument marshalling only: tensors are checked (device, dtype, contiguity) and their
addresses handed to the library.  PyTorch supplies device memory and streams, nothing else.
"""
from __future__ import annotations

import ctypes as C
import os
from array import array
from dataclasses import dataclass
from typing import Optional

import numpy as np
import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
GS_ROUTE_ACCUMULATE = 1


class DeviceStatus:
    BAD_INSTANCE = 1
    BAD_TYPE = 2
    BAD_VALUE = 4
    TIMEOUT = 8
    CAND_TRUNCATED = 16
    INTERNAL = 32


class GoodServeError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"libgoodserve error {code}: {message}")
        self.code = code


class _Instances(C.Structure):
    _fields_ = [("type_id", C.c_void_p), ("queued_prefill_tokens", C.c_void_p),
                ("decode_batch", C.c_void_p), ("free_kv_tokens", C.c_void_p),
                ("q_ema_ms", C.c_void_p), ("n_instances", C.c_int32)]


class _Types(C.Structure):
    _fields_ = [("prefill_ms_per_tok", C.c_void_p), ("tpot_a_ms", C.c_void_p),
                ("tpot_b_ms", C.c_void_p), ("n_types", C.c_int32)]


class _InstanceTable(C.Structure):
    _fields_ = [("q_ms", C.c_void_p), ("p_ms_per_tok", C.c_void_p), ("d_ms_per_tok", C.c_void_p),
                ("free_kv_tokens", C.c_void_p), ("n_instances", C.c_int32)]


class _ExpertRouter(C.Structure):
    _fields_ = [("n_experts", C.c_int32), ("top_k", C.c_int32), ("score", C.c_int32), ("n_groups", C.c_int32),
                ("top_groups", C.c_int32), ("group_top", C.c_int32), ("renormalise", C.c_int32), ("scale", C.c_float)]


class _InstancesMut(C.Structure):
    _fields_ = [("queued_prefill_tokens", C.c_void_p), ("decode_batch", C.c_void_p),
                ("free_kv_tokens", C.c_void_p), ("q_ema_ms", C.c_void_p),
                ("n_instances", C.c_int32)]


def library_path(counting: bool = False, checking: bool = False) -> str:
    name = "libgoodserve_count.so" if counting else "libgoodserve_debug.so" if checking else "libgoodserve.so"
    return os.path.join(_PKG, name)


_libs = {}


def _declare(lib):
    """Argument and result types of every entry point of include/goodserve.h."""
    vp, i32, i64, f32, u32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_uint
    lib.gs_create.argtypes = [C.POINTER(vp), C.c_int, C.c_int, C.c_int]
    lib.gs_destroy.argtypes = [vp]
    lib.gs_strerror.argtypes = [C.c_int]
    lib.gs_strerror.restype = C.c_char_p
    lib.gs_last_cuda_error.argtypes = [vp]
    lib.gs_device_status.argtypes = [vp, vp, C.POINTER(u32)]
    lib.gs_launch_count.argtypes = [vp]
    lib.gs_launch_count.restype = i64
    lib.gs_eval_counters.argtypes = [vp, vp, C.POINTER(C.c_uint64), C.c_int]
    lib.gs_eval_counters.restype = C.c_int
    route_args = [vp, vp, vp, vp, i64, C.POINTER(_Instances), C.POINTER(_Types), f32, vp, vp, vp, vp]
    lib.gs_route_batch.argtypes = route_args + [u32, vp]
    lib.gs_route_batch_host.argtypes = route_args + [vp]
    lib.gs_route_batch_host_deferred.argtypes = route_args + [vp]
    lib.gs_host_wait.argtypes = [vp, vp]
    lib.gs_route_batch_prefix.argtypes = [vp, vp, vp, vp, i64, vp, vp, C.c_int, i64, C.POINTER(_Instances),
                                          C.POINTER(_Types), f32, vp, vp, vp, vp, vp]
    lib.gs_route_batch_prefix.restype = C.c_int
    lib.gs_route_batch_direct.argtypes = [vp, vp, vp, vp, i64, C.POINTER(_InstanceTable), vp, vp, vp, vp, vp]
    lib.gs_route_batch_direct.restype = C.c_int
    lib.gs_ema_update.argtypes = [vp, f32, i32, vp, vp, vp, vp, vp, vp, vp]
    lib.gs_ema_update.restype = C.c_int
    lib.gs_route_sequential.argtypes = [vp, vp, vp, vp, i64, vp, C.POINTER(_InstancesMut), C.POINTER(_Types), f32,
                                        vp, vp, vp, vp, vp]
    lib.gs_route_sequential.restype = C.c_int
    lib.gs_advance_state.argtypes = [vp, C.POINTER(_InstancesMut), vp]
    risk_args = [vp, vp, vp, vp, vp, vp, i64, C.POINTER(_Instances), C.POINTER(_Types), vp, vp, i64, vp, vp]
    lib.gs_risk_scan.argtypes = risk_args
    lib.gs_risk_scan_host.argtypes = risk_args
    lib.gs_timing_enable.argtypes = [vp, C.c_int]
    lib.gs_timing_read.argtypes = [vp, C.c_int, C.POINTER(C.c_double), C.POINTER(i64)]
    lib.gs_reroute_candidates.argtypes = [vp, vp, vp, i64, vp, vp, vp, vp, vp, vp, i64, C.POINTER(_Instances),
                                          C.POINTER(_Types), f32, vp, vp, vp, vp, vp]
    lib.gs_reroute_candidates.restype = C.c_int
    lib.gs_risk_scan_noalloc.argtypes = [vp, vp, vp, vp, vp, i64, C.POINTER(_Instances), C.POINTER(_Types),
                                         vp, vp, i64, vp, vp, vp]
    lib.gs_risk_scan_noalloc.restype = C.c_int
    lib.gs_expert_route.argtypes = [vp, vp, C.c_int, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.gs_expert_route_backward.argtypes = [vp, vp, C.c_int, i64, i64, vp, vp, vp, vp, i64, vp]
    lib.gs_expert_linear.argtypes = [vp, C.c_int, vp, i64, i64, vp, vp, i32, i64, vp, i64, vp, i32, i32, u32, vp, i64, vp]
    lib.gs_expert_linear_backward.argtypes = [vp, C.c_int, vp, i64, vp, i64, i64, vp, vp, i32, i64, vp, i64, i32, i32, u32,
                                              vp, i64, vp, i64, vp, vp, i64, vp]
    lib.gs_expert_linear_backward_workspace.argtypes = [vp, i32, i64, i32, i32]
    lib.gs_expert_linear_backward_workspace.restype = i64
    lib.gs_expert_combine.argtypes = [vp, C.c_int, vp, i64, i64, vp, vp, i64, i32, i32, C.c_int, vp, i64, vp]
    lib.gs_expert_combine_backward.argtypes = [vp, C.c_int, C.c_int, vp, i64, vp, i64, i64, vp, vp, i64, i32, i32, u32,
                                               vp, i64, vp, vp]
    lib.gs_clip_grad_norm.argtypes = [vp, vp, i32, f32, vp, vp]
    for name in ("gs_expert_route", "gs_expert_route_backward", "gs_expert_linear", "gs_expert_linear_backward",
                 "gs_expert_combine", "gs_expert_combine_backward", "gs_clip_grad_norm"):
        getattr(lib, name).restype = C.c_int
    for name in ("gs_timing_enable", "gs_timing_read", "gs_create", "gs_destroy", "gs_last_cuda_error", "gs_device_status", "gs_route_batch",
                 "gs_route_batch_host", "gs_route_batch_host_deferred", "gs_host_wait", "gs_advance_state", "gs_risk_scan", "gs_risk_scan_host"):
        getattr(lib, name).restype = C.c_int
    return lib


def load_library(build_if_missing: bool = True, counting: bool = False, checking: bool = False):
    """Loads libgoodserve.so (building it with nvcc first if it is absent or stale).
    Raises if that fails -- there is no other implementation to fall back to.
    ``counting=True`` loads the measuring build instead (-DGS_COUNT_EVALS: the work counters
    behind gs_eval_counters tick; many times slower, for benchmarks only); ``checking=True`` the
    build with table index checks compiled in (-DGS_DEBUG; GS_DEV_INTERNAL reports a failure)."""
    kind = "counting" if counting else "checking" if checking else "regular"
    if kind in _libs:
        return _libs[kind]
    path = library_path(counting, checking)
    if build_if_missing:
        from .build import build_library
        try:
            build_library(counting=counting, checking=checking)
        except Exception as exc:                      # nvcc missing on a box that has the .so
            if not os.path.exists(path):
                raise RuntimeError(f"{os.path.basename(path)} is missing and could not be built: {exc}") from exc
    if not os.path.exists(path):
        raise RuntimeError(f"{path} not found; run paper_2605_16867_b200/build.py")
    _libs[kind] = _declare(C.CDLL(path))
    return _libs[kind]


def _dev_ptr(t: Optional[torch.Tensor], dtype: torch.dtype, n: Optional[int], name: str, device) -> Optional[int]:
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name}: expected a CUDA tensor")
    if t.device != device:
        raise ValueError(f"{name}: tensor is on {t.device}, context is on {device}")
    if t.dtype != dtype or not t.is_contiguous() or t.dim() != 1:
        raise TypeError(f"{name}: expected a contiguous 1-D {dtype} tensor, got {t.dtype} {tuple(t.shape)}")
    if n is not None and t.numel() < n:
        raise ValueError(f"{name}: needs {n} elements, has {t.numel()}")
    return t.data_ptr()


def _host_ptr(a, dtype, n: Optional[int], name: str) -> Optional[int]:
    if a is None:
        return None
    if isinstance(a, torch.Tensor):
        if a.is_cuda or not a.is_contiguous():
            raise TypeError(f"{name}: expected a contiguous host tensor")
        if n is not None and a.numel() < n:
            raise ValueError(f"{name}: needs {n} elements, has {a.numel()}")
        return a.data_ptr()
    if not isinstance(a, np.ndarray) or a.dtype != dtype or not a.flags.c_contiguous:
        raise TypeError(f"{name}: expected a contiguous numpy array of {dtype}")
    if n is not None and a.size < n:
        raise ValueError(f"{name}: needs {n} elements, has {a.size}")
    return a.ctypes.data


# the current stream's cudaStream_t (torch.cuda.current_stream builds an object around it)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_OPERANDS = (torch.bfloat16, torch.float16)


def _refuse(t, dtype, shape, name: str, index: int):
    """Says what is wrong with an argument that one of the checks below turned down."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.get_device() != index:
        raise TypeError(f"{name}: expected a tensor on cuda:{index}")
    if t.dtype is not dtype or (isinstance(shape, tuple) and t.dim() != len(shape)):
        raise TypeError(f"{name}: expected a {len(shape)}-D {dtype} tensor, got {t.dtype} {tuple(t.shape)}"
                        if isinstance(shape, tuple) else f"{name}: expected a {dtype} tensor, got {t.dtype}")
    if isinstance(shape, tuple) and tuple(t.shape) != shape:
        raise ValueError(f"{name}: expected {list(shape)}, got {list(t.shape)}")
    if not isinstance(shape, tuple) and t.numel() != shape:
        raise ValueError(f"{name}: needs {shape} elements, has {t.numel()}")
    raise TypeError(f"{name}: expected evenly spaced rows of consecutive elements, got strides {t.stride()}")


# (These run before every launch of a few microseconds: one expression on the way that is taken, and
# all explanations on the other one.)
def _array(t, dtype: torch.dtype, n: int, name: str, index: int) -> Optional[int]:
    """The address of a contiguous CUDA tensor of n elements, whatever its shape."""
    if t is None:
        return None
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.numel() == n and t.is_contiguous() and t.is_cuda
            and t.get_device() == index):
        _refuse(t, dtype, n, name, index)
    return t.data_ptr()


def _matrix(t, dtype: torch.dtype, rows: int, cols: int, name: str, index: int):
    """(address, row stride) of a row-major CUDA matrix; the rows may be further apart than they are wide."""
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == (rows, cols) and t.is_cuda and t.get_device() == index):
        _refuse(t, dtype, (rows, cols), name, index)
    ld, one = t.stride()
    if (one != 1 and cols > 1) or (ld < cols and rows > 1):
        _refuse(t, dtype, (rows, cols), name, index)
    return t.data_ptr(), ld if ld >= cols else (cols + 7) // 8 * 8


def _stack(t, dtype: torch.dtype, shape, name: str, index: int):
    """(address, row stride) of the experts' matrices [experts, out, in], experts out rows apart."""
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and len(shape) == 3 and t.is_cuda and t.get_device() == index):
        _refuse(t, dtype, tuple(shape) if len(shape) == 3 else (0, 0, 0), name, index)
    (e, o, i), (step, ld, one) = shape, t.stride()
    if o == 1:
        ld = step if e > 1 else max(ld, (i + 7) // 8 * 8)
    if (one != 1 and i > 1) or ld < i or (e > 1 and step != o * ld):
        _refuse(t, dtype, tuple(shape), name, index)
    return t.data_ptr(), ld


class ExpertRouter:
    """How a row of a gate's logits becomes choices and weights (gs_expert_router)."""

    def __init__(self, n_experts: int, top_k: int, score: str = "softmax", n_groups: int = 1, top_groups: int = 1,
                 group_top: int = 1, renormalise: bool = True, scale: float = 1.0):
        if score not in ("softmax", "sigmoid"):
            raise ValueError(f"score: expected 'softmax' or 'sigmoid', got {score!r}")
        self.n_experts, self.top_k = int(n_experts), int(top_k)
        self._struct = _ExpertRouter(self.n_experts, self.top_k, 1 if score == "sigmoid" else 0, int(n_groups),
                                     int(top_groups), int(group_top), 1 if renormalise else 0, float(scale))
        self._address = C.addressof(self._struct)


@dataclass
class InstancePool:
    """Device-resident pool description: per-instance state (SoA) and the type table."""
    type_id: torch.Tensor
    queued_prefill_tokens: torch.Tensor
    decode_batch: torch.Tensor
    free_kv_tokens: torch.Tensor
    q_ema_ms: torch.Tensor
    prefill_ms_per_tok: torch.Tensor
    tpot_a_ms: torch.Tensor
    tpot_b_ms: torch.Tensor

    @property
    def n_instances(self) -> int:
        return int(self.type_id.numel())

    @property
    def n_types(self) -> int:
        return int(self.prefill_ms_per_tok.numel())

    @staticmethod
    def from_host(types, inst, device) -> "InstancePool":
        def up(a):
            return torch.from_numpy(np.ascontiguousarray(a)).to(device)
        return InstancePool(up(inst.type_id), up(inst.queued_prefill_tokens), up(inst.decode_batch),
                            up(inst.free_kv_tokens), up(inst.q_ema_ms), up(types.prefill_ms_per_tok),
                            up(types.tpot_a_ms), up(types.tpot_b_ms))


class GoodServe:
    """One library context (gs_create / gs_destroy) bound to a CUDA device."""

    def __init__(self, device: int = 0, max_instances: int = 1024, max_types: int = 16, counting: bool = False,
                 checking: bool = False):
        if not torch.cuda.is_available():
            raise RuntimeError("GoodServe needs a CUDA device; there is no CPU implementation")
        self._lib = load_library(counting=counting, checking=checking)
        self.device, self._index = torch.device("cuda", device), int(device)
        torch.cuda.init()
        with torch.cuda.device(self.device):
            torch.zeros(1, device=self.device)          # make sure the primary context exists
        h = C.c_void_p()
        self._check(self._lib.gs_create(C.byref(h), device, max_instances, max_types))
        self._h = h
        self._deferred = None

    # -- plumbing ------------------------------------------------------------------------
    def _check(self, rc: int):
        if rc:
            raise GoodServeError(rc, self._lib.gs_strerror(rc).decode())

    def _stream(self, stream) -> Optional[int]:
        s = torch.cuda.current_stream(self.device) if stream is None else stream
        return s.cuda_stream or None

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            self._lib.gs_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _pool_structs(self, pool: InstancePool):
        M, Tn, dev = pool.n_instances, pool.n_types, self.device
        i32, f32 = torch.int32, torch.float32
        inst = _Instances(_dev_ptr(pool.type_id, i32, M, "type_id", dev),
                          _dev_ptr(pool.queued_prefill_tokens, i32, M, "queued_prefill_tokens", dev),
                          _dev_ptr(pool.decode_batch, i32, M, "decode_batch", dev),
                          _dev_ptr(pool.free_kv_tokens, i32, M, "free_kv_tokens", dev),
                          _dev_ptr(pool.q_ema_ms, f32, M, "q_ema_ms", dev), M)
        types = _Types(_dev_ptr(pool.prefill_ms_per_tok, f32, Tn, "prefill_ms_per_tok", dev),
                       _dev_ptr(pool.tpot_a_ms, f32, Tn, "tpot_a_ms", dev),
                       _dev_ptr(pool.tpot_b_ms, f32, Tn, "tpot_b_ms", dev), Tn)
        return inst, types

    @staticmethod
    def _host_pool_structs(types, inst):
        M, Tn = int(inst.type_id.shape[0]), int(types.prefill_ms_per_tok.shape[0])
        hi = _Instances(_host_ptr(inst.type_id, np.int32, M, "type_id"),
                        _host_ptr(inst.queued_prefill_tokens, np.int32, M, "queued_prefill_tokens"),
                        _host_ptr(inst.decode_batch, np.int32, M, "decode_batch"),
                        _host_ptr(inst.free_kv_tokens, np.int32, M, "free_kv_tokens"),
                        _host_ptr(inst.q_ema_ms, np.float32, M, "q_ema_ms"), M)
        ht = _Types(_host_ptr(types.prefill_ms_per_tok, np.float32, Tn, "prefill_ms_per_tok"),
                    _host_ptr(types.tpot_a_ms, np.float32, Tn, "tpot_a_ms"),
                    _host_ptr(types.tpot_b_ms, np.float32, Tn, "tpot_b_ms"), Tn)
        return hi, ht

    # -- C ABI, same names ----------------------------------------------------------------
    def route_batch(self, prompt_len, pred_decode_len, slo_ms, pool: InstancePool, ema_alpha: float,
                    out_instance_idx, out_est_e2e_ms, out_slack_ms, out_tier=None,
                    accumulate: bool = False, n_requests: Optional[int] = None, stream=None):
        n = int(prompt_len.numel()) if n_requests is None else int(n_requests)
        dev, i32, f32 = self.device, torch.int32, torch.float32
        inst, types = self._pool_structs(pool)
        self._check(self._lib.gs_route_batch(
            self._h, _dev_ptr(prompt_len, i32, n, "prompt_len", dev),
            _dev_ptr(pred_decode_len, i32, n, "pred_decode_len", dev),
            _dev_ptr(slo_ms, f32, n, "slo_ms", dev), n, C.byref(inst), C.byref(types),
            float(ema_alpha), _dev_ptr(out_instance_idx, i32, n, "out_instance_idx", dev),
            _dev_ptr(out_est_e2e_ms, f32, n, "out_est_e2e_ms", dev),
            _dev_ptr(out_slack_ms, f32, n, "out_slack_ms", dev),
            _dev_ptr(out_tier, torch.uint8, n, "out_tier", dev),
            GS_ROUTE_ACCUMULATE if accumulate else 0, self._stream(stream)))

    def route_batch_prefix(self, prompt_len, pred_decode_len, slo_ms, prefix_inst, prefix_hit_len,
                           n_slots: int, slot_stride: int, pool: InstancePool, ema_alpha: float,
                           out_instance_idx, out_est_e2e_ms, out_slack_ms, out_tier=None,
                           n_requests: Optional[int] = None, stream=None):
        """``prefix_inst`` / ``prefix_hit_len``: 1-D int32 CUDA tensors of n_slots * slot_stride
        entries, slot k of request r at k * slot_stride + r."""
        n = int(prompt_len.numel()) if n_requests is None else int(n_requests)
        dev, i32, f32 = self.device, torch.int32, torch.float32
        inst, types = self._pool_structs(pool)
        n_hits = max(int(n_slots), 0) * int(slot_stride)
        self._check(self._lib.gs_route_batch_prefix(
            self._h, _dev_ptr(prompt_len, i32, n, "prompt_len", dev),
            _dev_ptr(pred_decode_len, i32, n, "pred_decode_len", dev),
            _dev_ptr(slo_ms, f32, n, "slo_ms", dev), n,
            _dev_ptr(prefix_inst, i32, n_hits, "prefix_inst", dev),
            _dev_ptr(prefix_hit_len, i32, n_hits, "prefix_hit_len", dev), int(n_slots), int(slot_stride),
            C.byref(inst), C.byref(types),
            float(ema_alpha), _dev_ptr(out_instance_idx, i32, n, "out_instance_idx", dev),
            _dev_ptr(out_est_e2e_ms, f32, n, "out_est_e2e_ms", dev),
            _dev_ptr(out_slack_ms, f32, n, "out_slack_ms", dev),
            _dev_ptr(out_tier, torch.uint8, n, "out_tier", dev), self._stream(stream)))

    def route_batch_direct(self, prompt_len, pred_decode_len, slo_ms, q_ms, p_ms_per_tok, d_ms_per_tok,
                           free_kv_tokens, out_instance_idx, out_est_e2e_ms, out_slack_ms, out_tier=None,
                           n_requests: Optional[int] = None, n_instances: Optional[int] = None, stream=None):
        """Routing round against per-instance coefficients given directly (CUDA tensors)."""
        n = int(prompt_len.numel()) if n_requests is None else int(n_requests)
        M = int(q_ms.numel()) if n_instances is None else int(n_instances)
        dev, i32, f32 = self.device, torch.int32, torch.float32
        table = _InstanceTable(_dev_ptr(q_ms, f32, M, "q_ms", dev), _dev_ptr(p_ms_per_tok, f32, M, "p_ms_per_tok", dev),
                               _dev_ptr(d_ms_per_tok, f32, M, "d_ms_per_tok", dev),
                               _dev_ptr(free_kv_tokens, i32, M, "free_kv_tokens", dev), M)
        self._check(self._lib.gs_route_batch_direct(
            self._h, _dev_ptr(prompt_len, i32, n, "prompt_len", dev),
            _dev_ptr(pred_decode_len, i32, n, "pred_decode_len", dev),
            _dev_ptr(slo_ms, f32, n, "slo_ms", dev), n, C.byref(table),
            _dev_ptr(out_instance_idx, i32, n, "out_instance_idx", dev),
            _dev_ptr(out_est_e2e_ms, f32, n, "out_est_e2e_ms", dev),
            _dev_ptr(out_slack_ms, f32, n, "out_slack_ms", dev),
            _dev_ptr(out_tier, torch.uint8, n, "out_tier", dev), self._stream(stream)))

    def ema_update(self, alpha: float, obs_q_ms, obs_p_ms_per_tok, obs_d_ms_per_tok, q_ms, p_ms_per_tok,
                   d_ms_per_tok, n_instances: Optional[int] = None, stream=None):
        """In-place EMA step of the coefficient columns; a ``None`` observation skips its column."""
        cols = [t for t in (q_ms, p_ms_per_tok, d_ms_per_tok, obs_q_ms, obs_p_ms_per_tok, obs_d_ms_per_tok) if t is not None]
        M = int(cols[0].numel()) if n_instances is None else int(n_instances)
        dev, f32 = self.device, torch.float32
        self._check(self._lib.gs_ema_update(
            self._h, float(alpha), M, _dev_ptr(obs_q_ms, f32, M, "obs_q_ms", dev),
            _dev_ptr(obs_p_ms_per_tok, f32, M, "obs_p_ms_per_tok", dev),
            _dev_ptr(obs_d_ms_per_tok, f32, M, "obs_d_ms_per_tok", dev), _dev_ptr(q_ms, f32, M, "q_ms", dev),
            _dev_ptr(p_ms_per_tok, f32, M, "p_ms_per_tok", dev), _dev_ptr(d_ms_per_tok, f32, M, "d_ms_per_tok", dev),
            self._stream(stream)))

    def route_sequential(self, prompt_len, pred_decode_len, slo_ms, pool: InstancePool, ema_alpha: float,
                         out_instance_idx, out_est_e2e_ms, out_slack_ms, out_tier=None,
                         n_requests: Optional[int] = None, stream=None):
        """One request at a time; ``pool``'s state tensors are advanced in place."""
        n = int(prompt_len.numel()) if n_requests is None else int(n_requests)
        M, dev, i32, f32 = pool.n_instances, self.device, torch.int32, torch.float32
        _, types = self._pool_structs(pool)
        mut = _InstancesMut(_dev_ptr(pool.queued_prefill_tokens, i32, M, "queued_prefill_tokens", dev),
                            _dev_ptr(pool.decode_batch, i32, M, "decode_batch", dev),
                            _dev_ptr(pool.free_kv_tokens, i32, M, "free_kv_tokens", dev),
                            _dev_ptr(pool.q_ema_ms, f32, M, "q_ema_ms", dev), M)
        self._check(self._lib.gs_route_sequential(
            self._h, _dev_ptr(prompt_len, i32, n, "prompt_len", dev),
            _dev_ptr(pred_decode_len, i32, n, "pred_decode_len", dev),
            _dev_ptr(slo_ms, f32, n, "slo_ms", dev), n, _dev_ptr(pool.type_id, i32, M, "type_id", dev),
            C.byref(mut), C.byref(types), float(ema_alpha),
            _dev_ptr(out_instance_idx, i32, n, "out_instance_idx", dev),
            _dev_ptr(out_est_e2e_ms, f32, n, "out_est_e2e_ms", dev),
            _dev_ptr(out_slack_ms, f32, n, "out_slack_ms", dev),
            _dev_ptr(out_tier, torch.uint8, n, "out_tier", dev), self._stream(stream)))

    def advance_state(self, pool: InstancePool, stream=None):
        M, dev, i32 = pool.n_instances, self.device, torch.int32
        mut = _InstancesMut(_dev_ptr(pool.queued_prefill_tokens, i32, M, "queued_prefill_tokens", dev),
                            _dev_ptr(pool.decode_batch, i32, M, "decode_batch", dev),
                            _dev_ptr(pool.free_kv_tokens, i32, M, "free_kv_tokens", dev),
                            _dev_ptr(pool.q_ema_ms, torch.float32, M, "q_ema_ms", dev), M)
        self._check(self._lib.gs_advance_state(self._h, C.byref(mut), self._stream(stream)))

    def risk_scan(self, assigned_inst, generated_tokens, pred_len, elapsed_ms, slo_ms,
                  pool: InstancePool, out_flag_bits, out_cand_idx, out_cand_count,
                  cand_capacity: Optional[int] = None, n_active: Optional[int] = None, stream=None):
        n = int(assigned_inst.numel()) if n_active is None else int(n_active)
        cap = (0 if out_cand_idx is None else int(out_cand_idx.numel())) if cand_capacity is None else int(cand_capacity)
        dev, i32, f32 = self.device, torch.int32, torch.float32
        inst, types = self._pool_structs(pool)
        self._check(self._lib.gs_risk_scan(
            self._h, _dev_ptr(assigned_inst, i32, n, "assigned_inst", dev),
            _dev_ptr(generated_tokens, i32, n, "generated_tokens", dev),
            _dev_ptr(pred_len, i32, n, "pred_len", dev),
            _dev_ptr(elapsed_ms, f32, n, "elapsed_ms", dev), _dev_ptr(slo_ms, f32, n, "slo_ms", dev), n,
            C.byref(inst), C.byref(types),
            _dev_ptr(out_flag_bits, i32, (n + 31) // 32, "out_flag_bits", dev),
            _dev_ptr(out_cand_idx, i32, cap, "out_cand_idx", dev), cap,
            _dev_ptr(out_cand_count, torch.int64, 1, "out_cand_count", dev), self._stream(stream)))

    def reroute_candidates(self, cand_idx, cand_count, assigned_inst, generated_tokens, pred_len, elapsed_ms,
                           slo_ms, prompt_len, pool: InstancePool, ema_alpha: float,
                           out_new_instance, out_est_ms, out_slack_ms, out_tier=None,
                           cand_capacity: Optional[int] = None, stream=None):
        """gs_reroute_candidates: cand_idx / cand_count are risk_scan's device outputs."""
        cap = int(cand_idx.numel()) if cand_capacity is None else int(cand_capacity)
        n = int(assigned_inst.numel())
        dev, i32, f32 = self.device, torch.int32, torch.float32
        inst, types = self._pool_structs(pool)
        self._check(self._lib.gs_reroute_candidates(
            self._h, _dev_ptr(cand_idx, i32, cap, "cand_idx", dev),
            _dev_ptr(cand_count, torch.int64, 1, "cand_count", dev), cap,
            _dev_ptr(assigned_inst, i32, n, "assigned_inst", dev),
            _dev_ptr(generated_tokens, i32, n, "generated_tokens", dev),
            _dev_ptr(pred_len, i32, n, "pred_len", dev), _dev_ptr(elapsed_ms, f32, n, "elapsed_ms", dev),
            _dev_ptr(slo_ms, f32, n, "slo_ms", dev), _dev_ptr(prompt_len, i32, n, "prompt_len", dev), n,
            C.byref(inst), C.byref(types), float(ema_alpha),
            _dev_ptr(out_new_instance, i32, cap, "out_new_instance", dev),
            _dev_ptr(out_est_ms, f32, cap, "out_est_ms", dev),
            _dev_ptr(out_slack_ms, f32, cap, "out_slack_ms", dev),
            _dev_ptr(out_tier, torch.uint8, cap, "out_tier", dev), self._stream(stream)))

    def route_batch_host(self, prompt_len, pred_decode_len, slo_ms, types, inst, ema_alpha: float,
                         out_instance_idx, out_est_e2e_ms, out_slack_ms, out_tier=None, stream=None,
                         wait: bool = True):
        """Host-buffer variant: numpy arrays or (pinned) host tensors in and out.  With
        ``wait=False`` the call returns once everything is enqueued (gs_route_batch_host_deferred):
        the outputs are valid after ``host_wait()`` or the next host-buffer call has returned."""
        n = int(prompt_len.shape[0])
        hi, ht = self._host_pool_structs(types, inst)
        fn = self._lib.gs_route_batch_host if wait else self._lib.gs_route_batch_host_deferred
        if not wait:        # what the enqueued copies read and write stays referenced until the wait
            self._deferred = (prompt_len, pred_decode_len, slo_ms, types, inst, hi, ht,
                              out_instance_idx, out_est_e2e_ms, out_slack_ms, out_tier)
        self._check(fn(
            self._h, _host_ptr(prompt_len, np.int32, n, "prompt_len"),
            _host_ptr(pred_decode_len, np.int32, n, "pred_decode_len"),
            _host_ptr(slo_ms, np.float32, n, "slo_ms"), n, C.byref(hi), C.byref(ht), float(ema_alpha),
            _host_ptr(out_instance_idx, np.int32, n, "out_instance_idx"),
            _host_ptr(out_est_e2e_ms, np.float32, n, "out_est_e2e_ms"),
            _host_ptr(out_slack_ms, np.float32, n, "out_slack_ms"),
            _host_ptr(out_tier, np.uint8, n, "out_tier"), self._stream(stream)))

    def host_wait(self, stream=None):
        """Waits for what the host-buffer calls have enqueued (gs_host_wait)."""
        self._check(self._lib.gs_host_wait(self._h, self._stream(stream)))
        self._deferred = None

    def risk_scan_host(self, assigned_inst, generated_tokens, pred_len, elapsed_ms, slo_ms, types, inst,
                       out_flag_bits, out_cand_idx, stream=None) -> int:
        """Host-buffer variant; returns the true number of flagged requests."""
        n = int(assigned_inst.shape[0])
        cap = 0 if out_cand_idx is None else int(out_cand_idx.shape[0])
        hi, ht = self._host_pool_structs(types, inst)
        count = C.c_int64(0)
        self._check(self._lib.gs_risk_scan_host(
            self._h, _host_ptr(assigned_inst, np.int32, n, "assigned_inst"),
            _host_ptr(generated_tokens, np.int32, n, "generated_tokens"),
            _host_ptr(pred_len, np.int32, n, "pred_len"),
            _host_ptr(elapsed_ms, np.float32, n, "elapsed_ms"), _host_ptr(slo_ms, np.float32, n, "slo_ms"), n,
            C.byref(hi), C.byref(ht), _host_ptr(out_flag_bits, np.uint32, (n + 31) // 32, "out_flag_bits"),
            _host_ptr(out_cand_idx, np.int32, cap, "out_cand_idx"), cap,
            C.cast(C.byref(count), C.c_void_p), self._stream(stream)))
        return int(count.value)

    # -- the length predictor's operators, same names ---------------------------------------
    def expert_route(self, logits, router: ExpertRouter, out_expert, out_weight, out_offsets=None, out_row_token=None,
                     out_token_row=None, bias=None, stream=None):
        """gs_expert_route.  logits [tokens, experts] (float32, bfloat16 or float16; any row stride);
        out_expert, out_weight and out_token_row [tokens, top_k], out_offsets [experts + 1],
        out_row_token [tokens * top_k]; the last three together or not at all."""
        dev, i32 = self._index, torch.int32
        code = _DTYPES.get(logits.dtype)
        if code is None:
            raise TypeError(f"logits: expected float32, bfloat16 or float16, got {logits.dtype}")
        n, e, k = logits.shape[0], router.n_experts, router.top_k
        x, ld = _matrix(logits, logits.dtype, n, e, "logits", dev)
        self._check(self._lib.gs_expert_route(
            self._h, x, code, n, ld, _array(bias, torch.float32, e, "bias", dev), router._address,
            _array(out_expert, i32, n * k, "out_expert", dev), _array(out_weight, torch.float32, n * k, "out_weight", dev),
            _array(out_offsets, i32, e + 1, "out_offsets", dev), _array(out_row_token, i32, n * k, "out_row_token", dev),
            _array(out_token_row, i32, n * k, "out_token_row", dev), _raw_stream(dev) if stream is None else stream.cuda_stream))

    def expert_route_backward(self, logits, router: ExpertRouter, expert, d_weight, out_d_logits, stream=None):
        """gs_expert_route_backward: d_weight [tokens, top_k] to out_d_logits [tokens, experts]."""
        dev, n, e, k = self._index, logits.shape[0], router.n_experts, router.top_k
        code = _DTYPES.get(logits.dtype)
        if code is None:
            raise TypeError(f"logits: expected float32, bfloat16 or float16, got {logits.dtype}")
        x, ld = _matrix(logits, logits.dtype, n, e, "logits", dev)
        d, ld_d = _matrix(out_d_logits, logits.dtype, n, e, "out_d_logits", dev)
        self._check(self._lib.gs_expert_route_backward(
            self._h, x, code, n, ld, router._address, _array(expert, torch.int32, n * k, "expert", dev),
            _array(d_weight, torch.float32, n * k, "d_weight", dev), d, ld_d, _raw_stream(dev) if stream is None else stream.cuda_stream))

    def expert_linear(self, x, w, offsets, out, bias=None, row_token=None, relu: bool = False, stream=None):
        """gs_expert_linear: out[r] = act(x[row_token[r]] . w[e]^T + bias[e]) for the rows r of expert e.
        w [experts, out, in]; without row_token x has a row for every row of out."""
        dev, dt = self._index, x.dtype
        if dt not in _OPERANDS:
            raise TypeError(f"x: expected bfloat16 or float16, got {dt}")
        wp, ldw = _stack(w, dt, w.shape, "w", dev)
        e, o, i = w.shape
        rows, nx = out.shape[0], x.shape[0]
        xp, ldx = _matrix(x, dt, nx, i, "x", dev)
        yp, ldy = _matrix(out, dt, rows, o, "out", dev)
        self._check(self._lib.gs_expert_linear(
            self._h, _DTYPES[dt], xp, nx, ldx, _array(row_token, torch.int32, rows, "row_token", dev),
            _array(offsets, torch.int32, e + 1, "offsets", dev), e, rows, wp, ldw,
            _array(bias, torch.float32, e * o, "bias", dev), i, o, 1 if relu else 0, yp, ldy, _raw_stream(dev) if stream is None else stream.cuda_stream))

    def expert_linear_backward(self, dz, x, w, offsets, dx=None, dw=None, db=None, row_token=None,
                               relu_input: bool = False, stream=None):
        """gs_expert_linear_backward: fills those of dx [rows, in], dw [experts, out, in] (float32) and
        db [experts, out] (float32) that are given.  The partial sums' workspace comes from PyTorch's
        allocator, on the stream of the call."""
        dev, dt = self._index, dz.dtype
        if dt not in _OPERANDS:
            raise TypeError(f"dz: expected bfloat16 or float16, got {dt}")
        wp, ldw = _stack(w, dt, w.shape, "w", dev)
        e, o, i = w.shape
        rows, nx = dz.shape[0], x.shape[0]
        zp, ldz = _matrix(dz, dt, rows, o, "dz", dev)
        xp, ldx = _matrix(x, dt, nx, i, "x", dev)
        dxp = dwp = workspace = None
        lddx = lddw = need = 0
        if dx is not None:
            dxp, lddx = _matrix(dx, dt, rows, i, "dx", dev)
        if dw is not None:
            dwp, lddw = _stack(dw, torch.float32, w.shape, "dw", dev)
            need = self._lib.gs_expert_linear_backward_workspace(self._h, e, rows, i, o)
            if need > 0:
                # (from the pool of the stream that uses it: what another stream gave back there, that stream's
                # kernels may still be writing)
                with torch.cuda.stream(stream):
                    workspace = torch.empty(need, dtype=torch.uint8, device=self.device)
        self._check(self._lib.gs_expert_linear_backward(
            self._h, _DTYPES[dt], zp, ldz, xp, nx, ldx, _array(row_token, torch.int32, rows, "row_token", dev),
            _array(offsets, torch.int32, e + 1, "offsets", dev), e, rows, wp, ldw, i, o, 2 if relu_input else 0,
            dxp, lddx, dwp, lddw, _array(db, torch.float32, e * o, "db", dev),
            None if workspace is None else workspace.data_ptr(), max(need, 0), _raw_stream(dev) if stream is None else stream.cuda_stream))

    def expert_combine(self, y, token_row, out, weight=None, stream=None):
        """gs_expert_combine: out[n] = sum over j of weight[n, j] * y[token_row[n, j]]; out in y's dtype or float32."""
        dev, dt = self._index, y.dtype
        if dt not in _OPERANDS:
            raise TypeError(f"y: expected bfloat16 or float16, got {dt}")
        if out.dtype is not dt and out.dtype is not torch.float32:
            raise TypeError(f"out: expected {dt} or float32, got {out.dtype}")
        (n, k), (rows, f) = token_row.shape, y.shape
        yp, ldy = _matrix(y, dt, rows, f, "y", dev)
        op, ldo = _matrix(out, out.dtype, n, f, "out", dev)
        self._check(self._lib.gs_expert_combine(
            self._h, _DTYPES[dt], yp, rows, ldy, _array(token_row, torch.int32, n * k, "token_row", dev),
            _array(weight, torch.float32, n * k, "weight", dev), n, k, f, _DTYPES[out.dtype], op, ldo, _raw_stream(dev) if stream is None else stream.cuda_stream))

    def expert_combine_backward(self, d_out, y, token_row, dy=None, weight=None, d_weight=None, relu: bool = False,
                                stream=None):
        """gs_expert_combine_backward: fills those of dy [rows, features] and d_weight [tokens, top_k] that are given."""
        dev, dt = self._index, y.dtype
        if dt not in _OPERANDS:
            raise TypeError(f"y: expected bfloat16 or float16, got {dt}")
        if d_out.dtype is not dt and d_out.dtype is not torch.float32:
            raise TypeError(f"d_out: expected {dt} or float32, got {d_out.dtype}")
        (n, k), (rows, f) = token_row.shape, y.shape
        yp, ldy = _matrix(y, dt, rows, f, "y", dev)
        gp, ldg = _matrix(d_out, d_out.dtype, n, f, "d_out", dev)
        dyp, lddy = (None, 0) if dy is None else _matrix(dy, dt, rows, f, "dy", dev)
        self._check(self._lib.gs_expert_combine_backward(
            self._h, _DTYPES[dt], _DTYPES[d_out.dtype], gp, ldg, yp, rows, ldy,
            _array(token_row, torch.int32, n * k, "token_row", dev), _array(weight, torch.float32, n * k, "weight", dev),
            n, k, f, 2 if relu else 0, dyp, lddy, _array(d_weight, torch.float32, n * k, "d_weight", dev), _raw_stream(dev) if stream is None else stream.cuda_stream))

    def clip_grad_norm(self, grads, max_norm: float, out_norm, outs=None, write: bool = True, stream=None):
        """gs_clip_grad_norm over contiguous tensors (float32, bfloat16 or float16): scales them in place, or into
        ``outs``, so that their global norm is at most max_norm.  out_norm: one float32 on the device.  With
        ``write=False`` only the norm is computed."""
        if outs is not None and len(outs) != len(grads):
            raise ValueError(f"outs: needs {len(grads)} tensors, has {len(outs)}")
        flat, dev = [], self._index                    # four words for every gs_grad
        for k, g in enumerate(grads):
            code, n, p = _DTYPES.get(g.dtype), g.numel(), g.data_ptr()
            if code is None or not g.is_cuda or g.get_device() != dev or not g.is_contiguous():
                raise TypeError(f"grads[{k}]: expected a contiguous float32, bfloat16 or float16 tensor on cuda:{dev}")
            if outs is not None:
                o = outs[k]
                if o.dtype is not g.dtype or o.numel() != n or not o.is_cuda or o.get_device() != dev or not o.is_contiguous():
                    raise TypeError(f"outs[{k}]: expected a contiguous {g.dtype} tensor of {n} elements on cuda:{dev}")
                flat += (p, o.data_ptr(), n, code)
            else:
                flat += (p, p if write else 0, n, code)
        if outs is not None and not write:
            flat[1::4] = [0] * len(grads)
        table = array("q", flat)
        self._check(self._lib.gs_clip_grad_norm(self._h, table.buffer_info()[0], len(grads), float(max_norm),
                                                _array(out_norm, torch.float32, 1, "out_norm", dev),
                                                _raw_stream(dev) if stream is None else stream.cuda_stream))

    def device_status(self, stream=None) -> int:
        bits = C.c_uint(0)
        self._check(self._lib.gs_device_status(self._h, self._stream(stream), C.byref(bits)))
        return int(bits.value)

    def eval_counters(self, clear: bool = True, stream=None):
        """Work counters of the routing kernels (all zero unless the library was built with
        -DGS_COUNT_EVALS): exact scorings, row bounds, type bounds, queued, fallback, exhaustive."""
        out = (C.c_uint64 * 8)()
        self._check(self._lib.gs_eval_counters(self._h, self._stream(stream), out, 1 if clear else 0))
        return [int(v) for v in out]

    def launch_count(self) -> int:
        return int(self._lib.gs_launch_count(self._h))

    def timing_enable(self, on: bool):
        self._check(self._lib.gs_timing_enable(self._h, 1 if on else 0))

    def timing_read(self, kernel: int):
        """(total milliseconds, launches) of one kernel since timing was enabled."""
        ms, n = C.c_double(0.0), C.c_int64(0)
        self._check(self._lib.gs_timing_read(self._h, int(kernel), C.byref(ms), C.byref(n)))
        return float(ms.value), int(n.value)

    def last_cuda_error(self) -> int:
        return int(self._lib.gs_last_cuda_error(self._h))


NOALLOC_MAX_ACTIVE = 16_777_216


def risk_scan_noalloc(assigned_inst, generated_tokens, pred_len, elapsed_ms, slo_ms, pool: InstancePool,
                      out_flag_bits, out_cand_idx, out_cand_count, out_status_bits=None,
                      cand_capacity: Optional[int] = None, n_active: Optional[int] = None, stream=None):
    """gs_risk_scan_noalloc: the risk scan for callers that must not allocate device memory.

    Needs no GoodServe context (creating one allocates).  The scan's scratch is a fixed array
    inside the library, shared by every call on the same GPU, so calls on one GPU must not
    overlap; at most NOALLOC_MAX_ACTIVE requests per call.  Runs on the tensors' device, which
    must be the current CUDA device.  This wrapper allocates nothing either: every tensor,
    including the optional one-word ``out_status_bits`` (int32, zeroed by the caller), is the
    caller's.
    """
    lib = load_library()
    n = int(assigned_inst.numel()) if n_active is None else int(n_active)
    cap = (0 if out_cand_idx is None else int(out_cand_idx.numel())) if cand_capacity is None else int(cand_capacity)
    dev = assigned_inst.device
    if torch.cuda.current_device() != dev.index:
        raise ValueError("risk_scan_noalloc runs on the current device; make the tensors' device current")
    i32, f32 = torch.int32, torch.float32
    M, Tn = pool.n_instances, pool.n_types
    inst = _Instances(_dev_ptr(pool.type_id, i32, M, "type_id", dev),
                      _dev_ptr(pool.queued_prefill_tokens, i32, M, "queued_prefill_tokens", dev),
                      _dev_ptr(pool.decode_batch, i32, M, "decode_batch", dev),
                      _dev_ptr(pool.free_kv_tokens, i32, M, "free_kv_tokens", dev),
                      _dev_ptr(pool.q_ema_ms, f32, M, "q_ema_ms", dev), M)
    types = _Types(_dev_ptr(pool.prefill_ms_per_tok, f32, Tn, "prefill_ms_per_tok", dev),
                   _dev_ptr(pool.tpot_a_ms, f32, Tn, "tpot_a_ms", dev),
                   _dev_ptr(pool.tpot_b_ms, f32, Tn, "tpot_b_ms", dev), Tn)
    s = torch.cuda.current_stream(dev) if stream is None else stream
    rc = lib.gs_risk_scan_noalloc(
        _dev_ptr(assigned_inst, i32, n, "assigned_inst", dev),
        _dev_ptr(generated_tokens, i32, n, "generated_tokens", dev),
        _dev_ptr(pred_len, i32, n, "pred_len", dev),
        _dev_ptr(elapsed_ms, f32, n, "elapsed_ms", dev),
        _dev_ptr(slo_ms, f32, n, "slo_ms", dev), n,
        C.byref(inst), C.byref(types),
        _dev_ptr(out_flag_bits, i32, (n + 31) // 32, "out_flag_bits", dev),
        _dev_ptr(out_cand_idx, i32, cap, "out_cand_idx", dev), cap,
        _dev_ptr(out_cand_count, torch.int64, 1, "out_cand_count", dev),
        _dev_ptr(out_status_bits, i32, 1, "out_status_bits", dev), s.cuda_stream or None)
    if rc != 0:
        raise GoodServeError(rc, lib.gs_strerror(rc).decode())
