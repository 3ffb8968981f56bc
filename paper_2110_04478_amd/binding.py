"""ctypes binding of libthemis_hip.so: argument marshalling only.

PyTorch is used for device memory and the current HIP stream; every
computation happens in the library's kernels.  Loading fails loudly if the
library has not been built (python paper_2110_04478_amd/csrc/build.py).
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from dataclasses import dataclass
from typing import Optional

import numpy as np
import torch

from . import overlap

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libthemis_hip.so")

MAX_DIMS = 4
MAX_CHUNKS = 512

_vp = C.c_void_p


class _Batch(C.Structure):
    _fields_ = [
        ("n", C.c_uint64), ("max_chunks", C.c_uint32), ("threshold_mode", C.c_uint32),
        ("ndims", _vp), ("npus", _vp), ("bw", _vp), ("size_bytes", _vp), ("chunks", _vp),
        ("inter_policy", _vp), ("intra_policy", _vp), ("threshold", _vp),
        ("max_coll", C.c_uint32), ("n_coll", _vp), ("coll_size", _vp), ("release_time", _vp),
        ("fixed_delay", _vp), ("collective_type", _vp),
    ]


class _Rows(C.Structure):
    _fields_ = [("data", _vp), ("type", C.c_int32), ("inner", C.c_uint64),
                ("outer_stride", C.c_int64), ("inner_stride", C.c_int64)]


class _Gradient(C.Structure):
    _fields_ = [("in_", _vp), ("out", _vp), ("tensor", C.c_uint32), ("in_type", C.c_int32),
                ("out_type", C.c_int32), ("rows", C.c_uint64), ("cols", C.c_uint64),
                ("in_row_stride", C.c_int64), ("in_col_stride", C.c_int64),
                ("out_row_stride", C.c_int64), ("out_col_stride", C.c_int64)]


class _GradientPlan(C.Structure):
    _fields_ = [("n_tensors", C.c_uint64), ("n_pieces", C.c_uint64), ("image_bytes", C.c_uint64),
                ("workspace_bytes", C.c_uint64), ("in_bytes", C.c_uint64), ("has_out", C.c_uint32),
                ("strided", C.c_uint32), ("image", _vp)]


class _ExpertOrder(C.Structure):
    _fields_ = [("n", C.c_uint64), ("k", C.c_uint64), ("n_experts", C.c_uint64), ("capacity", C.c_uint64),
                ("place", _vp), ("counts", _vp), ("starts", _vp), ("source", _vp)]


_lib = None


def lib():
    """The loaded C ABI library; raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with "
                "`python paper_2110_04478_amd/csrc/build.py` (there is no CPU fallback)")
        L = C.CDLL(LIB_PATH)
        L.themis_version.restype = C.c_int
        L.themis_status_string.restype = C.c_char_p
        L.themis_status_string.argtypes = [C.c_int]
        L.themis_queue_entry_bytes.restype = C.c_int
        L.themis_queue_entry_bytes.argtypes = [C.c_uint32, C.c_uint32]
        L.themis_workspace_bytes.restype = C.c_size_t
        L.themis_workspace_bytes.argtypes = [C.c_uint64, C.c_uint32, C.c_uint32]
        L.themis_plan_batch.restype = C.c_int
        L.themis_plan_batch.argtypes = [C.POINTER(_Batch), _vp, _vp, _vp]
        L.themis_simulate_batch.restype = C.c_int
        L.themis_simulate_batch.argtypes = [C.POINTER(_Batch), _vp, _vp, _vp, _vp, _vp,
                                            C.c_size_t, _vp]
        L.themis_simulate_batch_noalloc.restype = C.c_int
        L.themis_simulate_batch_noalloc.argtypes = [C.POINTER(_Batch), _vp, _vp, _vp, _vp, _vp]
        L.themis_metrics_batch.restype = C.c_int
        L.themis_metrics_batch.argtypes = [C.POINTER(_Batch), _vp, _vp, _vp, _vp, _vp]
        L.themis_search_workspace_bytes.restype = C.c_size_t
        L.themis_search_workspace_bytes.argtypes = [C.c_uint64, C.c_uint64]
        L.themis_search_batch.restype = C.c_int
        L.themis_search_batch.argtypes = [C.POINTER(_Batch), C.c_uint64, _vp, _vp, _vp,
                                          C.c_size_t, _vp]
        L.themis_beam_workspace_bytes.restype = C.c_size_t
        L.themis_beam_workspace_bytes.argtypes = [C.c_uint64, C.c_uint32, C.c_uint32]
        L.themis_beam_search_batch.restype = C.c_int
        L.themis_beam_search_batch.argtypes = [C.POINTER(_Batch), C.c_uint32, _vp, _vp, _vp,
                                               C.c_size_t, _vp]
        L.themis_classify_batch.restype = C.c_int
        L.themis_classify_batch.argtypes = [C.POINTER(_Batch), _vp, _vp]
        L.themis_sweep_best.restype = C.c_int
        L.themis_sweep_best.argtypes = [C.c_uint64, C.c_int, C.c_int, _vp, C.c_int, _vp, _vp, _vp, _vp]
        L.themis_set_sweep_mapping.restype = C.c_int
        L.themis_set_sweep_mapping.argtypes = [C.c_int]
        L.themis_set_batch_mapping.restype = C.c_int
        L.themis_set_batch_mapping.argtypes = [C.c_int]
        L.themis_sweep.restype = C.c_int
        L.themis_sweep.argtypes = [C.POINTER(_Batch), C.c_int, _vp, C.c_int, C.c_uint, _vp,
                                   _vp, C.c_size_t, _vp]
        L.themis_sweep_scratch_bytes.restype = C.c_size_t
        L.themis_sweep_scratch_bytes.argtypes = [C.c_uint64, C.c_uint32, C.c_int, C.c_uint]
        L.themis_sweep_with_scratch.restype = C.c_int
        L.themis_sweep_with_scratch.argtypes = [C.POINTER(_Batch), C.c_int, _vp, C.c_int, C.c_uint,
                                                _vp, _vp, C.c_size_t, _vp, C.c_size_t, _vp]
        L.themis_embedding_lookup.restype = C.c_int
        L.themis_embedding_lookup.argtypes = [C.POINTER(_Rows), C.c_uint64, C.c_uint64, C.POINTER(_Rows),
                                              C.c_uint64, C.c_float, C.POINTER(_Rows), _vp]
        L.themis_embedding_grad_workspace_bytes.restype = C.c_size_t
        L.themis_embedding_grad_workspace_bytes.argtypes = [C.c_uint64, C.c_uint64, C.c_uint64]
        L.themis_embedding_grad.restype = C.c_int
        L.themis_embedding_grad.argtypes = [C.POINTER(_Rows), C.c_uint64, C.POINTER(_Rows), C.c_uint64,
                                            C.c_float, C.c_int64, C.c_int, C.POINTER(_Rows), C.c_uint64,
                                            _vp, C.c_size_t, _vp]
        L.themis_gradient_plan.restype = C.c_int
        L.themis_gradient_plan.argtypes = [C.POINTER(_Gradient), C.c_uint64, C.c_uint64,
                                           C.POINTER(_GradientPlan), _vp, C.c_size_t]
        L.themis_gradient_norm.restype = C.c_int
        L.themis_gradient_norm.argtypes = [C.POINTER(_GradientPlan), _vp, _vp, _vp, C.c_size_t, _vp]
        L.themis_gradient_clip.restype = C.c_int
        L.themis_gradient_clip.argtypes = [C.POINTER(_GradientPlan), C.c_double, _vp, _vp, _vp,
                                           C.c_size_t, _vp]
        rows, order = C.POINTER(_Rows), C.POINTER(_ExpertOrder)
        L.themis_expert_gate.restype = C.c_int
        L.themis_expert_gate.argtypes = [rows, C.c_uint64, C.c_uint64, C.c_uint64, C.c_int, rows, rows, _vp]
        L.themis_expert_gate_grad.restype = C.c_int
        L.themis_expert_gate_grad.argtypes = [rows, rows, C.c_uint64, rows, C.c_uint64, C.c_uint64, C.c_int,
                                              rows, _vp]
        L.themis_expert_sort_workspace_bytes.restype = C.c_size_t
        L.themis_expert_sort_workspace_bytes.argtypes = [C.c_uint64, C.c_uint64, C.c_uint64]
        L.themis_expert_sort.restype = C.c_int
        L.themis_expert_sort.argtypes = [rows, order, _vp, C.c_size_t, _vp]
        L.themis_expert_dispatch.restype = C.c_int
        L.themis_expert_dispatch.argtypes = [order, rows, C.c_uint64, rows, _vp]
        L.themis_expert_combine.restype = C.c_int
        L.themis_expert_combine.argtypes = [order, rows, C.c_uint64, rows, C.c_int, rows, _vp]
        L.themis_expert_combine_grad.restype = C.c_int
        L.themis_expert_combine_grad.argtypes = [order, rows, C.c_uint64, rows, rows, rows, rows, _vp]
        L.themis_dropout.restype = C.c_int
        L.themis_dropout.argtypes = [rows, C.c_uint64, C.c_uint64, C.c_double, C.c_uint64, C.c_uint64, _vp, rows,
                                     rows, _vp]
        _lib = L
    return _lib


class ThemisError(RuntimeError):
    def __init__(self, status: int, why: str = ""):
        self.status = status
        super().__init__(f"themis: {lib().themis_status_string(status).decode()} ({status}){why and ': ' + why}")


def _check(status: int):
    if status != 0:
        raise ThemisError(status)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else _vp(t.data_ptr())


def _stream() -> _vp:
    return _vp(torch.cuda.current_stream().cuda_stream)


@dataclass
class DeviceBatch:
    """A scenario batch resident in HBM (torch tensors own the memory)."""
    n: int
    max_chunks: int
    threshold_mode: int
    ndims: torch.Tensor
    npus: torch.Tensor
    bw: torch.Tensor
    size_bytes: torch.Tensor
    chunks: torch.Tensor
    inter_policy: torch.Tensor
    intra_policy: torch.Tensor
    threshold: torch.Tensor
    max_coll: int = 0
    n_coll: Optional[torch.Tensor] = None
    coll_size: Optional[torch.Tensor] = None
    release_time: Optional[torch.Tensor] = None
    fixed_delay: Optional[torch.Tensor] = None
    collective_type: Optional[torch.Tensor] = None

    @property
    def slots(self) -> int:
        return self.max_chunks * (self.max_coll if self.n_coll is not None else 1)

    @property
    def device(self):
        return self.ndims.device

    def c_struct(self) -> _Batch:
        return _Batch(self.n, self.max_chunks, self.threshold_mode, _ptr(self.ndims),
                      _ptr(self.npus), _ptr(self.bw), _ptr(self.size_bytes), _ptr(self.chunks),
                      _ptr(self.inter_policy), _ptr(self.intra_policy), _ptr(self.threshold),
                      self.max_coll, _ptr(self.n_coll), _ptr(self.coll_size),
                      _ptr(self.release_time), _ptr(self.fixed_delay),
                      _ptr(self.collective_type))


def to_device(b, device="cuda:0") -> DeviceBatch:
    """Copies a host workloads.ScenarioBatch into HBM."""
    def up(a, dt):
        if a is None:
            return None
        a = np.ascontiguousarray(a)
        if not a.flags.writeable:  # broadcast views: torch wants a writable source
            a = a.copy()
        if dt == torch.uint32:  # torch cannot build uint32 from numpy directly everywhere
            return torch.from_numpy(a.view(np.int32)).to(device).view(torch.uint32)
        return torch.from_numpy(a).to(device)
    return DeviceBatch(
        n=int(b.n), max_chunks=int(b.max_chunks), threshold_mode=int(b.threshold_mode),
        ndims=up(b.ndims, torch.uint8), npus=up(b.npus, torch.uint32), bw=up(b.bw, torch.float64),
        size_bytes=up(b.size_bytes, torch.float64), chunks=up(b.chunks, torch.uint32),
        inter_policy=up(b.inter_policy, torch.uint8), intra_policy=up(b.intra_policy, torch.uint8),
        threshold=up(b.threshold, torch.float64), max_coll=int(b.max_coll),
        n_coll=up(b.n_coll, torch.uint32), coll_size=up(b.coll_size, torch.float64),
        release_time=up(b.release_time, torch.float64),
        fixed_delay=up(getattr(b, "fixed_delay", None), torch.float64),
        collective_type=up(getattr(b, "collective_type", None), torch.uint8))


def themis_version() -> int:
    return lib().themis_version()


def themis_queue_entry_bytes(max_chunks: int, max_coll: int = 0) -> int:
    return lib().themis_queue_entry_bytes(max_chunks, max_coll)


def themis_workspace_bytes(n: int, max_chunks: int, max_coll: int = 0) -> int:
    return lib().themis_workspace_bytes(n, max_chunks, max_coll)


def themis_plan_batch(b: DeviceBatch, orders: Optional[torch.Tensor] = None,
                      loads: Optional[torch.Tensor] = None, want_loads: bool = True):
    """Alg. 1 for every scenario -> (orders u8[n, slots], loads f64[4, n] or None)."""
    if orders is None:
        orders = torch.empty((b.n, b.slots), dtype=torch.uint8, device=b.device)
    if loads is None and want_loads:
        loads = torch.empty((MAX_DIMS, b.n), dtype=torch.float64, device=b.device)
    s = b.c_struct()
    _check(lib().themis_plan_batch(C.byref(s), _ptr(orders), _ptr(loads), _stream()))
    return orders, loads


def themis_simulate_batch(b: DeviceBatch, orders: torch.Tensor,
                          t_done: Optional[torch.Tensor] = None,
                          queue_order: Optional[torch.Tensor] = None,
                          busy: Optional[torch.Tensor] = None,
                          workspace: Optional[torch.Tensor] = None,
                          want_queue_order: bool = True, want_busy: bool = True):
    """Queue simulation -> (t_done f64[n], queue_order [n,4,2*slots] or None,
    busy f64[4,n] or None)."""
    dev = b.device
    if t_done is None:
        t_done = torch.empty(b.n, dtype=torch.float64, device=dev)
    if queue_order is None and want_queue_order:
        eb = themis_queue_entry_bytes(b.max_chunks, b.max_coll if b.n_coll is not None else 0)
        queue_order = torch.empty((b.n, MAX_DIMS, 2 * b.slots),
                                  dtype=torch.uint8 if eb == 1 else torch.uint16, device=dev)
    if busy is None and want_busy:
        busy = torch.empty((MAX_DIMS, b.n), dtype=torch.float64, device=dev)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    s = b.c_struct()
    _check(lib().themis_simulate_batch(C.byref(s), _ptr(orders), _ptr(t_done), _ptr(queue_order),
                                       _ptr(busy), _ptr(workspace), ws_bytes, _stream()))
    return t_done, queue_order, busy


STATIC_SCRATCH_BYTES = 32 << 20


def themis_simulate_batch_noalloc(b: DeviceBatch, orders: torch.Tensor, t_done: torch.Tensor,
                                  queue_order: Optional[torch.Tensor],
                                  busy: Optional[torch.Tensor]):
    """themis_simulate_batch on the library's own scratch: every buffer is the
    caller's, nothing is allocated here or in the library."""
    s = b.c_struct()
    _check(lib().themis_simulate_batch_noalloc(C.byref(s), _ptr(orders), _ptr(t_done),
                                               _ptr(queue_order), _ptr(busy), _stream()))
    return t_done, queue_order, busy


def themis_sweep_scratch_bytes(n: int, max_chunks: int, n_thr: int, policy_mask: int) -> int:
    """Bytes of scratch a sweep of this size can use (0: none)."""
    return lib().themis_sweep_scratch_bytes(n, max_chunks, n_thr, policy_mask)


def themis_sweep(b: DeviceBatch, thr: torch.Tensor, policy_mask: int,
                 thr_per_scenario: bool = False, t_done: Optional[torch.Tensor] = None,
                 workspace: Optional[torch.Tensor] = None, scratch: Optional[torch.Tensor] = None):
    """Fused plan + simulate -> t_done f64[n, n_thr, n_pol].

    scratch: themis_sweep_scratch_bytes() bytes in which the thresholds that share a plan are
    listed; allocated for the call where it is not given, and done without (same results) where
    there is no room for it."""
    n_thr = int(thr.shape[0])
    n_pol = bin(policy_mask & 7).count("1")
    if t_done is None:
        t_done = torch.empty((b.n, n_thr, n_pol), dtype=torch.float64, device=b.device)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    # (a sweep of fewer evaluations is one turn of the GPU's wavefronts and has no use for the
    # list: not worth the call, 1 us of the 12 that a small sweep takes)
    if scratch is None and b.n * n_thr >= 8192:
        try:   # (stream-ordered: torch hands it on only behind this stream's work)
            scratch = alloc_workspace(themis_sweep_scratch_bytes(b.n, b.max_chunks, n_thr, policy_mask),
                                      b.device)
        except torch.OutOfMemoryError:
            pass
    need = 0 if scratch is None else scratch.numel() * scratch.element_size()
    s = b.c_struct()
    _check(lib().themis_sweep_with_scratch(C.byref(s), n_thr, _ptr(thr), 1 if thr_per_scenario else 0,
                                           policy_mask, _ptr(t_done), _ptr(workspace), ws_bytes,
                                           _ptr(scratch), need, _stream()))
    return t_done


MAPPING_AUTO, MAPPING_LANE, MAPPING_QUAD, MAPPING_WAVE = 0, 1, 2, 3


def themis_set_sweep_mapping(mapping: int) -> None:
    """One lane or four per evaluation (MAPPING_AUTO / _LANE / _QUAD) in themis_sweep, and in
    themis_simulate_batch (single collectives and traces) where it does not take a wavefront each;
    beyond 64 chunks there are only four.  Process-wide."""
    _check(lib().themis_set_sweep_mapping(int(mapping)))


def themis_set_batch_mapping(mapping: int) -> None:
    """Whether the planner and the simulation (single collectives and traces) take a wavefront per
    scenario: in small batches (MAPPING_AUTO), never (_LANE: one lane or four, as
    themis_set_sweep_mapping says) or wherever they can (_WAVE).  Process-wide."""
    _check(lib().themis_set_batch_mapping(int(mapping)))


def themis_metrics_batch(b: DeviceBatch, t_done: torch.Tensor, transfer: torch.Tensor,
                         utilization: Optional[torch.Tensor] = None,
                         ideal: Optional[torch.Tensor] = None):
    """Average bandwidth utilisation and Ideal time -> (utilization f64[n], ideal f64[n])."""
    if utilization is None:
        utilization = torch.empty(b.n, dtype=torch.float64, device=b.device)
    if ideal is None:
        ideal = torch.empty(b.n, dtype=torch.float64, device=b.device)
    s = b.c_struct()
    _check(lib().themis_metrics_batch(C.byref(s), _ptr(t_done), _ptr(transfer), _ptr(utilization),
                                      _ptr(ideal), _stream()))
    return utilization, ideal


def themis_beam_search_batch(b: DeviceBatch, width: int, workspace: Optional[torch.Tensor] = None):
    """Beam search over per-chunk orders -> (best_t f64[n], best_orders u8[n, max_chunks])."""
    best_t = torch.empty(b.n, dtype=torch.float64, device=b.device)
    best_orders = torch.empty((b.n, b.max_chunks), dtype=torch.uint8, device=b.device)
    if workspace is None:
        workspace = alloc_workspace(lib().themis_beam_workspace_bytes(b.n, b.max_chunks, width),
                                    b.device)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    s = b.c_struct()
    _check(lib().themis_beam_search_batch(C.byref(s), int(width), _ptr(best_t), _ptr(best_orders),
                                          _ptr(workspace), ws_bytes, _stream()))
    return best_t, best_orders


def themis_search_workspace_bytes(n: int, max_assignments: int) -> int:
    return lib().themis_search_workspace_bytes(n, max_assignments)


def themis_search_batch(b: DeviceBatch, max_assignments: int,
                        workspace: Optional[torch.Tensor] = None):
    """Exhaustive search over per-chunk orders -> (best_t f64[n], best_orders u8[n, max_chunks])."""
    best_t = torch.empty(b.n, dtype=torch.float64, device=b.device)
    best_orders = torch.empty((b.n, b.max_chunks), dtype=torch.uint8, device=b.device)
    if workspace is None:
        workspace = alloc_workspace(themis_search_workspace_bytes(b.n, max_assignments), b.device)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    s = b.c_struct()
    _check(lib().themis_search_batch(C.byref(s), max_assignments, _ptr(best_t), _ptr(best_orders),
                                     _ptr(workspace), ws_bytes, _stream()))
    return best_t, best_orders


def themis_classify_batch(b: DeviceBatch) -> torch.Tensor:
    """Bandwidth provisioning class of every dimension pair -> u8[6, n]."""
    classes = torch.empty((6, b.n), dtype=torch.uint8, device=b.device)
    s = b.c_struct()
    _check(lib().themis_classify_batch(C.byref(s), _ptr(classes), _stream()))
    return classes


def themis_sweep_best(t_done: torch.Tensor, baseline_col: int = -1):
    """Best threshold per scenario and scheduler of a sweep result f64[n, n_thr, n_pol]
    -> (best_t f64[n, n_pol], best_thr u32[n, n_pol], speedup f64[n, n_pol] or None)."""
    n, n_thr, n_pol = t_done.shape
    assert t_done.dtype == torch.float64 and t_done.is_contiguous()
    best_t = torch.empty((n, n_pol), dtype=torch.float64, device=t_done.device)
    best_thr = torch.empty((n, n_pol), dtype=torch.uint32, device=t_done.device)
    speedup = (torch.empty((n, n_pol), dtype=torch.float64, device=t_done.device)
               if baseline_col >= 0 else None)
    _check(lib().themis_sweep_best(n, n_thr, n_pol, _ptr(t_done), baseline_col, _ptr(best_t),
                                   _ptr(best_thr), _ptr(speedup), _stream()))
    return best_t, best_thr, speedup


def alloc_workspace(nbytes: int, device="cuda:0") -> Optional[torch.Tensor]:
    """Device scratch for the generic path (a plain byte tensor)."""
    if nbytes <= 0:
        return None
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


# -- gradients of an iteration ------------------------------------------------------------

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2, torch.int32: 3, torch.int64: 4}
INVALID_ARGUMENT = -1
UNSUPPORTED = -2


def _rows(t: torch.Tensor, lead: int, width: int) -> Optional[_Rows]:
    """t as rows of its last dimension (lead = t.dim() - 1, width elements) or of single elements
    (lead = t.dim(), width = 1), in the two levels of themis_rows; None where its strides need
    more."""
    if t.is_contiguous():
        return _Rows(t.data_ptr(), _TYPES[t.dtype], 1 << 31, 0, width)   # (one level)
    if width > 1 and t.stride(-1) != 1:
        return None
    levels = []   # (rows, stride), outermost first, merged where one stride covers both
    for n, s in zip(t.shape[:lead], t.stride()[:lead]):
        if n == 1:
            continue
        if levels and levels[-1][1] == n * s:
            levels[-1] = (levels[-1][0] * n, s)
        else:
            levels.append((n, s))
    if len(levels) > 2:
        return None
    outer = levels[0][1] if len(levels) == 2 else 0
    inner, step = levels[-1] if levels else (1, 0)
    return _Rows(t.data_ptr(), _TYPES[t.dtype], max(1, inner), outer, step)


def _read_rows(t: torch.Tensor, lead: int, width: int) -> tuple:
    """(rows, the tensor that holds them): t itself, or a copy where its strides are beyond
    what the library reads."""
    r = _rows(t, lead, width)
    if r is None:
        t = t.contiguous()
        r = _rows(t, lead, width)
    return r, t


def _need(ok: bool):
    if not ok:
        raise ThemisError(INVALID_ARGUMENT)


_FLOATS = frozenset((torch.float32, torch.bfloat16, torch.float16))
_INDEXES = frozenset((torch.int32, torch.int64))


# (0.3 us; what a call writes shares no memory with what it reads where their storages differ, and is
# looked at by _apart where not)
_one_storage = torch._C._is_alias_of


def _apart(out: torch.Tensor, *inputs) -> bool:
    return not overlap.shared([overlap.view_of(out)], [overlap.view_of(t) for t in inputs if t.numel()])


def _stream_here(device: int) -> int:
    """The current stream of this GPU, which has to be the current one.  (Through the raw
    handle: the stream object of torch.cuda.current_stream takes 2.7 us, a quarter of a call on
    a few rows.)"""
    _need(device == torch._C._cuda_getDevice())
    return torch._C._cuda_getCurrentRawStream(device)


def themis_embedding_lookup(table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0,
                            out: Optional[torch.Tensor] = None,
                            out_dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """scale * table[ids] -> [*ids.shape, width] of out's type (given by out or out_dtype;
    the table's otherwise).  A token number outside the table gives a row of NaN."""
    device = table.get_device()
    _need(device >= 0 and table.dim() == 2 and table.dtype in _FLOATS and ids.dtype in _INDEXES and
          ids.get_device() == device)
    vocab, width = table.shape
    shape = (*ids.shape, width)
    given = out is not None
    if not given:
        _need(out_dtype is None or out_dtype in _FLOATS)
        out = table.new_empty(shape, dtype=out_dtype)
    else:
        _need(out.dtype in _FLOATS and out.shape == shape and out.get_device() == device and
              out_dtype in (None, out.dtype))
    n = ids.numel()
    if n == 0 or width == 0:
        return out
    stream = _stream_here(device)
    rows_t, table = _read_rows(table, 1, width)
    rows_i, ids = _read_rows(ids, len(shape) - 1, 1)
    rows_o = _rows(out, len(shape) - 1, width)
    _need(rows_o is not None)
    if given and (_one_storage(out, table) or _one_storage(out, ids)):
        _need(_apart(out, table, ids))
    _check(lib().themis_embedding_lookup(rows_t, vocab, width, rows_i, n, scale, rows_o, stream))
    return out


@functools.lru_cache(maxsize=1024)   # (a function of the sizes alone; a call of the library takes 0.6 us)
def themis_embedding_grad_workspace_bytes(n: int, width: int, vocab: int) -> int:
    return lib().themis_embedding_grad_workspace_bytes(n, width, vocab)


def themis_embedding_grad(grad_out: torch.Tensor, ids: torch.Tensor, vocab: int, scale: float = 1.0,
                          ignored: int = -1, out: Optional[torch.Tensor] = None,
                          out_dtype: Optional[torch.dtype] = None, accumulate: bool = False,
                          workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The gradient of the table behind themis_embedding_lookup -> [vocab, width] of out's type
    (given by out or out_dtype; grad_out's otherwise), or added to out where `accumulate`.
    Tokens of number `ignored`, or outside the table, have no gradient."""
    device = grad_out.get_device()
    shape = grad_out.shape
    _need(device >= 0 and grad_out.dtype in _FLOATS and ids.dtype in _INDEXES and
          len(shape) >= 1 and shape[:-1] == ids.shape and ids.get_device() == device and
          vocab >= 0 and (out is not None or not accumulate) and
          (workspace is None or (workspace.get_device() == device and workspace.is_contiguous())))
    width = shape[-1]
    given = out is not None
    if not given:
        _need(out_dtype is None or out_dtype in _FLOATS)
        out = grad_out.new_empty((vocab, width), dtype=out_dtype)
    else:
        _need(out.dtype in _FLOATS and out.shape == (vocab, width) and
              out.get_device() == device and out_dtype in (None, out.dtype))
    n = ids.numel()
    if vocab == 0 or width == 0 or (n == 0 and accumulate):
        return out
    stream = _stream_here(device)
    rows_g, grad_out = _read_rows(grad_out, len(shape) - 1, width)
    rows_i, ids = _read_rows(ids, len(shape) - 1, 1)
    rows_o = _rows(out, 1, width)
    _need(rows_o is not None)
    if given and (_one_storage(out, grad_out) or _one_storage(out, ids)):
        _need(_apart(out, grad_out, ids))
    if workspace is None:
        need = themis_embedding_grad_workspace_bytes(n, width, vocab)
        if need:
            workspace = alloc_workspace(need, out.device)
    at, size = (None, 0) if workspace is None else (workspace.data_ptr(),
                                                    workspace.numel() * workspace.element_size())
    _check(lib().themis_embedding_grad(rows_g, width, rows_i, n, scale, ignored, int(accumulate),
                                       rows_o, vocab, at, size, stream))
    return out


@dataclass
class GradientPlan:
    """A list of gradients laid out for themis_gradient_norm / _clip.  It keeps the tensors, the
    device copy of the layout and the workspace, so calls on one plan must follow each other (one
    stream, or the caller's own ordering)."""
    grads: list
    out: Optional[list]
    image: torch.Tensor
    workspace: Optional[torch.Tensor]
    c_struct: _GradientPlan
    n_tensors: int
    streams: set   # raw handles: the one it was made on, and others that have used it

    @property
    def device(self):
        return self.image.device

    def stream(self) -> int:
        """The current stream; the plan's memory, once it is given up, waits for it."""
        stream = _stream_here(self.image.get_device())
        if stream not in self.streams:
            self.streams.add(stream)
            for t in (self.image, self.workspace):
                if t is not None:
                    t.record_stream(torch.cuda.current_stream())
        return stream

    @property
    def workspace_at(self) -> Optional[int]:
        return None if self.workspace is None else self.workspace.data_ptr()


def _views(g: torch.Tensor, o: Optional[torch.Tensor]):
    """g (and o, element for element) as views of two levels: yields (in offset, out offset,
    rows, cols, in row stride, in col stride, out row stride, out col stride), in elements."""
    so = o.stride() if o is not None else g.stride()
    dims = sorted(((abs(a), abs(b), n, a, b) for n, a, b in zip(g.shape, g.stride(), so) if n != 1),
                  reverse=True)
    merged = []   # (count, in stride, out stride), the longest steps first
    for _, _, n, a, b in dims:
        if merged and merged[-1][1] == n * a and merged[-1][2] == n * b:
            merged[-1] = (merged[-1][0] * n, a, b)
        else:
            merged.append((n, a, b))
    while len(merged) < 2:
        merged.insert(0, (1, 0, 0))
    offsets = [(0, 0)]
    for n, a, b in merged[:-2]:
        offsets = [(x + k * a, y + k * b) for x, y in offsets for k in range(n)]
    (rows, ra, rb), (cols, ca, cb) = merged[-2:]
    for x, y in offsets:
        yield x, y, rows, cols, ra, ca, rb, cb


def _targets_share(grads: list, outs: list) -> bool:
    """Whether some element of a target is given twice, or is one of a gradient that is not this
    target's own in place."""
    targets, others = [], []
    for g, o in zip(grads, outs):
        if o.numel() == 0:
            continue
        place = overlap.view_of(o)
        if not o.is_contiguous() and overlap.repeats(o):
            return True
        targets.append(place)
        if g is not o and (g.dtype != o.dtype or overlap.view_of(g) != place):
            others.append(overlap.view_of(g))
    return overlap.shared(targets, others)


def themis_gradient_plan(grads, out=None) -> GradientPlan:
    """Lays out a list of gradients for themis_gradient_norm and themis_gradient_clip.

    out: where the clipped gradients go, tensors of the gradients' shapes and any of the three
    types (parts of a flat bucket, say); the gradients themselves where it is not given.  Targets
    that share an element with each other, or with a gradient that is not theirs, are refused;
    gradients that share elements and have no other targets have norms alone.  Good for as long
    as the tensors stay where they are; their values may change.  (Host work: 482 tensors 2 ms.)"""
    grads = list(grads)
    _need(all(g.dtype in _FLOATS and g.is_cuda for g in grads) and
          len({g.device for g in grads}) <= 1)
    outs = grads if out is None else list(out)
    _need(len(outs) == len(grads) and
          all(o.dtype in _FLOATS and o.shape == g.shape and o.device == g.device for g, o in zip(grads, outs)))
    # (gradients that are their own targets and share elements, a broadcast or one given twice,
    # cannot be scaled in place: then only norms are to be had)
    twice = _targets_share(grads, outs)
    _need(out is None or not twice)
    plan = _GradientPlan()
    for with_out in ((False,) if twice else (True, False) if out is None else (True,)):
        parts = []
        for i, (g, o) in enumerate(zip(grads, outs)):
            if g.numel() == 0:
                continue
            gt, ot, ge, oe = _TYPES[g.dtype], _TYPES[o.dtype], g.element_size(), o.element_size()
            for x, y, rows, cols, ra, ca, rb, cb in _views(g, o):
                parts.append(_Gradient(g.data_ptr() + x * ge, o.data_ptr() + y * oe if with_out else None, i,
                                       gt, ot, rows, cols, ra, ca, rb, cb))
        array = (_Gradient * len(parts))(*parts)
        status = lib().themis_gradient_plan(array, len(parts), len(grads), plan, None, 0)
        if status != INVALID_ARGUMENT:
            break
    _check(status)
    image = np.empty((plan.image_bytes + 7) // 8, dtype=np.uint64)
    _check(lib().themis_gradient_plan(array, len(parts), len(grads), plan, image.ctypes.data,
                                      image.nbytes))
    device = grads[0].device if grads else torch.device("cuda", torch.cuda.current_device())
    streams = {torch._C._cuda_getCurrentRawStream(device.index)}
    on_device = torch.from_numpy(image.view(np.int64)).to(device)
    plan.image = on_device.data_ptr()
    return GradientPlan(grads, None if out is None else outs, on_device,
                        alloc_workspace(plan.workspace_bytes, device), plan, len(grads), streams)


def themis_gradient_norm(plan: GradientPlan):
    """Euclidean norms -> (total f32[1], norms f32[n_tensors])."""
    result = plan.image.new_empty(1 + plan.n_tensors, dtype=torch.float32)
    at = result.data_ptr()
    _check(lib().themis_gradient_norm(plan.c_struct, at, at + 4, plan.workspace_at,
                                      plan.c_struct.workspace_bytes, plan.stream()))
    return torch.split_with_sizes(result, (1, plan.n_tensors))


def themis_gradient_clip(plan: GradientPlan, max_norm: float):
    """The same, and the gradients times min(1, max_norm / norm) into the plan's targets
    -> (f32[2]: norm and factor, norms f32[n_tensors])."""
    result = plan.image.new_empty(2 + plan.n_tensors, dtype=torch.float32)
    at = result.data_ptr()
    _check(lib().themis_gradient_clip(plan.c_struct, max_norm, at, at + 8, plan.workspace_at,
                                      plan.c_struct.workspace_bytes, plan.stream()))
    return torch.split_with_sizes(result, (2, plan.n_tensors))


# -- an expert layer of the iteration, and dropout ----------------------------------------

def _result(given: Optional[torch.Tensor], like: torch.Tensor, shape, dtype: Optional[torch.dtype]) -> torch.Tensor:
    """`given`, checked, or a new tensor of this shape and type (like's where none is named)."""
    if given is None:
        _need(dtype is None or dtype in _FLOATS)
        return like.new_empty(shape, dtype=dtype)
    _need(given.dtype in _FLOATS and given.shape == shape and given.get_device() == like.get_device() and
          dtype in (None, given.dtype))
    return given


def _need_apart(out: Optional[torch.Tensor], *inputs):
    """What the caller gave to be written shares no memory with what is read."""
    if out is not None:
        for t in inputs:
            if t is not None and _one_storage(out, t):
                _need(_apart(out, t))


def _written_rows(t: torch.Tensor, width: int) -> _Rows:
    r = _rows(t, t.dim() - 1, width)
    _need(r is not None)
    return r


def _new_rows(t: torch.Tensor, width: int) -> _Rows:
    """The same of a tensor that this call has made."""
    return _Rows(t.data_ptr(), _TYPES[t.dtype], 1 << 31, 0, width)


def themis_expert_gate(logits: torch.Tensor, k: int, renormalize: bool = True,
                       out_dtype: torch.dtype = torch.float32, index_dtype: torch.dtype = torch.int32) -> tuple:
    """The k largest of the last dimension, equal ones in ascending order -> (weights [.., k]: their
    softmax, over the chosen alone or (renormalize=False) over all; experts [.., k]).  A logit of
    -inf is not chosen: a token with fewer than k others has experts -1 of weight 0 behind them."""
    device = logits.get_device()
    _need(device >= 0 and logits.dim() >= 1 and logits.dtype in _FLOATS and out_dtype in _FLOATS and
          index_dtype in _INDEXES)
    n_experts = logits.shape[-1]
    _need(0 <= k <= n_experts)
    shape = (*logits.shape[:-1], k)
    weights = logits.new_empty(shape, dtype=out_dtype)
    experts = logits.new_empty(shape, dtype=index_dtype)
    if weights.numel() == 0:
        return weights, experts
    stream = _stream_here(device)
    n = weights.numel() // k
    rows_l, logits = _read_rows(logits, len(shape) - 1, n_experts)
    _check(lib().themis_expert_gate(rows_l, n_experts, n, k, int(renormalize), _new_rows(weights, k),
                                    _new_rows(experts, k), stream))
    return weights, experts


def themis_expert_gate_grad(grad_weights: torch.Tensor, logits: torch.Tensor, experts: torch.Tensor,
                            renormalize: bool = True, out_dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """The gradient of the logits behind themis_expert_gate, of the logits' type unless out_dtype
    says another."""
    device = logits.get_device()
    _need(device >= 0 and logits.dim() >= 1 and logits.dtype in _FLOATS and grad_weights.dtype in _FLOATS and
          experts.dtype in _INDEXES and experts.dim() == logits.dim() and
          experts.shape[:-1] == logits.shape[:-1] and grad_weights.shape == experts.shape and
          grad_weights.get_device() == device and experts.get_device() == device and
          out_dtype in (None, *_FLOATS))
    grad = logits.new_empty(logits.shape, dtype=out_dtype)
    if grad.numel() == 0:
        return grad
    stream = _stream_here(device)
    lead, n_experts, k = logits.dim() - 1, logits.shape[-1], experts.shape[-1]
    rows_g, grad_weights = _read_rows(grad_weights, lead, k)
    rows_l, logits = _read_rows(logits, lead, n_experts)
    rows_e, experts = _read_rows(experts, lead, k)
    _check(lib().themis_expert_gate_grad(rows_g, rows_l, n_experts, rows_e, grad.numel() // n_experts, k,
                                         int(renormalize), _new_rows(grad, n_experts), stream))
    return grad


@dataclass
class ExpertOrder:
    """Pairs (token, its j-th expert) in the order of their experts (themis_expert_sort), pieces of one
    allocation; counts and starts may be changed once they are there, nothing here reads them.  A pair whose place is
    set to -1 afterwards has no part in sums, and its slot holds zeros where rows are written by slots."""
    place: torch.Tensor    # i32 [.., k]: slot of a pair, -1 for none
    counts: torch.Tensor   # i32 [n_experts]: pairs of an expert, those without a slot too
    starts: torch.Tensor   # i32 [n_experts + 1]: first slot of an expert; behind the last
    source: torch.Tensor   # i32 [slots]: the pair of a slot, token * k + j, -1 for none
    capacity: int          # slots of an expert; 0: packed
    slots: int
    shape: torch.Size      # of the tokens
    pairs: torch.Size      # of place
    device: int
    c_struct: _ExpertOrder
    streams: set           # raw handles: the one it was made on, and others that have used it

    def stream(self) -> int:
        """The current stream; the order's memory, once it is given up, waits for it."""
        stream = _stream_here(self.device)
        if stream not in self.streams:
            self.streams.add(stream)
            for t in (self.place, self.counts, self.starts, self.source):
                t.record_stream(torch.cuda.current_stream())
        return stream


@functools.lru_cache(maxsize=1024)
def themis_expert_sort_workspace_bytes(n: int, k: int, n_experts: int) -> int:
    return lib().themis_expert_sort_workspace_bytes(n, k, n_experts)


def themis_expert_sort(experts: torch.Tensor, n_experts: int, capacity: int = 0,
                       workspace: Optional[torch.Tensor] = None) -> ExpertOrder:
    """Orders the pairs of experts [.., k] by expert, an expert's in the tokens' order.

    capacity 0: the experts' pairs end to end, as many slots as pairs; else a buffer of this many
    slots for every expert, whose later pairs have none.  Numbers outside 0 .. n_experts-1 have no slot."""
    device = experts.get_device()
    _need(device >= 0 and experts.dim() >= 1 and experts.dtype in _INDEXES and n_experts >= 1 and capacity >= 0 and
          (workspace is None or (workspace.get_device() == device and workspace.is_contiguous())))
    _need_apart(workspace, experts)
    stream = _stream_here(device)
    k, pairs = experts.shape[-1], experts.numel()
    n = pairs // k if k else experts.shape[:-1].numel()
    slots = n_experts * capacity if capacity else pairs
    if max(n, k, pairs, slots, n_experts) >= 1 << 31:
        raise ThemisError(UNSUPPORTED)
    # (one allocation for all of it, the workspace too: a call on a few tokens is the host's time)
    own = 0 if workspace is not None else (themis_expert_sort_workspace_bytes(n, k, n_experts) + 15) // 16 * 4
    room = torch.empty(own + pairs + 2 * n_experts + 1 + slots, dtype=torch.int32, device=experts.device)
    first = room.data_ptr()
    at, size = (first, 4 * own) if workspace is None else (workspace.data_ptr(),
                                                           workspace.numel() * workspace.element_size())
    # (pieces with version numbers of their own: a caller may change the counts before a backward reads the places)
    _, place, counts, starts, source = torch.unsafe_split_with_sizes(room, (own, pairs, n_experts, n_experts + 1, slots))
    first += 4 * own
    order = _ExpertOrder(n, k, n_experts, capacity, first, first + 4 * pairs, first + 4 * (pairs + n_experts),
                         first + 4 * (pairs + 2 * n_experts + 1))
    shape = experts.shape
    rows_e, experts = _read_rows(experts, len(shape) - 1, k)
    _check(lib().themis_expert_sort(rows_e, order, at, size, stream))
    return ExpertOrder(place.view(shape), counts, starts, source, capacity, slots, shape[:-1], shape, device, order,
                       {stream})


def _slots_width(order: ExpertOrder, y: torch.Tensor) -> int:
    shape = y.shape
    _need(y.dtype in _FLOATS and len(shape) == 2 and shape[0] == order.slots and y.get_device() == order.device)
    return shape[1]


def _tokens_width(order: ExpertOrder, x: torch.Tensor) -> int:
    shape = x.shape
    _need(x.dtype in _FLOATS and len(shape) == len(order.pairs) and shape[:-1] == order.shape and
          x.get_device() == order.device)
    return shape[-1]


def _need_weights(order: ExpertOrder, weights: torch.Tensor):
    _need(weights.dtype in _FLOATS and weights.shape == order.pairs and weights.get_device() == order.device)


def themis_expert_dispatch(x: torch.Tensor, order: ExpertOrder, out: Optional[torch.Tensor] = None,
                           out_dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """The tokens' rows x [.., width] in the order of their experts -> [slots, width] of out's type
    (given by out or out_dtype; x's otherwise), zeros in the slots of no pair.  Its gradient is
    themis_expert_combine without weights."""
    width = _tokens_width(order, x)
    result = _result(out, x, (order.slots, width), out_dtype)
    if result.numel() == 0:
        return result
    _need_apart(out, x, order.place, order.source)
    stream = order.stream()
    rows_x, x = _read_rows(x, x.dim() - 1, width)
    _check(lib().themis_expert_dispatch(order.c_struct, rows_x, width, _written_rows(result, width), stream))
    return result


def themis_expert_combine(y: torch.Tensor, order: ExpertOrder, weights: Optional[torch.Tensor] = None,
                          out: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None,
                          accumulate: bool = False) -> torch.Tensor:
    """The sum of a token's rows of y [slots, width], times weights [.., k] -> [.., width] of out's
    type (given by out or out_dtype; y's otherwise), or added to out where `accumulate`.  Pairs
    without a slot have no part."""
    width = _slots_width(order, y)
    if weights is not None:
        _need_weights(order, weights)
    _need(out is not None or not accumulate)
    result = _result(out, y, (*order.shape, width), out_dtype)
    if result.numel() == 0:
        return result
    _need_apart(out, y, weights, order.place)
    stream = order.stream()
    rows_y, y = _read_rows(y, 1, width)
    rows_w = None
    if weights is not None:
        rows_w, weights = _read_rows(weights, len(order.shape), order.pairs[-1])
    _check(lib().themis_expert_combine(order.c_struct, rows_y, width, rows_w, int(accumulate),
                                       _written_rows(result, width), stream))
    return result


def themis_expert_combine_grad(grad_out: torch.Tensor, y: torch.Tensor, order: ExpertOrder, weights: torch.Tensor,
                               need_rows: bool = True, need_weights: bool = True) -> tuple:
    """The gradients behind themis_expert_combine with weights -> (of y [slots, width], of the
    weights [.., k]), each of its tensor's type, None where it is not needed."""
    width = _slots_width(order, y)
    _need_weights(order, weights)
    _need(_tokens_width(order, grad_out) == width)
    stream = order.stream()
    lead, k = len(order.shape), order.pairs[-1]
    rows = y.new_empty(y.shape) if need_rows else None
    products = weights.new_empty(order.pairs) if need_weights else None
    rows_g, grad_out = _read_rows(grad_out, lead, width)
    rows_y, y = _read_rows(y, 1, width)
    rows_w, weights = _read_rows(weights, lead, k)
    _check(lib().themis_expert_combine_grad(order.c_struct, rows_g, width, rows_y, rows_w,
                                            _new_rows(rows, width) if need_rows else None,
                                            _new_rows(products, k) if need_weights else None, stream))
    return rows, products


def _in_place(a: torch.Tensor, b: torch.Tensor) -> bool:
    return a.data_ptr() == b.data_ptr() and a.dtype == b.dtype and a.shape == b.shape and a.stride() == b.stride()


def themis_dropout(x: torch.Tensor, p: float, seed: int, call, add: Optional[torch.Tensor] = None,
                   out: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """add + x / (1 - p), elements of x dropped with probability p -> out's type (given by out,
    which may be x or add themselves, or out_dtype; add's or x's otherwise).

    What is dropped is a function of (seed, call, row, column), x as rows of its last dimension: the
    gradient of x is the same call on the result's gradient, without add.  call: a whole number, or a
    tensor of one 64 bit number on the GPU, read when the kernel runs (a captured graph draws another mask in
    every replay if the program moves it on)."""
    device = x.get_device()
    given = out is not None
    _need(device >= 0 and x.dim() >= 1 and x.dtype in _FLOATS and 0.0 <= p <= 1.0)
    if add is not None:
        _need(add.shape == x.shape and add.dtype in _FLOATS and add.get_device() == device)
        out_dtype = out_dtype or (None if given else add.dtype)
    call_at = None
    if isinstance(call, torch.Tensor):
        _need(call.dtype == torch.int64 and call.numel() == 1 and call.get_device() == device)
        call, call_at = 0, call
    out = _result(out, x, x.shape, out_dtype)
    _need(add is None or add.dtype == out.dtype)
    if out.numel() == 0:
        return out
    if given:
        for t in (x, add):
            if t is not None and _one_storage(out, t) and not _in_place(out, t):
                _need(_apart(out, t))
        _need_apart(out, call_at)
    stream = _stream_here(device)
    lead, width = x.dim() - 1, x.shape[-1]
    rows_o = _written_rows(out, width)
    rows_x, x = _read_rows(x, lead, width)
    rows_a = None
    if add is not None:
        rows_a, add = _read_rows(add, lead, width)
    _check(lib().themis_dropout(rows_x, x.numel() // width, width, p, seed & _ALL64, call & _ALL64,
                                None if call_at is None else call_at.data_ptr(), rows_a, rows_o, stream))
    return out


_ALL64 = (1 << 64) - 1
