"""ctypes marshalling for the railsched C ABI (include/railsched.h).

PyTorch is used for device memory and streams only: tensors are allocated with
torch, their data pointers and the current HIP stream are handed to the library.
There is no fallback: if librailsched.so cannot be loaded, importing a symbol
works but the first call raises.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "librailsched.so")
_lib = None

EXPORTS = (
    "railsched_version", "railsched_strerror", "railsched_check_capacity", "railsched_route_topk",
    "railsched_traffic_matrix_workspace_bytes", "railsched_traffic_matrix",
    "railsched_route_traffic_workspace_bytes", "railsched_route_traffic",
    "railsched_chunk_sort_workspace_bytes", "railsched_chunk_sort", "railsched_lpt_spray_workspace_bytes", "railsched_lpt_spray",
    "railsched_lpt_spray_chunkwise",
    "railsched_eval_workspace_bytes", "railsched_eval", "railsched_schedule_workspace_bytes", "railsched_schedule", "railsched_schedule_static", "railsched_transpose_matrix", "railsched_assign_policy",
    "railsched_port_round_robin_workspace_bytes", "railsched_port_round_robin",
    "railsched_route_logprobs", "railsched_route_logprobs_backward",
    "railsched_route_balance_workspace_bytes", "railsched_route_balance", "railsched_route_balance_backward",
    "railsched_route_distill", "railsched_route_distill_backward",
)


class RailschedError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {strerror(status)} (status {status})")


class _TopoStruct(C.Structure):
    _fields_ = [("nodes", C.c_int32), ("rails", C.c_int32), ("chunk_bytes", C.c_int64),
                ("rail_bw_Bps", C.c_int64), ("include_intra_node", C.c_int32), ("reserved", C.c_int32)]


@dataclass(frozen=True)
class Topo:
    """M nodes x N rails, chunk size C, rail rate R2 (Section 4.1 of the paper)."""
    nodes: int
    rails: int
    chunk_bytes: int
    rail_bw_Bps: int = 50_000_000_000
    include_intra_node: int = 0

    @property
    def G(self) -> int:
        return self.nodes * self.rails

    def c(self) -> _TopoStruct:
        return _TopoStruct(self.nodes, self.rails, self.chunk_bytes, self.rail_bw_Bps, self.include_intra_node, 0)


def lib_path() -> str:
    return _LIB_PATH


def load():
    """Load librailsched.so (building it first only if it is absent)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        from . import build as _build
        _build.build(force=True)
    lib = C.CDLL(_LIB_PATH)           # torch is imported above, so its HIP runtime is the one resolved
    lib.railsched_version.restype = C.c_char_p
    lib.railsched_strerror.restype = C.c_char_p
    lib.railsched_strerror.argtypes = [C.c_int]
    P, I32, I64, SZ, F32 = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t, C.c_float
    TP = C.POINTER(_TopoStruct)
    lib.railsched_route_topk.argtypes = [P, I64, I32, I32, P, P]
    lib.railsched_check_capacity.argtypes = [P, I32, TP, I64, C.POINTER(C.c_int64), P]
    lib.railsched_traffic_matrix_workspace_bytes.argtypes = [I32, I64, I32, TP]
    lib.railsched_traffic_matrix_workspace_bytes.restype = SZ
    lib.railsched_traffic_matrix.argtypes = [P, I32, I64, I32, P, I32, I32, I64, TP, P, P, SZ, P]
    lib.railsched_route_traffic_workspace_bytes.argtypes = [I32, I64, I32, I32, TP]
    lib.railsched_route_traffic_workspace_bytes.restype = SZ
    lib.railsched_route_traffic.argtypes = [P, I32, I64, I32, I32, P, I32, I64, TP, P, P, P, SZ, P]
    lib.railsched_chunk_sort_workspace_bytes.argtypes = [I32, TP]
    lib.railsched_chunk_sort_workspace_bytes.restype = SZ
    lib.railsched_chunk_sort.argtypes = [P, I32, TP, P, P, P, P, I64, P, SZ, P]
    lib.railsched_lpt_spray_workspace_bytes.argtypes = [I32, TP]
    lib.railsched_lpt_spray_workspace_bytes.restype = SZ
    lib.railsched_lpt_spray.argtypes = [P, P, I32, TP, I64, P, P, P, SZ, P]
    lib.railsched_lpt_spray_chunkwise.argtypes = [P, P, I32, TP, I64, P, P, P, SZ, P]
    lib.railsched_eval_workspace_bytes.argtypes = [I32, TP]
    lib.railsched_eval_workspace_bytes.restype = SZ
    lib.railsched_eval.argtypes = [P, P, P, P, P, I32, TP, I64, P, P, P, SZ, P]
    lib.railsched_schedule_workspace_bytes.argtypes = [I32, TP]
    lib.railsched_schedule_workspace_bytes.restype = SZ
    lib.railsched_schedule.argtypes = [P, I32, TP, P, P, P, P, I64, P, P, P, P, P, SZ, P]
    lib.railsched_schedule_static.argtypes = [P, I32, TP, P, P, P, P, I64, P, P, P, P, P]
    lib.railsched_schedule_static.restype = C.c_int
    lib.railsched_transpose_matrix.argtypes = [P, I32, TP, P, P]
    lib.railsched_assign_policy.argtypes = [I32, C.c_uint64, P, P, P, I32, TP, I64, P, P, P]
    lib.railsched_port_round_robin_workspace_bytes.argtypes = [I32, TP, I64]
    lib.railsched_port_round_robin_workspace_bytes.restype = SZ
    lib.railsched_port_round_robin.argtypes = [P, P, I32, TP, I32, I64, P, P, SZ, P]
    lib.railsched_port_round_robin.restype = C.c_int
    lib.railsched_transpose_matrix.restype = C.c_int
    lib.railsched_assign_policy.restype = C.c_int
    for fn in ("railsched_check_capacity", "railsched_route_topk", "railsched_traffic_matrix", "railsched_route_traffic",
               "railsched_chunk_sort", "railsched_lpt_spray", "railsched_lpt_spray_chunkwise", "railsched_eval",
               "railsched_schedule"):
        getattr(lib, fn).restype = C.c_int
    lib.railsched_route_logprobs.argtypes = [P, I32, I64, I32, I64, F32, P, P, I32, I32, P, P, P, P, P, P]
    lib.railsched_route_logprobs_backward.argtypes = [P, I32, I64, I32, I64, F32, P, P, I32, P, P, P, I32, P, I64, P]
    lib.railsched_route_balance_workspace_bytes.argtypes = [I64, I32, I32]
    lib.railsched_route_balance_workspace_bytes.restype = SZ
    lib.railsched_route_balance.argtypes = [P, I32, I64, I32, I64, P, P, I32, P, I32, F32, P, P, P, P, P, SZ, P]
    lib.railsched_route_balance_backward.argtypes = [P, I32, I64, I32, I64, P, I32, P, I32, F32, P, P, P, I32, P, I64, P]
    lib.railsched_route_distill.argtypes = [P, I32, I64, I32, I64, F32, P, P, P, P, I32, P, P]
    lib.railsched_route_distill_backward.argtypes = [P, I32, I64, I32, I64, F32, P, P, P, P, I32, P, I32, P, I64, P]
    for fn in ("railsched_route_logprobs", "railsched_route_logprobs_backward", "railsched_route_balance", "railsched_route_balance_backward",
               "railsched_route_distill", "railsched_route_distill_backward"):
        getattr(lib, fn).restype = C.c_int
    _lib = lib
    return lib


def version() -> str:
    return load().railsched_version().decode()


def strerror(status: int) -> str:
    return load().railsched_strerror(int(status)).decode()


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _dev(t: torch.Tensor, dtype, name: str) -> torch.Tensor:
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _check(status: int, where: str):
    if status != 0:
        raise RailschedError(status, where)


def _ws(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def check_capacity(chunk_off: torch.Tensor, batch: int, topo: Topo, capacity: int) -> int:
    """Waits for the current stream, returns the chunk count; raises RailschedError(RAILSCHED_ERR_CAPACITY) if it
    exceeds `capacity` (the one synchronising call of the library)."""
    _dev(chunk_off, torch.int64, "chunk_off")
    total = C.c_int64(0)
    t = topo.c()
    rc = load().railsched_check_capacity(_ptr(chunk_off), batch, C.byref(t), capacity, C.byref(total), _stream())
    if rc != 0:
        err = RailschedError(rc, "railsched_check_capacity")
        err.total = int(total.value)
        raise err
    return int(total.value)


# ---------------------------------------------------------------------------------- stage 1
def route_topk(logits: torch.Tensor, k: int, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """[rows][E] fp32 -> [rows][k] int32 indices of the k largest logits, lowest index on ties."""
    _dev(logits, torch.float32, "logits")
    rows, E = logits.shape
    if out is None:
        out = torch.empty((rows, k), dtype=torch.int32, device=logits.device)
    _dev(out, torch.int32, "out")
    _check(load().railsched_route_topk(_ptr(logits), rows, E, k, _ptr(out), _stream()), "railsched_route_topk")
    return out


# ---------------------------------------------------------------------------------- stage 2
def traffic_matrix_workspace_bytes(batch: int, tokens_per_gpu: int, k: int, topo: Topo) -> int:
    t = topo.c()
    return int(load().railsched_traffic_matrix_workspace_bytes(batch, tokens_per_gpu, k, C.byref(t)))


def traffic_matrix(topk_idx: torch.Tensor, batch: int, tokens_per_gpu: int, expert_gpu: torch.Tensor,
                   payload_bytes: int, topo: Topo, out: Optional[torch.Tensor] = None,
                   ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """top-k indices + expert placement -> D1 [batch][G][G] int64 bytes."""
    _dev(topk_idx, torch.int32, "topk_idx")
    _dev(expert_gpu, torch.int32, "expert_gpu")
    k = topk_idx.shape[1]
    E, R = expert_gpu.shape
    G = topo.G
    if topk_idx.shape[0] != batch * G * tokens_per_gpu:
        raise ValueError("topk_idx must hold batch*G*tokens_per_gpu rows")
    if out is None:
        out = torch.empty((batch, G, G), dtype=torch.int64, device=topk_idx.device)
    _dev(out, torch.int64, "out")
    if ws is None:
        ws = _ws(traffic_matrix_workspace_bytes(batch, tokens_per_gpu, k, topo), topk_idx.device)
    t = topo.c()
    _check(load().railsched_traffic_matrix(_ptr(topk_idx), batch, tokens_per_gpu, k, _ptr(expert_gpu), E, R,
                                           payload_bytes, C.byref(t), _ptr(out), _ptr(ws), ws.numel(), _stream()),
           "railsched_traffic_matrix")
    return out


def route_traffic_workspace_bytes(batch: int, tokens_per_gpu: int, E: int, k: int, topo: Topo) -> int:
    t = topo.c()
    return int(load().railsched_route_traffic_workspace_bytes(batch, tokens_per_gpu, E, k, C.byref(t)))


def route_traffic(logits: torch.Tensor, k: int, batch: int, tokens_per_gpu: int, expert_gpu: torch.Tensor,
                  payload_bytes: int, topo: Topo, want_idx: bool = True,
                  out: Optional[Tuple[Optional[torch.Tensor], torch.Tensor]] = None, ws: Optional[torch.Tensor] = None):
    """Stages 1 and 2 in one call: (topk_idx or None, D1)."""
    _dev(logits, torch.float32, "logits")
    _dev(expert_gpu, torch.int32, "expert_gpu")
    rows, E = logits.shape
    E2, R = expert_gpu.shape
    G = topo.G
    if E2 != E:
        raise ValueError("expert_gpu must have one row per expert")
    if rows != batch * G * tokens_per_gpu:
        raise ValueError("logits must hold batch*G*tokens_per_gpu rows")
    if out is None:
        idx = torch.empty((rows, k), dtype=torch.int32, device=logits.device) if want_idx else None
        D1 = torch.empty((batch, G, G), dtype=torch.int64, device=logits.device)
    else:
        idx, D1 = out
    if idx is not None:
        _dev(idx, torch.int32, "topk_idx")
    _dev(D1, torch.int64, "D1")
    if ws is None:
        ws = _ws(route_traffic_workspace_bytes(batch, tokens_per_gpu, E, k, topo), logits.device)
    t = topo.c()
    _check(load().railsched_route_traffic(_ptr(logits), batch, tokens_per_gpu, E, k, _ptr(expert_gpu), R, payload_bytes,
                                          C.byref(t), None if idx is None else _ptr(idx), _ptr(D1), _ptr(ws), ws.numel(),
                                          _stream()),
           "railsched_route_traffic")
    return idx, D1


# ---------------------------------------------------------------------------------- stage 3
def chunk_sort_workspace_bytes(batch: int, topo: Topo) -> int:
    t = topo.c()
    return int(load().railsched_chunk_sort_workspace_bytes(batch, C.byref(t)))


def eval_workspace_bytes(batch: int, topo: Topo) -> int:
    t = topo.c()
    return int(load().railsched_eval_workspace_bytes(batch, C.byref(t)))


def chunk_count(D1: torch.Tensor, topo: Topo, ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Count query: chunk_off [batch*M+1] int64 only."""
    _dev(D1, torch.int64, "D1")
    batch = D1.shape[0]
    off = torch.empty(batch * topo.nodes + 1, dtype=torch.int64, device=D1.device)
    if ws is None:
        ws = _ws(chunk_sort_workspace_bytes(batch, topo), D1.device)
    t = topo.c()
    _check(load().railsched_chunk_sort(_ptr(D1), batch, C.byref(t), _ptr(off), None, None, None, 0,
                                       _ptr(ws), ws.numel(), _stream()), "railsched_chunk_sort(count)")
    return off


def chunk_total(D1: torch.Tensor, topo: Topo, ws: Optional[torch.Tensor] = None) -> int:
    """Count query followed by the one synchronising call: the number of chunks stage 3 will produce for D1."""
    off = chunk_count(D1, topo, ws)
    return check_capacity(off, D1.shape[0], topo, (1 << 62))


def chunk_sort(D1: torch.Tensor, topo: Topo, want_perm: bool = True, capacity: Optional[int] = None,
               out=None, ws: Optional[torch.Tensor] = None):
    """D1 -> (chunk_off, chunk_w, chunk_flow, perm|None), every instance sorted by descending weight.

    Without `capacity` a count query runs first and the host waits for the total (one
    synchronisation) to size the record arrays.  With `capacity` (and optionally preallocated
    `out` = (chunk_off, chunk_w, chunk_flow, perm)) the call is fully asynchronous; the record
    arrays are left untouched if the total exceeds the capacity.
    """
    _dev(D1, torch.int64, "D1")
    batch = D1.shape[0]
    dev = D1.device
    if ws is None:
        ws = _ws(chunk_sort_workspace_bytes(batch, topo), dev)
    if capacity is None:
        capacity = chunk_total(D1, topo, ws)
    if out is None:
        off = torch.empty(batch * topo.nodes + 1, dtype=torch.int64, device=dev)
        w = torch.empty(max(capacity, 1), dtype=torch.int32, device=dev)
        flow = torch.empty(max(capacity, 1), dtype=torch.int32, device=dev)
        perm = torch.empty(max(capacity, 1), dtype=torch.int32, device=dev) if want_perm else None
    else:
        off, w, flow, perm = out
    t = topo.c()
    _check(load().railsched_chunk_sort(_ptr(D1), batch, C.byref(t), _ptr(off), _ptr(w), _ptr(flow), _ptr(perm),
                                       capacity, _ptr(ws), ws.numel(), _stream()), "railsched_chunk_sort")
    return off, w, flow, perm


# ---------------------------------------------------------------------------------- stage 4
def lpt_spray_workspace_bytes(batch: int, topo: Topo) -> int:
    t = topo.c()
    return int(load().railsched_lpt_spray_workspace_bytes(batch, C.byref(t)))


def lpt_spray(chunk_off: torch.Tensor, chunk_w: torch.Tensor, batch: int, topo: Topo, out=None, chunkwise: bool = False,
              capacity: Optional[int] = None, ws="auto"):
    """Greedy least-loaded-rail assignment per instance -> (rail uint8 [capacity], S int64 [batch][M][N]).
    chunkwise=True calls railsched_lpt_spray_chunkwise (same result, no closed-form periods).
    capacity = records chunk_w and rail hold (default: the length of chunk_w).
    ws: workspace tensor, None for none, "auto" to allocate one here (instances are then taken longest first)."""
    _dev(chunk_off, torch.int64, "chunk_off")
    if chunk_w.dtype not in (torch.int32, torch.uint32):
        raise ValueError("chunk_w must be a 32-bit integer tensor")
    if capacity is None:
        capacity = chunk_w.numel()
    if out is None:
        rail = torch.empty(max(capacity, 1), dtype=torch.uint8, device=chunk_off.device)
        S = torch.empty((batch, topo.nodes, topo.rails), dtype=torch.int64, device=chunk_off.device)
    else:
        rail, S = out
    if min(chunk_w.numel(), rail.numel()) < capacity:
        raise ValueError("chunk_w and rail must hold `capacity` records")
    t = topo.c()
    if isinstance(ws, str):
        ws = _ws(lpt_spray_workspace_bytes(batch, topo), chunk_off.device)
    fn = load().railsched_lpt_spray_chunkwise if chunkwise else load().railsched_lpt_spray
    _check(fn(_ptr(chunk_off), _ptr(chunk_w), batch, C.byref(t), capacity, _ptr(rail), _ptr(S), _ptr(ws),
              0 if ws is None else ws.numel(), _stream()), "railsched_lpt_spray")
    return rail, S


# ---------------------------------------------------------------------------------- stage 5
def eval(chunk_off, chunk_w, chunk_flow, rail, S, batch: int, topo: Topo, out=None,  # noqa: A001
         ws: Optional[torch.Tensor] = None, capacity: Optional[int] = None):
    """Receive loads R [batch][M][N] and stats [batch][8] (see include/railsched.h).
    capacity = records the per-chunk arrays hold (default: the shortest of them)."""
    dev = chunk_off.device
    if capacity is None:
        capacity = min(chunk_w.numel(), chunk_flow.numel(), rail.numel())
    if out is None:
        R = torch.empty((batch, topo.nodes, topo.rails), dtype=torch.int64, device=dev)
        stats = torch.empty((batch, 8), dtype=torch.int64, device=dev)
    else:
        R, stats = out
    if ws is None:
        ws = _ws(eval_workspace_bytes(batch, topo), dev)
    t = topo.c()
    _check(load().railsched_eval(_ptr(chunk_off), _ptr(chunk_w), _ptr(chunk_flow), _ptr(rail), _ptr(S), batch,
                                 C.byref(t), capacity, _ptr(R), _ptr(stats), _ptr(ws), ws.numel(), _stream()), "railsched_eval")
    return R, stats


evaluate = eval

POLICIES = {"nic_direct": 0, "flow_hash": 1, "random_spray": 2, "round_robin": 3}


def transpose_matrix(D1: torch.Tensor, topo: Topo, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Traffic of the second all-to-all: D1T[b][d][s] = D1[b][s][d]."""
    _dev(D1, torch.int64, "D1")
    if out is None:
        out = torch.empty_like(D1)
    t = topo.c()
    _check(load().railsched_transpose_matrix(_ptr(D1), D1.shape[0], C.byref(t), _ptr(out), _stream()),
           "railsched_transpose_matrix")
    return out


def assign_policy(policy, seed: int, chunk_off, chunk_w, chunk_flow, batch: int, topo: Topo, out=None,
                  capacity: Optional[int] = None):
    """Rails under a comparison scheme ("nic_direct", "flow_hash", "random_spray", "round_robin") -> (rail, S)."""
    if capacity is None:
        capacity = min(chunk_w.numel(), chunk_flow.numel())
    if out is None:
        rail = torch.empty(max(capacity, 1), dtype=torch.uint8, device=chunk_off.device)
        S = torch.empty((batch, topo.nodes, topo.rails), dtype=torch.int64, device=chunk_off.device)
    else:
        rail, S = out
    t = topo.c()
    pol = POLICIES[policy] if isinstance(policy, str) else int(policy)
    if rail.numel() < capacity:
        raise ValueError("rail must hold `capacity` records")
    _check(load().railsched_assign_policy(pol, seed, _ptr(chunk_off), _ptr(chunk_w), _ptr(chunk_flow), batch, C.byref(t),
                                          capacity, _ptr(rail), _ptr(S), _stream()), "railsched_assign_policy")
    return rail, S


# ---------------------------------------------------------------------------------- whole path
def schedule_workspace_bytes(batch: int, topo: Topo) -> int:
    t = topo.c()
    return int(load().railsched_schedule_workspace_bytes(batch, C.byref(t)))


def schedule(D1: torch.Tensor, topo: Topo, capacity: int, want_perm: bool = True, out=None, ws: Optional[torch.Tensor] = None):
    """Stages 3-5 in one call: (chunk_off, chunk_w, chunk_flow, perm, rail, S, R, stats)."""
    _dev(D1, torch.int64, "D1")
    batch = D1.shape[0]
    M, N = topo.nodes, topo.rails
    dev = D1.device
    if out is None:
        n = max(capacity, 1)
        out = (torch.empty(batch * M + 1, dtype=torch.int64, device=dev), torch.empty(n, dtype=torch.int32, device=dev),
               torch.empty(n, dtype=torch.int32, device=dev), torch.empty(n, dtype=torch.int32, device=dev) if want_perm else None,
               torch.empty(n, dtype=torch.uint8, device=dev), torch.empty((batch, M, N), dtype=torch.int64, device=dev),
               torch.empty((batch, M, N), dtype=torch.int64, device=dev), torch.empty((batch, 8), dtype=torch.int64, device=dev))
    off, w, flow, perm, rail, S, R, stats = out
    if ws is None:
        ws = _ws(schedule_workspace_bytes(batch, topo), dev)
    t = topo.c()
    _check(load().railsched_schedule(_ptr(D1), batch, C.byref(t), _ptr(off), _ptr(w), _ptr(flow), _ptr(perm), capacity, _ptr(rail),
                                     _ptr(S), _ptr(R), _ptr(stats), _ptr(ws), ws.numel(), _stream()), "railsched_schedule")
    return out


STATIC_SCRATCH_BYTES = 4 << 20


def schedule_static(D1: torch.Tensor, topo: Topo, capacity: int, out):
    """railsched_schedule_static: stages 3-5 with the library's own static scratch buffer instead of a workspace.
    `out` = (chunk_off, chunk_w, chunk_flow, perm or None, rail, S, R, stats), preallocated: nothing is allocated here."""
    _dev(D1, torch.int64, "D1")
    off, w, flow, perm, rail, S, R, stats = out
    t = topo.c()
    _check(load().railsched_schedule_static(_ptr(D1), D1.shape[0], C.byref(t), _ptr(off), _ptr(w), _ptr(flow), _ptr(perm), capacity,
                                            _ptr(rail), _ptr(S), _ptr(R), _ptr(stats), _stream()), "railsched_schedule_static")
    return out


class Plan:
    """Preallocated buffers for repeated passes of the whole path over same-shaped batches
    (no allocation and no host synchronisation inside step())."""

    def __init__(self, topo: Topo, batch: int, capacity: int, device, rows: int = 0, k: int = 0, want_perm: bool = True):
        self.topo, self.batch, self.capacity = topo, batch, capacity
        M, N, G = topo.nodes, topo.rails, topo.G
        i32, i64 = torch.int32, torch.int64
        self.topk_idx = torch.empty((rows, k), dtype=i32, device=device) if rows else None
        self.D1 = torch.empty((batch, G, G), dtype=i64, device=device)
        self.chunk_off = torch.empty(batch * M + 1, dtype=i64, device=device)
        self.chunk_w = torch.empty(max(capacity, 1), dtype=i32, device=device)
        self.chunk_flow = torch.empty(max(capacity, 1), dtype=i32, device=device)
        self.perm = torch.empty(max(capacity, 1), dtype=i32, device=device) if want_perm else None
        self.rail = torch.empty(max(capacity, 1), dtype=torch.uint8, device=device)
        self.S = torch.empty((batch, M, N), dtype=i64, device=device)
        self.R = torch.empty((batch, M, N), dtype=i64, device=device)
        self.stats = torch.empty((batch, 8), dtype=i64, device=device)
        self.ws_sort = _ws(chunk_sort_workspace_bytes(batch, topo), device)
        self.ws_eval = _ws(eval_workspace_bytes(batch, topo), device)
        self.ws_sched = _ws(schedule_workspace_bytes(batch, topo), device)
        self.ws_lpt = _ws(lpt_spray_workspace_bytes(batch, topo), device)
        self.ws_tm = None

    def route(self, logits, tokens_per_gpu, expert_gpu, payload_bytes):
        k = self.topk_idx.shape[1]
        if self.ws_tm is None:
            self.ws_tm = _ws(traffic_matrix_workspace_bytes(self.batch, tokens_per_gpu, k, self.topo), logits.device)
        route_topk(logits, k, out=self.topk_idx)
        traffic_matrix(self.topk_idx, self.batch, tokens_per_gpu, expert_gpu, payload_bytes, self.topo, out=self.D1, ws=self.ws_tm)
        return self.D1

    def schedule_one_call(self, D1=None):
        """Stages 3-5 through railsched_schedule (same outputs as schedule())."""
        D1 = self.D1 if D1 is None else D1
        schedule(D1, self.topo, self.capacity, out=(self.chunk_off, self.chunk_w, self.chunk_flow, self.perm, self.rail, self.S,
                                                   self.R, self.stats), ws=self.ws_sched)
        return self.stats

    def schedule(self, D1=None):
        """Stages 3-5 through the three calls; like schedule_one_call, fills S, R and stats with -1 (and touches no
        per-chunk array) if the batch yields more chunks than the plan's capacity."""
        D1 = self.D1 if D1 is None else D1
        chunk_sort(D1, self.topo, capacity=self.capacity,
                   out=(self.chunk_off, self.chunk_w, self.chunk_flow, self.perm), ws=self.ws_sort)
        lpt_spray(self.chunk_off, self.chunk_w, self.batch, self.topo, out=(self.rail, self.S), capacity=self.capacity, ws=self.ws_lpt)
        eval(self.chunk_off, self.chunk_w, self.chunk_flow, self.rail, self.S, self.batch, self.topo,
             out=(self.R, self.stats), ws=self.ws_eval, capacity=self.capacity)
        return self.stats


def port_round_robin(chunk_off, rail, batch: int, topo: Topo, ports: int, capacity: Optional[int] = None, out=None, ws=None):
    """Port (queue pair) of every chunk: round robin per rail inside each instance -> uint8 [chunks]."""
    if capacity is None:
        capacity = rail.numel()
    t = topo.c()
    if ws is None:
        ws = _ws(load().railsched_port_round_robin_workspace_bytes(batch, C.byref(t), capacity), chunk_off.device)
    port = torch.empty(max(capacity, 1), dtype=torch.uint8, device=chunk_off.device) if out is None else out
    _check(load().railsched_port_round_robin(_ptr(chunk_off), _ptr(rail), batch, C.byref(t), ports, capacity, _ptr(port),
                                             _ptr(ws), ws.numel(), _stream()), "railsched_port_round_robin")
    return port


# ---------------------------------------------------------------------------------- a router in training
# No part of torch's autograd: outputs are detached, also of logits that require a gradient.  The _backward calls give the logits' gradient, which goes on by
# logits.backward(gradient).
DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


def _int32(v: int, name: str) -> int:
    """v, refused where 32 bits do not hold it: the library would see another number."""
    if not -(1 << 31) <= v < 1 << 31:
        raise ValueError(f"{name} must fit 32 bits, got {v}")
    return v


class _Rows:
    """Checks of the operators on a router's logits: tensors on one device, launches on that device's current stream."""
    __slots__ = ("logits", "device", "dtype", "rows", "E", "head")

    def __init__(self, logits: torch.Tensor):
        if not logits.is_cuda:
            raise ValueError("logits must be a device tensor")
        self.dtype = logits.dtype
        code = DTYPES.get(self.dtype)
        if code is None:
            raise ValueError(f"logits must be torch.float32, bfloat16 or float16, got {logits.dtype}")
        self.logits, self.device = logits, logits.device
        self.rows, self.E, ld = self._strided(logits, "logits")
        self.head = (logits.data_ptr(), code, self.rows, self.E, ld)        # how every entry point's arguments begin

    @staticmethod
    def _strided(t: torch.Tensor, name: str):
        shape = t.shape
        if len(shape) != 2:
            raise ValueError(f"{name} must have two dimensions")
        rows, E = shape
        ld, step = t.stride()
        if step != 1 and E > 1:
            raise ValueError(f"the values of a row of {name} must be next to each other")
        if rows <= 1:
            ld = max(E, 1)
        if ld < E:
            raise ValueError(f"the rows of {name} must not overlap")
        return rows, E, ld

    @staticmethod
    def width(t: Optional[torch.Tensor], name: str) -> int:
        if t is None:
            return 0
        if t.dim() != 2:
            raise ValueError(f"{name} must have two dimensions")
        return _int32(t.shape[1], f"the width of {name}")

    def arg(self, t: Optional[torch.Tensor], dtype, shape, name: str):
        """The address of a contiguous tensor of this type and shape on the logits' device; None for None."""
        if t is None:
            return None
        if t.dtype is dtype and t.shape == shape and t.device == self.device and t.is_contiguous():
            return t.data_ptr()
        if t.device != self.device:
            raise ValueError(f"{name} must be on {self.device}")
        if t.dtype != dtype:
            raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
        if t.shape != shape:
            raise ValueError(f"{name} must have the shape {tuple(shape)}, got {tuple(t.shape)}")
        raise ValueError(f"{name} must be contiguous")

    def mask(self, t: Optional[torch.Tensor]):
        if t is None:
            return None
        if t.dtype == torch.bool:
            t = t.view(torch.uint8)
        return self.arg(t, torch.uint8, (self.rows,), "row_mask")

    def new(self, shape, dtype=torch.float32):
        return self.logits.new_empty(shape, dtype=dtype)

    def gradient(self, out: Optional[torch.Tensor], accumulate: bool):
        """(d_logits, its address, its row stride)"""
        if out is None:
            if accumulate:
                raise ValueError("accumulate needs `out`, the gradient to add to")
            out = self.logits.new_empty((self.rows, self.E))
            return out, out.data_ptr(), max(self.E, 1)
        if out.device != self.device or out.dtype != self.dtype or out.shape != (self.rows, self.E):
            raise ValueError(f"out must be {self.dtype} of shape {(self.rows, self.E)} on {self.device}")
        return out, out.data_ptr(), self._strided(out, "out")[2]

    def call(self, name: str, *args):
        """Runs an entry point on the current stream of the logits' device."""
        fn, at = getattr(load(), name), self.device.index
        if torch.cuda.current_device() == at:
            rc = fn(*args, _raw_stream(at))
        else:
            with torch.cuda.device(at):
                rc = fn(*args, _raw_stream(at))
        _check(rc, name)


# the handle of a device's current stream: 0.1 us where torch hands it out as a number, 2.7 us through a Stream object, of 8 us that a call takes
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda at: torch.cuda.current_stream(at).cuda_stream)


def route_logprobs(logits: torch.Tensor, topk_idx: Optional[torch.Tensor] = None, alternatives: int = 0, temperature: float = 1.0,
                   row_mask: Optional[torch.Tensor] = None, out=None):
    """Log probabilities of the experts topk_idx [rows][k], log-sum-exp and entropy of every row, and its `alternatives` most likely
    experts: (logp or None, lse, entropy, alt_idx or None, alt_logp or None).  logits may be a view with a row stride.
    out: a tuple of the same five, preallocated (lse and entropy may be None there: not computed).
    The outputs are detached from autograd: route_logprobs_backward gives the logits' gradient."""
    r = _Rows(logits)
    k, m = r.width(topk_idx, "topk_idx"), _int32(alternatives, "alternatives")
    if out is None:
        out = (r.new((r.rows, k)) if k else None, r.new(r.rows), r.new(r.rows), r.new((r.rows, m), torch.int32) if m > 0 else None,
               r.new((r.rows, m)) if m > 0 else None)
        to = [None if t is None else t.data_ptr() for t in out]
    else:
        logp, lse, entropy, alt_idx, alt_logp = out
        to = (r.arg(logp, torch.float32, (r.rows, k), "logp"), r.arg(lse, torch.float32, (r.rows,), "lse"),
              r.arg(entropy, torch.float32, (r.rows,), "entropy"), r.arg(alt_idx, torch.int32, (r.rows, m), "alt_idx"),
              r.arg(alt_logp, torch.float32, (r.rows, m), "alt_logp"))
    r.call("railsched_route_logprobs", *r.head, temperature, r.mask(row_mask), r.arg(topk_idx, torch.int32, (r.rows, k), "topk_idx"), k, m, *to)
    return out


def route_logprobs_backward(logits: torch.Tensor, topk_idx: Optional[torch.Tensor] = None, d_logp: Optional[torch.Tensor] = None,
                            d_lse: Optional[torch.Tensor] = None, d_entropy: Optional[torch.Tensor] = None, temperature: float = 1.0,
                            row_mask: Optional[torch.Tensor] = None, accumulate: bool = False, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The gradient of the logits from those of logp, lse and entropy (None: 0).  accumulate: added to `out`."""
    r = _Rows(logits)
    k = r.width(topk_idx, "topk_idx")
    out, to, ld_d = r.gradient(out, accumulate)
    r.call("railsched_route_logprobs_backward", *r.head, temperature, r.mask(row_mask), r.arg(topk_idx, torch.int32, (r.rows, k), "topk_idx"), k,
           r.arg(d_logp, torch.float32, (r.rows, k), "d_logp"), r.arg(d_lse, torch.float32, (r.rows,), "d_lse"),
           r.arg(d_entropy, torch.float32, (r.rows,), "d_entropy"), int(accumulate), to, ld_d)
    return out


def route_balance_workspace_bytes(rows: int, groups: int, E: int) -> int:
    return int(load().railsched_route_balance_workspace_bytes(rows, groups, E))


def _groups(r: _Rows, groups: int, group_off: Optional[torch.Tensor]):
    if group_off is None:
        return _int32(groups, "groups"), None
    if group_off.dim() != 1 or group_off.shape[0] < 1:
        raise ValueError("group_off must hold groups + 1 offsets")
    return group_off.shape[0] - 1, r.arg(group_off, torch.int64, group_off.shape, "group_off")


def route_balance(logits: torch.Tensor, topk_idx: torch.Tensor, groups: int = 1, group_off: Optional[torch.Tensor] = None, coef: float = 1.0,
                  row_mask: Optional[torch.Tensor] = None, out=None, ws: Optional[torch.Tensor] = None):
    """Balance loss of groups of rows: (counts [groups][E] int64, tokens [groups] int64, prob_sum [groups][E], loss [groups]).
    The groups are `groups` equal parts of the rows, or with group_off (int64 offsets) the rows between neighbouring offsets.
    The outputs are detached from autograd: route_balance_backward gives the logits' gradient."""
    r = _Rows(logits)
    n, off = _groups(r, groups, group_off)
    k = r.width(topk_idx, "topk_idx")
    if out is None:
        out = (r.new((n, r.E), torch.int64), r.new(n, torch.int64), r.new((n, r.E)), r.new(n))
        to = [t.data_ptr() for t in out]
    else:
        counts, tokens, prob_sum, loss = out
        to = (r.arg(counts, torch.int64, (n, r.E), "counts"), r.arg(tokens, torch.int64, (n,), "tokens"),
              r.arg(prob_sum, torch.float32, (n, r.E), "prob_sum"), r.arg(loss, torch.float32, (n,), "loss"))
    if ws is None:
        ws = _ws(route_balance_workspace_bytes(r.rows, n, r.E), r.device)
    r.call("railsched_route_balance", *r.head, r.mask(row_mask), r.arg(topk_idx, torch.int32, (r.rows, k), "topk_idx"), k, off, n, coef, *to,
           r.arg(ws, torch.uint8, ws.shape, "ws"), ws.numel())
    return out


def route_balance_backward(logits: torch.Tensor, k: int, counts: torch.Tensor, tokens: torch.Tensor, d_loss: torch.Tensor,
                           group_off: Optional[torch.Tensor] = None, coef: float = 1.0, row_mask: Optional[torch.Tensor] = None,
                           accumulate: bool = False, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The gradient of the logits from that of the losses, with the counts and tokens of route_balance (or their sums over ranks).
    Rows of no group (before the first offset, behind the last one) are left as they are in `out`, and 0 without `out`."""
    r = _Rows(logits)
    n, off = _groups(r, counts.shape[0], group_off)
    how = 2 if out is None and off is not None else int(accumulate)        # 2: rows of no group are set to 0
    out, to, ld_d = r.gradient(out, accumulate)
    r.call("railsched_route_balance_backward", *r.head, r.mask(row_mask), _int32(k, "k"), off, n, coef, r.arg(counts, torch.int64, (n, r.E), "counts"),
           r.arg(tokens, torch.int64, (n,), "tokens"), r.arg(d_loss, torch.float32, (n,), "d_loss"), how, to, ld_d)
    return out


def route_distill(logits: torch.Tensor, teacher_idx: torch.Tensor, teacher_logits: torch.Tensor, teacher_lse: Optional[torch.Tensor] = None,
                  temperature: float = 1.0, row_mask: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Divergence of every row's distribution from the teacher's list [rows][K] (and, with teacher_lse, the rest of the teacher's mass).
    temperature: 2^-8 to 2^8.  The outputs are detached from autograd: route_distill_backward gives the logits' gradient."""
    r = _Rows(logits)
    K = r.width(teacher_idx, "teacher_idx")
    if out is None:
        out = r.new(r.rows)
    else:
        r.arg(out, torch.float32, (r.rows,), "out")
    r.call("railsched_route_distill", *r.head, temperature, r.mask(row_mask), r.arg(teacher_idx, torch.int32, (r.rows, K), "teacher_idx"),
           r.arg(teacher_logits, torch.float32, (r.rows, K), "teacher_logits"), r.arg(teacher_lse, torch.float32, (r.rows,), "teacher_lse"), K,
           out.data_ptr())
    return out


def route_distill_backward(logits: torch.Tensor, teacher_idx: torch.Tensor, teacher_logits: torch.Tensor, d_loss: torch.Tensor,
                           teacher_lse: Optional[torch.Tensor] = None, temperature: float = 1.0, row_mask: Optional[torch.Tensor] = None,
                           accumulate: bool = False, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The gradient of the logits from that of route_distill's losses."""
    r = _Rows(logits)
    K = r.width(teacher_idx, "teacher_idx")
    out, to, ld_d = r.gradient(out, accumulate)
    r.call("railsched_route_distill_backward", *r.head, temperature, r.mask(row_mask),
           r.arg(teacher_idx, torch.int32, (r.rows, K), "teacher_idx"), r.arg(teacher_logits, torch.float32, (r.rows, K), "teacher_logits"),
           r.arg(teacher_lse, torch.float32, (r.rows,), "teacher_lse"), K, r.arg(d_loss, torch.float32, (r.rows,), "d_loss"),
           int(accumulate), to, ld_d)
    return out
