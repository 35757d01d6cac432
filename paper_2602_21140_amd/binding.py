"""ctypes binding of librevive.so: argument marshalling only.

Function names and argument order follow include/revive.h.  torch is used for device memory
(tensors whose data_ptr() is handed to the library) and for the stream handle; no step of the
layer is computed here.  There is no fallback: if the library is missing, loading raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, List, Optional, Sequence, Tuple

import numpy as np
import torch

_PKG_DIR = os.path.dirname(os.path.abspath(__file__))
_LIB_NAME = "librevive.so"
_lib = None
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # private to torch: another one may not have it

SCORE_FN = {"softmax": 0, "sigmoid": 1}
DTYPE = {"fp32": 0, "bf16": 1}
TORCH_DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16}

KERNEL_NAMES = ["router_gemm", "route_topk", "dispatch_index",
                "dispatch_permute", "ffn_tiles", "ffn_gate_up", "ffn_down", "ffn_shared_gate_up",
                "ffn_shared_down", "combine", "expert_counts", "mx_quantize", "mx_gate_up", "mx_down"]


class ReviveError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{_status_name(status)} ({status}): {message}")
        self.status = status


class Config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in
                ("T_max", "H", "E", "k", "I", "I_shared", "n_ranks", "slots_per_rank", "max_replicas",
                 "score_fn", "n_group", "topk_group", "dtype")] + [("route_scale", C.c_float)]


class MapStats(C.Structure):
    _fields_ = [(n, C.c_int32) for n in
                ("n_live_slots", "n_live_experts", "n_lost_experts", "n_degraded_experts")]

    def as_dict(self) -> Dict[str, int]:
        return {n: int(getattr(self, n)) for n, _ in self._fields_}


def lib_path() -> str:
    return os.path.join(_PKG_DIR, _LIB_NAME)


def lib() -> C.CDLL:
    """Load librevive.so (once) and declare its prototypes."""
    global _lib
    if _lib is not None:
        return _lib
    path = lib_path()
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it first (python -m paper_2602_21140_amd.build); "
                          "there is no fallback path")
    L = C.CDLL(path)
    vp, i32, sz = C.c_void_p, C.c_int32, C.c_size_t
    P = C.POINTER
    protos = {
        "revive_create": (C.c_int, [P(Config), P(vp)]),
        "revive_destroy": (C.c_int, [vp]),
        "revive_workspace_bytes": (C.c_int, [vp, P(sz)]),
        "revive_bind_workspace": (C.c_int, [vp, vp, sz]),
        "revive_set_placement": (C.c_int, [vp, vp]),
        "revive_update_map": (C.c_int, [vp, vp, vp, P(MapStats)]),
        "revive_update_map_experts": (C.c_int, [vp, vp, vp, vp, P(MapStats)]),
        "revive_get_map": (C.c_int, [vp, vp, vp, vp]),
        "revive_build_map_experts": (C.c_int, [P(Config), vp, vp, vp, vp, vp, vp, P(MapStats)]),
        "revive_compact_ranks": (C.c_int, [vp, i32, i32, i32]),
        "revive_mask_every_nth": (C.c_int, [i32, i32, vp]),
        "revive_mask_most_activated": (C.c_int, [vp, i32, i32, vp]),
        "revive_expert_counts": (C.c_int, [vp, vp, i32, vp, vp]),
        "revive_build_map": (C.c_int, [P(Config), vp, vp, vp, vp, vp, P(MapStats)]),
        "revive_route": (C.c_int, [vp, vp, vp, vp, i32, i32, vp, vp, vp, vp]),
        "revive_route_biased": (C.c_int, [vp, vp, vp, vp, i32, vp, i32, i32, vp, vp, vp, vp]),
        "revive_dispatch_index": (C.c_int, [vp, vp, i32, vp, vp, vp, vp]),
        "revive_mx_quantize": (C.c_int, [vp, i32, C.c_int64, i32, C.c_int64, vp, vp, vp]),
        "revive_mx_dequantize": (C.c_int, [vp, vp, C.c_int64, i32, i32, vp, C.c_int64, vp]),
        "revive_mx_packed_bytes": (C.c_int, [i32, i32, P(sz)]),
        "revive_mx_pack": (C.c_int, [vp, vp, i32, i32, vp, vp]),
        "revive_mx_expert_ffn": (C.c_int, [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp]),
        "revive_dispatch": (C.c_int, [vp, vp, vp, i32, vp, vp, vp, vp, vp]),
        "revive_set_token_offset": (C.c_int, [vp, C.c_int64]),
        "revive_get_rank_map": (C.c_int, [vp, vp, vp]),
        "revive_rank_offsets": (C.c_int, [vp, vp, vp, vp]),
        "revive_dispatch_static": (C.c_int, [vp, vp, vp, i32, vp, vp, vp, vp, vp]),
        "revive_expert_ffn": (C.c_int, [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp]),
        "revive_shared_ffn": (C.c_int, [vp, vp, vp, vp, vp, i32, vp]),
        "revive_combine": (C.c_int, [vp, vp, vp, vp, vp, i32, vp, vp]),
        "revive_graph_begin": (C.c_int, [vp, vp]),
        "revive_graph_end": (C.c_int, [vp, vp, P(vp)]),
        "revive_graph_launch": (C.c_int, [vp, vp]),
        "revive_graph_exec_id": (C.c_size_t, [vp]),
        "revive_graph_destroy": (C.c_int, [vp]),
        "revive_set_kernel_timing": (C.c_int, [vp, i32]),
        "revive_kernel_time": (C.c_int, [vp, i32, P(C.c_double), P(C.c_int64)]),
        "revive_reset_kernel_times": (C.c_int, [vp]),
        "revive_kernel_name": (C.c_char_p, [i32]),
        "revive_last_error": (C.c_char_p, [vp]),
        "revive_status_name": (C.c_char_p, [C.c_int]),
    }
    for name, (res, args) in protos.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    _lib = L
    return L


EXPORTS = ["revive_create", "revive_destroy", "revive_workspace_bytes", "revive_bind_workspace",
           "revive_set_placement", "revive_update_map", "revive_update_map_experts", "revive_get_map", "revive_build_map",
           "revive_build_map_experts", "revive_compact_ranks", "revive_mask_every_nth", "revive_mask_most_activated", "revive_expert_counts",
           "revive_get_rank_map", "revive_rank_offsets", "revive_set_token_offset",
           "revive_route_biased", "revive_dispatch_index", "revive_mx_quantize", "revive_mx_dequantize", "revive_mx_packed_bytes",
           "revive_mx_pack", "revive_mx_expert_ffn",
           "revive_route", "revive_dispatch", "revive_dispatch_static", "revive_expert_ffn", "revive_shared_ffn", "revive_combine",
           "revive_graph_begin", "revive_graph_end", "revive_graph_launch", "revive_graph_exec_id",
           "revive_graph_destroy", "revive_set_kernel_timing", "revive_kernel_time",
           "revive_reset_kernel_times", "revive_kernel_name", "revive_last_error", "revive_status_name"]


def _status_name(status: int) -> str:
    return lib().revive_status_name(status).decode()


def make_config(cfg, T_max: Optional[int] = None, route_scale: float = 1.0) -> Config:
    """C config from a synth.LayerConfig-like object (any object with the same field names)."""
    return Config(T_max=cfg.T if T_max is None else T_max, H=cfg.H, E=cfg.E, k=cfg.k, I=cfg.I,
                  I_shared=cfg.I_shared, n_ranks=cfg.n_ranks, slots_per_rank=cfg.slots_per_rank,
                  max_replicas=cfg.max_replicas, score_fn=SCORE_FN[cfg.score_fn], n_group=cfg.n_group,
                  topk_group=cfg.topk_group, dtype=DTYPE[cfg.dtype], route_scale=route_scale)


def compact_ranks(logical_rank, failed_device: int, switched_device: int = -1) -> np.ndarray:
    """revive_compact_ranks on a copy of logical_rank (int32[n]); raises on bad input."""
    r = np.array(logical_rank, dtype=np.int32)
    rc = lib().revive_compact_ranks(r.ctypes.data, r.shape[0], failed_device, switched_device)
    if rc != 0:
        raise ReviveError(rc, lib().revive_last_error(None).decode())
    return r


def mask_every_nth(E: int, n: int) -> np.ndarray:
    """revive_mask_every_nth: uint8[E], 1 for the experts whose index is a multiple of n."""
    m = np.zeros(E, dtype=np.uint8)
    rc = lib().revive_mask_every_nth(E, n, m.ctypes.data)
    if rc != 0:
        raise ReviveError(rc, lib().revive_last_error(None).decode())
    return m


def mask_most_activated(counts: np.ndarray, n_fail: int) -> np.ndarray:
    """revive_mask_most_activated: uint8[E], 1 for the n_fail most frequently activated experts."""
    c = np.ascontiguousarray(counts, dtype=np.int64)
    m = np.zeros(c.shape[0], dtype=np.uint8)
    rc = lib().revive_mask_most_activated(c.ctypes.data, c.shape[0], n_fail, m.ctypes.data)
    if rc != 0:
        raise ReviveError(rc, lib().revive_last_error(None).decode())
    return m


def build_map_host(cfg, phys_to_logical: np.ndarray, rank_failed: np.ndarray, route_scale: float = 1.0,
                   expert_failed: Optional[np.ndarray] = None):
    """revive_build_map(_experts): the library's host-side map construction, no GPU needed.

    Returns (status, l2p_table [E, max_replicas], l2p_count [E], slot_alive [P], stats dict)."""
    c = make_config(cfg, route_scale=route_scale)
    p2l = np.ascontiguousarray(phys_to_logical, dtype=np.int32)
    failed = np.ascontiguousarray(rank_failed, dtype=np.uint8)
    assert p2l.shape[0] == cfg.n_ranks * cfg.slots_per_rank and failed.shape[0] == cfg.n_ranks
    table = np.zeros((cfg.E, cfg.max_replicas), dtype=np.int32)
    count = np.zeros(cfg.E, dtype=np.int32)
    alive = np.zeros(p2l.shape[0], dtype=np.uint8)
    stats = MapStats()
    ef = None if expert_failed is None else np.ascontiguousarray(expert_failed, dtype=np.uint8)
    rc = lib().revive_build_map_experts(C.byref(c), p2l.ctypes.data, failed.ctypes.data,
                                        None if ef is None else ef.ctypes.data, table.ctypes.data,
                                        count.ctypes.data, alive.ctypes.data, C.byref(stats))
    return rc, table, count, alive, stats.as_dict()


def pack_router(w_router: torch.Tensor) -> torch.Tensor:
    """[H, E] router matrix -> the library's output-major [E, H] layout."""
    return w_router.t().contiguous()


TILE_ROWS, TILE_K = 128, 32   # tiled weight layout of bf16 layers (include/revive.h)


def _tile(w: torch.Tensor) -> torch.Tensor:
    """[rows, K] -> the tiled layout [ceil(rows/128)*128, K] (same storage order as
    [rows/128][K/32][128][32]); rows zero-padded to a multiple of 128."""
    rows, K = w.shape
    assert K % TILE_K == 0
    pad = -rows % TILE_ROWS
    if pad:
        w = torch.cat([w, w.new_zeros(pad, K)], dim=0)
    rp = rows + pad
    return w.reshape(rp // TILE_ROWS, TILE_ROWS, K // TILE_K, TILE_K).permute(0, 2, 1, 3).contiguous().reshape(rp, K)


def _untile(t: torch.Tensor, rows: int) -> torch.Tensor:
    rp, K = t.shape
    w = t.reshape(rp // TILE_ROWS, K // TILE_K, TILE_ROWS, TILE_K).permute(0, 2, 1, 3).reshape(rp, K)
    return w[:rows]


def padded_rows(rows: int) -> int:
    return rows + (-rows % TILE_ROWS)


def pack_expert(gate: torch.Tensor, up: torch.Tensor, down: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
    """Math-layout expert matrices (gate/up [H, I], down [I, H]) -> the library's layouts.

    fp32: w_gate_up = [gate^T; up^T] as [2I, H], w_down = down^T as [H, I].
    bf16: the same matrices in the tiled layout (each of gate^T, up^T, down^T tiled separately)."""
    if gate.dtype == torch.bfloat16:
        return torch.cat([_tile(gate.t()), _tile(up.t())], dim=0).contiguous(), _tile(down.t())
    return torch.cat([gate.t(), up.t()], dim=0).contiguous(), down.t().contiguous()


def unpack_expert(w_gate_up: torch.Tensor, w_down: torch.Tensor, H: int, I: int):
    """Inverse of pack_expert: (gate [H, I], up [H, I], down [I, H])."""
    if w_gate_up.dtype == torch.bfloat16:
        ip = padded_rows(I)
        return (_untile(w_gate_up[:ip], I).t(), _untile(w_gate_up[ip:], I).t(), _untile(w_down, H).t())
    return w_gate_up[:I].t(), w_gate_up[I:].t(), w_down.t()


# ---- microscaled 4-bit floats --------------------------------------------------------------------

MX_BLOCK = 32


def _current_stream(stream: Optional[torch.cuda.Stream]) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    # without the Stream object that torch.cuda.current_stream() makes: that took 2.6 us of each of the four calls of an
    # eager step (64 tokens, H = 256, fp32: 33 -> 24 us)
    return _raw_stream(torch.cuda.current_device())


def _check_free(rc: int):
    """Status of a call that has no context."""
    if rc != 0:
        raise ReviveError(rc, lib().revive_last_error(None).decode())


_MX_DTYPE = {torch.float32: DTYPE["fp32"], torch.bfloat16: DTYPE["bf16"]}


def _mx_check_form(codes: torch.Tensor, scales: torch.Tensor, rows: int, n: int):
    """codes [rows, 16 n] and scales [rows, n], contiguous uint8."""
    if (codes.dtype is not torch.uint8 or scales.dtype is not torch.uint8 or codes.shape != (rows, 16 * n) or scales.shape != (rows, n)
            or not codes.is_contiguous() or not scales.is_contiguous() or not codes.is_cuda or not scales.is_cuda):
        raise ValueError(f"codes {codes.dtype} {tuple(codes.shape)} and scales {scales.dtype} {tuple(scales.shape)}: contiguous uint8 "
                         f"{(rows, 16 * n)} and {(rows, n)} in device memory expected")


def _mx_rows(x: torch.Tensor, what: str):
    """(library dtype, rows, K, elements between rows) of a matrix whose rows are contiguous and do not overlap."""
    dtype = _MX_DTYPE.get(x.dtype)
    if dtype is None:
        raise TypeError(f"{what}: microscaled numbers are made of and into float32 and bfloat16, not {x.dtype}")
    shape, stride = x.shape, x.stride()
    if len(shape) != 2 or not x.is_cuda:
        raise ValueError(f"{what} is a matrix in device memory")
    rows, K = shape
    ld = stride[0] if rows > 1 else K
    if ld < K or (K > 1 and stride[1] != 1):
        raise ValueError(f"{what} is a matrix whose rows are contiguous and do not overlap")
    return dtype, rows, K, ld


# Both calls' checks are kept short: with a query each for what several of them need, a call took 2 us more.
def mx_quantize(x: torch.Tensor, out=None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """revive_mx_quantize: x [rows, K] fp32 or bf16 (rows may be strided) -> (codes [rows, 16 n], scales [rows, n]), n =
    ceil(K / 32) blocks of 32."""
    dtype, rows, K, ld = _mx_rows(x, "x")
    n = (K + MX_BLOCK - 1) // MX_BLOCK
    if out is None:
        out = (torch.empty(rows, 16 * n, dtype=torch.uint8, device=x.device), torch.empty(rows, n, dtype=torch.uint8, device=x.device))
    codes, scales = out
    _mx_check_form(codes, scales, rows, n)
    _check_free(lib().revive_mx_quantize(x.data_ptr(), dtype, rows, K, ld, codes.data_ptr(), scales.data_ptr(), _current_stream(stream)))
    return codes, scales


def mx_dequantize(codes: torch.Tensor, scales: torch.Tensor, K: Optional[int] = None, dtype=torch.bfloat16, out=None,
                  stream=None) -> torch.Tensor:
    """revive_mx_dequantize: the numbers that codes and scales stand for, [rows, K] (default: all of the blocks, or out's)."""
    if out is None:
        rows, n = scales.shape
        out = torch.empty(rows, MX_BLOCK * n if K is None else K, dtype=dtype, device=codes.device)
    code, rows, width, ld = _mx_rows(out, "out")
    if K is not None and width != K:
        raise ValueError(f"out {tuple(out.shape)}: {K} columns expected")
    _mx_check_form(codes, scales, rows, (width + MX_BLOCK - 1) // MX_BLOCK)
    _check_free(lib().revive_mx_dequantize(codes.data_ptr(), scales.data_ptr(), rows, width, code, out.data_ptr(), ld, _current_stream(stream)))
    return out


def mx_packed_bytes(rows: int, K: int) -> int:
    n = C.c_size_t()
    _check_free(lib().revive_mx_packed_bytes(rows, K, C.byref(n)))
    return n.value


def mx_pack(codes: torch.Tensor, scales: torch.Tensor, out=None, stream=None) -> torch.Tensor:
    """revive_mx_pack: an output-major weight matrix' codes and scales -> uint8 in the order that the 4-bit FFN reads."""
    if scales.dim() != 2:
        raise ValueError("codes and scales are matrices")
    rows, K = scales.shape[0], scales.shape[1] * MX_BLOCK
    _mx_check_form(codes, scales, rows, scales.shape[1])
    n = mx_packed_bytes(rows, K)
    if out is None:
        out = torch.empty(n, dtype=torch.uint8, device=codes.device)
    if out.dtype != torch.uint8 or out.numel() != n or not out.is_contiguous() or not out.is_cuda:
        raise ValueError(f"out: {n} contiguous bytes in device memory expected")
    _check_free(lib().revive_mx_pack(codes.data_ptr(), scales.data_ptr(), rows, K, out.data_ptr(), _current_stream(stream)))
    return out


def mx_pack_expert(gate: torch.Tensor, up: torch.Tensor, down: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
    """Math-layout expert matrices (gate/up [H, I], down [I, H], fp32 or bf16) -> (w_gate_up, w_down), quantised along each
    product's K and packed."""
    g, u, d = (mx_pack(*mx_quantize(w.t().contiguous())) for w in (gate, up, down))
    return torch.cat([g, u]), d


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


class ReviveLayer:
    """One MoE layer context.  Methods mirror the C calls one to one; tensors are allocated here
    (torch owns the memory) and handed to the library by pointer."""

    def __init__(self, cfg, device="cuda:0", T_max: Optional[int] = None, route_scale: float = 1.0):
        self.L = lib()
        self.cfg = cfg
        self.device = torch.device(device)
        self.dtype = TORCH_DTYPE[cfg.dtype]
        self.T_max = cfg.T if T_max is None else T_max
        self.P = cfg.n_ranks * cfg.slots_per_rank
        self._ctx = C.c_void_p()
        self._cfg_c = make_config(cfg, self.T_max, route_scale)
        with torch.cuda.device(self.device):
            rc = self.L.revive_create(C.byref(self._cfg_c), C.byref(self._ctx))
            if rc != 0:
                raise ReviveError(rc, self.L.revive_last_error(None).decode())
            nbytes = C.c_size_t()
            self._check(self.L.revive_workspace_bytes(self._ctx, C.byref(nbytes)))
            self.workspace = torch.empty(max(256, nbytes.value), dtype=torch.uint8, device=self.device)
            self._check(self.L.revive_bind_workspace(self._ctx, self.workspace.data_ptr(), self.workspace.numel()))
        self._w_tabs = None
        self._mx_tabs = None
        self._graphs: List[C.c_void_p] = []

    # -- plumbing --------------------------------------------------------------------------
    def _check(self, rc: int):
        if rc != 0:
            raise ReviveError(rc, self.L.revive_last_error(self._ctx).decode())

    _stream = staticmethod(_current_stream)

    def close(self):
        if self._ctx:
            for g in self._graphs:
                self.L.revive_graph_destroy(g)
            self._graphs = []
            self.L.revive_destroy(self._ctx)
            self._ctx = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def empty(self, *shape, dtype=None) -> torch.Tensor:
        return torch.empty(*shape, dtype=self.dtype if dtype is None else dtype, device=self.device)

    # -- map -------------------------------------------------------------------------------
    def set_placement(self, phys_to_logical: np.ndarray):
        p2l = np.ascontiguousarray(phys_to_logical, dtype=np.int32)
        assert p2l.shape == (self.P,)
        self.phys_to_logical = p2l
        self._check(self.L.revive_set_placement(self._ctx, p2l.ctypes.data))

    def update_map(self, rank_failed: np.ndarray, stream=None, expert_failed: Optional[np.ndarray] = None) -> Dict[str, int]:
        failed = np.ascontiguousarray(rank_failed, dtype=np.uint8)
        assert failed.shape == (self.cfg.n_ranks,)
        stats = MapStats()
        if expert_failed is None:
            self._check(self.L.revive_update_map(self._ctx, failed.ctypes.data, self._stream(stream), C.byref(stats)))
        else:
            ef = np.ascontiguousarray(expert_failed, dtype=np.uint8)
            assert ef.shape == (self.cfg.E,)
            self._check(self.L.revive_update_map_experts(self._ctx, failed.ctypes.data, ef.ctypes.data,
                                                         self._stream(stream), C.byref(stats)))
        return stats.as_dict()

    def expert_counts(self, topk_logical, T: int, counts=None, stream=None):
        """counts[e] += activations of e in topk_logical [T, k]; counts: int64 [E] on the device."""
        if counts is None:
            counts = torch.zeros(self.cfg.E, dtype=torch.int64, device=self.device)
        self._check(self.L.revive_expert_counts(self._ctx, _ptr(topk_logical), T, _ptr(counts), self._stream(stream)))
        return counts

    def update_map_status(self, rank_failed: np.ndarray, stream=None) -> int:
        """As update_map but returns the status code instead of raising."""
        failed = np.ascontiguousarray(rank_failed, dtype=np.uint8)
        return self.L.revive_update_map(self._ctx, failed.ctypes.data, self._stream(stream), None)

    def get_map(self):
        table = np.zeros((self.cfg.E, self.cfg.max_replicas), dtype=np.int32)
        count = np.zeros(self.cfg.E, dtype=np.int32)
        alive = np.zeros(self.P, dtype=np.uint8)
        self._check(self.L.revive_get_map(self._ctx, table.ctypes.data, count.ctypes.data, alive.ctypes.data))
        return table, count, alive

    def set_token_offset(self, first_token: int):
        """revive_set_token_offset: x is rows [first_token, first_token + T) of a larger batch."""
        self._check(self.L.revive_set_token_offset(self._ctx, int(first_token)))

    def get_rank_map(self):
        """(logical_rank int32[R], n_live_ranks) of the map in force (host copies)."""
        lr = np.zeros(self.cfg.n_ranks, dtype=np.int32)
        n = C.c_int32()
        self._check(self.L.revive_get_rank_map(self._ctx, lr.ctypes.data, C.byref(n)))
        return lr, int(n.value)

    def rank_offsets(self, slot_offsets, out=None, stream=None):
        """revive_rank_offsets: int32[R+1] compacted rank segment boundaries of a dispatched buffer."""
        if out is None:
            out = self.empty(self.cfg.n_ranks + 1, dtype=torch.int32)
        self._check(self.L.revive_rank_offsets(self._ctx, _ptr(slot_offsets), _ptr(out), self._stream(stream)))
        return out

    # -- weights ---------------------------------------------------------------------------
    def set_expert_weights(self, w_gate_up: Sequence[Optional[torch.Tensor]], w_down: Sequence[Optional[torch.Tensor]]):
        """Per-slot packed weights (lists of P tensors, None for empty slots) -> device pointer tables."""
        assert len(w_gate_up) == self.P and len(w_down) == self.P
        for gu, dn in zip(w_gate_up, w_down):
            if gu is not None:
                tiled = self.dtype == torch.bfloat16
                gu_rows = 2 * (padded_rows(self.cfg.I) if tiled else self.cfg.I)
                dn_rows = padded_rows(self.cfg.H) if tiled else self.cfg.H
                assert gu.shape == (gu_rows, self.cfg.H) and gu.dtype == self.dtype and gu.is_contiguous()
                assert dn.shape == (dn_rows, self.cfg.I) and dn.dtype == self.dtype and dn.is_contiguous()
        self._w_keep = (list(w_gate_up), list(w_down))
        gu_tab = torch.tensor([0 if t is None else t.data_ptr() for t in w_gate_up], dtype=torch.int64)
        dn_tab = torch.tensor([0 if t is None else t.data_ptr() for t in w_down], dtype=torch.int64)
        self._w_tabs = (gu_tab.to(self.device), dn_tab.to(self.device))

    def set_mx_expert_weights(self, w_gate_up: Sequence[Optional[torch.Tensor]], w_down: Sequence[Optional[torch.Tensor]]):
        """Per-slot packed 4-bit weights (mx_pack_expert; lists of P tensors, None for empty slots) -> device pointer tables."""
        assert len(w_gate_up) == self.P and len(w_down) == self.P
        n_gu, n_dn = 2 * mx_packed_bytes(self.cfg.I, self.cfg.H), mx_packed_bytes(self.cfg.H, self.cfg.I)
        for w, n in [(w, n_gu) for w in w_gate_up] + [(w, n_dn) for w in w_down]:
            if w is not None:
                assert w.dtype == torch.uint8 and w.numel() == n and w.is_contiguous() and w.is_cuda and w.data_ptr() % 16 == 0
        assert all((a is None) == (b is None) for a, b in zip(w_gate_up, w_down)), "a slot has both of its matrices or none"
        I_shared = self.cfg.I_shared
        self._mx_shared_bytes = (2 * mx_packed_bytes(I_shared, self.cfg.H), mx_packed_bytes(self.cfg.H, I_shared)) if I_shared else None
        self._mx_keep = (list(w_gate_up), list(w_down))
        self._mx_tabs = tuple(torch.tensor([0 if w is None else w.data_ptr() for w in ws], dtype=torch.int64).to(self.device)
                              for ws in (w_gate_up, w_down))

    # -- data path -------------------------------------------------------------------------
    def route(self, x, w_router, T: int, logits=None, logits_given=False, out=None, stream=None):
        k = self.cfg.k
        if logits is None:
            logits = self.empty(T, self.cfg.E, dtype=torch.float32)
        if out is None:
            out = (self.empty(T, k, dtype=torch.int32), self.empty(T, k, dtype=torch.float32),
                   self.empty(T, k, dtype=torch.int32))
        top_l, top_w, top_p = out
        self._check(self.L.revive_route(self._ctx, _ptr(x), _ptr(w_router), _ptr(logits), int(bool(logits_given)), T,
                                        _ptr(top_l), _ptr(top_w), _ptr(top_p), self._stream(stream)))
        return logits, top_l, top_w, top_p

    def route_biased(self, x, w_router, bias, T: int, renormalise=True, logits=None, logits_given=False, out=None, stream=None):
        """revive_route_biased: experts chosen by score + bias (fp32 [E]), weighted by the score."""
        k, E = self.cfg.k, self.cfg.E
        if bias.dtype is not torch.float32 or bias.numel() != E or not bias.is_contiguous() or not bias.is_cuda:
            raise ValueError(f"bias: {E} contiguous float32 in device memory expected")
        if logits is None:
            logits = self.empty(T, E, dtype=torch.float32)
        if out is None:
            out = (self.empty(T, k, dtype=torch.int32), self.empty(T, k, dtype=torch.float32),
                   self.empty(T, k, dtype=torch.int32))
        top_l, top_w, top_p = out
        if logits.dtype is not torch.float32 or logits.numel() < T * E or not logits.is_contiguous() or not logits.is_cuda:
            raise ValueError(f"logits {logits.dtype} {tuple(logits.shape)}: contiguous float32 {(T, E)} in device memory expected")
        self._check(self.L.revive_route_biased(self._ctx, _ptr(x), _ptr(w_router), logits.data_ptr(), 1 if logits_given else 0, bias.data_ptr(),
                                               1 if renormalise else 0, T, top_l.data_ptr(), top_w.data_ptr(), top_p.data_ptr(), _current_stream(stream)))
        return logits, top_l, top_w, top_p

    def dispatch_index(self, topk_phys, T: int, out=None, stream=None):
        """revive_dispatch_index: (slot_offsets, dst_row, src_of) without permuted rows."""
        N = T * self.cfg.k
        if out is None:
            out = (self.empty(self.P + 1, dtype=torch.int32), self.empty(N, dtype=torch.int32), self.empty(N, dtype=torch.int32))
        slot_offsets, dst_row, src_of = out
        if N and (topk_phys.dtype is not torch.int32 or topk_phys.numel() < N or not topk_phys.is_contiguous() or not topk_phys.is_cuda):
            raise ValueError(f"topk_phys {topk_phys.dtype} {tuple(topk_phys.shape)}: contiguous int32 {(T, self.cfg.k)} in device memory expected")
        self._check(self.L.revive_dispatch_index(self._ctx, _ptr(topk_phys), T, _ptr(slot_offsets), _ptr(dst_row), _ptr(src_of),
                                                 self._stream(stream)))
        return slot_offsets, dst_row, src_of

    def dispatch(self, x, topk_phys, T: int, out=None, stream=None, static_scratch=False):
        """revive_dispatch, or with static_scratch revive_dispatch_static (which needs `out`: it is
        for callers that allocate nothing)."""
        N = T * self.cfg.k
        if out is None:
            assert not static_scratch, "the allocation-free entry point takes caller-owned outputs"
            out = (self.empty(N, self.cfg.H), self.empty(self.P + 1, dtype=torch.int32),
                   self.empty(N, dtype=torch.int32), self.empty(N, dtype=torch.int32))
        x_perm, slot_offsets, dst_row, src_of = out
        fn = self.L.revive_dispatch_static if static_scratch else self.L.revive_dispatch
        self._check(fn(self._ctx, _ptr(x), _ptr(topk_phys), T, _ptr(x_perm), _ptr(slot_offsets),
                                           _ptr(dst_row), _ptr(src_of), self._stream(stream)))
        return x_perm, slot_offsets, dst_row, src_of

    def expert_ffn(self, x_perm, slot_offsets, T: int, x=None, w_sh_gate_up=None, w_sh_down=None, out=None,
                   shared=True, stream=None):
        assert self._w_tabs is not None, "set_expert_weights first"
        N = T * self.cfg.k
        use_shared = shared and w_sh_gate_up is not None
        if out is None:
            out = (self.empty(N, self.cfg.H), self.empty(T, self.cfg.H) if use_shared else None)
        y_perm, y_shared = out
        self._check(self.L.revive_expert_ffn(self._ctx, _ptr(x_perm), _ptr(slot_offsets), _ptr(self._w_tabs[0]),
                                             _ptr(self._w_tabs[1]), _ptr(y_perm), _ptr(x) if use_shared else None,
                                             _ptr(w_sh_gate_up) if use_shared else None,
                                             _ptr(w_sh_down) if use_shared else None,
                                             _ptr(y_shared) if use_shared else None, T, self._stream(stream)))
        return y_perm, y_shared

    def mx_expert_ffn(self, x, src_of, slot_offsets, T: int, w_sh_gate_up=None, w_sh_down=None, out=None, stream=None):
        """revive_mx_expert_ffn: (y_perm, y_shared) of the 4-bit experts; x [T, H] as it came, rows found through src_of."""
        # Checks in three expressions and addresses without _ptr: of the 10.1 us of the smallest call the checks are 1.3.
        assert self._mx_tabs is not None, "set_mx_expert_weights first"
        N, H = T * self.cfg.k, self.cfg.H
        if (x.dtype is not torch.bfloat16 or x.shape[-1] != H or x.numel() < T * H or not x.is_contiguous() or not x.is_cuda
                or src_of.dtype is not torch.int32 or src_of.numel() < N or not src_of.is_contiguous() or not src_of.is_cuda
                or slot_offsets.dtype is not torch.int32 or slot_offsets.numel() <= self.P or not slot_offsets.is_contiguous() or not slot_offsets.is_cuda):
            raise ValueError(f"x {x.dtype} {tuple(x.shape)}, src_of {src_of.dtype} {tuple(src_of.shape)}, slot_offsets {slot_offsets.dtype} "
                             f"{tuple(slot_offsets.shape)}: contiguous bfloat16 {(T, H)} and int32 {N} and {self.P + 1} in device memory expected")
        gate_up = down = shared = None
        if w_sh_gate_up is not None:
            n = self._mx_shared_bytes  # None: no shared expert
            if (n is None or w_sh_down is None or w_sh_gate_up.dtype is not torch.uint8 or w_sh_gate_up.numel() != n[0] or not w_sh_gate_up.is_contiguous()
                    or not w_sh_gate_up.is_cuda or w_sh_down.dtype is not torch.uint8 or w_sh_down.numel() != n[1] or not w_sh_down.is_contiguous()
                    or not w_sh_down.is_cuda):
                raise ValueError(f"the shared expert's weights: {'none' if n is None else n} contiguous bytes of gate and up, and of down, in device memory expected")
            gate_up, down = w_sh_gate_up.data_ptr(), w_sh_down.data_ptr()
        if out is None:
            out = (self.empty(N, H), self.empty(T, H) if gate_up is not None else None)
        y_perm, y_shared = out
        if y_perm.dtype is not torch.bfloat16 or y_perm.numel() < N * H or not y_perm.is_contiguous() or not y_perm.is_cuda:
            raise ValueError(f"y_perm {y_perm.dtype} {tuple(y_perm.shape)}: contiguous bfloat16 {(N, H)} in device memory expected")
        if gate_up is not None:
            if y_shared is None or y_shared.dtype is not torch.bfloat16 or y_shared.numel() < T * H or not y_shared.is_contiguous() or not y_shared.is_cuda:
                raise ValueError(f"y_shared: contiguous bfloat16 {(T, H)} in device memory expected, the shared expert's weights are given")
            shared = y_shared.data_ptr()
        tabs = self._mx_tabs
        self._check(self.L.revive_mx_expert_ffn(self._ctx, x.data_ptr(), src_of.data_ptr(), slot_offsets.data_ptr(), tabs[0].data_ptr(), tabs[1].data_ptr(),
                                                y_perm.data_ptr(), gate_up, down, shared, T, _current_stream(stream)))
        return y_perm, y_shared

    def shared_ffn(self, x, w_sh_gate_up, w_sh_down, T: int, out=None, stream=None):
        if out is None:
            out = self.empty(T, self.cfg.H)
        self._check(self.L.revive_shared_ffn(self._ctx, _ptr(x), _ptr(w_sh_gate_up), _ptr(w_sh_down), _ptr(out), T,
                                             self._stream(stream)))
        return out

    def combine(self, y_perm, dst_row, topk_weight, y_shared, T: int, out=None, stream=None):
        if out is None:
            out = self.empty(T, self.cfg.H)
        self._check(self.L.revive_combine(self._ctx, _ptr(y_perm), _ptr(dst_row), _ptr(topk_weight), _ptr(y_shared), T,
                                          _ptr(out), self._stream(stream)))
        return out

    # -- graph replay ----------------------------------------------------------------------
    def graph_begin(self, stream: torch.cuda.Stream):
        self._check(self.L.revive_graph_begin(self._ctx, stream.cuda_stream))

    def graph_end(self, stream: torch.cuda.Stream) -> C.c_void_p:
        g = C.c_void_p()
        self._check(self.L.revive_graph_end(self._ctx, stream.cuda_stream, C.byref(g)))
        self._graphs.append(g)
        return g

    def graph_launch(self, g, stream: torch.cuda.Stream):
        rc = self.L.revive_graph_launch(g, stream.cuda_stream)
        if rc != 0:
            raise ReviveError(rc, self.L.revive_last_error(None).decode())

    def graph_exec_id(self, g) -> int:
        return int(self.L.revive_graph_exec_id(g))

    # -- timing ----------------------------------------------------------------------------
    def set_kernel_timing(self, enabled: bool):
        self._check(self.L.revive_set_kernel_timing(self._ctx, int(enabled)))

    def reset_kernel_times(self):
        self._check(self.L.revive_reset_kernel_times(self._ctx))

    def kernel_times(self) -> Dict[str, Tuple[float, int]]:
        """{kernel name: (total ms, launches)} since the last reset."""
        out = {}
        for i, name in enumerate(KERNEL_NAMES):
            ms, n = C.c_double(), C.c_int64()
            self._check(self.L.revive_kernel_time(self._ctx, i, C.byref(ms), C.byref(n)))
            out[name] = (ms.value, n.value)
        return out
