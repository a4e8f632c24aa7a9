"""Thin ctypes binding of libemr's C ABI (include/emr.h), same names, no compute.

Device buffers are torch tensors (passed by data_ptr); streams are torch
streams. Every step of the path runs in libemr's kernels: this module only
marshals arguments, allocates caller-owned buffers for the convenience
wrappers and turns status codes into exceptions. There is no fallback: if the
library has not been built, loading it raises.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import os
from dataclasses import dataclass

import numpy as np
import torch

from . import _build

EMR_OK, EMR_ERR_ARG, EMR_ERR_CYCLE, EMR_ERR_RANGE, EMR_ERR_CAPACITY, EMR_ERR_CUDA, EMR_ERR_TIMEOUT, \
    EMR_ERR_ALLOC = range(8)
EMR_MAX_DEPTH = 14
EMR_EAGER, EMR_GATED = 0, 1
CONN_F, CONN_B, CONN_L, CONN_S, CONN_ALL = 1, 2, 4, 8, 15
SUBSTRATE_FEEDFORWARD, SUBSTRATE_HH, SUBSTRATE_BACKWARD, SUBSTRATE_LATERAL, SUBSTRATE_SELF, SUBSTRATE_FULL = range(6)
TYPE_CODES = ("forward", "backward", "lateral", "self")
_M = EMR_MAX_DEPTH + 2

_lib = None


class EmrError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__("%s: %s (status %d)" % (what, strerror(status) if _lib else "?", status))


class Grid(C.Structure):
    _fields_ = [("D", C.c_int32), ("reserved", C.c_int32), ("n_total", C.c_int64), ("n_halo", C.c_int64),
                ("n_words", C.c_int64), ("chunk", C.c_int64), ("level_off", C.c_int64 * _M),
                ("halo_off", C.c_int64 * _M), ("word_off", C.c_int64 * _M)]


class QueryC(C.Structure):
    _fields_ = [("S", C.c_int32), ("per_genome", C.c_int32), ("a_host", C.c_void_p), ("b_host", C.c_void_p),
                ("side_host", C.c_void_p), ("count_host", C.c_void_p), ("a_dev", C.c_void_p),
                ("b_dev", C.c_void_p), ("side_dev", C.c_void_p), ("count_dev", C.c_void_p)]


def lib() -> C.CDLL:
    """Load libemr (after torch, so both share one CUDA runtime). Raises if it is not built."""
    global _lib
    if _lib is None:
        if not os.path.exists(_build.LIB):
            raise RuntimeError("libemr is not built (%s missing): run __graft_entry__.build()" % _build.LIB)
        _lib = C.CDLL(_build.LIB)
        vp, i32, i64, f32, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_size_t
        sig = {
            "emr_grid_build": [i32, i64, vp],
            "emr_index_to_ij": [i64, vp, vp, vp],
            "emr_pack_size": [i32, vp, vp, vp],
            "emr_pack_population": [i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp, vp],
            "emr_pack_info": [vp, vp, vp, vp],
            "emr_partition_genomes": [vp, vp, i32, vp],
            "emr_eval_workspace_size": [vp, vp, vp],
            "emr_eval_prepare": [vp, vp, vp, vp, sz, vp],
            "emr_eval": [vp, vp, vp, vp, vp, vp, sz, vp],
            "emr_grid_chunk": [vp, i64, vp, vp, vp],
            "emr_eval_chunk": [vp, vp, vp, i64, vp, vp, vp, sz, vp],
            "emr_variance_filter": [vp, vp, vp, i32, i32, f32, f32, f32, i32, vp, vp, vp, vp, vp],
            "emr_mask_combine": [vp, vp, vp, i32, i32, vp, vp],
            "emr_eval_filter": [vp, vp, vp, f32, f32, f32, vp, vp, vp, vp, sz, vp],
            "emr_eval_filter_noalloc": [vp, vp, vp, vp, f32, f32, f32, vp, vp, vp, vp],
            "emr_stream_workspace_size": [vp, vp, vp, i64, vp],
            "emr_stream": [vp, vp, vp, vp, f32, f32, f32, vp, sz, i64, vp, vp, i64, vp, vp, i64, vp],
            "emr_stream_mode": [vp, vp, vp, vp, f32, f32, f32, i32, i32, vp, sz, i64, vp, vp, i64, vp, vp, i64, vp],
            "emr_mask_combine_types": [vp, vp, vp, vp, i32, i32, i32, vp, vp],
            "emr_conn_types": [vp, vp, vp, vp, i32, i64, vp, vp],
            "emr_scale_weights": [vp, vp, i32, i64, f32, f32, vp],
            "emr_subtree_workspace_size": [vp, i32, vp],
            "emr_subtree_split": [vp, vp, i32, f32, vp, vp, vp, sz, vp],
            "emr_eval_filter_tiles": [vp, vp, vp, f32, f32, f32, vp, vp, vp, vp, sz, vp],
            "emr_select": [vp, vp, vp, vp, vp, vp, sz, vp, i32, i32, vp, vp, i64, vp, vp, vp, sz, vp],
            "emr_select_workspace_size": [vp, i32, vp],
            "emr_discover_workspace_size": [vp, vp, vp, vp],
            "emr_discover": [vp, vp, vp, vp, f32, f32, f32, i32, i32, vp, sz, vp, vp, i64, vp, vp, vp],
            "emr_copy_async": [vp, vp, sz, vp],
            "emr_substrate_config": [i32, vp, vp],
            "emr_assemble_workspace_size": [vp, i32, i32, i32, vp, i64, vp],
            "emr_assemble": [vp, vp, i32, vp, vp, i32, vp, vp, vp, f32, f32, f32, i32, i32, i32, i32, vp, sz, i64,
                             vp, vp, i64, vp, vp, vp, vp, vp, i64, vp, vp],
            "emr_cache_create": [sz, vp],
            "emr_cache_destroy": [vp],
            "emr_cache_clear": [vp],
            "emr_cache_stats": [vp, vp, vp, vp, vp],
            "emr_ann_forward": [i32, i32, i32, i32, vp, vp, vp, vp, vp, i32, vp, i32, vp, vp],
            "emr_compact_workspace_size": [vp, i32, vp],
            "emr_compact": [vp, vp, vp, i32, vp, vp, i64, vp, vp, vp, sz, vp],
            "emr_compact_records": [vp, vp, vp, vp, sz, vp, vp, vp, i64, vp, vp, vp, sz, vp],
            "emr_q8_size": [i32, i64, i64, vp, vp],
            "emr_q8_quantize": [vp, i32, i32, i64, i64, i64, i64, i64, vp, vp, vp],
            "emr_q8_quantize_held": [vp, i32, i32, i64, i64, i64, i64, i64, vp, vp, vp],
            "emr_q8_transpose": [vp, vp, vp],
            "emr_q8_dequantize": [vp, vp, i32, vp],
            "emr_q8_slope_workspace_size": [i32, i64, i64, vp],
            "emr_q8_slope": [vp, i32, i32, i64, i64, vp, vp, vp, vp, i32, vp, sz, vp],
            "emr_q8_matmul": [vp, vp, vp, i32, i32, vp, i32, vp, vp],
            "emr_dense_forward_room": [vp, i32, i64, i32, vp, vp, vp],
            "emr_dense_forward": [vp, vp, i32, i32, i64, i64, i64, i64, vp, i32, i32, vp, vp, vp, vp],
            "emr_dense_backward_room": [vp, i32, i64, vp],
            "emr_dense_backward": [vp, vp, i32, i32, i64, vp, vp, vp, vp, vp, i32, vp, sz, vp],
            "emr_device_error": [vp, vp],
            "emr_sample": [vp, i32, i32, i64, i64, vp, i64, vp, f32, vp, i32, vp, f32, vp, f32, vp, vp, vp],
            "emr_q4_size": [i32, i64, i64, i32, vp],
            "emr_q4_quantize": [vp, i32, i64, i64, i64, vp, vp],
            "emr_q4_pack": [vp, i64, i64, i64, vp, i64, i64, i64, vp, vp],
            "emr_q4_dequantize": [vp, vp, i32, vp],
            "emr_q4_matmul_room": [vp, i32, i32, i64, i64, i64, i64, vp, vp],
            "emr_q4_matmul": [vp, i32, i32, i64, i64, i64, i64, vp, vp, i32, vp, i32, vp, sz, vp],
            "emr_log_probs": [vp, i32, i32, i64, i64, vp, vp, f32, i32, vp, vp, vp, vp, vp],
            "emr_log_probs_grad": [vp, i32, i32, i64, i64, vp, vp, f32, vp, f32, vp, f32, vp, vp, vp, i32, i64, vp],
            "emr_distill": [vp, i32, i32, i64, i64, vp, vp, i32, i32, vp, f32, i32, vp, f32, vp, vp, i32, i64, vp],
            "emr_version": [],
            "emr_probe_alu": [i32, i32, i32, vp, vp, vp, vp],
        }
        for name, args in sig.items():
            f = getattr(_lib, name)
            f.argtypes = args
            f.restype = C.c_int32
        _lib.emr_pack_release.argtypes = []
        _lib.emr_pack_release.restype = None
        _lib.emr_strerror.argtypes = [C.c_int32]
        _lib.emr_strerror.restype = C.c_char_p
    return _lib


def strerror(status: int) -> str:
    return lib().emr_strerror(status).decode()


def _check(status: int, what: str):
    if status != EMR_OK:
        raise EmrError(status, what)


def _ptr(x):
    if x is None:
        return None
    if isinstance(x, torch.Tensor):
        return C.c_void_p(x.data_ptr())
    if isinstance(x, np.ndarray):
        return x.ctypes.data_as(C.c_void_p)
    return x


def _stream(stream):
    s = stream if stream is not None else torch.cuda.current_stream()
    return C.c_void_p(s.cuda_stream)


# ---- a1 -----------------------------------------------------------------------

def grid_build(D: int, chunk: int = 0) -> Grid:
    g = Grid()
    _check(lib().emr_grid_build(D, chunk, C.byref(g)), "emr_grid_build")
    return g


def index_to_ij(gidx: int):
    d, i, j = C.c_int32(), C.c_int32(), C.c_int32()
    _check(lib().emr_index_to_ij(gidx, C.byref(d), C.byref(i), C.byref(j)), "emr_index_to_ij")
    return d.value, i.value, j.value


# ---- a2 -----------------------------------------------------------------------

def _pop_ptrs(pop):
    """Addresses of a Population's ten arrays, kept on the object together with the arrays
    themselves (so an address never outlives its array); a field that now holds another
    array is looked up again."""
    arrays = (pop.node_ptr, pop.node_id, pop.node_kind, pop.node_act, pop.node_bias, pop.conn_ptr,
              pop.conn_src, pop.conn_dst, pop.conn_w, pop.conn_enabled)
    cache = getattr(pop, "_emr_ptrs", None)
    if cache is None or any(a is not b for a, b in zip(cache[0], arrays)):
        cache = (arrays, tuple(int(a.ctypes.data) for a in arrays))
        try:
            object.__setattr__(pop, "_emr_ptrs", cache)
        except AttributeError:
            pass
    return cache[1]


def _range_ptrs(pop, genomes):
    """P and the ten array addresses for genomes [g0, g1) of pop (the whole population when
    genomes is None): node_ptr and conn_ptr offset to g0, the other arrays unchanged."""
    ptr = _pop_ptrs(pop)
    if genomes is None:
        return pop.P, ptr
    g0, g1 = int(genomes[0]), int(genomes[1])
    if not 0 <= g0 < g1 <= pop.P:
        raise ValueError("genome range [%d, %d) outside [0, %d)" % (g0, g1, pop.P))
    return g1 - g0, (ptr[0] + 8 * g0,) + ptr[1:5] + (ptr[5] + 8 * g0,) + ptr[6:]


def pack_size(pop, genomes=None) -> int:
    """Upper bound of the packed blob's bytes for a workloads.Population (emr_pack_size)."""
    n = C.c_size_t()
    P, ptr = _range_ptrs(pop, genomes)
    _check(lib().emr_pack_size(P, ptr[0], ptr[5], C.byref(n)), "emr_pack_size")
    return int(n.value)


def pack_population(pop, out=None, genomes=None) -> np.ndarray:
    """Packed blob (numpy uint8) of a workloads.Population, or of its genomes [g0, g1) when
    genomes = (g0, g1); written into `out` (a contiguous uint8 array, e.g. a view of pinned
    memory) when given, else into a new array."""
    L = lib()
    n = C.c_size_t()
    P, ptr = _range_ptrs(pop, genomes)
    _check(L.emr_pack_size(P, ptr[0], ptr[5], C.byref(n)), "emr_pack_size")
    if out is not None:
        if out.dtype != np.uint8 or not out.flags.c_contiguous or len(out) < n.value:
            raise ValueError("out: contiguous uint8 array of at least %d bytes" % n.value)
        buf = out
    else:
        buf = np.empty(n.value + 16, np.uint8)   # the packer clears what it uses
    used, bad = C.c_size_t(), C.c_int32()
    st = L.emr_pack_population(P, *ptr, int(buf.ctypes.data), len(buf), C.byref(used), C.byref(bad))
    if st != EMR_OK:
        e = EmrError(st, "emr_pack_population (genome %d)" % bad.value)
        e.bad_genome = bad.value
        raise e
    return buf[:used.value]


def pack_release() -> None:
    """Join the packer's worker threads and free its kept buffers (emr_pack_release)."""
    lib().emr_pack_release()


def partition_genomes(pack: np.ndarray, query, n_parts: int) -> np.ndarray:
    """Contiguous genome ranges of balanced cost (emr_partition_genomes): int32 [n_parts + 1],
    part k = genomes [g[k], g[k+1])."""
    g = np.zeros(n_parts + 1, np.int32)
    q = query.c
    _check(lib().emr_partition_genomes(_ptr(pack), C.byref(q), n_parts, _ptr(g)), "emr_partition_genomes")
    return g


def pack_info(pack: np.ndarray):
    P, mo, mi = C.c_int32(), C.c_int32(), C.c_int32()
    _check(lib().emr_pack_info(_ptr(pack), C.byref(P), C.byref(mo), C.byref(mi)), "emr_pack_info")
    return P.value, mo.value, mi.value


@dataclass
class Query:
    """Host and device copies of the query slots (workloads.Sources)."""
    a: np.ndarray
    b: np.ndarray
    side: np.ndarray
    count: np.ndarray | None
    a_dev: torch.Tensor
    b_dev: torch.Tensor
    side_dev: torch.Tensor
    count_dev: torch.Tensor | None
    S: int
    per_genome: bool

    @property
    def c(self) -> QueryC:
        q = QueryC()
        q.S, q.per_genome = self.S, 1 if self.per_genome else 0
        q.a_host, q.b_host, q.side_host = (self.a.ctypes.data, self.b.ctypes.data, self.side.ctypes.data)
        q.count_host = self.count.ctypes.data if self.count is not None else None
        q.a_dev, q.b_dev, q.side_dev = (self.a_dev.data_ptr(), self.b_dev.data_ptr(), self.side_dev.data_ptr())
        q.count_dev = self.count_dev.data_ptr() if self.count_dev is not None else None
        return q


def make_query(sources, device="cuda") -> Query:
    a = np.ascontiguousarray(sources.a, np.float32)
    b = np.ascontiguousarray(sources.b, np.float32)
    s = np.ascontiguousarray(sources.side, np.int32)
    cnt = None if sources.count is None else np.ascontiguousarray(sources.count, np.int32)
    dev = lambda x: torch.from_numpy(x).to(device) if x is not None else None
    return Query(a, b, s, cnt, dev(a), dev(b), dev(s), dev(cnt), int(a.shape[-1]), a.ndim == 2)


# ---- workspace sizes ------------------------------------------------------------

def eval_workspace_size(pack: np.ndarray, query: Query) -> int:
    n = C.c_size_t()
    q = query.c
    _check(lib().emr_eval_workspace_size(_ptr(pack), C.byref(q), C.byref(n)), "emr_eval_workspace_size")
    return n.value


def compact_workspace_size(grid: Grid, n_pairs: int) -> int:
    n = C.c_size_t()
    _check(lib().emr_compact_workspace_size(C.byref(grid), n_pairs, C.byref(n)), "emr_compact_workspace_size")
    return n.value


# ---- a3..a6 -----------------------------------------------------------------------

def eval_prepare(pack, pack_dev, query: Query, ws, stream=None):
    q = query.c
    _check(lib().emr_eval_prepare(_ptr(pack), _ptr(pack_dev), C.byref(q), _ptr(ws), C.c_size_t(ws.numel()),
                                  _stream(stream)), "emr_eval_prepare")


def eval(pack, query: Query, grid: Grid, out, out_halo, ws, stream=None):
    q = query.c
    _check(lib().emr_eval(_ptr(pack), C.byref(q), C.byref(grid), _ptr(out), _ptr(out_halo), _ptr(ws),
                          C.c_size_t(ws.numel()), _stream(stream)), "emr_eval")


def grid_chunk(grid: Grid, chunk_idx: int = 0):
    """(number of chunks, first global index, end global index) of chunk chunk_idx (emr_grid_chunk)."""
    n, lo, hi = C.c_int64(), C.c_int64(), C.c_int64()
    _check(lib().emr_grid_chunk(C.byref(grid), chunk_idx, C.byref(n), C.byref(lo), C.byref(hi)), "emr_grid_chunk")
    return n.value, lo.value, hi.value


def eval_chunk(pack, query: Query, grid: Grid, chunk_idx: int, out, out_halo, ws, stream=None):
    """emr_eval_chunk: CPPN outputs of one chunk, out [pairs, chunk positions]."""
    q = query.c
    _check(lib().emr_eval_chunk(_ptr(pack), C.byref(q), C.byref(grid), chunk_idx, _ptr(out), _ptr(out_halo),
                                _ptr(ws), ws.numel(), _stream(stream)), "emr_eval_chunk")

def variance_filter(out, out_halo, grid: Grid, P: int, S: int, theta: float, band: float, w_min: float, mode: int,
                    mask, split, band_bits, var_dbg=None, stream=None):
    _check(lib().emr_variance_filter(_ptr(out), _ptr(out_halo), C.byref(grid), P, S, theta, band, w_min, mode,
                                     _ptr(mask), _ptr(split), _ptr(band_bits), _ptr(var_dbg), _stream(stream)),
           "emr_variance_filter")


def mask_combine(split, band_bits, grid: Grid, n_pairs: int, mode: int, mask, stream=None):
    _check(lib().emr_mask_combine(_ptr(split), _ptr(band_bits), C.byref(grid), n_pairs, mode, _ptr(mask),
                                  _stream(stream)), "emr_mask_combine")


def eval_filter(pack, query: Query, grid: Grid, theta: float, band: float, w_min: float, split, band_bits, out, ws,
                stream=None):
    q = query.c
    _check(lib().emr_eval_filter(_ptr(pack), C.byref(q), C.byref(grid), theta, band, w_min, _ptr(split),
                                 _ptr(band_bits), _ptr(out), _ptr(ws), C.c_size_t(ws.numel()), _stream(stream)),
           "emr_eval_filter")


def eval_filter_noalloc(pack, pack_dev, query: Query, grid: Grid, theta: float, band: float, w_min: float, split,
                        band_bits, out, stream=None):
    """emr_eval_filter_noalloc: prepare + fused evaluation in libemr's static device scratch."""
    q = query.c
    _check(lib().emr_eval_filter_noalloc(_ptr(pack), _ptr(pack_dev), C.byref(q), C.byref(grid), theta, band, w_min,
                                         _ptr(split), _ptr(band_bits), _ptr(out), _stream(stream)),
           "emr_eval_filter_noalloc")


def stream_workspace_size(pack, query: Query, grid: Grid, chunk_cap: int) -> int:
    n = C.c_size_t()
    q = query.c
    _check(lib().emr_stream_workspace_size(_ptr(pack), C.byref(q), C.byref(grid), chunk_cap, C.byref(n)),
           "emr_stream_workspace_size")
    return n.value


def stream(pack, pack_dev, query: Query, grid: Grid, theta: float, band: float, w_min: float, ws, chunk_cap: int,
           h_idx, h_w, counts, offsets, timeout_ms: int = 0, stream=None, mode: int = EMR_EAGER,
           types: int = CONN_ALL):
    """emr_stream (eager, every type) or emr_stream_mode: chunked discovery; lists land in the
    (pinned) host tensors h_idx / h_w."""
    q = query.c
    if mode == EMR_EAGER and types == CONN_ALL:
        _check(lib().emr_stream(_ptr(pack), _ptr(pack_dev), C.byref(q), C.byref(grid), theta, band, w_min, _ptr(ws),
                                C.c_size_t(ws.numel()), chunk_cap, _ptr(h_idx), _ptr(h_w), h_idx.numel(),
                                _ptr(counts), _ptr(offsets), timeout_ms, _stream(stream)), "emr_stream")
        return
    _check(lib().emr_stream_mode(_ptr(pack), _ptr(pack_dev), C.byref(q), C.byref(grid), theta, band, w_min, mode,
                                 types, _ptr(ws), C.c_size_t(ws.numel()), chunk_cap, _ptr(h_idx), _ptr(h_w),
                                 h_idx.numel(), _ptr(counts), _ptr(offsets), timeout_ms, _stream(stream)),
           "emr_stream_mode")


def dense_tiles(D: int) -> int:
    """Dense tiles of a depth-D grid: one for depths 0..4, then the 64 x 64 blocks of depths 5..D."""
    return 1 + sum(4 ** (d - 5) for d in range(5, D + 1))


def eval_filter_tiles(pack, query: Query, grid: Grid, theta: float, band: float, w_min: float, split, band_bits,
                      tile_flags, ws, stream=None):
    q = query.c
    _check(lib().emr_eval_filter_tiles(_ptr(pack), C.byref(q), C.byref(grid), theta, band, w_min, _ptr(split),
                                       _ptr(band_bits), _ptr(tile_flags), _ptr(ws), C.c_size_t(ws.numel()),
                                       _stream(stream)), "emr_eval_filter_tiles")


def select_workspace_size(grid: Grid, n_pairs: int) -> int:
    n = C.c_size_t()
    _check(lib().emr_select_workspace_size(C.byref(grid), n_pairs, C.byref(n)), "emr_select_workspace_size")
    return n.value


def select(split, band_bits, tile_flags, pack, query: Query, eval_ws, grid: Grid, mode: int, types: int, idx, w,
           cap: int, counts, offsets, ws, stream=None):
    """emr_select: combine + compaction + kept weights over the flagged tiles only."""
    q = query.c
    _check(lib().emr_select(_ptr(split), _ptr(band_bits), _ptr(tile_flags), _ptr(pack), C.byref(q), _ptr(eval_ws),
                            C.c_size_t(eval_ws.numel()), C.byref(grid), mode, types, _ptr(idx), _ptr(w), cap,
                            _ptr(counts), _ptr(offsets), _ptr(ws), C.c_size_t(ws.numel()), _stream(stream)),
           "emr_select")


def discover_workspace_size(pack, query: Query, grid: Grid) -> int:
    n = C.c_size_t()
    q = query.c
    _check(lib().emr_discover_workspace_size(_ptr(pack), C.byref(q), C.byref(grid), C.byref(n)),
           "emr_discover_workspace_size")
    return n.value


def discover(pack, pack_dev, query: Query, grid: Grid, theta: float, band: float, w_min: float, mode: int,
             types: int, ws, idx, w, cap: int, counts, offsets, stream=None, qc=None):
    """emr_discover: the whole path (records, fused evaluation and filter, selection) in one call.
    qc: a QueryC from query.c, to reuse across calls."""
    q = qc if qc is not None else query.c
    _check(lib().emr_discover(_ptr(pack), _ptr(pack_dev), C.byref(q), C.byref(grid), theta, band, w_min, mode, types,
                              _ptr(ws), C.c_size_t(ws.numel()), _ptr(idx), _ptr(w), cap, _ptr(counts),
                              _ptr(offsets), _stream(stream)), "emr_discover")


def copy_async(dst, src, nbytes: int, stream=None):
    """emr_copy_async: nbytes from src to dst (tensors, numpy arrays or addresses; host buffers
    pinned) on the stream."""
    _check(lib().emr_copy_async(_ptr(dst), _ptr(src), C.c_size_t(nbytes), _stream(stream)), "emr_copy_async")


def mask_combine_types(split, band_bits, query: Query, grid: Grid, n_pairs: int, mode: int, types: int, mask,
                       stream=None):
    q = query.c
    _check(lib().emr_mask_combine_types(_ptr(split), _ptr(band_bits), C.byref(q), C.byref(grid), n_pairs, mode,
                                        types, _ptr(mask), _stream(stream)), "emr_mask_combine_types")


def subtree_workspace_size(grid: Grid, n_pairs: int) -> int:
    n = C.c_size_t()
    _check(lib().emr_subtree_workspace_size(C.byref(grid), n_pairs, C.byref(n)), "emr_subtree_workspace_size")
    return n.value


def subtree_split(out, grid: Grid, n_pairs: int, theta: float, split, ws, var_out=None, stream=None):
    """emr_subtree_split: split plane from the variance over each cell's depth-D descendants."""
    _check(lib().emr_subtree_split(_ptr(out), C.byref(grid), n_pairs, theta, _ptr(split), _ptr(var_out), _ptr(ws),
                                   C.c_size_t(ws.numel()), _stream(stream)), "emr_subtree_split")


def scale_weights(w, offsets, n_pairs: int, cap: int, w_thr: float, w_max: float, stream=None):
    """emr_scale_weights: HyperNEAT's thresholded linear weight scaling of list weights, in place."""
    _check(lib().emr_scale_weights(_ptr(w), _ptr(offsets), n_pairs, cap, w_thr, w_max, _stream(stream)),
           "emr_scale_weights")


def conn_types(idx, offsets, query: Query, grid: Grid, n_pairs: int, cap: int, type_out, stream=None):
    """emr_conn_types: type code (0 F, 1 B, 2 L, 3 S) of every list entry into the device uint8 tensor."""
    q = query.c
    _check(lib().emr_conn_types(_ptr(idx), _ptr(offsets), C.byref(q), C.byref(grid), n_pairs, cap, _ptr(type_out),
                                _stream(stream)), "emr_conn_types")


def substrate_config(config: int):
    """(enabled EMR_CONN_* bits, hidden-to-hidden rounds on) of a Section 6 substrate configuration."""
    t, h = C.c_int32(), C.c_int32()
    _check(lib().emr_substrate_config(config, C.byref(t), C.byref(h)), "emr_substrate_config")
    return t.value, h.value


def compact(mask, out, grid: Grid, n_pairs: int, idx, w, cap: int, counts, offsets, ws, stream=None):
    _check(lib().emr_compact(_ptr(mask), _ptr(out), C.byref(grid), n_pairs, _ptr(idx), _ptr(w), cap, _ptr(counts),
                             _ptr(offsets), _ptr(ws), C.c_size_t(ws.numel()), _stream(stream)), "emr_compact")


def compact_records(mask, pack, query: Query, eval_ws, grid: Grid, idx, w, cap: int, counts, offsets, ws,
                    stream=None):
    """emr_compact_records: lists with the kept weights recomputed from the prepared records."""
    q = query.c
    _check(lib().emr_compact_records(_ptr(mask), _ptr(pack), C.byref(q), _ptr(eval_ws),
                                     C.c_size_t(eval_ws.numel()), C.byref(grid), _ptr(idx), _ptr(w), cap,
                                     _ptr(counts), _ptr(offsets), _ptr(ws), C.c_size_t(ws.numel()),
                                     _stream(stream)), "emr_compact_records")


# ---- network assembly and the substrate ANN ----------------------------------------------

@dataclass
class Networks:
    """Assembled substrate networks (host arrays, layout of emr_assemble)."""
    n_in: int
    n_out: int
    node_off: np.ndarray   # int64 [P + 1]
    hidden: np.ndarray     # int32 global grid indices
    conn_off: np.ndarray   # int64 [P + 1]
    src: np.ndarray        # int32
    dst: np.ndarray        # int32
    w: np.ndarray          # float32
    type: np.ndarray       # uint8
    _dev: tuple | None = None  # device copies made by ann_forward

    @property
    def P(self) -> int:
        return len(self.node_off) - 1

    def genome(self, g: int):
        """(hidden positions, src, dst, w, type) of genome g."""
        h = self.hidden[self.node_off[g]:self.node_off[g + 1]]
        c = slice(self.conn_off[g], self.conn_off[g + 1])
        return h, self.src[c], self.dst[c], self.w[c], self.type[c]


class Cache:
    """emr_cache: connection lists reused across emr_assemble calls (owned handle)."""

    def __init__(self, max_bytes: int = 1 << 30):
        h = C.c_void_p()
        _check(lib().emr_cache_create(max_bytes, C.byref(h)), "emr_cache_create")
        self.handle = h

    def stats(self):
        v = [C.c_int64() for _ in range(4)]
        _check(lib().emr_cache_stats(self.handle, *[C.byref(x) for x in v]), "emr_cache_stats")
        return dict(zip(("hits", "misses", "entries", "bytes"), (x.value for x in v)))

    def clear(self):
        _check(lib().emr_cache_clear(self.handle), "emr_cache_clear")

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.emr_cache_destroy(self.handle)
            self.handle = None


def assemble(pack, pack_dev, in_xy, out_xy, grid: Grid, theta: float, band: float, w_min: float = 0.0,
             mode: int = EMR_EAGER, types: int = CONN_ALL, rounds: int = 1, slots_max: int = 256,
             list_cap: int = 1 << 24, hidden_cap: int = 1 << 22, conn_cap: int = 1 << 24, stream=None,
             cache: Cache | None = None) -> Networks:
    """emr_assemble: substrate networks of every genome (device workspace allocated here)."""
    in_xy = np.ascontiguousarray(in_xy, np.float32).reshape(-1, 2)
    out_xy = np.ascontiguousarray(out_xy, np.float32).reshape(-1, 2)
    ix, iy = np.ascontiguousarray(in_xy[:, 0]), np.ascontiguousarray(in_xy[:, 1])
    ox, oy = np.ascontiguousarray(out_xy[:, 0]), np.ascontiguousarray(out_xy[:, 1])
    n = C.c_size_t()
    _check(lib().emr_assemble_workspace_size(_ptr(pack), len(ix), len(ox), slots_max, C.byref(grid), list_cap,
                                             C.byref(n)), "emr_assemble_workspace_size")
    ws = torch.empty(n.value, dtype=torch.uint8, device="cuda")
    P = pack_info(pack)[0]
    node_off = np.zeros(P + 1, np.int64)
    conn_off = np.zeros(P + 1, np.int64)
    hidden = np.zeros(hidden_cap, np.int32)
    src = np.zeros(conn_cap, np.int32)
    dst = np.zeros(conn_cap, np.int32)
    w = np.zeros(conn_cap, np.float32)
    ty = np.zeros(conn_cap, np.uint8)
    _check(lib().emr_assemble(_ptr(pack), _ptr(pack_dev), len(ix), _ptr(ix), _ptr(iy), len(ox), _ptr(ox), _ptr(oy),
                              C.byref(grid), theta, band, w_min, mode, types, rounds, slots_max, _ptr(ws),
                              C.c_size_t(ws.numel()), list_cap, _ptr(node_off), _ptr(hidden), hidden_cap,
                              _ptr(conn_off), _ptr(src), _ptr(dst), _ptr(w), _ptr(ty), conn_cap,
                              cache.handle if cache is not None else None, _stream(stream)),
           "emr_assemble")
    nh, nc = int(node_off[-1]), int(conn_off[-1])
    return Networks(len(ix), len(ox), node_off, hidden[:nh].copy(), conn_off, src[:nc].copy(), dst[:nc].copy(),
                    w[:nc].copy(), ty[:nc].copy())


def ann_forward(nets: Networks, patterns, steps: int, device="cuda", stream=None, out=None):
    """emr_ann_forward: outputs [P, K, n_out] (device tensor) of every network on patterns [K, n_in].
    The networks' arrays are copied to the device once and kept with them."""
    dev = torch.device(device)
    if getattr(nets, "_dev", None) is None or nets._dev[0] != dev:
        t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)
        nets._dev = (dev, t(nets.node_off), t(nets.conn_off), t(nets.src), t(nets.dst), t(nets.w))
    _, node_off, conn_off, src, dst, w = nets._dev
    pat = patterns if isinstance(patterns, torch.Tensor) else \
        torch.as_tensor(np.ascontiguousarray(patterns, np.float32).reshape(-1, nets.n_in), device=dev)
    K = pat.shape[0]
    if out is None:
        out = torch.zeros(nets.P, K, nets.n_out, dtype=torch.float32, device=dev)
    max_hidden = int(np.max(np.diff(nets.node_off))) if nets.P else 0
    _check(lib().emr_ann_forward(nets.P, nets.n_in, nets.n_out, max_hidden, _ptr(node_off), _ptr(conn_off),
                                 _ptr(src), _ptr(dst), _ptr(w), K, _ptr(pat), steps, _ptr(out), _stream(stream)),
           "emr_ann_forward")
    return out


# ---- dense substrate layers in 8-bit floating point ----------------------------------------

ACT_IDENTITY, ACT_SIGMOID, ACT_TANH, ACT_GAUSS, ACT_SIN, ACT_ABS = range(6)
EMR_F32, EMR_BF16, EMR_F16 = range(3)
_DTYPES = {torch.float32: EMR_F32, torch.bfloat16: EMR_BF16, torch.float16: EMR_F16}


class Q8C(C.Structure):
    _fields_ = [("batch", C.c_int32), ("reserved", C.c_int32), ("rows", C.c_int64), ("cols", C.c_int64),
                ("values", C.c_void_p), ("scales", C.c_void_p)]


class DenseC(C.Structure):
    _fields_ = [("w", Q8C), ("wt", Q8C), ("bias", C.c_void_p), ("act", C.c_int32), ("reserved", C.c_int32)]


def _dtype(t, what: str) -> int:
    d = _DTYPES.get(t)
    if d is None:
        raise ValueError("%s: float32, bfloat16 or float16 is wanted, got %s" % (what, t))
    return d


def _counted(n: int, what: str):
    """Refuses a count that the library's 32 bits do not hold: passed on, it would be another one."""
    if n > 0x7fffffff:
        raise EmrError(EMR_ERR_RANGE, what)


def _matrices(x, what: str):
    """x as [batch, rows, cols] on the GPU (a view)."""
    if not isinstance(x, torch.Tensor) or x.dim() not in (2, 3):
        raise ValueError("%s: a tensor of two or three dimensions is wanted" % what)
    if not x.is_cuda:
        raise ValueError("%s: a tensor on the GPU is wanted" % what)
    return x if x.dim() == 3 else x.unsqueeze(0)


_NOTHING = contextlib.nullcontext()


def _away(dev, stream):
    """What a call on tensors of the GPU `dev` has to enter before it allocates and launches, None where it is
    there: the library works on the current GPU, and allocations belong to the current stream (the caching
    allocator reuses memory by stream)."""
    if stream is None:
        return None if dev.index == torch.cuda.current_device() else torch.cuda.device(dev)
    if stream.device != dev:
        raise ValueError("stream: one of %s is wanted, where the tensors are, got one of %s" % (dev, stream.device))
    here = dev.index == torch.cuda.current_device() and stream == torch.cuda.current_stream(dev)
    return None if here else torch.cuda.stream(stream)


def _on(dev, stream):
    """The same for a with statement."""
    return _away(dev, stream) or _NOTHING


def _lend(dev, *tensors):
    """Memory that this module allocated on one stream is used by the current one: the allocator gives it to no one
    else before that work is done."""
    s = torch.cuda.current_stream(dev)
    for t in tensors:
        if t is not None:
            t.record_stream(s)


def _together(dev, *others):
    """Operands are read and written on one GPU."""
    if dev.type != "cuda" or any(x is not None and x.device != dev for x in others):
        raise ValueError("operands on one GPU are wanted, got them on %s" %
                         ", ".join(str(d) for d in [dev] + [x.device for x in others if x is not None]))


def _q8_bytes(batch: int, rows: int, cols: int):
    """(bytes of the values, bytes of the scales) of an emr_q8 (emr_q8_size)."""
    blocks = (cols + 127) // 128
    return batch * rows * blocks * 128, batch * ((rows + 127) // 128) * ((blocks + 3) // 4) * 512


class Q8:
    """Matrices [batch, rows, cols] in 8-bit floating point with one power-of-two scale for each block of
    128 columns of a row (emr_q8): values uint8 (e4m3 codes, [batch, rows, cols rounded up to 128]) and scales
    uint8 (tiles of 128 rows x 4 blocks) are parts of one piece of memory, `data`."""

    def __init__(self, batch: int, rows: int, cols: int, device="cuda"):
        n, m = C.c_size_t(), C.c_size_t()
        _check(lib().emr_q8_size(batch, rows, cols, C.byref(n), C.byref(m)), "emr_q8_size")
        self.batch, self.rows, self.cols = batch, rows, cols
        self.data = torch.empty(n.value + m.value, dtype=torch.uint8, device=device)
        p = self.data.data_ptr()
        self.c = Q8C(batch, 0, rows, cols, p, p + n.value)
        self._split = n.value

    @classmethod
    def of(cls, data, batch: int, rows: int, cols: int):
        """The matrices that `data` (uint8, values then scales) holds."""
        q = cls.__new__(cls)
        n, m = _q8_bytes(batch, rows, cols)
        if data.dtype != torch.uint8 or data.numel() < n + m or not data.is_contiguous():
            raise ValueError("data: a contiguous uint8 tensor of %d values is wanted" % (n + m))
        q.batch, q.rows, q.cols, q.data, q._split = batch, rows, cols, data, n
        q.c = Q8C(batch, 0, rows, cols, data.data_ptr(), data.data_ptr() + n)
        return q

    @property
    def values(self):
        return self.data[:self._split]

    @property
    def scales(self):
        return self.data[self._split:]

    @property
    def ref(self):
        return C.byref(self.c)

    @property
    def device(self):
        return self.data.device

    @property
    def shape(self):
        return self.batch, self.rows, self.cols


def _ref(q):
    return q.ref if q is not None else None


def q8_quantize(x, q: Q8 | None = None, qt: Q8 | None = None, stream=None):
    """emr_q8_quantize: x [batch, rows, cols] or [rows, cols], any strides, into q (blocks along the columns)
    and, or instead, qt (the transpose, blocks along the rows). With neither, a new q. Returns (q, qt)."""
    x = _matrices(x, "x")
    _together(x.device, q, qt)
    with _on(x.device, stream):
        if q is None and qt is None:
            q = Q8(*x.shape, device=x.device)
        _check(lib().emr_q8_quantize(x.data_ptr(), _dtype(x.dtype, "x"), *x.shape, *x.stride(), _ref(q), _ref(qt),
                                     _stream(stream)), "emr_q8_quantize")
    return q, qt


def q8_quantize_held(x, stream=None):
    """emr_q8_quantize_held: (q, qt) of x, qt made of the values that q holds."""
    x = _matrices(x, "x")
    with _on(x.device, stream):
        q, qt = Q8(*x.shape, device=x.device), Q8(x.shape[0], x.shape[2], x.shape[1], device=x.device)
        _check(lib().emr_q8_quantize_held(x.data_ptr(), _dtype(x.dtype, "x"), *x.shape, *x.stride(), q.ref, qt.ref,
                                          _stream(stream)), "emr_q8_quantize_held")
    return q, qt


def q8_transpose(q: Q8, qt: Q8 | None = None, stream=None) -> Q8:
    """emr_q8_transpose: the transpose of what q holds, with blocks along q's rows."""
    _together(q.device, qt)
    with _on(q.device, stream):
        if qt is None:
            qt = Q8(q.batch, q.cols, q.rows, device=q.device)
        _check(lib().emr_q8_transpose(q.ref, qt.ref, _stream(stream)), "emr_q8_transpose")
    return qt


def q8_dequantize(q: Q8, dtype=torch.float32, stream=None):
    """emr_q8_dequantize: the values that q stands for, a new [batch, rows, cols] tensor."""
    _together(q.device)
    with _on(q.device, stream):
        out = torch.empty(q.shape, dtype=dtype, device=q.device)
        _check(lib().emr_q8_dequantize(q.ref, out.data_ptr(), _dtype(dtype, "dtype"), _stream(stream)),
               "emr_q8_dequantize")
    return out


def q8_matmul(a: Q8, w: Q8, bias=None, act: int = ACT_IDENTITY, out_dtype=torch.float32, slope: Q8 | None = None,
              sum_batch: bool = False, out=None, stream=None):
    """emr_q8_matmul: act(a w^T + bias), [batch, a.rows, w.rows] ([1, ...] with sum_batch). An operand of
    batch 1 serves every batch; slope receives act'(z) in 8 bits. If a device-side wait gives up, the result is
    undefined and only device_error tells."""
    batch = max(a.batch, w.batch)
    shape = (1 if sum_batch else batch, a.rows, w.rows)
    if bias is not None and (bias.dtype != torch.float32 or not bias.is_contiguous() or
                             bias.numel() != batch * w.rows or bias.device != a.device):
        raise ValueError("bias: a contiguous float32 tensor [batch, rows of w] on the operands' GPU is wanted")
    _together(a.device, w, slope)
    with _on(a.device, stream):
        if out is None:
            out = torch.empty(shape, dtype=out_dtype, device=a.device)
        elif tuple(out.shape) != shape or not out.is_contiguous() or out.device != a.device:
            raise ValueError("out: a contiguous tensor %s is wanted" % (shape,))
        _check(lib().emr_q8_matmul(a.ref, w.ref, _ptr(bias), act, 1 if sum_batch else 0, out.data_ptr(),
                                   _dtype(out.dtype, "out"), _ref(slope), _stream(stream)), "emr_q8_matmul")
    return out


def q8_slope(dy, d: Q8 | None, dz: Q8 | None = None, dzt: Q8 | None = None, db=None, stream=None):
    """emr_q8_slope: dz = dy * d into dz and, transposed, dzt, and its column sums into db [batch, cols]."""
    dy = _matrices(dy, "dy")
    batch, rows, cols = dy.shape
    if db is not None and (db.numel() != batch * cols or not db.is_contiguous() or db.device != dy.device):
        raise ValueError("db: a contiguous tensor [batch, cols] is wanted")
    _together(dy.device, d, dz, dzt)
    n = C.c_size_t()
    with _on(dy.device, stream):
        dy, ws = dy.contiguous(), None
        if db is not None:
            _check(lib().emr_q8_slope_workspace_size(batch, rows, cols, C.byref(n)), "emr_q8_slope_workspace_size")
            ws = torch.empty(n.value, dtype=torch.uint8, device=dy.device)
        _check(lib().emr_q8_slope(dy.data_ptr(), _dtype(dy.dtype, "dy"), batch, rows, cols, _ref(d), _ref(dz),
                                  _ref(dzt), _ptr(db), _dtype(db.dtype, "db") if db is not None else 0, _ptr(ws),
                                  C.c_size_t(n.value), _stream(stream)), "emr_q8_slope")


def device_error(stream=None) -> int:
    """emr_device_error: 0, or the number of a device-side wait that gave up since the last call, on the stream's
    GPU (the current one). After a number, call again until it is 0: several kernels' waits are told one a call."""
    code = C.c_int32()
    with _on(stream.device, stream) if stream is not None else _NOTHING:
        _check(lib().emr_device_error(C.byref(code), _stream(stream)), "emr_device_error")
    return code.value


class Saved:
    """What a training step keeps between the passes, in 8 bits: xt, the transpose [nx, k, m] of x, as the weight
    gradient reads it, and slope, act'(z) [nets, m, n] (None: identity). nx, m: batch and rows of x."""

    def __init__(self, layer, nx: int, m: int, data, split: int, home: int | None = None):
        # one piece of memory: xt, then, from `split` on (0: none), slope; home: the stream that it was allocated on
        self._layer, self.nx, self.m, self._data, self._split, self._home = layer, nx, m, data, split, home

    @property
    def xt(self) -> Q8:
        return Q8.of(self._data[:self._split or None], self.nx, self._layer.k, self.m)

    @property
    def slope(self) -> Q8 | None:
        return Q8.of(self._data[self._split:], self._layer.nets, self.m, self._layer.n) if self._split else None


class DenseLayer:
    """y = act(x w^T + b) for one network, or for a batch of networks with weights of their own, in 8-bit
    floating point with 32-bit sums: a HyperNEAT substrate that connects every source to every position
    (w: outputs x sources, any strides, so the transpose of emr_eval's materialised [slots, positions] output
    is taken as it is).

    w [n, k] or [nets, n, k] (float32, bfloat16, float16), b [n] or [nets, n] float32 or None. x is [m, k],
    [1, m, k] (shared by all networks) or [nets, m, k]; results are three-dimensional. The layer keeps the
    weights in 8 bits (with train=True also their transpose, which the backward pass reads), not w itself:
    after an update of w call set_weights. A training step keeps x and act'(z) in 8 bits, 2 bytes in all for
    each pair, and takes its gradients from those and from the weights as they are laid out when backward is
    called.

    The kernels' waits on the device are bounded. None is expected to give up; if one does, the results of that
    call are undefined, no exception is raised, and device_error tells (it waits for the stream).
    """

    def __init__(self, w, b=None, act: int = ACT_IDENTITY, train: bool = False, stream=None):
        w = _matrices(w, "w")
        if not ACT_IDENTITY <= act <= ACT_ABS:
            raise ValueError("act: one of ACT_* is wanted, got %r" % (act,))
        self.nets, self.n, self.k = w.shape
        self.act, self.train, self.device = act, train, w.device
        with _on(w.device, stream):
            self.w8 = Q8(*w.shape, device=w.device)
            self.w8t = Q8(self.nets, self.k, self.n, device=w.device) if train else None
            self._home = torch._C._cuda_getCurrentRawStream(w.device.index)
        self.c = DenseC(self.w8.c, self.w8t.c if train else Q8C(), None, act, 0)
        self._ref = C.byref(self.c)
        self._room, self._kept, self._back = {}, {}, {}
        self._w8 = self.w8.ref, self.w8t.ref if train else None
        self.set_weights(w, b, stream)

    def set_weights(self, w, b=None, stream=None):
        """Lay out new weights (same shape) and keep the bias (None: no bias)."""
        w = _matrices(w, "w")
        dev = self.device
        if w.shape != (self.nets, self.n, self.k) or w.device != dev:
            raise ValueError("w: shape %s on %s is wanted" % ((self.nets, self.n, self.k), dev))
        kind = _DTYPES.get(w.dtype)
        if kind is None:
            _dtype(w.dtype, "w")
        away = _away(dev, stream)
        if away is not None:
            with away:
                return self.set_weights(w, b)
        if b is not None:
            if b.dtype != torch.float32 or b.numel() != self.nets * self.n or b.device != dev:
                raise ValueError("b: a float32 tensor [%d, %d] on the layer's GPU is wanted" % (self.nets, self.n))
            b = b.contiguous()
        q, qt = self._w8
        raw = torch._C._cuda_getCurrentRawStream(dev.index)
        if raw != self._home:
            _lend(dev, self.w8.data, self.w8t.data if qt else None)
        _check(lib().emr_q8_quantize(w.data_ptr(), kind, self.nets, self.n, self.k, *w.stride(), q, qt, raw), "emr_q8_quantize")
        self.b = b
        self.c.bias = b.data_ptr() if b is not None else None

    def _needs_room(self, nx, m):
        """Bytes that a forward pass without keep needs for x in 8 bits (emr_dense_forward_room)."""
        got = self._room.get((nx, m))
        if got is None:
            a, b, c = C.c_size_t(), C.c_size_t(), C.c_size_t()
            _check(lib().emr_dense_forward_room(self._ref, nx, m, 0, C.byref(a), C.byref(b), C.byref(c)),
                   "emr_dense_forward_room")
            if len(self._room) > 64:
                self._room.clear()
            got = self._room[(nx, m)] = a.value
        return got

    def _kept_bytes(self, nx, m):
        """Bytes of x in 8 bits, of its transpose and of the slopes (0: identity) in a training step."""
        got = self._kept.get((nx, m))
        if got is None:
            if len(self._kept) > 64:
                self._kept.clear()
            slope = sum(_q8_bytes(self.nets, m, self.n)) if self.act != ACT_IDENTITY else 0
            got = self._kept[(nx, m)] = sum(_q8_bytes(nx, m, self.k)), sum(_q8_bytes(nx, self.k, m)), slope
        return got

    def _forward(self, x, out_dtype, stream, keep):
        x = _matrices(x, "x")
        nx, m, k = x.shape
        dev = self.device
        if k != self.k or (nx != 1 and nx != self.nets) or x.device != dev:
            raise ValueError("x: [m, %d], [1, m, %d] or [%d, m, %d] on the layer's GPU is wanted, got %s" %
                             (self.k, self.k, self.nets, self.k, tuple(x.shape)))
        kind, out_kind = _DTYPES.get(x.dtype), _DTYPES.get(out_dtype)
        if kind is None or out_kind is None:
            _dtype(x.dtype, "x"), _dtype(out_dtype, "out_dtype")
        if m == 0:
            if keep:
                raise ValueError("x: at least one row is wanted for training")
            return torch.empty(self.nets, 0, self.n, dtype=out_dtype, device=dev), None, 0, None
        away = _away(dev, stream)
        if away is not None:
            with away:
                return self._forward(x, out_dtype, None, keep)
        out = torch.empty((self.nets, m, self.n), dtype=out_dtype, device=dev)
        kept = xp = tp = sp = None
        split = 0
        if keep:
            room, xt_bytes, slope_bytes = self._kept_bytes(nx, m)
            kept = torch.empty(xt_bytes + slope_bytes, dtype=torch.uint8, device=dev)
            tp = kept.data_ptr()
            if slope_bytes:
                split, sp = xt_bytes, tp + xt_bytes
        else:
            room = self._needs_room(nx, m)
        if room:
            xq = torch.empty(room, dtype=torch.uint8, device=dev)
            xp = xq.data_ptr()
        raw = torch._C._cuda_getCurrentRawStream(dev.index)
        if raw != self._home:
            _lend(dev, self.w8.data, self.b)
        status = _lib.emr_dense_forward(self._ref, x.data_ptr(), kind, nx, m, *x.stride(), out.data_ptr(), out_kind,
                                        1 if keep else 0, xp, tp, sp, raw)
        if status:
            _check(status, "emr_dense_forward")
        return out, kept, split, raw

    def forward(self, x, out_dtype=torch.float32, stream=None):
        """y [nets, m, n] of out_dtype. m = 0 gives an empty result."""
        return self._forward(x, out_dtype, stream, False)[0]

    def forward_train(self, x, out_dtype=torch.float32, stream=None):
        """(y, saved): saved holds x and act'(z) in 8 bits for backward."""
        if not self.train:
            raise ValueError("forward_train: the layer was made with train=False")
        y, kept, split, home = self._forward(x, out_dtype, stream, True)
        return y, Saved(self, x.shape[0] if x.dim() == 3 else 1, y.shape[1], kept, split, home)

    def backward(self, dy, saved: Saved, out_dtype=torch.float32, stream=None):
        """(dx, dw, db) of out_dtype for dy [nets, m, n]: dx [1 or nets, m, k] as forward_train took x (summed
        over the networks where x was shared), dw [nets, n, k], db [nets, n] (also without a bias)."""
        dy = _matrices(dy, "dy")
        nx, m, dev = saved.nx, saved.m, self.device
        if dy.shape != (self.nets, m, self.n) or dy.device != dev:
            raise ValueError("dy: shape %s on %s is wanted, got %s" % ((self.nets, m, self.n), dev, tuple(dy.shape)))
        if saved._layer is not self:
            raise ValueError("saved: of another layer")
        kind, out_kind = _DTYPES.get(dy.dtype), _DTYPES.get(out_dtype)
        if kind is None or out_kind is None:
            _dtype(dy.dtype, "dy"), _dtype(out_dtype, "out_dtype")
        away = _away(dev, stream)
        if away is not None:
            with away:
                return self.backward(dy, saved, out_dtype)
        dy = dy.contiguous()
        room = self._back.get((nx, m))
        if room is None:
            n = C.c_size_t()
            _check(_lib.emr_dense_backward_room(self._ref, nx, m, C.byref(n)), "emr_dense_backward_room")
            if len(self._back) > 64:
                self._back.clear()
            room = self._back[(nx, m)] = n.value
        dx = torch.empty((nx, m, self.k), dtype=out_dtype, device=dev)
        dw = torch.empty((self.nets, self.n, self.k), dtype=out_dtype, device=dev)
        db = torch.empty((self.nets, self.n), dtype=out_dtype, device=dev)
        ws = torch.empty(room, dtype=torch.uint8, device=dev)
        kept, split = saved._data.data_ptr(), saved._split
        raw = torch._C._cuda_getCurrentRawStream(dev.index)
        if raw != saved._home:
            _lend(dev, saved._data)
        if raw != self._home:
            _lend(dev, self.w8t.data)
        status = _lib.emr_dense_backward(self._ref, dy.data_ptr(), kind, nx, m, kept, kept + split if split else None,
                                         dx.data_ptr(), dw.data_ptr(), db.data_ptr(), out_kind, ws.data_ptr(), room, raw)
        if status:
            _check(status, "emr_dense_backward")
        return dx, dw, db


# ---- sampling from scores -------------------------------------------------------------------

def _per_row(v, rows: int, dtype, device, what: str):
    """Address of a device array of a parameter given for each row."""
    _check_per_row(v, rows, dtype, device, what)
    return v.data_ptr()


def _check_per_row(v, rows: int, dtype, device, what: str):
    if v.shape != (rows,) or v.dtype != dtype or v.device != device or not v.is_contiguous():
        raise ValueError("%s: a number or a contiguous %s tensor [%d] on the scores' GPU is wanted" % (what, dtype, rows))


def sample(scores, noise, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, stream=None):
    """emr_sample: one index for each row of scores [rows, n] (or [n]; float32, bfloat16, float16), drawn with
    the given Exp(1) noise (float32, same shape). Parameters are numbers, or tensors [rows] (float32; top_k
    int32). Returns (index int32 [rows], log probability float32 [rows])."""
    if not isinstance(scores, torch.Tensor) or scores.dim() not in (1, 2) or not scores.is_cuda:
        raise ValueError("scores: a tensor [rows, n] or [n] on the GPU is wanted")
    dev = scores.device
    if noise.shape != scores.shape or noise.dtype is not torch.float32 or noise.device != dev:
        raise ValueError("noise: a float32 tensor in the shape of scores on the same GPU is wanted")
    away = _away(dev, stream)
    if away is not None:
        with away:
            return sample(scores, noise, temperature, top_k, top_p, min_p)
    if scores.dim() == 1:
        scores, noise = scores.unsqueeze(0), noise.unsqueeze(0)
    rows, n = scores.shape
    _counted(rows, "rows")
    kind = _DTYPES.get(scores.dtype)
    if kind is None:
        _dtype(scores.dtype, "scores")
    tp = kp = pp = qp = None
    if isinstance(temperature, torch.Tensor):
        tp, temperature = _per_row(temperature, rows, torch.float32, dev, "temperature"), 0.0
    if isinstance(top_k, torch.Tensor):
        kp, top_k = _per_row(top_k, rows, torch.int32, dev, "top_k"), 0
    if isinstance(top_p, torch.Tensor):
        pp, top_p = _per_row(top_p, rows, torch.float32, dev, "top_p"), 0.0
    if isinstance(min_p, torch.Tensor):
        qp, min_p = _per_row(min_p, rows, torch.float32, dev, "min_p"), 0.0
    s_row, s_col = scores.stride()
    e_row, e_col = noise.stride()
    if s_col != 1:
        scores = scores.contiguous()
        s_row = n
    if e_col != 1:
        noise = noise.contiguous()
        e_row = n
    index = torch.empty(rows, dtype=torch.int32, device=dev)
    logp = torch.empty(rows, dtype=torch.float32, device=dev)
    if rows:
        status = lib().emr_sample(scores.data_ptr(), kind, rows, n, s_row, noise.data_ptr(), e_row, tp, temperature, kp,
                                  top_k, pp, top_p, qp, min_p, index.data_ptr(), logp.data_ptr(),
                                  torch._C._cuda_getCurrentRawStream(dev.index))
        if status:
            _check(status, "emr_sample")
    return index, logp


# ---- products with 4-bit weights ---------------------------------------------------------------

class Q4C(C.Structure):
    _fields_ = [("batch", C.c_int32), ("group", C.c_int32), ("rows", C.c_int64), ("cols", C.c_int64), ("data", C.c_void_p)]


class Q4:
    """Matrices [batch, rows, cols] of 4-bit codes (-8 to 7) with one bfloat16 scale for each `group` (32, 64 or 128) columns of a
    row (emr_q4), in one piece of memory, `data` (uint8): what a layer that only answers keeps of its weights."""

    def __init__(self, batch: int, rows: int, cols: int, group: int = 32, device="cuda", data=None):
        _counted(batch, "batch")
        n = C.c_size_t()
        _check(lib().emr_q4_size(batch, rows, cols, group, C.byref(n)), "emr_q4_size")
        if data is None:
            data = torch.empty(n.value, dtype=torch.uint8, device=device)
        elif data.dtype != torch.uint8 or data.numel() < n.value or not data.is_contiguous():
            raise ValueError("data: a contiguous uint8 tensor of %d values is wanted" % n.value)
        self.batch, self.rows, self.cols, self.group, self.data = batch, rows, cols, group, data
        self.c = Q4C(batch, group, rows, cols, data.data_ptr())
        self.ref = C.byref(self.c)
        self._home = None  # the stream that this module allocated data on

    @classmethod
    def of(cls, data, batch: int, rows: int, cols: int, group: int = 32):
        """The matrices that `data` (uint8, as another Q4's) holds."""
        return cls(batch, rows, cols, group, data=data)

    @property
    def device(self):
        return self.data.device

    @property
    def shape(self):
        return self.batch, self.rows, self.cols


def _new_q4(shape, group: int, dev) -> Q4:
    if group not in (32, 64, 128):
        raise ValueError("group: 32, 64 or 128 is wanted, got %r" % (group,))
    q = Q4(*shape, group, device=dev)
    q._home = torch._C._cuda_getCurrentRawStream(dev.index)
    return q


def q4_quantize(w, group: int = 32, stream=None) -> Q4:
    """emr_q4_quantize: w [batch, rows, cols] or [rows, cols] (float32, bfloat16, float16; any strides) in 4 bits."""
    w = _matrices(w, "w")
    kind = _dtype(w.dtype, "w")
    with _on(w.device, stream):
        q = _new_q4(w.shape, group, w.device)
        _check(lib().emr_q4_quantize(w.data_ptr(), kind, *w.stride(), q.ref, _stream(stream)), "emr_q4_quantize")
    return q


def q4_pack(codes, scales, group: int = 32, stream=None) -> Q4:
    """emr_q4_pack: given codes (int8 -8 to 7, [batch, rows, cols] or [rows, cols]) and scales (bfloat16, [..., rows, cols / group
    rounded up]) as a Q4."""
    codes, scales = _matrices(codes, "codes"), _matrices(scales, "scales")
    batch, rows, cols = codes.shape
    if group not in (32, 64, 128):
        raise ValueError("group: 32, 64 or 128 is wanted, got %r" % (group,))
    if codes.dtype != torch.int8:
        raise ValueError("codes: int8 is wanted, got %s" % codes.dtype)
    if scales.dtype != torch.bfloat16 or scales.shape != (batch, rows, (cols + group - 1) // group):
        raise ValueError("scales: a bfloat16 tensor %s is wanted" % ((batch, rows, (cols + group - 1) // group),))
    _together(codes.device, scales)
    with _on(codes.device, stream):
        q = _new_q4(codes.shape, group, codes.device)
        _check(lib().emr_q4_pack(codes.data_ptr(), *codes.stride(), scales.data_ptr(), *scales.stride(), q.ref, _stream(stream)),
               "emr_q4_pack")
    return q


def q4_dequantize(q: Q4, dtype=torch.float32, stream=None):
    """emr_q4_dequantize: the values that q stands for, a new [batch, rows, cols] tensor."""
    _together(q.device)
    kind = _dtype(dtype, "dtype")
    with _on(q.device, stream):
        raw = torch._C._cuda_getCurrentRawStream(q.device.index)
        if q._home is not None and raw != q._home:
            _lend(q.device, q.data)
        out = torch.empty(q.shape, dtype=dtype, device=q.device)
        _check(lib().emr_q4_dequantize(q.ref, out.data_ptr(), kind, raw), "emr_q4_dequantize")
    return out


def q4_matmul(x, w: Q4, bias=None, act: int = ACT_IDENTITY, out_dtype=torch.float32, out=None, stream=None):
    """emr_q4_matmul: act(x w^T + bias), [batch, m, w.rows], for x [batch, m, cols], [1, m, cols] or [m, cols] (float32, bfloat16,
    float16; any strides). An operand of batch 1 serves every batch. bias: float32 [batch, w.rows] or None. Made for the few rows
    that a layer answers at a time. m = 0 gives an empty result."""
    x = _matrices(x, "x")
    nx, m, k = x.shape
    dev = x.device
    if k != w.cols or (nx != 1 and w.batch != 1 and nx != w.batch) or nx < 1:
        raise ValueError("x: [m, %d], [1, m, %d] or [%d, m, %d] is wanted, got %s" % (w.cols, w.cols, w.batch, w.cols, tuple(x.shape)))
    batch = max(nx, w.batch)
    _counted(nx, "batch")
    kind = _DTYPES.get(x.dtype)
    if kind is None:
        _dtype(x.dtype, "x")
    if not ACT_IDENTITY <= act <= ACT_ABS:
        raise ValueError("act: one of ACT_* is wanted, got %r" % (act,))
    if bias is not None and (bias.dtype != torch.float32 or not bias.is_contiguous() or bias.numel() != batch * w.rows or
                             bias.device != dev):
        raise ValueError("bias: a contiguous float32 tensor [%d, %d] on the operands' GPU is wanted" % (batch, w.rows))
    if w.data.device != dev:
        _together(dev, w)
    shape = (batch, m, w.rows)
    if out is not None and (tuple(out.shape) != shape or not out.is_contiguous() or out.device != dev):
        raise ValueError("out: a contiguous tensor %s is wanted" % (shape,))
    out_kind = _dtype(out_dtype if out is None else out.dtype, "out")
    away = _away(dev, stream)
    if away is not None:
        with away:
            return q4_matmul(x, w, bias, act, out_dtype, out)
    if out is None:
        out = torch.empty(shape, dtype=out_dtype, device=dev)
    if m:
        raw = torch._C._cuda_getCurrentRawStream(dev.index)
        if w._home is not None and raw != w._home:
            _lend(dev, w.data)
        L, x_args, ws, room = lib(), (x.data_ptr(), kind, nx, m, *x.stride(), w.ref), None, 0
        if m > 8:
            n = C.c_size_t()
            _check(L.emr_q4_matmul_room(*x_args, C.byref(n)), "emr_q4_matmul_room")
            room = n.value
            if room:
                ws = torch.empty(room, dtype=torch.uint8, device=dev)
        status = L.emr_q4_matmul(*x_args, bias.data_ptr() if bias is not None else None, act, out.data_ptr(), out_kind,
                                 ws.data_ptr() if room else None, room, raw)
        if status:
            _check(status, "emr_q4_matmul")
    return out


# ---- log probabilities of answers ------------------------------------------------------------

MAX_TOP = 256


@dataclass
class LogProbs:
    """What log_probs gives, tensors [rows] and [rows, top]; None for what was not asked for."""
    logp: torch.Tensor | None
    entropy: torch.Tensor
    top_index: torch.Tensor | None
    top_logp: torch.Tensor | None


def _scores(scores):
    """(rows, n, row stride, emr_dtype) of scores [rows, n] or [n]; the stride is None where columns are no neighbours and a
    copy is wanted."""
    if not isinstance(scores, torch.Tensor) or not scores.is_cuda:
        raise ValueError("scores: a tensor [rows, n] or [n] on the GPU is wanted")
    shape = scores.shape
    if len(shape) == 2:
        rows, n = shape
        stride, col = scores.stride()
    elif len(shape) == 1:
        rows, n = 1, shape[0]
        stride, col = n, scores.stride(0)
    else:
        raise ValueError("scores: a tensor [rows, n] or [n] on the GPU is wanted")
    if n < 1:
        raise ValueError("scores: rows of at least one entry are wanted")
    _counted(rows, "rows")
    kind = _DTYPES.get(scores.dtype)
    if kind is None:
        _dtype(scores.dtype, "scores")
    return rows, n, stride if col == 1 or n == 1 else None, kind


def _check_number_or_rows(v, rows: int, dev, what: str):
    if type(v) is not float and isinstance(v, torch.Tensor):
        _check_per_row(v, rows, torch.float32, dev, what)


def _number_or_rows(v):
    """(address, number) of a float parameter that is given for each row or for all."""
    return (None, v) if type(v) is float else (v.data_ptr(), 0.0) if isinstance(v, torch.Tensor) else (None, float(v))


def _check_targets(targets, rows: int, dev):
    if not isinstance(targets, torch.Tensor):
        raise ValueError("targets: an int32 tensor [%d] on the scores' GPU is wanted" % rows)
    _check_per_row(targets, rows, torch.int32, dev, "targets")


def log_probs(scores, targets=None, temperature=1.0, top=0, stream=None) -> LogProbs:
    """emr_log_probs: log probabilities of the answers targets (int32 [rows], below 0: none) under scores [rows, n] (or [n];
    float32, bfloat16, float16), the rows' entropies, and the `top` (up to MAX_TOP) best answers of each row with
    theirs. temperature: a number, or a float32 tensor [rows]."""
    rows, n, stride, kind = _scores(scores)
    dev = scores.device
    if not 0 <= top <= MAX_TOP:
        raise ValueError("top: 0 to %d is wanted, got %r" % (MAX_TOP, top))
    if targets is not None:
        _check_targets(targets, rows, dev)
    _check_number_or_rows(temperature, rows, dev, "temperature")
    away = _away(dev, stream)
    if away is not None:
        with away:
            return log_probs(scores, targets, temperature, top)
    if stride is None:
        scores, stride = scores.contiguous(), n
    entropy = torch.empty(rows, dtype=torch.float32, device=dev)
    logp = index = best = tp = lp = ip = bp = None
    if targets is not None:
        logp = torch.empty_like(entropy)
        tp, lp = targets.data_ptr(), logp.data_ptr()
    if top:
        best = torch.empty((rows, top), dtype=torch.float32, device=dev)
        index = torch.empty_like(best, dtype=torch.int32)
        ip, bp = index.data_ptr(), best.data_ptr()
    if rows:
        hp, heat = _number_or_rows(temperature)
        status = lib().emr_log_probs(scores.data_ptr(), kind, rows, n, stride, tp, hp, heat, top, lp, entropy.data_ptr(), ip, bp,
                                     torch._C._cuda_getCurrentRawStream(dev.index))
        if status:
            _check(status, "emr_log_probs")
    return LogProbs(logp, entropy, index, best)


def log_probs_grad(scores, targets, dlogp, dentropy=None, temperature=1.0, out_dtype=None, stream=None):
    """emr_log_probs_grad: (dscores, logp, entropy), the gradient of sum(dlogp logp + dentropy entropy) in the shape of scores,
    of out_dtype (None: the scores' type), with the values that log_probs gives. dlogp and dentropy: numbers, or float32
    tensors [rows]; dentropy None: 0. The loss of a step of cross entropy is -logp with dlogp = -1 / rows."""
    rows, n, stride, kind = _scores(scores)
    dev, shape = scores.device, scores.shape
    _check_targets(targets, rows, dev)
    _check_number_or_rows(dlogp, rows, dev, "dlogp")
    if dentropy is None:
        dentropy = 0.0
    _check_number_or_rows(dentropy, rows, dev, "dentropy")
    _check_number_or_rows(temperature, rows, dev, "temperature")
    out_kind = _dtype(scores.dtype if out_dtype is None else out_dtype, "out_dtype")
    away = _away(dev, stream)
    if away is not None:
        with away:
            return log_probs_grad(scores, targets, dlogp, dentropy, temperature, out_dtype)
    if stride is None:
        scores, stride = scores.contiguous(), n
    dscores = torch.empty(shape, dtype=out_dtype or scores.dtype, device=dev)
    logp = torch.empty(rows, dtype=torch.float32, device=dev)
    entropy = torch.empty_like(logp)
    if rows:
        status = lib().emr_log_probs_grad(scores.data_ptr(), kind, rows, n, stride, targets.data_ptr(), *_number_or_rows(temperature),
                                          *_number_or_rows(dlogp), *_number_or_rows(dentropy), logp.data_ptr(), entropy.data_ptr(),
                                          dscores.data_ptr(), out_kind, n, torch._C._cuda_getCurrentRawStream(dev.index))
        if status:
            _check(status, "emr_log_probs_grad")
    return dscores, logp, entropy


# ---- distillation ------------------------------------------------------------------------------

def _distill(scores, index, logp, dloss, temperature, tail, out_dtype, stream):
    rows, n, stride, kind = _scores(scores)
    dev, shape = scores.device, scores.shape
    if not isinstance(index, torch.Tensor) or index.dtype is not torch.int32 or index.dim() != 2 or index.shape[0] != rows or \
            index.device != dev or not 1 <= index.shape[1] <= MAX_TOP:
        raise ValueError("index: an int32 tensor [%d, 1 to %d] on the scores' GPU is wanted" % (rows, MAX_TOP))
    if not isinstance(logp, torch.Tensor) or logp.shape != index.shape or logp.device != dev:
        raise ValueError("logp: a tensor in the shape of index on the scores' GPU is wanted")
    k, t_kind = index.shape[1], _dtype(logp.dtype, "logp")
    _check_number_or_rows(temperature, rows, dev, "temperature")
    if not isinstance(temperature, torch.Tensor) and not temperature > 0:
        raise ValueError("temperature: a number above 0 is wanted, got %r" % (temperature,))
    grad = dloss is not None
    if grad:
        _check_number_or_rows(dloss, rows, dev, "dloss")
    out_kind = _dtype(scores.dtype if out_dtype is None else out_dtype, "out_dtype") if grad else 0
    away = _away(dev, stream)
    if away is not None:
        with away:
            return _distill(scores, index, logp, dloss, temperature, tail, out_dtype, None)
    if stride is None:
        scores, stride = scores.contiguous(), n
    index, logp = index.contiguous(), logp.contiguous()
    dscores = torch.empty(shape, dtype=out_dtype or scores.dtype, device=dev) if grad else None
    loss = torch.empty(rows, dtype=torch.float32, device=dev)
    if rows:
        status = lib().emr_distill(scores.data_ptr(), kind, rows, n, stride, index.data_ptr(), logp.data_ptr(), t_kind, k,
                                   *_number_or_rows(temperature), 1 if tail else 0, *_number_or_rows(dloss if grad else 0.0), loss.data_ptr(), dscores.data_ptr() if grad else None, out_kind, n,
                                   torch._C._cuda_getCurrentRawStream(dev.index))
        if status:
            _check(status, "emr_distill")
    return dscores, loss


def distill(scores, index, logp, temperature=1.0, tail=True, stream=None):
    """emr_distill: the loss [rows] of scores [rows, n] (or [n]; float32, bfloat16, float16) against a teacher's best answers,
    as log_probs(teacher's scores, top=k) gives them: index int32 [rows, k] (below 0: none) and logp [rows, k] (float32,
    bfloat16, float16), log probabilities at the student's temperature. tail: what they leave over counts as one more answer; without it the teacher is
    softmax(logp) over them. temperature: a number above 0, or a float32 tensor [rows]."""
    return _distill(scores, index, logp, None, temperature, tail, None, stream)[1]


def distill_grad(scores, index, logp, dloss, temperature=1.0, tail=True, out_dtype=None, stream=None):
    """emr_distill: (dscores, loss), the gradient of sum(dloss loss) in the shape of scores, of out_dtype (None: the scores' type), with
    the loss that distill gives, in one pass. dloss: a number, or a float32 tensor [rows]."""
    if dloss is None:
        raise ValueError("dloss: a number or a float32 tensor [rows] is wanted")
    return _distill(scores, index, logp, dloss, temperature, tail, out_dtype, stream)


# ---- ALU probes (roofline denominators) -------------------------------------------------

PROBE_FFMA, PROBE_EX2, PROBE_RCP, PROBE_SIN = range(4)


def probe_alu(op: int, blocks: int, iters: int, stream=None):
    """(operations, milliseconds) of one probe launch (include/emr_probe.h)."""
    sink = torch.zeros(blocks, dtype=torch.float32, device="cuda")
    ops, ms = C.c_double(), C.c_float()
    _check(lib().emr_probe_alu(op, blocks, iters, C.byref(ops), C.byref(ms), _ptr(sink), _stream(stream)),
           "emr_probe_alu")
    return ops.value, ms.value


# ---- convenience: the whole path on caller-visible buffers --------------------------

class Discovery:
    """Buffers and calls for one (population, query, depth) configuration.

    run_fused(): CPPN outputs never materialised; the kept weights are recomputed at compaction
    (or, with sparse_out=True, written by the fused kernel where the band test passed).
    run_unfused(): CPPN outputs materialised, then filtered.
    """

    def __init__(self, pop, sources, D: int, theta: float, band: float, w_min: float = 0.0,
                 mode: int = EMR_EAGER, cap: int | None = None, materialise: bool = False, device="cuda",
                 types: int = CONN_ALL):
        self.device = torch.device(device)
        self.pack = pack_population(pop)
        self.pack_dev = torch.from_numpy(self.pack).to(self.device)
        self.query = make_query(sources, self.device)
        self.grid = grid_build(D)
        self.P, self.S = pop.P, self.query.S
        self.n_pairs = self.P * self.S
        self.theta, self.band, self.w_min, self.mode, self.types = theta, band, w_min, mode, types
        g = self.grid
        u32 = dict(dtype=torch.int32, device=self.device)
        self.mask = torch.zeros(self.n_pairs, g.n_words, **u32)
        self.split = torch.zeros(self.n_pairs, g.n_words, **u32)
        self.band_bits = torch.zeros(self.n_pairs, g.n_words, **u32)
        self.out = (torch.zeros(self.n_pairs, g.n_total, dtype=torch.float32, device=self.device)
                    if materialise else None)
        self.out_halo = (torch.zeros(self.n_pairs, g.n_halo, dtype=torch.float32, device=self.device)
                         if materialise else None)
        self.var_dbg = None
        self.ws = torch.zeros(eval_workspace_size(self.pack, self.query), dtype=torch.uint8, device=self.device)
        self.cws = torch.zeros(compact_workspace_size(g, self.n_pairs), dtype=torch.uint8, device=self.device)
        self.cap = int(cap if cap is not None else min(self.n_pairs * g.n_total, 1 << 27))
        self.idx = torch.zeros(self.cap, dtype=torch.int32, device=self.device)
        self.w = torch.zeros(self.cap, dtype=torch.float32, device=self.device)
        self.counts = torch.zeros(self.n_pairs, dtype=torch.int64, device=self.device)
        self.offsets = torch.zeros(self.n_pairs + 1, dtype=torch.int64, device=self.device)

    def prepare(self, stream=None):
        eval_prepare(self.pack, self.pack_dev, self.query, self.ws, stream)

    def _materialise(self):
        if self.out is None:
            self.out = torch.zeros(self.n_pairs, self.grid.n_total, dtype=torch.float32, device=self.device)
        if self.out_halo is None:
            self.out_halo = torch.zeros(self.n_pairs, self.grid.n_halo, dtype=torch.float32, device=self.device)

    def run_fused(self, sparse_out: bool = False, stream=None):
        """emr_eval_prepare, emr_eval_filter, emr_mask_combine, emr_compact_records
        (sparse_out: emr_eval_filter writes band-passing outputs, emr_compact reads them)."""
        self.prepare(stream)
        if sparse_out:
            self._materialise()
        eval_filter(self.pack, self.query, self.grid, self.theta, self.band, self.w_min, self.split,
                    self.band_bits, self.out if sparse_out else None, self.ws, stream)
        self.combine(stream)
        if sparse_out:
            compact(self.mask, self.out, self.grid, self.n_pairs, self.idx, self.w, self.cap, self.counts,
                    self.offsets, self.cws, stream)
        else:
            compact_records(self.mask, self.pack, self.query, self.ws, self.grid, self.idx, self.w, self.cap,
                            self.counts, self.offsets, self.cws, stream)

    def run_select(self, stream=None):
        """emr_eval_prepare, emr_eval_filter_tiles, emr_select (no mask plane)."""
        if getattr(self, "tile_flags", None) is None:
            self.tile_flags = torch.zeros(self.n_pairs, dense_tiles(self.grid.D), dtype=torch.uint8,
                                          device=self.device)
            self.sws = torch.zeros(select_workspace_size(self.grid, self.n_pairs), dtype=torch.uint8,
                                   device=self.device)
        self.prepare(stream)
        eval_filter_tiles(self.pack, self.query, self.grid, self.theta, self.band, self.w_min, self.split,
                          self.band_bits, self.tile_flags, self.ws, stream)
        select(self.split, self.band_bits, self.tile_flags, self.pack, self.query, self.ws, self.grid, self.mode,
               self.types, self.idx, self.w, self.cap, self.counts, self.offsets, self.sws, stream)

    def run_discover(self, stream=None):
        """emr_discover: the whole path in one call on its own workspace."""
        if getattr(self, "dws", None) is None:
            self.dws = torch.zeros(discover_workspace_size(self.pack, self.query, self.grid), dtype=torch.uint8,
                                   device=self.device)
        discover(self.pack, self.pack_dev, self.query, self.grid, self.theta, self.band, self.w_min, self.mode,
                 self.types, self.dws, self.idx, self.w, self.cap, self.counts, self.offsets, stream)

    def combine(self, stream=None):
        """emr_mask_combine, or emr_mask_combine_types when a connection-type filter is set."""
        if self.types == CONN_ALL:
            mask_combine(self.split, self.band_bits, self.grid, self.n_pairs, self.mode, self.mask, stream)
        else:
            mask_combine_types(self.split, self.band_bits, self.query, self.grid, self.n_pairs, self.mode,
                               self.types, self.mask, stream)

    def conn_types(self, stream=None):
        """Type codes of the current lists (device uint8 tensor of cap entries)."""
        t = torch.zeros(self.cap, dtype=torch.uint8, device=self.device)
        conn_types(self.idx, self.offsets, self.query, self.grid, self.n_pairs, self.cap, t, stream)
        return t

    def run_unfused(self, with_var: bool = False, stream=None):
        """emr_eval_prepare, emr_eval, emr_variance_filter, emr_compact."""
        self._materialise()
        if with_var and self.var_dbg is None:
            self.var_dbg = torch.zeros(self.n_pairs, self.grid.n_total, dtype=torch.float32, device=self.device)
        self.prepare(stream)
        eval(self.pack, self.query, self.grid, self.out, self.out_halo, self.ws, stream)
        variance_filter(self.out, self.out_halo, self.grid, self.P, self.S, self.theta, self.band, self.w_min,
                        self.mode, self.mask, self.split, self.band_bits, self.var_dbg if with_var else None,
                        stream)
        if self.types != CONN_ALL:
            self.combine(stream)
        compact(self.mask, self.out, self.grid, self.n_pairs, self.idx, self.w, self.cap, self.counts,
                self.offsets, self.cws, stream)

    def lists(self):
        """Host copies: per pair (idx, w) arrays, ascending global index."""
        off = self.offsets.cpu().numpy()
        total = int(off[-1])
        if total > self.cap:
            raise EmrError(EMR_ERR_CAPACITY, "compaction capacity %d < %d" % (self.cap, total))
        idx = self.idx[:total].cpu().numpy()
        w = self.w[:total].cpu().numpy()
        return [(idx[off[r]:off[r + 1]], w[off[r]:off[r + 1]]) for r in range(self.n_pairs)]


# ---- inspection of a packed blob (layout of csrc/emr_internal.h) ----------------------

_HDR = np.dtype([("magic", "<u4"), ("version", "<u4"), ("P", "<i4"), ("max_nodes", "<i4"),
                 ("max_varying", "<i4", 2), ("max_vedges", "<i4", 2), ("max_edges", "<i4"), ("reserved", "<i4"),
                 ("off_genomes", "<u8"), ("off_nodes", "<u8"), ("off_edges", "<u8"), ("total", "<u8")])
_GEN = np.dtype([("node_beg", "<u4"), ("edge_beg", "<u4"), ("n_nodes", "<u2"), ("n_edges", "<u2"),
                 ("n_varying", "<u2", 2), ("n_vedges", "<u2", 2), ("cost", "<u4", 2), ("n_joint", "<u2", 2)])
_NODE = np.dtype([("act", "u1"), ("vary", "u1"), ("axes", "u1"), ("reserved", "u1"), ("edge_beg", "<u2"), ("edge_cnt", "<u2"),
                  ("bias", "<f4"), ("w_in", "<f4", 5)])
_EDGE = np.dtype([("src", "<u2"), ("reserved", "<u2"), ("w", "<f4")])


def pack_records(pack: np.ndarray):
    """(header, genome table, node records, edge records) of a packed blob, as numpy views. The node
    and edge arrays are the blob's whole sections: genome g's records start at its node_beg and
    edge_beg (the slots past its n_nodes and n_edges are zero)."""
    raw = np.ascontiguousarray(pack).tobytes()
    h = np.frombuffer(raw[:_HDR.itemsize], _HDR)[0]
    P = int(h["P"])
    gs = np.frombuffer(raw, _GEN, P, int(h["off_genomes"]))
    nn = (int(h["off_edges"]) - int(h["off_nodes"])) // _NODE.itemsize
    ne = (int(h["total"]) - int(h["off_edges"])) // _EDGE.itemsize
    return h, gs, np.frombuffer(raw, _NODE, nn, int(h["off_nodes"])), np.frombuffer(raw, _EDGE, ne,
                                                                                    int(h["off_edges"]))
