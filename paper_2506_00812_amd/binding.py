"""Thin Python binding of the C ABI in ``include/vecflow.h``.

Argument marshalling only: every step of the search path runs in the HIP
library.  PyTorch supplies device memory (tensors) and the current HIP stream.
There is no CPU fallback: if ``libvecflow.so`` is missing, loading fails loudly.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
import struct

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libvecflow.so")

VF_U8, VF_F32, VF_BF16, VF_F16 = 0, 1, 2, 3
ARR = dict(S=0, O_HS=1, O_LS=2, M_HS=3, M_LS=4, G_HS=5, GO_LS=6, X_LS=7, BITSET=8)
_ARR_DTYPE = dict(S=np.int64, O_HS=np.int64, O_LS=np.int64, M_HS=np.int32, M_LS=np.int32, G_HS=np.int32,
                  GO_LS=np.int64, X_LS=np.uint8, BITSET=np.uint32)

EXPORTED_SYMBOLS = ("vf_build_index", "vf_search", "vf_search_exact", "vf_index_export", "vf_index_stats",
                    "vf_index_free", "vf_last_error", "vf_profile_enable", "vf_profile_read", "vf_search_multi",
                    "vf_build_index_opt", "vf_tune", "vf_debug_route", "vf_search_noalloc", "vf_serve_begin", "vf_serve_submit",
                    "vf_serve_poll", "vf_serve_end", "vf_serve_run", "vf_search_ex",
                    "vf_linear", "vf_linear_backward", "vf_linear_workspace", "vf_debug_linear", "vf_layer_norm", "vf_layer_norm_backward",
                    "vf_layer_norm_workspace", "vf_log_probs", "vf_log_probs_backward", "vf_log_probs_workspace",
                    "vf_adamw_step", "vf_adamw_moments")

ALLOC_FN = C.CFUNCTYPE(C.c_void_p, C.c_size_t, C.c_void_p)
FREE_FN = C.CFUNCTYPE(None, C.c_void_p, C.c_void_p)


class VfAllocator(C.Structure):
    _fields_ = [("alloc", ALLOC_FN), ("free", FREE_FN), ("ctx", C.c_void_p)]


class VfStats(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("n", "n_HS", "n_LS", "n_groups_LS")] + \
               [(n, C.c_int32) for n in ("dim", "dtype", "n_labels", "T", "graph_degree", "n_graph_labels",
                                         "n_scan_labels", "chunks_per_vector")] + \
               [(n, C.c_int64) for n in ("bytes_graph", "bytes_maps", "bytes_x_ls", "bytes_bitsets", "bytes_meta",
                                         "bytes_total", "bytes_x_ls_bf16")]


class VfProfile(C.Structure):
    _fields_ = [("scan_ms", C.c_float), ("seed_ms", C.c_float), ("beam_ms", C.c_float), ("scan_ms_sum", C.c_double),
                ("seed_ms_sum", C.c_double), ("beam_ms_sum", C.c_double), ("calls", C.c_int64)] + \
               [(n, C.c_int64) for n in ("nq", "n_scan_queries", "n_graph_queries", "n_scan_items",
                                         "scan_list_entries", "scan_pairs", "beam_scored", "beam_expanded",
                                         "beam_tested", "n_seed_tiles", "seed_pairs", "seed_tile_seeds",
                                         "seeds_on_matrix_cores", "seed_rescored", "seed_fallbacks", "beam_gathered",
                                         "scan_kernel", "seed_selected", "seed_run_keys", "scan_fallbacks")] + \
               [(n, C.c_double) for n in ("host_plan_ms_sum", "host_blob_ms_sum", "host_launch_ms_sum", "host_wait_ms_sum")]


class VfSearchParams(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("k", "itopk", "width", "iters", "n_seeds", "and_scan_limit")] + \
               [("reserved", C.c_int32 * 2)]


class VfServeParams(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("k", "itopk", "width", "iters", "n_seeds", "n_workers", "ring_slots", "waves_per_worker")] + \
               [(n, C.c_int64) for n in ("max_jobs", "idle_polls")]


class VfAdamwTensor(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("param", "grad", "master", "m", "v", "m_scale", "v_scale")] + \
               [("n", C.c_int64), ("weight_decay", C.c_double)] + \
               [(n, C.c_int32) for n in ("param_type", "grad_type", "state_bits", "reserved")]


class VfAdamwParams(C.Structure):
    _fields_ = [(n, C.c_double) for n in ("lr", "beta1", "beta2", "eps", "grad_scale")] + [("step", C.c_int64)]


class VecflowError(RuntimeError):
    pass


_lib = None


def load_library():
    """dlopen the in-tree HIP library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise VecflowError(f"{LIB_PATH} is missing: run `python -m paper_2506_00812_amd.build` "
                               "(there is no CPU fallback)")
        L = C.CDLL(LIB_PATH)
        p, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
        L.vf_build_index.restype = C.c_int
        L.vf_build_index.argtypes = [p, C.c_int, i64, i32, p, p, i32, i32, i32, C.POINTER(VfAllocator), p, C.POINTER(p)]
        L.vf_build_index_opt.restype = C.c_int
        L.vf_build_index_opt.argtypes = [p, C.c_int, i64, i32, p, p, i32, i32, i32, i32, i32, C.POINTER(VfAllocator), p,
                                         C.POINTER(p)]
        L.vf_tune.restype = C.c_int
        L.vf_tune.argtypes = [p, C.c_char_p, C.c_double]
        L.vf_debug_route.restype = C.c_int
        L.vf_debug_route.argtypes = [p, i32, i32, i64, p, p, i32, i32, p, p, p, p, i64, p, i64, p, p]
        L.vf_search.restype = C.c_int
        L.vf_search.argtypes = [p, p, i64, p, p, i32, i32, i32, i32, i32, p, p, p]
        L.vf_search_noalloc.restype = C.c_int
        L.vf_search_noalloc.argtypes = [p, p, i64, p, p, i32, i32, i32, i32, i32, p, p, p]
        L.vf_serve_begin.restype = C.c_int
        L.vf_serve_begin.argtypes = [p, C.POINTER(VfServeParams), C.POINTER(p)]
        L.vf_serve_submit.restype = C.c_int
        L.vf_serve_submit.argtypes = [p, p, p, i32, C.POINTER(i64)]
        L.vf_serve_poll.restype = C.c_int
        L.vf_serve_poll.argtypes = [p, i64, p, p, C.POINTER(i32)]
        L.vf_serve_end.restype = C.c_int
        L.vf_serve_end.argtypes = [p, C.POINTER(i64), C.POINTER(i32)]
        L.vf_serve_run.restype = C.c_int
        L.vf_serve_run.argtypes = [p, p, i64, p, p, i32, p, p, p]
        L.vf_search_ex.restype = C.c_int
        L.vf_search_ex.argtypes = [p, p, i64, p, p, C.POINTER(VfSearchParams), p, p, p]
        L.vf_search_exact.restype = C.c_int
        L.vf_search_exact.argtypes = [p, p, i64, p, p, i32, p, p, p]
        L.vf_index_export.restype = C.c_int
        L.vf_index_export.argtypes = [p, C.c_int, p, C.POINTER(C.c_size_t)]
        L.vf_index_stats.restype = C.c_int
        L.vf_index_stats.argtypes = [p, C.POINTER(VfStats)]
        L.vf_search_multi.restype = C.c_int
        L.vf_search_multi.argtypes = [p, p, C.c_int64, p, p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                      C.c_int32, p, p, p]
        L.vf_profile_enable.restype = C.c_int
        L.vf_profile_enable.argtypes = [p, C.c_int]
        L.vf_profile_read.restype = C.c_int
        L.vf_profile_read.argtypes = [p, C.POINTER(VfProfile), p]
        sz = C.c_size_t
        for name, args in dict(
                vf_linear=[i32, i64, i64, i64, p, i64, p, i64, p, i32, p, i64, p, i64, p, i64, p, sz, p],
                vf_linear_backward=[i32, i64, i64, i64, p, i64, p, i64, p, i64, p, i64, i32, p, i64, p, i64, p, p, sz, p],
                vf_linear_workspace=[i32, i64, i64, i64, i32, i32, C.POINTER(sz)],
                vf_debug_linear=[i32, i64, i64, i64, i32, i32, C.POINTER(i32), C.POINTER(i32)],
                vf_layer_norm=[i32, i64, i64, p, i64, p, p, C.c_double, p, i64, p, p, p],
                vf_layer_norm_backward=[i32, i64, i64, p, i64, p, i64, p, p, p, p, i64, p, p, p, sz, p],
                vf_layer_norm_workspace=[i32, i64, i64, C.POINTER(sz)],
                vf_log_probs=[i32, i64, i64, p, i64, p, i32, p, p, p, p, p, p, sz, p],
                vf_log_probs_backward=[i32, i64, i64, p, i64, p, p, p, p, p, p, i64, p],
                vf_log_probs_workspace=[i32, i64, i64, i32, C.POINTER(sz)],
                vf_adamw_step=[p, i32, C.POINTER(VfAdamwParams), p, p],
                vf_adamw_moments=[p, i32, p, p, p]).items():
            getattr(L, name).restype = C.c_int
            getattr(L, name).argtypes = args
        L.vf_index_free.restype = None
        L.vf_index_free.argtypes = [p]
        L.vf_last_error.restype = C.c_char_p
        L.vf_last_error.argtypes = []
        _lib = L
    return _lib


def _check(rc):
    if rc != 0:
        raise VecflowError(f"vecflow error {rc}: {load_library().vf_last_error().decode()}")


def _np_ptr(a):
    return a.ctypes.data_as(C.c_void_p)


def _stream_handle(stream=None):
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return C.c_void_p(s.cuda_stream)


def _dtype_code(t):
    import torch
    if t.dtype == torch.uint8:
        return VF_U8
    if t.dtype == torch.float32:
        return VF_F32
    raise VecflowError(f"unsupported dtype {t.dtype}")


class TorchAllocator:
    """vf_allocator backed by PyTorch's caching allocator: the index and its workspaces then live in memory that
    torch accounts for and reuses.  Blocks are requested on the stream of the call in progress (the binding sets
    it before every library call); the library frees a block only after the work that used it has completed."""

    def __init__(self, device):
        import torch
        self._torch = torch
        self.device = device
        self.stream = 0
        self.live = {}            # address -> bytes
        self.n_alloc = self.n_free = 0

        def _alloc(nbytes, _ctx):
            try:
                ptr = torch.cuda.caching_allocator_alloc(int(nbytes), device=self.device, stream=self.stream)
            except Exception:      # out of memory: the library reports VF_ENOMEM
                return None
            self.live[ptr] = int(nbytes)
            self.n_alloc += 1
            return ptr

        def _free(ptr, _ctx):
            try:
                if self.live.pop(ptr, None) is not None:
                    self.n_free += 1
                    torch.cuda.caching_allocator_delete(ptr)
            except Exception:      # interpreter shutdown: torch may be gone, the process is ending anyway
                pass

        self._alloc_cb, self._free_cb = ALLOC_FN(_alloc), FREE_FN(_free)   # kept alive with this object
        self.struct = VfAllocator(self._alloc_cb, self._free_cb, None)

    def live_bytes(self):
        return sum(self.live.values())


class Index:
    """Handle of a built index.  Keeps the vector tensor alive (the library references it)."""

    def __init__(self, handle, vectors, allocator=None):
        self._h = handle
        self.vectors = vectors
        self.allocator = allocator   # keeps the callbacks alive as long as the library may call them
        self._free = load_library().vf_index_free  # bound here: module globals may be gone at interpreter exit

    def _enter(self, stream=None):
        """Before a library call that may allocate: blocks come from the pool of the call's stream."""
        if self.allocator is not None:
            import torch
            s = stream if stream is not None else torch.cuda.current_stream()
            self.allocator.stream = s.cuda_stream

    def tune(self, name: str, value):
        """Experiment / test switch of this index (vf_tune)."""
        self._enter()
        _check(load_library().vf_tune(self._h, name.encode(), float(value)))

    def __del__(self):
        self.free()

    def free(self):
        if getattr(self, "_h", None):
            self._free(self._h)
            self._h = None

    def stats(self) -> dict:
        st = VfStats()
        _check(load_library().vf_index_stats(self._h, C.byref(st)))
        return {n: getattr(st, n) for n, _ in VfStats._fields_}

    def profile_enable(self, on=True, serial: bool = False, exact_counts: bool = False):
        """serial=True also runs the IVF-BFS and IVF-Graph launches one after the other; exact_counts=True has a
        small kernel count, before every call with AND queries, the seeds that pass each query's predicate."""
        mode = (2 if serial else 1) if on else 0
        _check(load_library().vf_profile_enable(self._h, mode | (4 if (on and exact_counts) else 0)))

    def profile_read(self, per_query: bool = False):
        """Durations and work counters of the last profiled search; waits for it."""
        pf = VfProfile()
        L = load_library()
        if per_query:
            # nq is only known after a first read
            _check(L.vf_profile_read(self._h, C.byref(pf), None))
            cn = np.zeros((pf.nq, 4), dtype=np.int32)
            _check(L.vf_profile_read(self._h, C.byref(pf), _np_ptr(cn)))
        else:
            cn = None
            _check(L.vf_profile_read(self._h, C.byref(pf), None))
        out = {n: getattr(pf, n) for n, _ in VfProfile._fields_}
        return (out, cn) if per_query else out

    def export(self, name: str) -> np.ndarray:
        L = load_library()
        nbytes = C.c_size_t(0)
        _check(L.vf_index_export(self._h, ARR[name], None, C.byref(nbytes)))
        dt = np.dtype(_ARR_DTYPE[name])
        out = np.empty(nbytes.value // dt.itemsize, dtype=dt)
        if nbytes.value:
            _check(L.vf_index_export(self._h, ARR[name], _np_ptr(out), C.byref(nbytes)))
        return out


def debug_route(S, T, qlabel_offsets, qlabel_ids, tile_rows=16, seg_groups=16):
    """Host-only routing and scan work list for posting-list sizes S (vf_debug_route); no device is touched."""
    L = load_library()
    S = np.ascontiguousarray(S, dtype=np.int32)
    off = np.ascontiguousarray(qlabel_offsets, dtype=np.int64)
    ids = np.ascontiguousarray(qlabel_ids, dtype=np.int32)
    nq = len(off) - 1
    searched, method, n_others = (np.empty(nq, dtype=np.int32) for _ in range(3))
    counts = np.zeros(6, dtype=np.int64)
    args = [_np_ptr(S), len(S), int(T), nq, _np_ptr(off), _np_ptr(ids), int(tile_rows), int(seg_groups),
            _np_ptr(searched), _np_ptr(method), _np_ptr(n_others)]
    _check(L.vf_debug_route(*args, None, 0, None, 0, None, _np_ptr(counts)))      # sizes only
    items = np.zeros((max(int(counts[2]), 1), 8), dtype=np.int64)
    merges = np.zeros((max(int(counts[3]), 1), 5), dtype=np.int64)
    qrow = np.zeros(max(nq, 1), dtype=np.int32)
    _check(L.vf_debug_route(*args, _np_ptr(items), len(items), _np_ptr(merges), len(merges), _np_ptr(qrow),
                            _np_ptr(counts)))
    n_g, n_s, n_items, n_merges, part_rows, max_nseg = (int(c) for c in counts)
    return dict(searched=searched, method=method, n_others=n_others, items=items[:n_items], merges=merges[:n_merges],
                scan_rows=qrow[:n_s], graph_queries=qrow[n_s:n_s + n_g], part_rows=part_rows, max_nseg=max_nseg)


GRAPH_KNN, GRAPH_PRUNED = 0, 1


def tune_defaults(name: str, value):
    """Process-wide default of an experiment / test switch: indexes built afterwards start from it."""
    _check(load_library().vf_tune(None, name.encode(), float(value)))


def build_index(vectors, label_offsets, label_ids, n_labels, T, graph_degree, stream=None, graph_kind=GRAPH_KNN,
                knn_degree=0, torch_allocator=True) -> Index:
    """vectors: CUDA tensor [n, dim] uint8/float32 (contiguous); labels: host CSR arrays.
    graph_kind=GRAPH_PRUNED: graphs of degree knn_degree (0 = the default) reduced to graph_degree by
    rank-based pruning and reverse edges (vf_build_index_opt).
    torch_allocator: the index takes its device memory from PyTorch's caching allocator (False: hipMalloc)."""
    L = load_library()
    if not vectors.is_cuda or not vectors.is_contiguous() or vectors.dim() != 2:
        raise VecflowError("vectors must be a contiguous 2-D CUDA tensor")
    off = np.ascontiguousarray(label_offsets, dtype=np.int64)
    ids = np.ascontiguousarray(label_ids, dtype=np.int32)
    if off.shape[0] != vectors.shape[0] + 1:
        raise VecflowError("label_offsets must have n + 1 entries")
    h = C.c_void_p()
    al = None
    if torch_allocator:
        import torch
        al = TorchAllocator(vectors.device)
        al.stream = (stream if stream is not None else torch.cuda.current_stream()).cuda_stream
    al_ref = C.byref(al.struct) if al is not None else None
    if graph_kind == GRAPH_KNN and knn_degree == 0:
        _check(L.vf_build_index(C.c_void_p(vectors.data_ptr()), _dtype_code(vectors), vectors.shape[0],
                                vectors.shape[1], _np_ptr(off), _np_ptr(ids), int(n_labels), int(T), int(graph_degree),
                                al_ref, _stream_handle(stream), C.byref(h)))
    else:
        _check(L.vf_build_index_opt(C.c_void_p(vectors.data_ptr()), _dtype_code(vectors), vectors.shape[0],
                                    vectors.shape[1], _np_ptr(off), _np_ptr(ids), int(n_labels), int(T),
                                    int(graph_degree), int(graph_kind), int(knn_degree), al_ref, _stream_handle(stream),
                                    C.byref(h)))
    return Index(h, vectors, al)


def _prep_queries(index, queries, qlabel_offsets, qlabel_ids):
    if not queries.is_cuda or not queries.is_contiguous() or queries.dim() != 2:
        raise VecflowError("queries must be a contiguous 2-D CUDA tensor")
    if queries.dtype != index.vectors.dtype or queries.shape[1] != index.vectors.shape[1]:
        raise VecflowError("queries must match the index dtype and dim")
    off = np.ascontiguousarray(qlabel_offsets, dtype=np.int64)
    ids = np.ascontiguousarray(qlabel_ids, dtype=np.int32)
    if off.shape[0] != queries.shape[0] + 1:
        raise VecflowError("qlabel_offsets must have nq + 1 entries")
    return off, ids


def search(index: Index, queries, qlabel_offsets, qlabel_ids, k, itopk=64, width=1, iters=32, n_seeds=0,
           out_ids=None, out_dists=None, stream=None, and_scan_limit=0):
    """Asynchronous on the (current) stream; returns (ids int64 [nq,k], dists float32 [nq,k]) CUDA tensors.
    and_scan_limit > 0: vf_search_ex with selectivity-aware routing of AND queries."""
    import torch
    off, ids = _prep_queries(index, queries, qlabel_offsets, qlabel_ids)
    nq = queries.shape[0]
    if out_ids is None:
        out_ids = torch.empty((nq, k), dtype=torch.int64, device=queries.device)
    if out_dists is None:
        out_dists = torch.empty((nq, k), dtype=torch.float32, device=queries.device)
    index._enter(stream)
    if and_scan_limit:
        prm = VfSearchParams(int(k), int(itopk), int(width), int(iters), int(n_seeds), int(and_scan_limit))
        _check(load_library().vf_search_ex(index._h, C.c_void_p(queries.data_ptr()), nq, _np_ptr(off), _np_ptr(ids),
                                           C.byref(prm), C.c_void_p(out_ids.data_ptr()), C.c_void_p(out_dists.data_ptr()),
                                           _stream_handle(stream)))
        return out_ids, out_dists
    _check(load_library().vf_search(index._h, C.c_void_p(queries.data_ptr()), nq, _np_ptr(off), _np_ptr(ids), int(k),
                                    int(itopk), int(width), int(iters), int(n_seeds),
                                    C.c_void_p(out_ids.data_ptr()), C.c_void_p(out_dists.data_ptr()),
                                    _stream_handle(stream)))
    return out_ids, out_dists


def search_noalloc(index: Index, queries, qlabel_offsets, qlabel_ids, k, out_ids, out_dists, itopk=64, width=1,
                   iters=32, n_seeds=0, stream=None):
    """vf_search_noalloc: the same search with every temporary in the library's fixed scratch array; the caller
    passes the output tensors, nothing is allocated on the way.  Asynchronous on the (current) stream."""
    off, ids = _prep_queries(index, queries, qlabel_offsets, qlabel_ids)
    nq = queries.shape[0]
    if tuple(out_ids.shape) != (nq, k) or tuple(out_dists.shape) != (nq, k):
        raise VecflowError("out_ids / out_dists must be [nq, k]")
    _check(load_library().vf_search_noalloc(index._h, C.c_void_p(queries.data_ptr()), nq, _np_ptr(off), _np_ptr(ids),
                                            int(k), int(itopk), int(width), int(iters), int(n_seeds),
                                            C.c_void_p(out_ids.data_ptr()), C.c_void_p(out_dists.data_ptr()),
                                            _stream_handle(stream)))
    return out_ids, out_dists


EBUSY = -5


class Server:
    """A serving session (vf_serve_*): a resident kernel that answers single queries from a job ring."""

    def __init__(self, index: Index, k, itopk=32, width=1, iters=8, n_seeds=0, n_workers=0, ring_slots=0, max_jobs=0,
                 idle_polls=0, waves_per_worker=0):
        self.index, self.k = index, int(k)
        prm = VfServeParams(int(k), int(itopk), int(width), int(iters), int(n_seeds), int(n_workers), int(ring_slots),
                            int(waves_per_worker), int(max_jobs), int(idle_polls))
        h = C.c_void_p()
        index._enter()
        if index.allocator is not None:   # its blocks follow the current stream's order; the session uses them on a stream of its own
            import torch
            torch.cuda.current_stream().synchronize()
        _check(load_library().vf_serve_begin(index._h, C.byref(prm), C.byref(h)))
        self._h = h
        self._np_dtype = np.uint8 if _dtype_code(index.vectors) == VF_U8 else np.float32
        self.dim = index.vectors.shape[1]

    def submit(self, query, labels):
        """query: host array [dim]; labels: 1..8 ids.  Returns the job id, or None when the ring is full."""
        q = np.ascontiguousarray(query, dtype=self._np_dtype)
        if q.shape != (self.dim,):
            raise VecflowError("query must have dim elements")
        lab = np.ascontiguousarray(labels, dtype=np.int32).reshape(-1)
        job = C.c_int64(-1)
        rc = load_library().vf_serve_submit(self._h, _np_ptr(q), _np_ptr(lab), len(lab), C.byref(job))
        if rc == EBUSY:
            return None
        _check(rc)
        return job.value

    def poll(self, job):
        """(ids, dists) of a completed job, else None."""
        ids = np.empty(self.k, dtype=np.int64)
        d = np.empty(self.k, dtype=np.float32)
        done = C.c_int32(0)
        _check(load_library().vf_serve_poll(self._h, int(job), _np_ptr(ids), _np_ptr(d), C.byref(done)))
        return (ids, d) if done.value else None

    def run(self, queries, qlabel_offsets, qlabel_ids, in_flight=64):
        """A host batch through the session, one job per query (vf_serve_run): (ids, dists, latency_us)."""
        q = np.ascontiguousarray(queries, dtype=self._np_dtype)
        off = np.ascontiguousarray(qlabel_offsets, dtype=np.int64)
        lab = np.ascontiguousarray(qlabel_ids, dtype=np.int32)
        nq = q.shape[0]
        ids = np.empty((nq, self.k), dtype=np.int64)
        d = np.empty((nq, self.k), dtype=np.float32)
        lat = np.empty(nq, dtype=np.float32)
        _check(load_library().vf_serve_run(self._h, _np_ptr(q), nq, _np_ptr(off), _np_ptr(lab), int(in_flight),
                                           _np_ptr(ids), _np_ptr(d), _np_ptr(lat)))
        return ids, d, lat

    def end(self):
        """Stops the kernel and releases the session; returns (jobs completed, exit reason)."""
        if self._h is None:
            return None
        n, why = C.c_int64(0), C.c_int32(0)
        h, self._h = self._h, None
        _check(load_library().vf_serve_end(h, C.byref(n), C.byref(why)))
        return n.value, why.value

    def __del__(self):
        try:
            self.end()
        except Exception:
            pass


NOALLOC_SCRATCH_BYTES, NOALLOC_MAX_QUERIES = 8 << 20, 1024
AND_GREEDY, AND_PARALLEL, OR = 0, 1, 2
MULTI_EXACT = 0x100


def search_multi(index: Index, queries, qlabel_offsets, qlabel_ids, mode, k, itopk=64, width=1, iters=32, n_seeds=0,
                 out_ids=None, out_dists=None, stream=None):
    """OR queries and the parallel AND policy: one search per query label, merged.  Asynchronous."""
    import torch
    off, ids = _prep_queries(index, queries, qlabel_offsets, qlabel_ids)
    nq = queries.shape[0]
    if out_ids is None:
        out_ids = torch.empty((nq, k), dtype=torch.int64, device=queries.device)
    if out_dists is None:
        out_dists = torch.empty((nq, k), dtype=torch.float32, device=queries.device)
    index._enter(stream)
    _check(load_library().vf_search_multi(index._h, C.c_void_p(queries.data_ptr()), nq, _np_ptr(off), _np_ptr(ids),
                                          int(mode), int(k), int(itopk), int(width), int(iters), int(n_seeds),
                                          C.c_void_p(out_ids.data_ptr()), C.c_void_p(out_dists.data_ptr()),
                                          _stream_handle(stream)))
    return out_ids, out_dists


def search_exact(index: Index, queries, qlabel_offsets, qlabel_ids, k, stream=None):
    """Exact filtered top-k (ground truth).  Synchronises the stream."""
    import torch
    off, ids = _prep_queries(index, queries, qlabel_offsets, qlabel_ids)
    nq = queries.shape[0]
    out_ids = torch.empty((nq, k), dtype=torch.int64, device=queries.device)
    out_dists = torch.empty((nq, k), dtype=torch.float32, device=queries.device)
    index._enter(stream)
    _check(load_library().vf_search_exact(index._h, C.c_void_p(queries.data_ptr()), nq, _np_ptr(off), _np_ptr(ids),
                                          int(k), C.c_void_p(out_ids.data_ptr()), C.c_void_p(out_dists.data_ptr()),
                                          _stream_handle(stream)))
    return out_ids, out_dists


# ---------------------------------------------------------------- operators of a query encoder
#
# Tensors are CUDA tensors of one device, the current one.  Matrices are 2-D with neighbouring columns (stride(1) == 1); rows may be
# slices of a wider matrix.  Everything is enqueued on the current stream (or `stream`), where outputs and workspaces
# are allocated too; nothing synchronises.

ACTIVATIONS = dict(none=0, relu=1, gelu=2, silu=3)
ADAMW_BLOCK = 256
LOG_PROBS_MAX_TOP = 64

# Filled on first use (torch is imported lazily here): torch, the codes of its float types, the current stream's handle.
_torch = _codes = _raw_stream = None


def _use_torch():
    global _torch, _codes, _raw_stream
    import torch
    _codes = {torch.float32: VF_F32, torch.bfloat16: VF_BF16, torch.float16: VF_F16}
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)     # (a Stream object costs more than a small kernel's launch)
    _raw_stream = raw or (lambda device: torch.cuda.current_stream(device).cuda_stream)
    _torch = torch


def _first(t, what, stream):
    """(type code, dtype, device, stream handle) of a call, from its first tensor, which must be on the current device."""
    if _torch is None:
        _use_torch()
    T = t.dtype
    code = _codes.get(T)
    if code is None:
        raise VecflowError(f"{what}: unsupported dtype {T}")
    dev = t.get_device()
    if dev < 0 or dev != _torch.cuda.current_device():
        raise VecflowError(f"{what} must be a CUDA tensor on the current device")
    return code, T, dev, _raw_stream(dev) if stream is None else stream.cuda_stream


def _matrix(t, what, T, dev, rows=None, cols=None):
    """Distance of two rows of a matrix argument, which must have the dtype, device and sizes given."""
    if t.dtype != T or t.get_device() != dev or t.dim() != 2:
        raise VecflowError(f"{what} must be a 2-D CUDA tensor of {T} on the same device")
    n, d = t.shape
    if (rows is not None and n != rows) or (cols is not None and d != cols):
        raise VecflowError(f"{what} must have shape [{n if rows is None else rows}, {d if cols is None else cols}], not {list(t.shape)}")
    ld, step = t.stride()
    if step != 1 and d > 1:
        raise VecflowError(f"{what} must have neighbouring columns (stride(1) == 1)")
    if n <= 1:
        return d
    if ld < d:
        raise VecflowError(f"{what} must not have overlapping rows")
    return ld


def _vector(t, what, T, dev, n):
    """Address of a vector argument; None stays None."""
    if t is None:
        return None
    if t.dtype != T or t.get_device() != dev or t.numel() != n or t.dim() != 1 or not t.is_contiguous():
        raise VecflowError(f"{what} must be a contiguous CUDA tensor [{n}] of {T} on the same device")
    return t.data_ptr()


def _empty(like, shape, T, stream):
    """Memory on the call's stream, so that it returns to the pool in that stream's order."""
    if stream is None:
        return like.new_empty(shape, dtype=T)
    with _torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=T)


@functools.lru_cache(maxsize=4096)
def _size_of(name, *args):
    """What a vf_*_workspace function says for these sizes (it depends on nothing else)."""
    n = C.c_size_t(0)
    _check(getattr(load_library(), name)(*args, C.byref(n)))
    return n.value


def _workspace(like, nbytes, stream):
    """(tensor, address): the tensor has to live until the call has been made, its memory is then the stream's to reuse."""
    if nbytes == 0:
        return None, None
    t = _empty(like, (nbytes,), _torch.uint8, stream)
    return t, t.data_ptr()


def _activation(name):
    act = ACTIVATIONS.get(name)
    if act is None:
        raise VecflowError(f"unknown activation {name!r}: one of {sorted(ACTIVATIONS)}")
    return act


def linear(x, weight, bias=None, residual=None, activation="none", save=False, out=None, stream=None):
    """act(x weight^T + bias) + residual for x [m, k], weight [n, k] (vf_linear).  save=True: (y, z) with the
    pre-activation z that linear_backward reads.  `out` may be the residual's own memory."""
    L = load_library()
    code, T, dev, handle = _first(x, "x", stream)
    act = _activation(activation)
    ldx = _matrix(x, "x", T, dev)
    m, k = x.shape
    ldw = _matrix(weight, "weight", T, dev, None, k)
    n = weight.shape[0]
    pb = _vector(bias, "bias", T, dev, n)
    ldr = 0 if residual is None else _matrix(residual, "residual", T, dev, m, n)
    if out is None:
        out, ldy = _empty(x, (m, n), T, stream), n
    else:
        ldy = _matrix(out, "out", T, dev, m, n)
    z = _empty(x, (m, n), T, stream) if save else None
    nw = _size_of("vf_linear_workspace", code, m, n, k, act, 0)
    _ws, pw = _workspace(x, nw, stream)
    _check(L.vf_linear(code, m, n, k, x.data_ptr(), ldx, weight.data_ptr(), ldw, pb, act,
                       None if residual is None else residual.data_ptr(), ldr, out.data_ptr(), ldy,
                       z.data_ptr() if save else None, n, pw, nw, handle))
    return (out, z) if save else out


def linear_backward(dy, x, weight, z=None, activation="none", bias=True, dx=True, dweight=True, stream=None):
    """Gradients (dx, dweight, dbias) of linear from dy [m, n] (vf_linear_backward); the residual's gradient is dy itself.
    What is not asked for is None.  z: the pre-activation, needed for any activation but "none"."""
    L = load_library()
    code, T, dev, handle = _first(dy, "dy", stream)
    act = _activation(activation)
    lddy = _matrix(dy, "dy", T, dev)
    m, n = dy.shape
    ldx = _matrix(x, "x", T, dev, m)
    k = x.shape[1]
    ldw = _matrix(weight, "weight", T, dev, n, k)
    if act and z is None:
        raise VecflowError(f"linear_backward needs z, the pre-activation, for activation {activation!r}")
    ldz = _matrix(z, "z", T, dev, m, n) if act else 0
    gx = _empty(dy, (m, k), T, stream) if dx else None
    gw = _empty(dy, (n, k), T, stream) if dweight else None
    gb = _empty(dy, (n,), T, stream) if bias else None
    nw = _size_of("vf_linear_workspace", code, m, n, k, act, 1)
    _ws, pw = _workspace(dy, nw, stream)
    _check(L.vf_linear_backward(code, m, n, k, dy.data_ptr(), lddy, x.data_ptr(), ldx, weight.data_ptr(), ldw,
                                z.data_ptr() if act else None, ldz, act, gx.data_ptr() if dx else None, k,
                                gw.data_ptr() if dweight else None, k, gb.data_ptr() if bias else None, pw, nw, handle))
    return gx, gw, gb


def debug_linear(dtype, m, n, k, product=0, direct=True):
    """(tiling, splits) of a product of the linear layer (vf_debug_linear); dtype: VF_F32, VF_BF16 or VF_F16."""
    tiling, splits = C.c_int32(), C.c_int32()
    _check(load_library().vf_debug_linear(dtype, m, n, k, product, int(direct), C.byref(tiling), C.byref(splits)))
    return tiling.value, splits.value


def layer_norm(x, weight=None, bias=None, eps=1e-5, save=False, out=None, stream=None):
    """(x - mean) / sqrt(variance + eps) weight + bias per row of x [m, d] (vf_layer_norm).  save=True: (y, mean, rstd).
    `out` may be x's own memory."""
    L = load_library()
    code, T, dev, handle = _first(x, "x", stream)
    ldx = _matrix(x, "x", T, dev)
    m, d = x.shape
    pg, pb = _vector(weight, "weight", T, dev, d), _vector(bias, "bias", T, dev, d)
    if out is None:
        out, ldy = _empty(x, (m, d), T, stream), d
    else:
        ldy = _matrix(out, "out", T, dev, m, d)
    if not save:
        _check(L.vf_layer_norm(code, m, d, x.data_ptr(), ldx, pg, pb, eps, out.data_ptr(), ldy, None, None, handle))
        return out
    mean, rstd = _empty(x, (2, m), _torch.float32, stream).unbind(0)
    _check(L.vf_layer_norm(code, m, d, x.data_ptr(), ldx, pg, pb, eps, out.data_ptr(), ldy, mean.data_ptr(), rstd.data_ptr(),
                           handle))
    return out, mean, rstd


def layer_norm_backward(dy, x, mean, rstd, weight=None, dx=True, dweight=True, dbias=True, out=None, stream=None):
    """Gradients (dx, dweight, dbias) of layer_norm from dy [m, d] (vf_layer_norm_backward).  What is not asked for is
    None.  `out`: where dx goes, dy's own memory if need be."""
    L = load_library()
    code, T, dev, handle = _first(dy, "dy", stream)
    lddy = _matrix(dy, "dy", T, dev)
    m, d = dy.shape
    ldx = _matrix(x, "x", T, dev, m, d)
    pm, pr = _vector(mean, "mean", _torch.float32, dev, m), _vector(rstd, "rstd", _torch.float32, dev, m)
    pg = _vector(weight, "weight", T, dev, d)
    if dx and out is None:
        out = _empty(dy, (m, d), T, stream)
    ldo = _matrix(out, "out", T, dev, m, d) if dx else 0
    gw = _empty(dy, (d,), T, stream) if dweight else None
    gb = _empty(dy, (d,), T, stream) if dbias else None
    nw = _size_of("vf_layer_norm_workspace", code, m, d) if dweight or dbias else 0
    _ws, pw = _workspace(dy, nw, stream)
    _check(L.vf_layer_norm_backward(code, m, d, dy.data_ptr(), lddy, x.data_ptr(), ldx, pm, pr, pg,
                                    out.data_ptr() if dx else None, ldo, gw.data_ptr() if dweight else None,
                                    gb.data_ptr() if dbias else None, pw, nw, handle))
    return out if dx else None, gw, gb


def log_probs(logits, targets=None, top=0, stream=None):
    """Log probabilities over the vocabulary of logits [m, v] (vf_log_probs): (logp, entropy, lse) or, with top > 0,
    (logp, entropy, lse, top_ids, top_logp); float32 [m], int32 / float32 [m, top].  targets: int32 [m], -1 for none;
    logp is None without them."""
    L = load_library()
    code, T, dev, handle = _first(logits, "logits", stream)
    ld = _matrix(logits, "logits", T, dev)
    m, v = logits.shape
    top = int(top)
    if not 0 <= top <= LOG_PROBS_MAX_TOP:
        raise VecflowError(f"top must be 0 .. {LOG_PROBS_MAX_TOP}")
    f32, i32 = _torch.float32, _torch.int32
    pt = _vector(targets, "targets", i32, dev, m)
    logp, entropy, lse = _empty(logits, (3, m), f32, stream).unbind(0)
    ids = _empty(logits, (m, top), i32, stream) if top else None
    tlp = _empty(logits, (m, top), f32, stream) if top else None
    nw = _size_of("vf_log_probs_workspace", code, m, v, top)
    _ws, pw = _workspace(logits, nw, stream)
    _check(L.vf_log_probs(code, m, v, logits.data_ptr(), ld, pt, top, None if targets is None else logp.data_ptr(),
                          entropy.data_ptr(), lse.data_ptr(), ids.data_ptr() if top else None,
                          tlp.data_ptr() if top else None, pw, nw, handle))
    if targets is None:
        logp = None
    return (logp, entropy, lse, ids, tlp) if top else (logp, entropy, lse)


def log_probs_backward(logits, lse, targets=None, d_logp=None, entropy=None, d_entropy=None, out=None, stream=None):
    """Gradient with respect to the logits from those of logp and entropy (vf_log_probs_backward); `out` may be the
    logits' own memory.  p = exp(logits - lse) has lse's rounding, 2^-24 |lse|, as a relative error."""
    L = load_library()
    code, T, dev, handle = _first(logits, "logits", stream)
    ld = _matrix(logits, "logits", T, dev)
    m, v = logits.shape
    f32 = _torch.float32
    if (targets is None) != (d_logp is None) or (entropy is None) != (d_entropy is None):
        raise VecflowError("targets and d_logp go together, and entropy and d_entropy")
    if out is None:
        out, ldd = _empty(logits, (m, v), T, stream), v
    else:
        ldd = _matrix(out, "out", T, dev, m, v)
    _check(L.vf_log_probs_backward(code, m, v, logits.data_ptr(), ld, _vector(lse, "lse", f32, dev, m),
                                   _vector(targets, "targets", _torch.int32, dev, m), _vector(d_logp, "d_logp", f32, dev, m),
                                   _vector(entropy, "entropy", f32, dev, m), _vector(d_entropy, "d_entropy", f32, dev, m),
                                   out.data_ptr(), ldd, handle))
    return out


def adamw_state(param, bits=32):
    """Moments before the first step: (m, v) float32, or with bits=8 (m int8, v uint8, m_scale, v_scale)."""
    import torch
    n = param.numel()
    if bits == 32:
        return tuple(torch.zeros(n, dtype=torch.float32, device=param.device) for _ in range(2))
    if bits != 8:
        raise VecflowError("bits must be 32 or 8")
    blocks = -(-n // ADAMW_BLOCK)
    return (torch.zeros(n, dtype=torch.int8, device=param.device), torch.zeros(n, dtype=torch.uint8, device=param.device),
            torch.zeros(blocks, dtype=torch.float32, device=param.device),
            torch.zeros(blocks, dtype=torch.float32, device=param.device))


def _flat(t, what, kinds, dev, n):
    if t.dtype not in kinds or t.get_device() != dev or t.numel() != n or not t.is_contiguous():
        raise VecflowError(f"adamw: {what} must be a contiguous tensor of {n} elements of {' or '.join(map(str, kinds))} "
                           "on the current device")
    return t.data_ptr()


_ADAMW_ITEM = struct.Struct("@7Pqd4i")     # VfAdamwTensor, field by field: one pack per tensor costs a tenth of its assignments


def _adamw_moments_of(ms, vs, m_scales, v_scales):
    """Per tensor (elements, state bits, addresses of m, v, m_scale, v_scale), and the device."""
    if _torch is None:
        _use_torch()
    count = len(ms)
    for other in (vs, m_scales, v_scales):
        if other is not None and len(other) != count:
            raise VecflowError("adamw: the lists must have one entry per tensor")
    if (m_scales is None) != (v_scales is None):
        raise VecflowError("adamw: m_scales and v_scales go together")
    F, I8, U8 = (_torch.float32,), (_torch.int8,), (_torch.uint8,)
    dev = _torch.cuda.current_device() if count else -1
    out = []
    for i, m in enumerate(ms):
        n = m.numel()
        if m.dtype == F[0]:
            out.append((n, 32, _flat(m, "a first moment", F, dev, n), _flat(vs[i], "a second moment", F, dev, n), 0, 0))
            continue
        if m_scales is None or m_scales[i] is None or v_scales[i] is None:
            raise VecflowError(f"adamw: tensor {i}: moments in 8 bits need scales")
        blocks = -(-n // ADAMW_BLOCK)
        out.append((n, 8, _flat(m, "a first moment", I8, dev, n), _flat(vs[i], "a second moment", U8, dev, n),
                    _flat(m_scales[i], "a scale", F, dev, blocks), _flat(v_scales[i], "a scale", F, dev, blocks)))
    return out, dev


def adamw_step(params, grads, ms, vs, step, lr, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0, grad_scale=1.0, masters=None,
               m_scales=None, v_scales=None, skip=None, stream=None):
    """One AdamW step over lists of tensors, in place (vf_adamw_step).  params: float32, bfloat16 or float16, with a
    float32 master each if `masters` is given (entries may be None); ms, vs: the moments of adamw_state, in 8 bits with
    their scales; weight_decay: one number or one per tensor; step counts from 1; skip: int32 CUDA tensor [1], the step
    changes nothing if it is not 0 when the work runs."""
    count = len(params)
    if len(grads) != count or len(ms) != count or (masters is not None and len(masters) != count):
        raise VecflowError("adamw: the lists must have one entry per tensor")
    decay = weight_decay if isinstance(weight_decay, (list, tuple)) else [weight_decay] * count
    if len(decay) != count:
        raise VecflowError("adamw: weight_decay must be one number or one per tensor")
    moments, dev = _adamw_moments_of(ms, vs, m_scales, v_scales)
    if count == 0:
        return
    items, F, pack = [], (_torch.float32,), _ADAMW_ITEM.pack
    for i, p in enumerate(params):
        n, bits, pm, pv, pms, pvs = moments[i]
        g, w = grads[i], None if masters is None else masters[i]
        items.append(pack(_flat(p, "a parameter", _codes, dev, n), _flat(g, "a gradient", _codes, dev, n),
                          0 if w is None else _flat(w, "a master", F, dev, n), pm, pv, pms, pvs, n, decay[i],
                          _codes[p.dtype], _codes[g.dtype], bits, 0))
    prm = VfAdamwParams(lr, betas[0], betas[1], eps, grad_scale, step)
    handle = _raw_stream(dev) if stream is None else stream.cuda_stream
    _check(load_library().vf_adamw_step(b"".join(items), count, C.byref(prm), _vector(skip, "skip", _torch.int32, dev, 1), handle))


def adamw_moments(ms, vs, m_scales=None, v_scales=None, stream=None):
    """The moments as float32 tensors: lists (m, v) (vf_adamw_moments)."""
    moments, dev = _adamw_moments_of(ms, vs, m_scales, v_scales)
    count = len(ms)
    if count == 0:
        return [], []
    items = b"".join([_ADAMW_ITEM.pack(0, 0, 0, pm, pv, pms, pvs, n, 0.0, 0, 0, bits, 0) for n, bits, pm, pv, pms, pvs in moments])
    sizes = [t[0] for t in moments]
    at = [0]
    for n in sizes:
        at.append(at[-1] + n)
    outs, ptrs = [], []
    for _ in range(2):
        whole = _empty(ms[0], (at[-1],), _torch.float32, stream)
        base = whole.data_ptr()
        outs.append(list(whole.split(sizes)))
        ptrs.append((C.c_void_p * count)(*[base + 4 * a for a in at[:-1]]))
    handle = _raw_stream(dev) if stream is None else stream.cuda_stream
    _check(load_library().vf_adamw_moments(items, count, ptrs[0], ptrs[1], handle))
    return outs[0], outs[1]
