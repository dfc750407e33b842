"""Thin ctypes binding of libgrand.so (the C ABI in include/grand.h).

Argument marshalling only: every step of the update and search path runs in
the library's HIP kernels.  Arrays may be numpy arrays (host memory) or
torch tensors (host or device memory); device tensors are passed by their
data pointer, and the library runs on torch's current HIP stream.
"""
from __future__ import annotations

import ctypes
import os
from typing import Any, NamedTuple, Optional

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libgrand.so")
INVALID = 0xFFFFFFFF

OK, E_ARG, E_ID, E_CAPACITY, E_DEVICE, E_OOM, E_STATE = 0, -1, -2, -3, -4, -5, -6
VAMANA, CAGRA = 0, 1
F32, U8 = 0, 1
BF16, F16 = 2, 3
L2, IP, MIPS = 0, 1, 2
ALPHA_ON_DIST, ALPHA_ON_L2 = 0, 1
CAS_GROUPED, CAS_RACING = 0, 1
REV_FULL, REV_BATCH = 0, 1
INDEG_SCAN, INDEG_REV_BATCH, INDEG_REV_FULL = 0, 1, 2
STATIC_SCRATCH_BYTES = 8 << 20   # GRAND_STATIC_SCRATCH_BYTES

PHASES = ["validate", "stage", "search_insert", "bootstrap", "prune_fwd", "group", "rebuild", "search_delete",
          "reverse", "repair", "clear", "medoid", "search_query", "cagra_detour", "cagra_pickone"]

EXPORTED = ["grand_default_params", "grand_create", "grand_destroy", "grand_set_stream", "grand_insert_batch",
            "grand_build_cagra", "grand_delete_batch", "grand_search", "grand_search_static", "grand_count_in_edges", "grand_reader_create",
            "grand_reader_search", "grand_reader_destroy", "grand_reader_last_error", "grand_export_graph", "grand_import_graph", "grand_set_timing",
            "grand_set_counting", "grand_stats", "grand_reset_stats", "grand_last_error",
            "grand_default_cache_params", "grand_cache_create", "grand_cache_destroy", "grand_cache_set_stream", "grand_cache_check",
            "grand_cache_last_error", "grand_cache_append", "grand_cache_attend", "grand_cache_attend_ids", "grand_cache_evict",
            "grand_cache_append_packed", "grand_cache_attend_sinks", "grand_cache_attend_packed", "grand_cache_attend_ids_packed",
            "grand_packed_read", "grand_packed_copy", "grand_pages_fork", "grand_pages_grow", "grand_pages_release", "grand_pages_compact",
            "grand_pages_copy"]


class GrandError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"grand status {code}: {msg}")
        self.code = code


class Params(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("algo", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("metric", ctypes.c_int32), ("dim", ctypes.c_uint32), ("capacity", ctypes.c_uint32),
                ("R", ctypes.c_uint32), ("L_build", ctypes.c_uint32), ("P", ctypes.c_uint32),
                ("c", ctypes.c_uint32), ("k_repair", ctypes.c_uint32), ("max_iters", ctypes.c_uint32),
                ("alpha", ctypes.c_float), ("prune_rule", ctypes.c_int32), ("cas_mode", ctypes.c_int32),
                ("rev_mode", ctypes.c_int32), ("max_batch", ctypes.c_uint32), ("mips_norm", ctypes.c_float),
                ("device", ctypes.c_int32),
                ("stream", ctypes.c_void_p)]


class Stats(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("timing_enabled", ctypes.c_uint32),
                ("inserted", ctypes.c_uint64), ("deleted", ctypes.c_uint64), ("queried", ctypes.c_uint64),
                ("search_hops", ctypes.c_uint64 * 3), ("search_evals", ctypes.c_uint64 * 3),
                ("fwd_evals", ctypes.c_uint64), ("fwd_prunes", ctypes.c_uint64),
                ("rebuild_evals", ctypes.c_uint64), ("rebuild_prunes", ctypes.c_uint64), ("dirty", ctypes.c_uint64),
                ("rebuild_records", ctypes.c_uint64), ("records", ctypes.c_uint64), ("rev_edges", ctypes.c_uint64),
                ("repair_evals", ctypes.c_uint64), ("rebuild_rows", ctypes.c_uint64),
                ("repair_rows", ctypes.c_uint64), ("repair_records", ctypes.c_uint64),
                ("search_distinct", ctypes.c_uint64 * 3), ("search_capped", ctypes.c_uint64 * 3),
                ("phase_ms", ctypes.c_double * len(PHASES)), ("phase_calls", ctypes.c_uint64 * len(PHASES))]


class CacheParams(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32), ("q_heads", ctypes.c_uint32),
                ("kv_heads", ctypes.c_uint32), ("head_dim", ctypes.c_uint32), ("page_size", ctypes.c_uint32),
                ("device", ctypes.c_int32), ("stream", ctypes.c_void_p)]


class Pages(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("n_pages", ctypes.c_uint32),
                ("page_stride", ctypes.c_int64), ("slot_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class PackedPages(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scales", ctypes.c_void_p), ("v_scales", ctypes.c_void_p),
                ("n_pages", ctypes.c_uint32), ("page_stride", ctypes.c_int64), ("slot_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("scale_page_stride", ctypes.c_int64), ("scale_slot_stride", ctypes.c_int64), ("scale_head_stride", ctypes.c_int64)]


class Rows(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class Weights(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("seq_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class Seqs(ctypes.Structure):
    _fields_ = [("n_seq", ctypes.c_uint32), ("n_tokens", ctypes.c_uint32), ("max_q", ctypes.c_uint32),
                ("max_k", ctypes.c_uint32), ("table", ctypes.c_void_p), ("table_stride", ctypes.c_int64),
                ("max_pages", ctypes.c_uint32), ("q_start", ctypes.c_void_p), ("lens", ctypes.c_void_p)]


_lib = None


def load_library(path: str = LIB_PATH):
    """Loads libgrand.so; raises if it has not been built (there is no
    fallback implementation)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with paper_2608_21163_amd/build.py")
    # One HIP runtime per process: torch ships its own libamdhip64 with the
    # same soname as the system one libgrand.so links.  Loading torch first
    # makes libgrand bind to torch's copy; loading libgrand first would pull
    # in the system copy, and torch's later initialisation then finds no GPU.
    try:
        import torch  # noqa: F401
    except ImportError:
        pass
    lib = ctypes.CDLL(path)
    P, U32, I32, U64 = ctypes.c_void_p, ctypes.c_uint32, ctypes.c_int32, ctypes.c_uint64
    lib.grand_default_params.argtypes = [P]
    lib.grand_create.argtypes = [P, P]
    lib.grand_destroy.argtypes = [P]
    lib.grand_set_stream.argtypes = [P, P]
    lib.grand_insert_batch.argtypes = [P, P, P, U32]
    lib.grand_build_cagra.restype = I32
    lib.grand_build_cagra.argtypes = [P, P, P, U32, P, U32, U32, U32]
    lib.grand_delete_batch.argtypes = [P, P, U32]
    lib.grand_search.argtypes = [P, P, U32, U32, U32, P, P]
    lib.grand_search_static.argtypes = [P, P, U32, U32, U32, P, P]
    lib.grand_count_in_edges.argtypes = [P, P, U32, I32, P, P]
    lib.grand_reader_create.argtypes = [P, P, P]
    lib.grand_reader_search.argtypes = [P, P, U32, U32, U32, P, P]
    lib.grand_reader_destroy.argtypes = [P]
    lib.grand_reader_last_error.argtypes = [P]
    lib.grand_reader_last_error.restype = ctypes.c_char_p
    lib.grand_export_graph.argtypes = [P, P, P, P, P, P, P, P]
    lib.grand_import_graph.argtypes = [P, P, P, P, P, U32]
    lib.grand_set_timing.argtypes = [P, I32]
    lib.grand_set_counting.argtypes = [P, I32]
    lib.grand_stats.argtypes = [P, P, ctypes.c_size_t]
    lib.grand_reset_stats.argtypes = [P]
    lib.grand_last_error.argtypes = [P]
    lib.grand_last_error.restype = ctypes.c_char_p
    lib.grand_default_cache_params.argtypes = [P]
    lib.grand_cache_create.argtypes = [P, P]
    lib.grand_cache_destroy.argtypes = [P]
    lib.grand_cache_set_stream.argtypes = [P, P]
    lib.grand_cache_check.argtypes = [P]
    lib.grand_cache_last_error.argtypes = [P]
    lib.grand_cache_last_error.restype = ctypes.c_char_p
    F, I64 = ctypes.c_float, ctypes.c_int64
    lib.grand_cache_append.argtypes = [P, P, P, P, P]
    lib.grand_cache_attend.argtypes = [P, P, P, P, F, I32, U32, P, P, P, P]
    lib.grand_cache_attend_ids.argtypes = [P, U32, P, P, P, U32, I64, I64, F, P, P, P, P]
    lib.grand_cache_evict.argtypes = [P, P, U32, U32, P, P, U32, U32, P, P, P, P, P]
    lib.grand_cache_append_packed.argtypes = [P, P, P, P, P]
    lib.grand_cache_attend_sinks.argtypes = [P, P, P, P, F, I32, U32, U32, P, P, P, P]
    lib.grand_cache_attend_packed.argtypes = [P, P, P, P, F, I32, U32, U32, P, P, P, P]
    lib.grand_cache_attend_ids_packed.argtypes = [P, U32, P, P, P, U32, I64, I64, F, P, P, P, P]
    lib.grand_packed_read.argtypes = [P, U32, P, P, P, P]
    lib.grand_packed_copy.argtypes = [P, U32, P, P, P]
    lib.grand_pages_fork.argtypes = [P, P, U32, P, I32, U32, P, P, P, P]
    lib.grand_pages_grow.argtypes = [P, P, P, U32, P, P, P, P, P, P]
    lib.grand_pages_release.argtypes = [P, U32, U32, P, I64, P, I32, U32, P, P, P, P]
    lib.grand_pages_compact.argtypes = [P, P, U32, P, P, P, P, P, P]
    lib.grand_pages_copy.argtypes = [P, U32, P, P, P]
    for name in EXPORTED:
        if name not in ("grand_default_params", "grand_last_error", "grand_reader_last_error",
                        "grand_default_cache_params", "grand_cache_last_error"):
            getattr(lib, name).restype = I32
    _lib = lib
    return lib


def _is_torch(x) -> bool:
    return type(x).__module__.startswith("torch")


def _ptr(x):
    """Data pointer of a numpy array or torch tensor (must be contiguous)."""
    if x is None:
        return None
    if _is_torch(x):
        assert x.is_contiguous()
        return x.data_ptr()
    assert x.flags["C_CONTIGUOUS"]
    return x.ctypes.data


def _np(x, dtype):
    return np.ascontiguousarray(x, dtype=dtype)


def params_from_config(cfg, device: int = 0, max_batch: int = 10000, rev_mode: int = REV_BATCH) -> Params:
    """grand_params from a workloads.IndexConfig."""
    p = Params()
    load_library().grand_default_params(ctypes.byref(p))
    p.algo = CAGRA if cfg.algo == "cagra" else VAMANA
    p.dtype = U8 if cfg.dtype == "u8" else F32
    p.metric = {"l2": L2, "ip": IP, "mips": MIPS}[cfg.metric]
    p.mips_norm = getattr(cfg, "mips_norm", 0.0)
    p.dim, p.capacity, p.R, p.L_build = cfg.dim, cfg.capacity, cfg.R, cfg.L_build
    p.P, p.c, p.k_repair, p.max_iters = cfg.P, cfg.c, cfg.k_repair, cfg.max_iters
    p.alpha = cfg.alpha
    p.prune_rule = ALPHA_ON_L2 if cfg.prune_rule == "alpha_on_l2" else ALPHA_ON_DIST
    p.cas_mode = CAS_RACING if cfg.cas_mode == "racing" else CAS_GROUPED
    p.rev_mode = rev_mode
    p.max_batch = max_batch
    p.device = device
    return p


class Reader:
    """grand_reader_create ... grand_reader_destroy: searches that may run on
    another host thread while the index is updated (ctypes releases the
    GIL during the call)."""

    def __init__(self, index: "GrandIndex", stream: Optional[int] = None):
        self.lib = index.lib
        self.index = index
        h = ctypes.c_void_p()
        rc = self.lib.grand_reader_create(index.h, None if stream is None else ctypes.c_void_p(stream),
                                          ctypes.byref(h))
        if rc != OK:
            raise GrandError(rc, index.last_error())
        self.h = h

    def search(self, queries, k: int, beam: int, out_ids=None, out_dists=None):
        if not _is_torch(queries):
            queries = _np(queries, self.index.np_dtype)
        nq = int(queries.shape[0])
        if out_ids is None:
            out_ids = np.zeros((nq, k), np.uint32)
            out_dists = np.zeros((nq, k), np.float32)
        rc = self.lib.grand_reader_search(self.h, _ptr(queries), nq, k, beam, _ptr(out_ids), _ptr(out_dists))
        if rc != OK:
            raise GrandError(rc, self.lib.grand_reader_last_error(self.h).decode())
        return out_ids, out_dists

    def close(self):
        if getattr(self, "h", None):
            self.lib.grand_reader_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class GrandIndex:
    """One index on one GPU (grand_create ... grand_destroy)."""

    def __init__(self, params: Params, stream: Optional[int] = None):
        self.lib = load_library()
        self.params = params
        if stream is not None:
            params.stream = stream
        h = ctypes.c_void_p()
        rc = self.lib.grand_create(ctypes.byref(params), ctypes.byref(h))
        if rc != OK:
            raise GrandError(rc, "grand_create failed")
        self.h = h
        self.np_dtype = np.uint8 if params.dtype == U8 else np.float32

    @classmethod
    def from_config(cls, cfg, **kw):
        stream = kw.pop("stream", None)
        return cls(params_from_config(cfg, **kw), stream=stream)

    def close(self):
        if getattr(self, "h", None):
            self.lib.grand_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc: int) -> int:
        if rc != OK:
            raise GrandError(rc, self.last_error())
        return rc

    def last_error(self) -> str:
        return self.lib.grand_last_error(self.h).decode()

    def set_stream(self, stream: int):
        self._check(self.lib.grand_set_stream(self.h, ctypes.c_void_p(stream)))

    def insert(self, ids, vecs, check: bool = True) -> int:
        if not _is_torch(ids):
            ids = _np(ids, np.uint32)
        if not _is_torch(vecs):
            vecs = _np(vecs, self.np_dtype)
        n = int(ids.shape[0])
        rc = self.lib.grand_insert_batch(self.h, _ptr(vecs), _ptr(ids), n)
        return self._check(rc) if check else rc

    def build_cagra(self, ids, vecs, init, knn: int, iters: int, sample: int, check: bool = True) -> int:
        """CAGRA graph construction over this empty CAGRA index; init is
        n x knn batch positions (the random initial neighbour lists)."""
        if not _is_torch(ids):
            ids = _np(ids, np.uint32)
        if not _is_torch(vecs):
            vecs = _np(vecs, self.np_dtype)
        if not _is_torch(init):
            init = _np(init, np.uint32)
        n = int(ids.shape[0])
        if tuple(init.shape) != (n, knn):
            raise ValueError("init must be n x knn")
        rc = self.lib.grand_build_cagra(self.h, _ptr(vecs), _ptr(ids), n, _ptr(init), knn, iters, sample)
        return self._check(rc) if check else rc

    def delete(self, ids, check: bool = True) -> int:
        if not _is_torch(ids):
            ids = _np(ids, np.uint32)
        rc = self.lib.grand_delete_batch(self.h, _ptr(ids), int(ids.shape[0]))
        return self._check(rc) if check else rc

    def search(self, queries, k: int, beam: int, out_ids=None, out_dists=None):
        """Returns (ids, dists); with out_* given (e.g. device tensors) the
        results are written there."""
        if not _is_torch(queries):
            queries = _np(queries, self.np_dtype)
        nq = int(queries.shape[0])
        if out_ids is None:
            out_ids = np.zeros((nq, k), np.uint32)
            out_dists = np.zeros((nq, k), np.float32)
        self._check(self.lib.grand_search(self.h, _ptr(queries), nq, k, beam, _ptr(out_ids), _ptr(out_dists)))
        return out_ids, out_dists

    def search_static(self, queries, k: int, beam: int, out_ids=None, out_dists=None, check: bool = True):
        """grand_search_static: the search without any device allocation.
        Returns (ids, dists), or the status code when check is False."""
        if not _is_torch(queries):
            queries = _np(queries, self.np_dtype)
        nq = int(queries.shape[0])
        if out_ids is None:
            out_ids = np.zeros((nq, k), np.uint32)
            out_dists = np.zeros((nq, k), np.float32)
        rc = self.lib.grand_search_static(self.h, _ptr(queries), nq, k, beam, _ptr(out_ids), _ptr(out_dists))
        if not check:
            return rc
        self._check(rc)
        return out_ids, out_dists

    def count_in_edges(self, ids, method: int):
        """grand_count_in_edges: (counts, GPU milliseconds of the method)."""
        ids = _np(ids, np.uint32)
        out = np.zeros(ids.shape[0], np.uint32)
        ms = ctypes.c_float(0.0)
        self._check(self.lib.grand_count_in_edges(self.h, _ptr(ids), ids.shape[0], method, _ptr(out),
                                                  ctypes.byref(ms)))
        return out, float(ms.value)

    def search_rc(self, queries, k: int, beam: int) -> int:
        q = _np(queries, self.np_dtype)
        ids = np.zeros((max(q.shape[0], 1), max(k, 1)), np.uint32)
        d = np.zeros_like(ids, dtype=np.float32)
        return self.lib.grand_search(self.h, _ptr(q), q.shape[0], k, beam, _ptr(ids), _ptr(d))

    def export(self, with_reverse: bool = False) -> dict:
        p = self.params
        cap, R = p.capacity, p.R
        adj = np.zeros((cap, R), np.uint32)
        deg = np.zeros(cap, np.uint32)
        act = np.zeros(cap, np.uint8)
        med = np.zeros(1, np.uint32)
        out = dict(adj=adj, deg=deg, active=act)
        if with_reverse:
            offs = np.zeros(cap + 1, np.uint32)
            nnz = np.zeros(1, np.uint64)
            self._check(self.lib.grand_export_graph(self.h, _ptr(adj), _ptr(deg), _ptr(act), _ptr(med), _ptr(offs),
                                                    None, _ptr(nnz)))
            srcs = np.zeros(max(int(nnz[0]), 1), np.uint32)
            self._check(self.lib.grand_export_graph(self.h, None, None, None, None, _ptr(offs), _ptr(srcs),
                                                    _ptr(nnz)))
            out["rev_offsets"] = offs
            out["rev_srcs"] = srcs[: int(nnz[0])]
        else:
            self._check(self.lib.grand_export_graph(self.h, _ptr(adj), _ptr(deg), _ptr(act), _ptr(med), None, None,
                                                    None))
        out["medoid"] = int(med[0])
        return out

    def import_graph(self, vecs, adj, deg, active, medoid: int):
        if not _is_torch(vecs):
            vecs = _np(vecs, self.np_dtype)
        self._check(self.lib.grand_import_graph(self.h, _ptr(vecs), _ptr(_np(adj, np.uint32)),
                                                _ptr(_np(deg, np.uint32)), _ptr(_np(active, np.uint8)),
                                                int(medoid)))

    def set_timing(self, on: bool = True):
        self._check(self.lib.grand_set_timing(self.h, 1 if on else 0))

    def set_counting(self, on: bool = True):
        self._check(self.lib.grand_set_counting(self.h, 1 if on else 0))

    def reset_stats(self):
        self._check(self.lib.grand_reset_stats(self.h))

    def stats(self) -> dict:
        s = Stats()
        self._check(self.lib.grand_stats(self.h, ctypes.byref(s), ctypes.sizeof(Stats)))
        arrays = ("search_hops", "search_evals", "search_distinct", "search_capped", "phase_ms", "phase_calls")
        out = {n: getattr(s, n) for n, _ in Stats._fields_ if n not in arrays}
        for i, w in enumerate(("insert", "delete", "query")):
            out[f"hops_{w}"] = s.search_hops[i]
            out[f"evals_{w}"] = s.search_evals[i]
            out[f"distinct_{w}"] = s.search_distinct[i]
            out[f"capped_{w}"] = s.search_capped[i]
        out["phase_ms"] = {n: s.phase_ms[i] for i, n in enumerate(PHASES)}
        out["phase_calls"] = {n: s.phase_calls[i] for i, n in enumerate(PHASES)}
        return out


class Sequences:
    """The sequences of cache calls (grand_seqs); holds the tensors it names.
    Calls do not change it.  n_tokens is None where each call's rows say."""

    def __init__(self, table, lens, q_start, n_tokens: Optional[int], max_q: int, max_k: int):
        self.tensors = (table, lens, q_start)
        self.n_seq, self.max_pages, self.n_tokens = table.shape[0], table.shape[1], n_tokens
        self.max_q, self.max_k = max_q, max_k
        self.c = Seqs(table.shape[0], n_tokens or 0, max_q, max_k, table.data_ptr(), table.stride(0), table.shape[1],
                      None if q_start is None else q_start.data_ptr(), lens.data_ptr())
        self.ref = ctypes.byref(self.c)


class Packed(NamedTuple):
    """Keys or values of a pool held in 4 bits (grand_packed): codes (pages,
    page_size, kv_heads, 16 * blocks) and scales (pages, page_size, kv_heads,
    blocks), uint8 views of any layout whose last axis is contiguous, rows of codes aligned to
    16 bytes; blocks = ceil(head_dim / 32)."""
    codes: Any
    scales: Any


class Cache:
    """The key/value-cache operators on one GPU (grand_cache_create ...
    grand_cache_destroy).  Every tensor is a torch tensor of that GPU; the
    calls enqueue work on the cache's stream and return.  Results that a call
    makes belong to that stream, as if allocated under it; memory that other
    streams read or write is ordered, and kept until then, by the caller.

    Queries, results, new keys and values are (tokens, heads, head_dim), pages
    (pages, page_size, kv_heads, head_dim) views of any layout whose rows are
    contiguous and 16-byte aligned, or two Packed.  Ids, lengths and starts are 32-bit
    integers; INVALID is -1 in an int32 tensor.  The operators serve: there is
    no backward pass, and results carry no gradient, whatever the arguments
    require."""

    def __init__(self, dtype: str = "bf16", q_heads: int = 32, kv_heads: int = 8, head_dim: int = 128, page_size: int = 16,
                 device: int = 0, stream: Optional[int] = None):
        import torch
        self.lib = load_library()
        p = CacheParams()
        self.lib.grand_default_cache_params(ctypes.byref(p))
        try:
            p.dtype, self.torch_dtype = {"bf16": (BF16, torch.bfloat16), "f16": (F16, torch.float16)}[dtype]
        except KeyError:
            raise ValueError(f"dtype must be 'bf16' or 'f16', not {dtype!r}") from None
        p.q_heads, p.kv_heads, p.head_dim, p.page_size, p.device = q_heads, kv_heads, head_dim, page_size, device
        p.stream = stream
        self.params = p
        h = ctypes.c_void_p()
        rc = self.lib.grand_cache_create(ctypes.byref(p), ctypes.byref(h))
        if rc != OK:
            raise GrandError(rc, "grand_cache_create failed")
        self.h = h
        self._torch, self._device = torch, torch.device("cuda", device)
        self._current = torch._C._cuda_getCurrentRawStream  # 0.1 us, a Stream object 1
        self._own_stream(stream)
        self._q, self._kv, self._dim, self._page = q_heads, kv_heads, head_dim, page_size
        self._page_shape = (page_size, kv_heads, head_dim)
        blocks = -(-head_dim // 32)
        self._code_shape, self._scale_shape = (page_size, kv_heads, 16 * blocks), (page_size, kv_heads, blocks)
        self._int = (torch.int32, torch.uint32)
        # argument structs, filled anew by every call
        self._args = {n: Rows() for n in ("q", "out", "k", "v", "prior")}
        self._args.update(pages=Pages(), packed=PackedPages(), weights=Weights(), weights_out=Weights())
        self._refs = {n: ctypes.byref(a) for n, a in self._args.items()}
        self._seqs = Seqs()
        self._seqs_ref, self._seqs_at = ctypes.byref(self._seqs), ctypes.addressof(self._seqs)

    def close(self):
        if getattr(self, "h", None):
            self.lib.grand_cache_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc: int) -> int:
        if rc != OK:
            raise GrandError(rc, self.last_error())
        return rc

    def last_error(self) -> str:
        return self.lib.grand_cache_last_error(self.h).decode()

    def set_stream(self, stream: int):
        self._check(self.lib.grand_cache_set_stream(self.h, ctypes.c_void_p(stream)))
        self._own_stream(stream)

    def _own_stream(self, stream):
        self._raw = stream or 0
        cuda = self._torch.cuda
        self._stream = cuda.ExternalStream(stream, device=self._device) if stream else cuda.default_stream(self._device)

    def check(self):
        """Waits for the stream; raises if a kernel found an id, a length or
        a start out of range since the last check."""
        self._check(self.lib.grand_cache_check(self.h))

    # ------------------------------------------------------------ arguments
    def _ints(self, name, x, shape):
        if x.dtype not in self._int or not x.is_cuda or x.shape != shape:
            raise ValueError(f"{name} must be a 32-bit integer tensor {shape} on the GPU")
        if x.shape and x.shape[-1] > 1 and x.stride(-1) != 1:
            raise ValueError(f"{name} must be contiguous along its last axis")

    def _rows(self, name, x, heads, tokens):
        stride = x.stride()
        if x.dtype != self.torch_dtype or x.shape != (tokens, heads, self._dim) or not x.is_cuda or stride[2] != 1:
            raise ValueError(f"{name} must be ({tokens}, {heads}, {self._dim}) {self.torch_dtype} on the GPU, contiguous "
                             "along its last axis")
        r = self._args[name]
        r.p, r.token_stride, r.head_stride = x.data_ptr(), stride[0], stride[1]
        return self._refs[name]

    def _packed(self, k, v):
        if not isinstance(v, Packed):
            raise ValueError("k_pages and v_pages must both be Packed")
        g = self._args["packed"]
        g.k, g.v, pages, (g.page_stride, g.slot_stride, g.head_stride) = self._packed_part("codes", k.codes, v.codes, self._code_shape)
        g.k_scales, g.v_scales, g.n_pages, (g.scale_page_stride, g.scale_slot_stride, g.scale_head_stride) = self._packed_part(
            "scales", k.scales, v.scales, self._scale_shape)
        if pages != g.n_pages:
            raise ValueError("codes and scales must have as many pages")
        return self._refs["packed"]

    def _packed_part(self, what, k, v, want):
        shape, stride, u8 = k.shape, k.stride(), self._torch.uint8
        if (k.dtype != u8 or v.dtype != u8 or shape[1:] != want or v.shape != shape or not k.is_cuda or not v.is_cuda
                or (want[2] > 1 and (stride[3] != 1 or v.stride(3) != 1))):
            raise ValueError(f"{what} of k_pages and v_pages must be (pages, {', '.join(map(str, want))}) uint8 on the GPU, contiguous "
                             "along their last axis")
        if v.stride() != stride and any(n > 1 and a != b for n, a, b in zip(shape, stride, v.stride())):
            raise ValueError(f"{what} of k_pages and v_pages must have the same strides")
        return k.data_ptr(), v.data_ptr(), shape[0], stride[:3]

    def _pages(self, k, v):
        if isinstance(v, Packed):
            raise ValueError("k_pages and v_pages must both be Packed")
        shape, stride = k.shape, k.stride()
        if (k.dtype != self.torch_dtype or v.dtype != self.torch_dtype or shape[1:] != self._page_shape or v.shape != shape
                or not k.is_cuda or not v.is_cuda or stride[3] != 1):
            raise ValueError(f"k_pages and v_pages must be (pages, {self._page}, {self._kv}, {self._dim}) {self.torch_dtype} on the "
                             "GPU, contiguous along their last axis")
        if v.stride() != stride and any(n > 1 and a != b for n, a, b in zip(shape, stride, v.stride())):
            raise ValueError("k_pages and v_pages must have the same strides")
        g = self._args["pages"]
        g.k, g.v, g.n_pages = k.data_ptr(), v.data_ptr(), shape[0]
        g.page_stride, g.slot_stride, g.head_stride = stride[:3]
        return self._refs["pages"]

    def _weights(self, name, w, n_seq, least, heads=None):
        if (w.dtype != self._torch.float32 or w.dim() != 3 or w.shape[0] != n_seq or not w.is_cuda or w.shape[2] < least
                or (heads is not None and w.shape[1] != heads) or (w.shape[2] > 1 and w.stride(2) != 1)):
            raise ValueError(f"{name} must be ({n_seq}, heads, at least {least}) float32 on the GPU, contiguous along its last axis")
        a = self._args[name]
        a.p, a.seq_stride, a.head_stride = w.data_ptr(), w.stride(0), w.stride(1)
        return self._refs[name]

    def _empty(self, shape, dtype):
        """Memory for a result: of the cache's stream, as memory that the current
        one has given back may still be in use there."""
        if self._current(self._device.index) == self._raw:
            return self._torch.empty(shape, dtype=dtype, device=self._device)
        with self._torch.cuda.stream(self._stream):
            return self._torch.empty(shape, dtype=dtype, device=self._device)

    def _out(self, tokens):
        return self._empty((tokens, self._q, self._dim), self.torch_dtype)

    def _lse(self, lse, tokens):
        if lse is None:
            return self._empty((tokens, self._q), self._torch.float32)
        if lse.dtype != self._torch.float32 or lse.shape != (tokens, self._q) or not lse.is_contiguous() or not lse.is_cuda:
            raise ValueError(f"lse must be a contiguous ({tokens}, {self._q}) float32 tensor on the GPU")
        return lse

    # ------------------------------------------------------------ operators
    def sequences(self, table, lens, q_start=None, n_tokens: Optional[int] = None, max_q: int = 1,
                  max_k: Optional[int] = None) -> Sequences:
        """Describes the sequences of the calls that follow: table (sequences,
        pages) page ids, lens cached tokens (new ones included), q_start
        (sequences + 1) the new tokens' rows, or None for one each; max_q and
        max_k bound new and cached tokens of a sequence.  n_tokens is the number
        of rows that q, k and v must have; if not given, with q_start, it is
        that of each call's rows."""
        n = int(lens.shape[0])
        self._ints("lens", lens, (n,))
        if table.dim() != 2 or table.shape[0] != n:
            raise ValueError("table must have a row for every sequence")
        self._ints("table", table, tuple(table.shape))
        if q_start is not None:
            self._ints("q_start", q_start, (n + 1,))
        if max_k is None:
            max_k = int(table.shape[1]) * self._page
        if n_tokens is not None and (n_tokens < 0 or (q_start is None and n_tokens != n)):
            raise ValueError("n_tokens must be the number of sequences without q_start, and not negative")
        return Sequences(table, lens, q_start, n if q_start is None else n_tokens, max_q, max_k)

    def _tokens(self, s: Sequences, rows):
        """The rows of a call and its grand_seqs: the description itself, or a
        copy with their number."""
        if s.n_tokens is not None:
            return s.n_tokens, s.ref
        n = int(rows.shape[0])
        ctypes.memmove(self._seqs_at, s.ref, ctypes.sizeof(Seqs))
        self._seqs.n_tokens = n
        return n, self._seqs_ref

    def packed_pages(self, n_pages: int):
        """Keys and values of a new pool held in 4 bits: two Packed of zeros,
        heads outermost in a page."""
        def zeros(shape):
            with self._torch.cuda.stream(self._stream):
                return self._torch.zeros((n_pages, shape[1], shape[0], shape[2]), dtype=self._torch.uint8, device=self._device).transpose(1, 2)
        return tuple(Packed(zeros(self._code_shape), zeros(self._scale_shape)) for _ in range(2))

    def append(self, seqs: Sequences, k, v, k_pages, v_pages):
        """grand_cache_append, grand_cache_append_packed: the new tokens' keys and values go into their pages."""
        n, ref = self._tokens(seqs, k)
        rk, rv = self._rows("k", k, self._kv, n), self._rows("v", v, self._kv, n)
        if isinstance(k_pages, Packed):
            self._check(self.lib.grand_cache_append_packed(self.h, ref, rk, rv, self._packed(k_pages, v_pages)))
        else:
            self._check(self.lib.grand_cache_append(self.h, ref, rk, rv, self._pages(k_pages, v_pages)))

    def attend(self, seqs: Sequences, q, k_pages, v_pages, scale: Optional[float] = None, causal: bool = True, window: int = 0,
               weights=None, weights_out=None, out=None, lse=None, sinks: int = 0):
        """grand_cache_attend, grand_cache_attend_sinks, grand_cache_attend_packed:
        (out, lse), and with weights (sequences, kv_heads, at least max_k)
        also weights_out (weights itself if not given).  With a window every
        row sees the first `sinks` tokens too."""
        if not 0 <= sinks < 1 << 32:
            raise ValueError("sinks must be a number of tokens")
        n, ref = self._tokens(seqs, q)
        rq = self._rows("q", q, self._q, n)
        if out is None:
            out = self._out(n)
        ro = self._rows("out", out, self._q, n)
        lse = self._lse(lse, n)
        wi = wo = None
        if weights is not None:
            weights_out = weights if weights_out is None else weights_out
            wi = self._weights("weights", weights, seqs.n_seq, seqs.max_k, self._kv)
            wo = self._weights("weights_out", weights_out, seqs.n_seq, seqs.max_k, self._kv)
        elif weights_out is not None:
            raise ValueError("weights_out needs weights")
        if isinstance(k_pages, Packed):
            call, pages = self.lib.grand_cache_attend_packed, self._packed(k_pages, v_pages)
        else:
            call, pages = self.lib.grand_cache_attend_sinks, self._pages(k_pages, v_pages)
        self._check(call(self.h, ref, rq, pages, self._dim ** -0.5 if scale is None else scale, 1 if causal else 0, window, sinks, ro,
                         lse.data_ptr(), wi, wo))
        return (out, lse) if weights is None else (out, lse, weights_out)

    def attend_ids(self, q, k_pages, v_pages, ids, scale: Optional[float] = None, prior=None, out=None, lse=None):
        """grand_cache_attend_ids(_packed): one token per sequence over ids (sequences,
        q_heads, k), e.g. the results of GrandIndex.search; prior: (out, lse)
        of the same rows over other tokens.  Returns (out, lse)."""
        n = int(q.shape[0])
        rq = self._rows("q", q, self._q, n)
        if ids.dim() != 3:
            raise ValueError("ids must be (sequences, q_heads, k)")
        k, stride = int(ids.shape[2]), ids.stride()
        self._ints("ids", ids, (n, self._q, k))
        if out is None:
            out = self._out(n)
        ro = self._rows("out", out, self._q, n)
        lse = self._lse(lse, n)
        rp = zp = None
        if prior is not None:
            rp = self._rows("prior", prior[0], self._q, n)
            zp = self._lse(prior[1], n).data_ptr()
        if isinstance(k_pages, Packed):
            call, pages = self.lib.grand_cache_attend_ids_packed, self._packed(k_pages, v_pages)
        else:
            call, pages = self.lib.grand_cache_attend_ids, self._pages(k_pages, v_pages)
        self._check(call(
            self.h, n, rq, pages, ids.data_ptr(), k, stride[0], stride[1],
            self._dim ** -0.5 if scale is None else scale, rp, zp, ro, lse.data_ptr()))
        return out, lse

    def evict(self, seqs: Sequences, weights, budget, sinks: int = 0, recent: int = 0):
        """grand_cache_evict: (table, weights, lens, freed, n_freed), the kept
        pages of each sequence and the freed ones; budget is in pages."""
        n, pages = seqs.n_seq, seqs.max_pages
        wi = self._weights("weights", weights, n, seqs.max_k)
        self._ints("budget", budget, (n,))
        heads, cap = weights.shape[1], weights.shape[2]
        empty, i32 = self._empty, self._torch.int32
        table, freed = empty((n, pages), i32), empty((n, pages), i32)
        lens, n_freed = empty(n, i32), empty(n, i32)
        new = empty((n, heads, cap), self._torch.float32)
        wo = self._weights("weights_out", new, n, cap)
        self._check(self.lib.grand_cache_evict(self.h, seqs.ref, heads, cap, wi, budget.data_ptr(), sinks, recent, table.data_ptr(),
                                               wo, lens.data_ptr(), freed.data_ptr(), n_freed.data_ptr()))
        return table, new, lens, freed, n_freed

    def read(self, slots, k_pages, v_pages):
        """grand_packed_read: (keys, values), rows of listed slots as packed
        pages hold them; INVALID entries are rows of zeros."""
        n = int(slots.shape[0])
        self._ints("slots", slots, (n,))
        k, v = self._empty((n, self._kv, self._dim), self.torch_dtype), self._empty((n, self._kv, self._dim), self.torch_dtype)
        self._check(self.lib.grand_packed_read(self.h, n, slots.data_ptr(), self._packed(k_pages, v_pages), self._rows("k", k, self._kv, n),
                                               self._rows("v", v, self._kv, n)))
        return k, v

    # ------------------------------------------------------------ shared pages
    def _counts(self, refs, refs_out):
        """refs, and where they go: themselves if no other memory is given."""
        if refs.dim() != 1:
            raise ValueError("refs must have one entry for each page")
        refs_out = refs if refs_out is None else refs_out
        for name, x in (("refs", refs), ("refs_out", refs_out)):
            self._ints(name, x, refs.shape)
        return refs_out

    def fork(self, seqs: Sequences, parents, refs, drop: bool = False, refs_out=None):
        """grand_pages_fork: (table, lens, refs_out) of new sequences that go on
        from the rows `parents`; drop: the old ones are given up."""
        n = int(parents.shape[0])
        self._ints("parents", parents, (n,))
        refs_out = self._counts(refs, refs_out)
        table, lens = self._empty((n, seqs.max_pages), self._torch.int32), self._empty(n, self._torch.int32)
        self._check(self.lib.grand_pages_fork(self.h, seqs.ref, n, parents.data_ptr(), 1 if drop else 0, refs.shape[0], refs.data_ptr(),
                                              refs_out.data_ptr(), table.data_ptr(), lens.data_ptr()))
        return table, lens, refs_out

    def grow(self, seqs: Sequences, n_new, refs, refs_out=None):
        """grand_pages_grow: pages for n_new more tokens a sequence, in place in
        the table and the lens that seqs was made of: (table, lens, src, dst),
        src and dst for copy_pages."""
        n = seqs.n_seq
        self._ints("n_new", n_new, (n,))
        refs_out = self._counts(refs, refs_out)
        table, lens, _ = seqs.tensors
        src, dst = self._empty(n, self._torch.int32), self._empty(n, self._torch.int32)
        self._check(self.lib.grand_pages_grow(self.h, seqs.ref, n_new.data_ptr(), refs.shape[0], refs.data_ptr(), refs_out.data_ptr(),
                                              table.data_ptr(), lens.data_ptr(), src.data_ptr(), dst.data_ptr()))
        return table, lens, src, dst

    def release(self, ids, refs, counts=None, tokens: bool = False, refs_out=None):
        """grand_pages_release: (refs_out, freed, n_freed).  ids (rows, width):
        tables of ended sequences (counts their lens, with tokens) or the freed
        pages of evict (counts its n_freed), INVALID entries passed over."""
        if ids.dim() != 2:
            raise ValueError("ids must be (rows, width)")
        rows, width = int(ids.shape[0]), int(ids.shape[1])
        self._ints("ids", ids, (rows, width))
        if counts is not None:
            self._ints("counts", counts, (rows,))
        refs_out = self._counts(refs, refs_out)
        freed, n_freed = self._empty(min(refs.shape[0], rows * width), self._torch.int32), self._empty(1, self._torch.int32)
        self._check(self.lib.grand_pages_release(self.h, rows, width, ids.data_ptr(), ids.stride(0), None if counts is None else counts.data_ptr(),
                                                 1 if tokens else 0, refs.shape[0], refs.data_ptr(), refs_out.data_ptr(), freed.data_ptr(),
                                                 n_freed.data_ptr()))
        return refs_out, freed, n_freed

    def compact(self, seqs: Sequences, refs, refs_out=None):
        """grand_pages_compact: (table, refs_out, src, dst, n_moves), src and dst
        for copy_pages."""
        refs_out = self._counts(refs, refs_out)
        n, empty, i32 = int(refs.shape[0]), self._empty, self._torch.int32
        table, src, dst, moves = empty((seqs.n_seq, seqs.max_pages), i32), empty(n, i32), empty(n, i32), empty(1, i32)
        self._check(self.lib.grand_pages_compact(self.h, seqs.ref, n, refs.data_ptr(), refs_out.data_ptr(), table.data_ptr(), src.data_ptr(),
                                                 dst.data_ptr(), moves.data_ptr()))
        return table, refs_out, src, dst, moves

    def copy_pages(self, k_pages, v_pages, src, dst):
        """grand_pages_copy, grand_packed_copy: pages src go to pages dst, keys and
        values; INVALID entries are passed over."""
        n = int(src.shape[0])
        self._ints("src", src, (n,))
        self._ints("dst", dst, (n,))
        if isinstance(k_pages, Packed):
            call, pages = self.lib.grand_packed_copy, self._packed(k_pages, v_pages)
        else:
            call, pages = self.lib.grand_pages_copy, self._pages(k_pages, v_pages)
        self._check(call(self.h, n, src.data_ptr(), dst.data_ptr(), pages))
