"""ctypes binding of libpancake.so: the C-ABI entry points under their own names.

Argument marshalling only.  Every step of search / insert / build runs in the HIP
kernels behind the C ABI; PyTorch is used for device memory (tensors own the
buffers, including arenas) and for the current HIP stream.  There is no CPU
fallback: if the library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libpancake.so")

PK_METRIC_IP, PK_METRIC_L2 = 0, 1
PK_F32, PK_F16, PK_BF16, PK_I8, PK_F8, PK_F4 = 0, 1, 2, 3, 4, 6
PK_OK = 0
PK_ERR_INVALID_ARG, PK_ERR_BAD_HANDLE, PK_ERR_DIM_MISMATCH, PK_ERR_NOMEM, PK_ERR_HIP, PK_ERR_UNSUPPORTED = (
    -1, -2, -3, -4, -5, -6)
PK_ERR_WORKSPACE = -7
PK_NOALLOC_WORKSPACE_BYTES = 64 << 20

EXPORTS = ["pk_workspace_reserve", "pk_index_set_emit_cap", "pk_index_set_tile_cap", "pk_index_set_values_cap", "pk_search_noalloc", "pk_search_noalloc_bytes", "pk_search_levels", "pk_search_union", "pk_insert_multi", "pk_delete", "pk_index_split", "pk_index_centroids", "pk_list_ids", "pk_arena_bytes", "pk_index_build", "pk_index_add_arena", "pk_index_compact", "pk_kmeans", "pk_insert", "pk_insert_assigned", "pk_search",
           "pk_search_multi", "pk_coarse", "pk_scan_probes", "pk_index_stats", "pk_list_lengths", "pk_profile_begin",
           "pk_profile_end", "pk_index_free", "pk_kv_arena_bytes", "pk_kv_create", "pk_kv_free", "pk_kv_append", "pk_kv_read",
           "pk_kv_bounds", "pk_kv_attend", "pk_kv_attend_scored", "pk_kv_select", "pk_kv_attend_blocks", "pk_kv_pool_bytes", "pk_kv_pool_create", "pk_kv_pool_free", "pk_kv_pool_clear",
           "pk_kv_pool_adopt", "pk_kv_pool_grant", "pk_kv_pool_fork", "pk_kv_pool_release", "pk_kv_pool_compact", "pk_kv_pool_counts", "pk_kv_copy", "pk_strerror"]


class pk_config(C.Structure):
    _fields_ = [("d", C.c_int32), ("nlist", C.c_int32), ("metric", C.c_int32), ("storage", C.c_int32),
                ("page_vecs", C.c_int32), ("max_delta_pages", C.c_int32)]


class pk_stats(C.Structure):
    _fields_ = [("n_total", C.c_int64), ("n_inserted", C.c_int64), ("pages_total", C.c_int64),
                ("pages_used", C.c_int64), ("arena_bytes", C.c_int64), ("workspace_bytes", C.c_int64),
                ("workspace_grows", C.c_int64),
                ("max_list_len", C.c_int64), ("device_error", C.c_int32), ("n_arenas", C.c_int32)]


class pk_profile(C.Structure):
    _fields_ = [("launches", C.c_int32), ("coarse_ms", C.c_float), ("worklist_ms", C.c_float),
                ("scan_ms", C.c_float), ("select_ms", C.c_float), ("scanned_rows", C.c_int64),
                ("candidates", C.c_int64), ("tiles", C.c_int64), ("emitted", C.c_int64),
                ("overflowed", C.c_int64), ("max_emitted", C.c_int64), ("scan_hot_ms", C.c_float)]


class pk_kv_config(C.Structure):
    _fields_ = [("n_pages", C.c_int64), ("n_heads", C.c_int32), ("head_dim", C.c_int32), ("page_tokens", C.c_int32), ("storage", C.c_int32)]


class pk_kv_batch(C.Structure):
    _fields_ = [("tables", C.c_void_p), ("offsets", C.c_void_p), ("lens", C.c_void_p), ("table_stride", C.c_int64), ("n_seqs", C.c_int32), ("n_cols", C.c_int32),
                ("n_tokens", C.c_int32), ("max_new", C.c_int32), ("max_len", C.c_int32)]


class pk_rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64), ("dtype", C.c_int32)]


class pk_kv_scores(C.Structure):
    _fields_ = [("cap", C.c_float), ("slopes", C.c_void_p), ("starts", C.c_void_p), ("prefix", C.c_void_p)]


class pk_kv_tables(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride", C.c_int64), ("n_rows", C.c_int32), ("n_cols", C.c_int32)]


class PancakeError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {strerror(status)} ({status})")


_lib = None


def lib():
    """The loaded library; raises if it has not been built (python -m paper_2602_21477_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} is missing: build it with `python -m paper_2602_21477_amd.build`")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
        L.pk_arena_bytes.restype = C.c_size_t
        L.pk_arena_bytes.argtypes = [C.POINTER(pk_config), i64, i64]
        L.pk_index_build.argtypes = [C.POINTER(pk_config), vp, vp, vp, i64, vp, C.c_size_t, vp, C.POINTER(vp)]
        L.pk_index_add_arena.argtypes = [vp, vp, C.c_size_t, vp]
        L.pk_index_compact.argtypes = [vp, vp, C.c_size_t, vp]
        L.pk_index_split.argtypes = [vp, vp, C.c_size_t, i64, i32, C.POINTER(i32), vp]
        L.pk_index_centroids.argtypes = [vp, vp, vp]
        L.pk_list_ids.argtypes = [vp, i32, vp, i64, vp]
        L.pk_kmeans.argtypes = [vp, i64, i32, i32, i32, vp, vp, C.POINTER(C.c_double), vp]
        L.pk_insert.argtypes = [vp, vp, vp, i64, vp, vp]
        L.pk_insert_assigned.argtypes = [vp, vp, vp, i64, vp, vp]
        L.pk_insert_multi.argtypes = [C.POINTER(vp), i32, C.POINTER(i64), vp, vp, vp, vp]
        L.pk_delete.argtypes = [vp, vp, i64, C.POINTER(i64), vp]
        L.pk_search.argtypes = [vp, vp, i64, i32, i32, vp, vp, vp]
        L.pk_workspace_reserve.argtypes = [C.POINTER(vp), i32, i64, i32, i32, i64, vp]
        L.pk_index_set_emit_cap.argtypes = [vp, i32]
        L.pk_index_set_tile_cap.argtypes = [vp, i32]
        L.pk_index_set_values_cap.argtypes = [vp, i64]
        L.pk_search_noalloc.argtypes = [vp, vp, i64, i32, i32, vp, vp, vp]
        L.pk_search_noalloc_bytes.restype = C.c_size_t
        L.pk_search_noalloc_bytes.argtypes = [vp, i64, i32, i32]
        L.pk_search_multi.argtypes = [C.POINTER(vp), i32, C.POINTER(i64), vp, i32, i32, vp, vp, vp]
        L.pk_search_union.argtypes = [C.POINTER(vp), i32, vp, i64, i32, i32, vp, vp, vp, vp]
        L.pk_search_levels.argtypes = [C.POINTER(vp), i32, C.POINTER(i32), vp, i64, i32, vp, vp, vp, vp, vp]
        L.pk_coarse.argtypes = [vp, vp, i64, i32, vp, vp]
        L.pk_scan_probes.argtypes = [vp, vp, i64, i32, i32, vp, vp, vp, vp]
        L.pk_index_stats.argtypes = [vp, C.POINTER(pk_stats), vp]
        L.pk_list_lengths.argtypes = [vp, vp, vp]
        L.pk_profile_begin.argtypes = [vp, vp]
        L.pk_profile_end.argtypes = [vp, C.POINTER(pk_profile), vp]
        L.pk_index_free.argtypes = [vp]
        L.pk_kv_arena_bytes.restype = C.c_size_t
        L.pk_kv_arena_bytes.argtypes = [C.POINTER(pk_kv_config)]
        L.pk_kv_create.argtypes = [C.POINTER(pk_kv_config), vp, C.c_size_t, C.POINTER(vp)]
        L.pk_kv_free.argtypes = [vp]
        L.pk_kv_append.argtypes = [vp, C.POINTER(pk_kv_batch), C.POINTER(pk_rows), C.POINTER(pk_rows), vp]
        L.pk_kv_read.argtypes = [vp, C.POINTER(pk_kv_batch), vp, vp, i32, vp]
        L.pk_kv_bounds.argtypes = [vp, vp, i64, vp, vp, vp]
        L.pk_kv_attend.argtypes = [vp, C.POINTER(pk_kv_batch), C.POINTER(pk_rows), i32, C.c_float, i32, vp, vp, vp]
        L.pk_kv_attend_scored.argtypes = [vp, C.POINTER(pk_kv_batch), C.POINTER(pk_rows), i32, C.c_float, i32, C.POINTER(pk_kv_scores), vp, vp, vp]
        L.pk_kv_select.argtypes = [vp, C.POINTER(pk_kv_batch), C.POINTER(pk_rows), i32, i32, i32, i32, vp, vp]
        L.pk_kv_attend_blocks.argtypes = [vp, C.POINTER(pk_kv_batch), C.POINTER(pk_rows), i32, C.c_float, vp, i32, vp, vp, vp]
        tables = C.POINTER(pk_kv_tables)
        L.pk_kv_pool_bytes.restype = C.c_size_t
        L.pk_kv_pool_bytes.argtypes = [C.POINTER(pk_kv_config)]
        L.pk_kv_pool_create.argtypes = [vp, vp, C.c_size_t, C.POINTER(vp)]
        L.pk_kv_pool_free.argtypes = [vp]
        L.pk_kv_pool_clear.argtypes = [vp, vp]
        L.pk_kv_pool_adopt.argtypes = [vp, tables, vp]
        L.pk_kv_pool_grant.argtypes = [vp, C.POINTER(pk_kv_batch), vp, vp]
        L.pk_kv_pool_fork.argtypes = [vp, tables, vp, vp, vp, i32, vp]
        L.pk_kv_pool_release.argtypes = [vp, tables, vp, vp, i32, vp]
        L.pk_kv_pool_compact.argtypes = [vp, vp, tables, tables, vp, vp]
        L.pk_kv_pool_counts.argtypes = [vp, vp, vp]
        L.pk_kv_copy.argtypes = [vp, vp, vp, vp, i64, vp]
        L.pk_strerror.restype = C.c_char_p
        L.pk_strerror.argtypes = [C.c_int]
        for name in EXPORTS:
            if name not in ("pk_arena_bytes", "pk_strerror", "pk_search_noalloc_bytes", "pk_kv_arena_bytes", "pk_kv_pool_bytes"):
                getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


def strerror(status: int) -> str:
    return lib().pk_strerror(int(status)).decode()


def _check(status: int, what: str):
    if status != PK_OK:
        raise PancakeError(status, what)


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _dev(t, dtype, what):
    if t is None:
        return None
    if not (t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise ValueError(f"{what}: need a contiguous {dtype} CUDA tensor")
    return t.data_ptr()


def pk_arena_bytes(cfg: pk_config, n: int, n_insert_reserve: int) -> int:
    return int(lib().pk_arena_bytes(C.byref(cfg), int(n), int(n_insert_reserve)))


def pk_index_build(cfg: pk_config, centroids, vectors, ids, arena) -> int:
    """Returns the handle (an integer).  `arena` is a uint8 CUDA tensor the caller keeps alive."""
    n = 0 if vectors is None else vectors.shape[0]
    h = C.c_void_p()
    rc = lib().pk_index_build(C.byref(cfg), _dev(centroids, torch.float32, "centroids"),
                              _dev(vectors, torch.float32, "vectors"), _dev(ids, torch.int64, "ids"), n,
                              _dev(arena, torch.uint8, "arena"), arena.numel(), _stream(), C.byref(h))
    _check(rc, "pk_index_build")
    return h.value


def pk_index_add_arena(handle: int, arena):
    _check(lib().pk_index_add_arena(handle, _dev(arena, torch.uint8, "arena"), arena.numel(), _stream()),
           "pk_index_add_arena")


def pk_kmeans(vectors, centroids, iters: int, assign_out=None):
    """Lloyd iterations in place on `centroids`; returns the per-iteration objective (host floats)."""
    n, d = vectors.shape
    inertia = (C.c_double * iters)()
    _check(lib().pk_kmeans(_dev(vectors, torch.float32, "vectors"), n, d, centroids.shape[0], iters,
                           _dev(centroids, torch.float32, "centroids"), _dev(assign_out, torch.int32, "assign_out"),
                           inertia, _stream()), "pk_kmeans")
    return [float(v) for v in inertia]


def pk_insert_multi(handles, v_offsets, vectors, ids=None, assigned_lists=None):
    hs = (C.c_void_p * len(handles))(*handles)
    offs = (C.c_int64 * len(v_offsets))(*[int(v) for v in v_offsets])
    _check(lib().pk_insert_multi(hs, len(handles), offs, _dev(vectors, torch.float32, "vectors"),
                                 _dev(ids, torch.int64, "ids"), _dev(assigned_lists, torch.int32, "assigned_lists"),
                                 _stream()), "pk_insert_multi")


def pk_index_split(handle: int, arena, threshold: int, iters: int) -> int:
    n = C.c_int32(0)
    _check(lib().pk_index_split(handle, _dev(arena, torch.uint8, "arena"), arena.numel(), threshold, iters,
                                C.byref(n), _stream()), "pk_index_split")
    return int(n.value)


def pk_index_centroids(handle: int, out):
    _check(lib().pk_index_centroids(handle, _dev(out, torch.float32, "out"), _stream()), "pk_index_centroids")


def pk_list_ids(handle: int, lst: int, out):
    _check(lib().pk_list_ids(handle, lst, _dev(out, torch.int64, "out"), out.numel(), _stream()), "pk_list_ids")


def pk_delete(handle: int, ids) -> int:
    n = C.c_int64(0)
    _check(lib().pk_delete(handle, _dev(ids, torch.int64, "ids"), ids.shape[0], C.byref(n), _stream()), "pk_delete")
    return int(n.value)


def pk_index_compact(handle: int, arena):
    _check(lib().pk_index_compact(handle, _dev(arena, torch.uint8, "arena"), arena.numel(), _stream()),
           "pk_index_compact")


def pk_insert(handle: int, vectors, ids=None, assigned_lists=None):
    _check(lib().pk_insert(handle, _dev(vectors, torch.float32, "vectors"), _dev(ids, torch.int64, "ids"),
                           vectors.shape[0], _dev(assigned_lists, torch.int32, "assigned_lists"), _stream()),
           "pk_insert")


def pk_insert_assigned(handle: int, vectors, ids, lists):
    _check(lib().pk_insert_assigned(handle, _dev(vectors, torch.float32, "vectors"), _dev(ids, torch.int64, "ids"),
                                    vectors.shape[0], _dev(lists, torch.int32, "lists"), _stream()),
           "pk_insert_assigned")


def pk_search(handle: int, queries, k: int, nprobe: int, out_ids, out_dist):
    _check(lib().pk_search(handle, _dev(queries, torch.float32, "queries"), queries.shape[0], k, nprobe,
                           _dev(out_ids, torch.int64, "out_ids"), _dev(out_dist, torch.float32, "out_dist"),
                           _stream()), "pk_search")


def pk_workspace_reserve(handles, nq_max: int, k_max: int, nprobe_max: int, inserts_ahead: int = 0):
    hs = (C.c_void_p * len(handles))(*handles)
    _check(lib().pk_workspace_reserve(hs, len(handles), int(nq_max), int(k_max), int(nprobe_max), int(inserts_ahead),
                                      _stream()), "pk_workspace_reserve")


def pk_index_set_emit_cap(handle: int, entries: int):
    _check(lib().pk_index_set_emit_cap(handle, int(entries)), "pk_index_set_emit_cap")


def pk_index_set_tile_cap(handle: int, tiles: int):
    _check(lib().pk_index_set_tile_cap(handle, int(tiles)), "pk_index_set_tile_cap")


def pk_index_set_values_cap(handle: int, nbytes: int):
    _check(lib().pk_index_set_values_cap(handle, int(nbytes)), "pk_index_set_values_cap")


def pk_search_noalloc(handle: int, queries, k: int, nprobe: int, out_ids, out_dist):
    _check(lib().pk_search_noalloc(handle, _dev(queries, torch.float32, "queries"), queries.shape[0], k, nprobe,
                                   _dev(out_ids, torch.int64, "out_ids"), _dev(out_dist, torch.float32, "out_dist"),
                                   _stream()), "pk_search_noalloc")


def pk_search_noalloc_bytes(handle: int, nq: int, k: int, nprobe: int) -> int:
    return int(lib().pk_search_noalloc_bytes(handle, int(nq), int(k), int(nprobe)))


def pk_search_multi(handles, q_offsets, queries, k: int, nprobe: int, out_ids, out_dist):
    n = len(handles)
    hs = (C.c_void_p * n)(*handles)
    offs = (C.c_int64 * (n + 1))(*[int(o) for o in q_offsets])
    _check(lib().pk_search_multi(hs, n, offs, _dev(queries, torch.float32, "queries"), k, nprobe,
                                 _dev(out_ids, torch.int64, "out_ids"), _dev(out_dist, torch.float32, "out_dist"),
                                 _stream()), "pk_search_multi")


def pk_coarse(handle: int, queries, nprobe: int, out_probes):
    _check(lib().pk_coarse(handle, _dev(queries, torch.float32, "queries"), queries.shape[0], nprobe,
                           _dev(out_probes, torch.int32, "out_probes"), _stream()), "pk_coarse")


def pk_scan_probes(handle: int, queries, k: int, probes, out_ids, out_dist):
    _check(lib().pk_scan_probes(handle, _dev(queries, torch.float32, "queries"), queries.shape[0], k,
                                probes.shape[1], _dev(probes, torch.int32, "probes"),
                                _dev(out_ids, torch.int64, "out_ids"), _dev(out_dist, torch.float32, "out_dist"),
                                _stream()), "pk_scan_probes")


def pk_index_stats(handle: int) -> pk_stats:
    st = pk_stats()
    _check(lib().pk_index_stats(handle, C.byref(st), _stream()), "pk_index_stats")
    return st


def pk_list_lengths(handle: int, nlist: int):
    import numpy as np
    out = np.empty(nlist, dtype=np.int64)
    _check(lib().pk_list_lengths(handle, out.ctypes.data_as(C.c_void_p), _stream()), "pk_list_lengths")
    return out


def pk_profile_begin(handle: int):
    _check(lib().pk_profile_begin(handle, _stream()), "pk_profile_begin")


def pk_profile_end(handle: int) -> pk_profile:
    pr = pk_profile()
    _check(lib().pk_profile_end(handle, C.byref(pr), _stream()), "pk_profile_end")
    return pr


def pk_index_free(handle: int):
    _check(lib().pk_index_free(handle), "pk_index_free")


class Index:
    """Convenience owner of one handle and its arena tensors (no arithmetic here)."""

    def __init__(self, centroids, vectors, metric=PK_METRIC_IP, storage=PK_F32, ids=None, page_vecs=0,
                 max_delta_pages=0, insert_reserve=0, arena_bytes=None):
        nlist, d = centroids.shape
        self.cfg = pk_config(d, nlist, metric, storage, page_vecs, max_delta_pages)
        n = 0 if vectors is None else vectors.shape[0]
        if arena_bytes is None:
            arena_bytes = pk_arena_bytes(self.cfg, n, insert_reserve)
            if arena_bytes == 0:
                raise PancakeError(PK_ERR_INVALID_ARG, "pk_arena_bytes")
        self.device = centroids.device
        self.arenas = [torch.empty(arena_bytes, dtype=torch.uint8, device=self.device)]
        self.nlist, self.d = nlist, d
        self.handle = pk_index_build(self.cfg, centroids, vectors, ids, self.arenas[0])

    def add_arena(self, nbytes: int):
        t = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        pk_index_add_arena(self.handle, t)
        self.arenas.append(t)

    def compact(self, nbytes: int):
        """Moves the index into one new arena of nbytes; the old arena tensors are released."""
        t = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        pk_index_compact(self.handle, t)
        self.arenas = [t]

    def insert(self, vectors, ids=None, want_lists=False):
        out = torch.empty(vectors.shape[0], dtype=torch.int32, device=self.device) if want_lists else None
        pk_insert(self.handle, vectors, ids, out)
        return out

    def split(self, threshold: int, iters: int, nbytes: int) -> int:
        """IVF-Split into one new arena of nbytes; returns the number of lists split (nlist grows by it)."""
        t = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        n = pk_index_split(self.handle, t, threshold, iters)
        self.arenas = [t]
        self.nlist += n
        self.cfg.nlist = self.nlist
        return n

    def centroids(self):
        out = torch.empty((self.nlist, self.d), dtype=torch.float32, device=self.device)
        pk_index_centroids(self.handle, out)
        return out

    def list_ids(self, lst: int):
        n = int(self.list_lengths()[lst])
        out = torch.empty(max(n, 1), dtype=torch.int64, device=self.device)
        pk_list_ids(self.handle, lst, out[:n])
        return out[:n]

    def delete(self, ids) -> int:
        return pk_delete(self.handle, ids)

    def insert_assigned(self, vectors, lists, ids=None):
        pk_insert_assigned(self.handle, vectors, ids, lists)

    def search(self, queries, k, nprobe):
        ids = torch.empty((queries.shape[0], k), dtype=torch.int64, device=self.device)
        dist = torch.empty((queries.shape[0], k), dtype=torch.float32, device=self.device)
        pk_search(self.handle, queries, k, nprobe, ids, dist)
        return ids, dist

    def coarse(self, queries, nprobe):
        out = torch.empty((queries.shape[0], nprobe), dtype=torch.int32, device=self.device)
        pk_coarse(self.handle, queries, nprobe, out)
        return out

    def scan_probes(self, queries, k, probes):
        ids = torch.empty((queries.shape[0], k), dtype=torch.int64, device=self.device)
        dist = torch.empty((queries.shape[0], k), dtype=torch.float32, device=self.device)
        pk_scan_probes(self.handle, queries, k, probes, ids, dist)
        return ids, dist

    def stats(self):
        return pk_index_stats(self.handle)

    def reserve(self, nq_max, k_max, nprobe_max, inserts_ahead=0):
        pk_workspace_reserve([self.handle], nq_max, k_max, nprobe_max, inserts_ahead)

    def list_lengths(self):
        return pk_list_lengths(self.handle, self.nlist)

    def close(self):
        if self.handle:
            torch.cuda.synchronize(self.device)
            pk_index_free(self.handle)
            self.handle = None
            self.arenas = []

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def pk_search_union(handles, queries, k: int, nprobe: int, out_src, out_ids, out_dist):
    hs = (C.c_void_p * len(handles))(*handles)
    _check(lib().pk_search_union(hs, len(handles), _dev(queries, torch.float32, "queries"), queries.shape[0], k, nprobe,
                                 _dev(out_src, torch.int32, "out_src"), _dev(out_ids, torch.int64, "out_ids"),
                                 _dev(out_dist, torch.float32, "out_dist"), _stream()), "pk_search_union")


def pk_search_levels(handles, nprobes, queries, k: int, stop, out_level, out_ids, out_dist):
    hs = (C.c_void_p * len(handles))(*handles)
    nps = (C.c_int32 * len(handles))(*[int(x) for x in nprobes])
    _check(lib().pk_search_levels(hs, len(handles), nps, _dev(queries, torch.float32, "queries"), queries.shape[0], k,
                                  _dev(stop, torch.float32, "stop"), _dev(out_level, torch.int32, "out_level"),
                                  _dev(out_ids, torch.int64, "out_ids"), _dev(out_dist, torch.float32, "out_dist"),
                                  _stream()), "pk_search_levels")


def search_levels(indexes, nprobes, queries, k, stop):
    """Top level first; returns (level each query ended at, ids, values)."""
    dev = queries.device
    level = torch.empty(queries.shape[0], dtype=torch.int32, device=dev)
    ids = torch.empty((queries.shape[0], k), dtype=torch.int64, device=dev)
    dist = torch.empty((queries.shape[0], k), dtype=torch.float32, device=dev)
    pk_search_levels([ix.handle for ix in indexes], nprobes, queries, k, stop, level, ids, dist)
    return level, ids, dist


def search_union(indexes, queries, k, nprobe):
    dev = queries.device
    src = torch.empty((queries.shape[0], k), dtype=torch.int32, device=dev)
    ids = torch.empty((queries.shape[0], k), dtype=torch.int64, device=dev)
    dist = torch.empty((queries.shape[0], k), dtype=torch.float32, device=dev)
    pk_search_union([ix.handle for ix in indexes], queries, k, nprobe, src, ids, dist)
    return src, ids, dist


def search_multi(indexes, q_offsets, queries, k, nprobe):
    dev = queries.device
    ids = torch.empty((queries.shape[0], k), dtype=torch.int64, device=dev)
    dist = torch.empty((queries.shape[0], k), dtype=torch.float32, device=dev)
    pk_search_multi([ix.handle for ix in indexes], q_offsets, queries, k, nprobe, ids, dist)
    return ids, dist


# ------------------------------------------------------------------------------- key/value cache

# The current stream of a device without an object of torch's for it: 0.1 us instead of 2.7, of the 9 that a call took.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_of(device: int) -> int:
    return _raw_stream(device) if _raw_stream is not None else torch.cuda.current_stream(device).cuda_stream


ROW_TYPES = {torch.float32: PK_F32, torch.float16: PK_F16, torch.bfloat16: PK_BF16}


def pk_kv_arena_bytes(cfg: pk_kv_config) -> int:
    return int(lib().pk_kv_arena_bytes(C.byref(cfg)))


def pk_kv_create(cfg: pk_kv_config, arena) -> int:
    """Returns the handle (an integer).  `arena` is a uint8 CUDA tensor the caller keeps alive."""
    h = C.c_void_p()
    _check(lib().pk_kv_create(C.byref(cfg), _dev(arena, torch.uint8, "arena"), arena.numel(), C.byref(h)), "pk_kv_create")
    return h.value


def pk_kv_free(handle: int):
    _check(lib().pk_kv_free(handle), "pk_kv_free")


def _rows(t, what) -> pk_rows:
    """Rows [token, head, channel] of any strides, the channels side by side."""
    kind, stride = ROW_TYPES.get(t.dtype), t.stride()
    if kind is None or not t.is_cuda or len(stride) != 3 or (stride[2] != 1 and t.shape[2] > 1):
        raise ValueError(f"{what}: need a CUDA tensor [token, head, channel] of float32, float16 or bfloat16 with its channels side by side")
    return pk_rows(t.data_ptr(), stride[0], stride[1], kind)


def pk_kv_append(handle: int, batch: pk_kv_batch, k, v):
    _check(lib().pk_kv_append(handle, batch, _rows(k, "k"), _rows(v, "v"), _stream_of(k.get_device())), "pk_kv_append")


def pk_kv_read(handle: int, batch: pk_kv_batch, k_out, v_out):
    kind = ROW_TYPES.get(k_out.dtype)
    if kind is None:
        raise ValueError("k_out: need float32, float16 or bfloat16")
    _check(lib().pk_kv_read(handle, batch, _dev(k_out, k_out.dtype, "k_out"), _dev(v_out, k_out.dtype, "v_out"), kind, _stream_of(k_out.get_device())), "pk_kv_read")


def pk_kv_bounds(handle: int, pages, hi, lo):
    _check(lib().pk_kv_bounds(handle, _dev(pages, torch.int32, "pages"), pages.numel(), _dev(hi, torch.float32, "hi"), _dev(lo, torch.float32, "lo"),
                              _stream_of(pages.get_device())), "pk_kv_bounds")


def pk_kv_attend(handle: int, batch: pk_kv_batch, q, scale: float, window: int, out, lse=None):
    _check(lib().pk_kv_attend(handle, batch, _rows(q, "q"), q.shape[1], scale, window, _dev(out, q.dtype, "out"), _dev(lse, torch.float32, "lse"),
                              _stream_of(q.get_device())), "pk_kv_attend")


def pk_kv_attend_scored(handle: int, batch: pk_kv_batch, q, scale: float, window: int, cap: float, slopes, starts, prefix, out, lse=None):
    scores = pk_kv_scores(cap, _dev(slopes, torch.float32, "slopes"), _dev(starts, torch.int32, "starts"), _dev(prefix, torch.int32, "prefix"))
    _check(lib().pk_kv_attend_scored(handle, batch, _rows(q, "q"), q.shape[1], scale, window, scores, _dev(out, q.dtype, "out"), _dev(lse, torch.float32, "lse"),
                                     _stream_of(q.get_device())), "pk_kv_attend_scored")


def pk_kv_select(handle: int, batch: pk_kv_batch, q, n_blocks: int, sink: int, local: int, out_blocks):
    _check(lib().pk_kv_select(handle, batch, _rows(q, "q"), q.shape[1], n_blocks, sink, local, _dev(out_blocks, torch.int32, "out_blocks"), _stream_of(q.get_device())),
           "pk_kv_select")


def pk_kv_attend_blocks(handle: int, batch: pk_kv_batch, q, scale: float, blocks, out, lse=None):
    _check(lib().pk_kv_attend_blocks(handle, batch, _rows(q, "q"), q.shape[1], scale, _dev(blocks, torch.int32, "blocks"), blocks.shape[2],
                                     _dev(out, q.dtype, "out"), _dev(lse, torch.float32, "lse"), _stream_of(q.get_device())), "pk_kv_attend_blocks")


def pk_kv_pool_bytes(cfg: pk_kv_config) -> int:
    return int(lib().pk_kv_pool_bytes(C.byref(cfg)))


def pk_kv_pool_create(kv: int, memory) -> int:
    """Returns the handle (an integer).  `memory` is a uint8 CUDA tensor the caller keeps alive."""
    h = C.c_void_p()
    _check(lib().pk_kv_pool_create(kv, _dev(memory, torch.uint8, "memory"), memory.numel(), C.byref(h)), "pk_kv_pool_create")
    return h.value


def pk_kv_pool_free(pool: int):
    _check(lib().pk_kv_pool_free(pool), "pk_kv_pool_free")


def _tables(t, what="tables") -> pk_kv_tables:
    if t.dim() != 2 or not t.is_cuda or t.dtype != torch.int32 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{what}: need an int32 CUDA tensor [sequence, page] with its rows' entries side by side")
    return pk_kv_tables(t.data_ptr(), t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1]), t.shape[0], t.shape[1])


def pk_kv_pool_clear(pool: int, device: int):
    _check(lib().pk_kv_pool_clear(pool, _stream_of(device)), "pk_kv_pool_clear")


def pk_kv_pool_adopt(pool: int, tables):
    _check(lib().pk_kv_pool_adopt(pool, _tables(tables), _stream_of(tables.get_device())), "pk_kv_pool_adopt")


def pk_kv_pool_grant(pool: int, batch: pk_kv_batch, missing, device: int):
    _check(lib().pk_kv_pool_grant(pool, batch, _dev(missing, torch.int32, "missing"), _stream_of(device)), "pk_kv_pool_grant")


def pk_kv_pool_fork(pool: int, tables, lens, sources, targets):
    _check(lib().pk_kv_pool_fork(pool, _tables(tables), _dev(lens, torch.int32, "lens"), _dev(sources, torch.int32, "sources"), _dev(targets, torch.int32, "targets"), targets.shape[0],
                                 _stream_of(tables.get_device())), "pk_kv_pool_fork")


def pk_kv_pool_release(pool: int, tables, rows, keep=None):
    _check(lib().pk_kv_pool_release(pool, _tables(tables), _dev(rows, torch.int32, "rows"), _dev(keep, torch.int32, "keep"), rows.shape[0], _stream_of(tables.get_device())),
           "pk_kv_pool_release")


def pk_kv_pool_compact(pool: int, into: int, tables, out, missing=None):
    _check(lib().pk_kv_pool_compact(pool, into, _tables(tables), _tables(out, "out"), _dev(missing, torch.int32, "missing"), _stream_of(tables.get_device())), "pk_kv_pool_compact")


def pk_kv_pool_counts(pool: int, counts):
    _check(lib().pk_kv_pool_counts(pool, _dev(counts, torch.int32, "counts"), _stream_of(counts.get_device())), "pk_kv_pool_counts")


def pk_kv_copy(to: int, source: int, to_pages, from_pages):
    _check(lib().pk_kv_copy(to, source, _dev(to_pages, torch.int32, "to_pages"), _dev(from_pages, torch.int32, "from_pages"), to_pages.shape[0], _stream_of(to_pages.get_device())), "pk_kv_copy")


class KVBatch:
    """One step of a batch of sequences: page tables, row offsets and lengths on the GPU (int32; tensors that are kept and may
    change from step to step), and their bounds on the host."""

    def __init__(self, tables, offsets, lens, n_tokens, max_new, max_len):
        n = lens.shape[0]
        if tables.dim() != 2 or tables.shape[0] != n or offsets.shape != (n + 1,) or lens.dim() != 1:
            raise ValueError("a batch has tables [sequence, page], offsets [sequence + 1] and lens [sequence]")
        if not tables.is_cuda or tables.dtype != torch.int32 or (tables.shape[1] > 1 and tables.stride(1) != 1):
            raise ValueError("tables: need an int32 CUDA tensor with its rows' entries side by side")
        if offsets.device != tables.device or lens.device != tables.device:
            raise ValueError("tables, offsets and lens are on different devices")
        self.tables, self.offsets, self.lens, self.n_tokens, self.device = tables, offsets, lens, n_tokens, tables.get_device()
        self.c = pk_kv_batch(tables.data_ptr(), _dev(offsets, torch.int32, "offsets"), _dev(lens, torch.int32, "lens"),
                             tables.stride(0) if n > 1 else max(tables.stride(0), tables.shape[1]), n, tables.shape[1], n_tokens, max_new, max_len)


class KVCache:
    """Convenience owner of one cache's handle and its arena tensor (no arithmetic here).  Calls go to the current stream of the
    cache's device, which has to be the current device."""

    def __init__(self, n_pages, n_heads, head_dim, storage=PK_BF16, page_tokens=64, device="cuda"):
        self.cfg = pk_kv_config(n_pages, n_heads, head_dim, page_tokens, storage)
        self.handle = None
        need = pk_kv_arena_bytes(self.cfg)
        if need == 0:
            raise PancakeError(PK_ERR_INVALID_ARG, "pk_kv_arena_bytes")
        self.arena = torch.empty(need, dtype=torch.uint8, device=device)
        self.n_heads, self.head_dim, self.device = n_heads, head_dim, self.arena.get_device()
        with torch.cuda.device(self.arena.device):
            self.handle = pk_kv_create(self.cfg, self.arena)

    def _shape(self, t, batch, heads, what):
        s = t.shape
        if len(s) != 3 or s[0] != batch.n_tokens or s[2] != self.head_dim or (heads and s[1] != heads):
            raise ValueError(f"{what}: need [{batch.n_tokens}, {heads or 'heads'}, {self.head_dim}], got {list(s)}")
        if t.get_device() != self.device or batch.device != self.device:
            raise ValueError(f"{what} is on {t.device}, the batch on device {batch.device}, the cache on {self.arena.device}")

    def append(self, k, v, batch):
        """Writes the batch's new tokens, rows [token, head, channel] of any strides."""
        self._shape(k, batch, self.n_heads, "k")
        self._shape(v, batch, self.n_heads, "v")
        pk_kv_append(self.handle, batch.c, k, v)

    def read(self, batch, dtype):
        """Keys and values of the batch's tokens as they are stored, [token, head, channel] of dtype."""
        if batch.device != self.device:
            raise ValueError(f"the batch is on device {batch.device}, the cache on {self.arena.device}")
        k, v = torch.empty((2, batch.n_tokens, self.n_heads, self.head_dim), dtype=dtype, device=self.arena.device).unbind(0)
        pk_kv_read(self.handle, batch.c, k, v)
        return k, v

    def bounds(self, pages):
        """Largest and smallest stored key value of every channel of the pages, [page, head, channel]."""
        if pages.get_device() != self.device:
            raise ValueError(f"pages: is on {pages.device}, the cache on {self.arena.device}")
        hi, lo = torch.empty((2, pages.numel(), self.n_heads, self.head_dim), dtype=torch.float32, device=self.arena.device).unbind(0)
        pk_kv_bounds(self.handle, pages, hi, lo)
        return hi, lo

    def copy_pages(self, pages, source, source_pages):
        """Pages of another cache of the same shape and storage (or of this one), with their scales and bounds, over pages of this one."""
        if pages.dim() != 1 or pages.shape != source_pages.shape:
            raise ValueError(f"pages: need as many as there are source pages, got {list(pages.shape)} and {list(source_pages.shape)}")
        if not (pages.get_device() == source_pages.get_device() == self.device == source.device):
            raise ValueError(f"pages on {pages.device} and {source_pages.device}, caches on {self.arena.device} and {source.arena.device}")
        pk_kv_copy(self.handle, source.handle, pages, source_pages)

    def _outputs(self, q, want_lse):
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        return out, torch.empty(q.shape[:2], dtype=torch.float32, device=q.device) if want_lse else None

    def attend(self, q, batch, scale, window=0, want_lse=False, cap=0.0, slopes=None, starts=None, prefix=None):
        """Attention of the new tokens over their sequences: out, or (out, lse).  Scores are capped (cap tanh(score / cap)) where cap is not 0, and
        lessened by slopes [query head] times the distance; starts [token]: the first position that a token sees; prefix [sequence]: tokens that all see."""
        self._shape(q, batch, 0, "q")
        out, lse = self._outputs(q, want_lse)
        if cap == 0.0 and slopes is None and starts is None and prefix is None:
            pk_kv_attend(self.handle, batch.c, q, scale, window, out, lse)
        else:
            for what, t, n in (("slopes", slopes, q.shape[1]), ("starts", starts, batch.n_tokens), ("prefix", prefix, batch.lens.shape[0])):
                if t is not None and (t.shape != (n,) or t.get_device() != self.device):
                    raise ValueError(f"{what}: need [{n}] on {self.arena.device}, got {list(t.shape)} on {t.device}")
            pk_kv_attend_scored(self.handle, batch.c, q, scale, window, cap, slopes, starts, prefix, out, lse)
        return (out, lse) if want_lse else out

    def select(self, q, batch, n_blocks, sink=1, local=2):
        """Blocks that each new token attends to, [token, key/value head, n_blocks], ascending, padded with -1."""
        self._shape(q, batch, 0, "q")
        blocks = torch.empty((batch.n_tokens, self.n_heads, n_blocks), dtype=torch.int32, device=q.device)
        pk_kv_select(self.handle, batch.c, q, n_blocks, sink, local, blocks)
        return blocks

    def attend_blocks(self, q, blocks, batch, scale, want_lse=False):
        """Attention of the new tokens over listed blocks: out, or (out, lse)."""
        self._shape(q, batch, 0, "q")
        if blocks.dim() != 3 or blocks.shape[0] != batch.n_tokens or blocks.shape[1] != self.n_heads or blocks.get_device() != self.device:
            raise ValueError(f"blocks: need [{batch.n_tokens}, {self.n_heads}, blocks], got {list(blocks.shape)}")
        out, lse = self._outputs(q, want_lse)
        pk_kv_attend_blocks(self.handle, batch.c, q, scale, blocks, out, lse)
        return (out, lse) if want_lse else out

    def close(self):
        if self.handle:
            torch.cuda.synchronize(self.arena.device)
            pk_kv_free(self.handle)
            self.handle = None
            self.arena = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class KVPool:
    """The pages of a cache: who has them, and which are free (no arithmetic here).  Tables are int32 tensors [sequence, page] of the caller's, changed in place.  Calls
    go to the current stream of the cache's device, which has to be the current device."""

    def __init__(self, cache):
        self.handle = None
        self.cache, self.device = cache, cache.device
        self.memory = torch.empty(pk_kv_pool_bytes(cache.cfg), dtype=torch.uint8, device=cache.arena.device)
        with torch.cuda.device(cache.arena.device):
            self.handle = pk_kv_pool_create(cache.handle, self.memory)

    def _check(self, **tensors):
        """The cache is open, and everything on its device."""
        if self.cache.handle is None:
            raise ValueError("the pool's cache is closed")
        for what, t in tensors.items():
            if t is not None and t.get_device() != self.device:
                raise ValueError(f"{what} is on {t.device}, the pool on {self.memory.device}")

    def clear(self):
        """All pages are free."""
        self._check()
        pk_kv_pool_clear(self.handle, self.device)

    def adopt(self, tables):
        """Counts the pages of tables that were filled without the pool."""
        self._check(tables=tables)
        pk_kv_pool_adopt(self.handle, tables)

    def grant(self, batch):
        """Pages of their own for the batch's new tokens, shared ones copied first; batch.tables is changed.  Returns the number of entries that got none, an int32 tensor [1]."""
        self._check()
        if batch.device != self.device:
            raise ValueError(f"the batch is on device {batch.device}, the pool on {self.memory.device}")
        missing = batch.lens.new_empty(1)
        pk_kv_pool_grant(self.handle, batch.c, missing, self.device)
        return missing

    def fork(self, tables, lens, sources, targets):
        """Rows `targets` of the tables get the pages of rows `sources` (of lens tokens, by row of the tables)."""
        self._check(tables=tables, lens=lens, sources=sources, targets=targets)
        if lens.shape != (tables.shape[0],) or sources.dim() != 1 or sources.shape != targets.shape:
            raise ValueError("a fork has lens for every row of the tables, and as many sources as targets")
        pk_kv_pool_fork(self.handle, tables, lens, sources, targets)

    def release(self, tables, rows, keep=None):
        """Rows of the tables keep the pages of their first `keep` tokens (none where it is left out) and give up the others."""
        self._check(tables=tables, rows=rows, keep=keep)
        if rows.dim() != 1 or (keep is not None and keep.shape != rows.shape):
            raise ValueError("a release has a list of rows, and as many numbers of tokens to keep")
        pk_kv_pool_release(self.handle, tables, rows, keep)

    def compact(self, into, tables):
        """Moves the pages in use into the cache of another pool, side by side.  Returns the tables' new entries, and the number of pages that had no room, an int32 tensor [1]."""
        self._check(tables=tables)
        into._check()
        if into.device != self.device:
            raise ValueError(f"the other pool is on {into.memory.device}, this one on {self.memory.device}")
        out, missing = tables.new_empty(tables.shape), tables.new_empty(1)
        pk_kv_pool_compact(self.handle, into.handle, tables, out, missing)
        return out, missing

    def counts(self):
        """Owners of every page, int32 [page]: 0 for a free one."""
        self._check()
        counts = torch.empty(self.cache.cfg.n_pages, dtype=torch.int32, device=self.memory.device)
        pk_kv_pool_counts(self.handle, counts)
        return counts

    def close(self):
        if self.handle:
            torch.cuda.synchronize(self.memory.device)
            pk_kv_pool_free(self.handle)
            self.handle = None
            self.memory = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
