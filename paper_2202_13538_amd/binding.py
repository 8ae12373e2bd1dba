"""ctypes binding of libsurel's C ABI (see include/surel.h).

Argument marshalling only: tensors are passed as raw device pointers, outputs are allocated
with torch, and every step of the path runs in the library's HIP kernels.  There is no CPU
fallback: if ``libsurel.so`` has not been built, ``load()`` raises.
"""
from __future__ import annotations

import ctypes
import os
import platform

import torch

_PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG_DIR, "libsurel.so")

OK, E_NULL, E_RANGE, E_HIP, E_CAPACITY, E_CTX, E_DEVICE = 0, -1, -2, -3, -4, -5, -6
DEV_BAD_SEED, DEV_BAD_GRAPH, DEV_BAD_WALK, DEV_BAD_QUERY = 0x01, 0x02, 0x04, 0x08
DEV_SET_TOO_LARGE, DEV_CAPACITY, DEV_BAD_TABLE, DEV_BAD_SIZES = 0x10, 0x20, 0x40, 0x80
DEV_STALL, DEV_BAD_OFFSETS, DEV_BAD_BUCKET, DEV_BAD_LABEL = 0x100, 0x200, 0x400, 0x800
DEV_BAD_PAGE, DEV_BAD_LENGTH, DEV_NO_PAGE, DEV_BAD_CHOICE = 0x1000, 0x2000, 0x4000, 0x8000
MAX_NODES, MAX_STEPS, MAX_WALKS = 268435455, 15, 65535
MAX_WALK_ENTRIES, MAX_SET, MAX_TUPLE = 2048, 2048, 3
MAX_DISTINCT = 1 << 24
MAX_BATCH = 1 << 20
MAX_ROWS, MAX_HEAD_DIM, MAX_REACH, MAX_STRIDE = 1 << 30, 128, 1024, (1 << 24) - 8
MAX_CLASS_DIM, MAX_SEQS = 256, 1 << 24
NOALLOC_MAX_QUERIES = 1 << 20
BF16, FP16, FP32 = 0, 1, 2

(K_WALK, K_RPE_COUNT, K_RPE_FILL, K_JOIN_COUNT, K_JOIN_FILL, K_SCAN, K_WALK_RPE,
 K_EDGE_RECORDS, K_QUERY_IDS, K_PRUNE, K_BATCH, K_ATTENTION,
 K_ATTENTION_GRAD, K_LOSS, K_LOSS_GRAD, K_CACHE_PLAN, K_CACHE_STORE, K_CACHE_ATTENTION,
 K_SAMPLE, K_COUNT) = range(20)
KERNEL_NAMES = {K_WALK: "walk", K_RPE_COUNT: "rpe_count", K_RPE_FILL: "rpe_fill",
                K_JOIN_COUNT: "join_count", K_JOIN_FILL: "join_fill", K_SCAN: "scan",
                K_WALK_RPE: "walk_rpe", K_EDGE_RECORDS: "edge_records",
                K_QUERY_IDS: "query_ids", K_PRUNE: "prune", K_BATCH: "batch",
                K_ATTENTION: "attention", K_ATTENTION_GRAD: "attention_grad",
                K_LOSS: "loss", K_LOSS_GRAD: "loss_grad", K_CACHE_PLAN: "cache_plan",
                K_CACHE_STORE: "cache_store", K_CACHE_ATTENTION: "cache_attention",
                K_SAMPLE: "sample"}

_vp = ctypes.c_void_p
_i32, _i64, _u64 = ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64


class AttentionArgs(ctypes.Structure):
    """surel_attention_args"""
    _fields_ = [(n, _vp) for n in ("d_q", "d_k", "d_v")] + \
               [(n, _i64) for n in ("q_row", "q_head", "k_row", "k_head", "v_row", "v_head")] + \
               [(n, _vp) for n in ("d_q_off", "d_k_off")] + \
               [(n, _i64) for n in ("n_seqs", "n_q", "n_k")] + \
               [(n, _i32) for n in ("type", "heads", "kv_heads", "dim", "causal")] + \
               [("scale", ctypes.c_float), ("d_bias", _vp), ("d_bucket", _vp), ("n_buckets", _i32),
                ("reach", _i32)]


class Cache(ctypes.Structure):
    """surel_cache"""
    _fields_ = [("d_k", _vp), ("d_v", _vp)] + [(n, _i64) for n in ("page", "row", "head", "n_pages")] + \
               [(n, _i32) for n in ("page_rows", "type", "kv_heads", "dim")]


class CacheAttentionArgs(ctypes.Structure):
    """surel_cache_attention_args"""
    _fields_ = [("d_q", _vp), ("q_row", _i64), ("q_head", _i64), ("d_pages", _vp), ("d_length", _vp), ("n_seqs", _i64),
                ("max_pages", _i32), ("heads", _i32), ("scale", ctypes.c_float), ("d_bias", _vp), ("d_bucket", _vp),
                ("n_buckets", _i32), ("reach", _i32)]


# name -> (restype, argtypes); the order and types of include/surel.h
SIGNATURES = {
    "surel_create": (ctypes.c_int, [ctypes.POINTER(_vp), ctypes.c_int, _vp]),
    "surel_destroy": (None, [_vp]),
    "surel_strerror": (ctypes.c_char_p, [ctypes.c_int]),
    "surel_rpe_rows_bound": (_i64, [_i64, _i32, _i32]),
    "surel_sample_walks": (ctypes.c_int, [_vp, _vp, _vp, _i32, _i64, _vp, _i64, _i32, _i32,
                                          _u64, _vp, _vp]),
    "surel_build_rpe": (ctypes.c_int, [_vp, _vp, _i64, _i32, _i32, _i32, _vp, _i64, _vp, _vp,
                                       _vp, ctypes.POINTER(_i64)]),
    "surel_build_rpe_count": (ctypes.c_int, [_vp, _vp, _i64, _i32, _i32, _i32, _vp, _vp,
                                             ctypes.POINTER(_i64)]),
    "surel_build_rpe_fill": (ctypes.c_int, [_vp, _vp, _i64, _i32, _i32, _i32, _vp, _i64, _vp, _vp]),
    "surel_sample_walks_rpe": (ctypes.c_int, [_vp, _vp, _vp, _i32, _i64, _vp, _i64, _i32, _i32,
                                              _u64, _vp, _i64, _vp, _vp, _vp,
                                              ctypes.POINTER(_i64)]),
    "surel_sample_walks_rpe_ids": (ctypes.c_int, [_vp, _vp, _vp, _i32, _i64, _vp, _i64, _i32, _i32,
                                                  _u64, _vp, _i64, _vp, _vp, _vp, _vp, _i64, _vp,
                                                  ctypes.POINTER(_i64), ctypes.POINTER(_i64)]),
    "surel_join_queries": (ctypes.c_int, [_vp, _vp, _vp, _vp, _i64, _i32, _i32, _vp, _i64, _i32,
                                          _i64, _vp, _vp, _vp, ctypes.POINTER(_i64)]),
    "surel_join_queries_noalloc": (ctypes.c_int, [_vp, _vp, _vp, _vp, _i64, _i32, _i32, _vp, _i64,
                                                  _i32, _i64, _vp, _vp, _vp, ctypes.POINTER(_i64)]),
    "surel_join_count": (ctypes.c_int, [_vp, _vp, _vp, _i64, _i32, _vp, _i64, _i32, _vp,
                                        ctypes.POINTER(_i64)]),
    "surel_join_fill": (ctypes.c_int, [_vp, _vp, _vp, _vp, _i64, _i32, _i32, _vp, _i64, _i32, _vp,
                                       _i64, _vp, _vp]),
    "surel_join_query_ids": (ctypes.c_int, [_vp, _vp, _vp, _vp, _i64, _i32, _vp, _i64, _i32, _i64,
                                            _vp, _vp, _vp, ctypes.POINTER(_i64)]),
    "surel_query_rpe_ids": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp, _i64, _i64, _i32, _i32, _i32,
                                           _vp, _i64, _i32, _vp]),
    "surel_prune_rpe": (ctypes.c_int, [_vp, _vp, _i64, _i32, _i64, _vp, _vp,
                                       ctypes.POINTER(_i64)]),
    "surel_query_incidence": (ctypes.c_int, [_vp, _vp, _i64, _i32, _i32, _vp, _vp]),
    "surel_bfs_batches": (ctypes.c_int, [_vp, _vp, _i64, _i32, _i32, _vp, _vp, _vp, _i64, _i32,
                                         _i32, _i32, _vp, _vp, _vp, _vp]),
    "surel_attention": (ctypes.c_int, [_vp, ctypes.POINTER(AttentionArgs), _vp, _vp]),
    "surel_attention_grad": (ctypes.c_int, [_vp, ctypes.POINTER(AttentionArgs)] + 7 * [_vp]),
    "surel_softmax_loss": (ctypes.c_int, [_vp, _i32, _vp, _vp, _vp, _i64, _i32, _i32, _vp, _vp]),
    "surel_softmax_loss_grad": (ctypes.c_int, [_vp, _i32, _vp, _vp, _vp, _vp, _vp, _i64, _i32, _i32, _vp,
                                               _vp]),
    "surel_cache_plan": (ctypes.c_int, [_vp, _vp, _vp, _i64, _i64, _i32, _i32, _i64] + 7 * [_vp]),
    "surel_cache_store": (ctypes.c_int, [_vp, ctypes.POINTER(Cache), _vp, _vp, _i64, _i64, _i64, _i64, _vp, _i64]),
    "surel_cache_attention": (ctypes.c_int, [_vp, ctypes.POINTER(Cache), ctypes.POINTER(CacheAttentionArgs), _vp, _vp]),
    "surel_sample_classes": (ctypes.c_int, [_vp, _i32, _vp, _i64, _i64, _i32] + 7 * [_vp]),
    "surel_set_spin_limit": (ctypes.c_int, [_vp, ctypes.c_uint32]),
    "surel_check": (ctypes.c_int, [_vp, ctypes.POINTER(ctypes.c_uint32)]),
    "surel_profile_enable": (ctypes.c_int, [_vp, ctypes.c_int]),
    "surel_profile_read": (ctypes.c_int, [_vp, ctypes.c_int, ctypes.POINTER(ctypes.c_double),
                                          ctypes.POINTER(_i64)]),
}

_lib = None


class SurelError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = load().surel_strerror(status).decode()
        super().__init__(f"{where}: {msg} (status {status})")


def load() -> ctypes.CDLL:
    """Load libsurel.so.  Raises if it is missing: there is no other implementation."""
    global _lib, _ptr
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is not built; run `python -m paper_2202_13538_amd.build` "
                "(hipcc cross-compiles for gfx950, no GPU needed)")
        _ptr = _checks_of_arguments()
        lib = ctypes.CDLL(LIB_PATH)
        for name, (restype, argtypes) in SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = restype
            fn.argtypes = argtypes
        _lib = lib
    return _lib


def _ptr_in_python(t: torch.Tensor | None, dtype: torch.dtype, what: str) -> int | None:
    if t is None:
        return None
    if t.dtype != dtype:
        raise TypeError(f"{what} must be {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{what} must live on the GPU")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return t.data_ptr()


_ptr = _ptr_in_python  # load() puts the one of host/marshal.cpp in its place


def _checks_of_arguments():
    """_ptr in native code, or in Python where _marshal.so is not built or is one for another torch or
    Python (which need not fail to load, but reads tensors through other headers)."""
    try:
        from . import _marshal
    except ImportError:
        return _ptr_in_python
    if getattr(_marshal, "built_for", None) != f"{torch.__version__} {platform.python_version()}":
        return _ptr_in_python
    _marshal.otherwise(_ptr_in_python)
    return _marshal.ptr


class Context:
    """Owns one ``surel_ctx`` bound to a device and a HIP stream (torch's current one)."""

    def __init__(self, device: int | torch.device | None = None,
                 stream: torch.cuda.Stream | None = None):
        if device is None:
            device = torch.cuda.current_device()
        self.device = torch.device("cuda", device) if isinstance(device, int) else device
        if stream is None:
            stream = torch.cuda.current_stream(self.device)
        self.stream = stream
        self._h = _vp()
        rc = load().surel_create(ctypes.byref(self._h), self.device.index or 0,
                                 _vp(stream.cuda_stream))
        if rc != OK:
            raise SurelError(rc, "surel_create")

    @property
    def handle(self) -> ctypes.c_void_p:
        return self._h

    def check(self) -> int:
        """Synchronise and return the device error word (also clears it)."""
        flags = ctypes.c_uint32(0)
        rc = load().surel_check(self._h, ctypes.byref(flags))
        if rc not in (OK, E_DEVICE):
            raise SurelError(rc, "surel_check")
        return flags.value

    def set_spin_limit(self, spins: int) -> None:
        rc = load().surel_set_spin_limit(self._h, spins)
        if rc != OK:
            raise SurelError(rc, "surel_set_spin_limit")

    def profile(self, on: bool) -> None:
        rc = load().surel_profile_enable(self._h, 1 if on else 0)
        if rc != OK:
            raise SurelError(rc, "surel_profile_enable")

    def profile_read(self) -> dict:
        """{kernel name: (total ms, launches)} since profiling was switched on."""
        out = {}
        for kid, name in KERNEL_NAMES.items():
            ms = ctypes.c_double(0.0)
            n = _i64(0)
            rc = load().surel_profile_read(self._h, kid, ctypes.byref(ms), ctypes.byref(n))
            if rc != OK:
                raise SurelError(rc, "surel_profile_read")
            out[name] = (ms.value, n.value)
        return out

    def close(self):
        if self._h:
            load().surel_destroy(self._h)
            self._h = _vp()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def rpe_rows_bound(n_seeds: int, M: int, m: int) -> int:
    return load().surel_rpe_rows_bound(n_seeds, M, m)


def sample_walks(ctx: Context, row_ptr: torch.Tensor, col_idx: torch.Tensor,
                 seeds: torch.Tensor, M: int, m: int, rng_seed: int = 0,
                 out: torch.Tensor | None = None,
                 set_sizes: torch.Tensor | None = None) -> torch.Tensor:
    """walks int32[n_seeds][M][m+1] on the GPU; ``set_sizes`` (int32[n_seeds], optional)
    receives the number of distinct nodes of every seed's walks."""
    n_nodes = row_ptr.numel() - 1
    n_seeds = seeds.numel()
    if out is None:
        out = torch.empty((n_seeds, M, m + 1), dtype=torch.int32, device=row_ptr.device)
    elif out.numel() != n_seeds * M * (m + 1):
        raise ValueError("out has the wrong size")
    rc = load().surel_sample_walks(
        ctx.handle, _ptr(row_ptr, torch.int32, "row_ptr"), _ptr(col_idx, torch.int32, "col_idx"),
        n_nodes, col_idx.numel(), _ptr(seeds, torch.int32, "seeds"), n_seeds, M, m,
        _u64(rng_seed), _ptr(out, torch.int32, "walks"),
        _ptr(set_sizes, torch.int32, "set_sizes"))
    if rc != OK:
        raise SurelError(rc, "surel_sample_walks")
    return out


def build_rpe_raw(ctx: Context, walks: torch.Tensor, n_nodes: int, cap_rows: int,
                  rpe_off: torch.Tensor, rpe_ids: torch.Tensor | None,
                  rpe_cnt: torch.Tensor | None, want_rows: bool = True,
                  set_sizes: torch.Tensor | None = None):
    """One call of surel_build_rpe into caller buffers.  Returns (status, rows or None)."""
    n_seeds, M, L = walks.shape
    rows = _i64(-1)
    rc = load().surel_build_rpe(
        ctx.handle, _ptr(walks, torch.int32, "walks"), n_seeds, M, L - 1, n_nodes,
        _ptr(set_sizes, torch.int32, "set_sizes"), cap_rows,
        _ptr(rpe_off, torch.int64, "rpe_off"), _ptr(rpe_ids, torch.int32, "rpe_ids"),
        _ptr(rpe_cnt, torch.uint16, "rpe_cnt"), ctypes.byref(rows) if want_rows else None)
    return rc, (rows.value if want_rows else None)


def build_rpe(ctx: Context, walks: torch.Tensor, n_nodes: int, cap_rows: int | None = None,
              set_sizes: torch.Tensor | None = None):
    """(rpe_off int64[n_seeds+1], rpe_ids int32[R], rpe_cnt uint16[R][m+1]) on the GPU.

    ``cap_rows=None`` sizes the outputs with a counting call first; a number allocates that
    many rows up front (``rpe_rows_bound`` always suffices for sampled walks) and returns
    views of the first R rows.
    """
    n_seeds, M, L = walks.shape
    dev = walks.device
    off = torch.empty(n_seeds + 1, dtype=torch.int64, device=dev)
    if cap_rows is None:
        rc, rows = build_rpe_raw(ctx, walks, n_nodes, 0, off, None, None, set_sizes=set_sizes)
        if rc != OK:
            raise SurelError(rc, "surel_build_rpe (count)")
        cap_rows = rows
    ids = torch.empty(cap_rows, dtype=torch.int32, device=dev)
    cnt = torch.empty((cap_rows, L), dtype=torch.uint16, device=dev)
    rc, rows = build_rpe_raw(ctx, walks, n_nodes, cap_rows, off, ids, cnt, set_sizes=set_sizes)
    if rc != OK:
        raise SurelError(rc, "surel_build_rpe")
    return off, ids[:rows], cnt[:rows]


def build_rpe_count(ctx: Context, walks: torch.Tensor, n_nodes: int, rpe_off: torch.Tensor,
                    set_sizes: torch.Tensor | None = None, want_rows: bool = True):
    """surel_build_rpe_count: the table's layout only.  Returns (status, rows or None)."""
    n_seeds, M, L = walks.shape
    rows = _i64(-1)
    rc = load().surel_build_rpe_count(
        ctx.handle, _ptr(walks, torch.int32, "walks"), n_seeds, M, L - 1, n_nodes,
        _ptr(set_sizes, torch.int32, "set_sizes"), _ptr(rpe_off, torch.int64, "rpe_off"),
        ctypes.byref(rows) if want_rows else None)
    return rc, (rows.value if want_rows else None)


def build_rpe_fill(ctx: Context, walks: torch.Tensor, n_nodes: int, rpe_off: torch.Tensor,
                   cap_rows: int, rpe_ids: torch.Tensor, rpe_cnt: torch.Tensor) -> int:
    """surel_build_rpe_fill: the rows only, at the offsets given.  Returns the status."""
    n_seeds, M, L = walks.shape
    return load().surel_build_rpe_fill(
        ctx.handle, _ptr(walks, torch.int32, "walks"), n_seeds, M, L - 1, n_nodes,
        _ptr(rpe_off, torch.int64, "rpe_off"), cap_rows, _ptr(rpe_ids, torch.int32, "rpe_ids"),
        _ptr(rpe_cnt, torch.uint16, "rpe_cnt"))


def sample_walks_rpe_raw(ctx: Context, row_ptr: torch.Tensor, col_idx: torch.Tensor,
                         seeds: torch.Tensor, M: int, m: int, rng_seed: int, walks: torch.Tensor,
                         cap_rows: int, rpe_off: torch.Tensor, rpe_ids: torch.Tensor | None,
                         rpe_cnt: torch.Tensor | None, want_rows: bool = True):
    """One call of surel_sample_walks_rpe into caller buffers.  Returns (status, rows or None)."""
    n_seeds = seeds.numel()
    if walks.numel() != n_seeds * M * (m + 1):
        raise ValueError("walks has the wrong size")
    rows = _i64(-1)
    rc = load().surel_sample_walks_rpe(
        ctx.handle, _ptr(row_ptr, torch.int32, "row_ptr"), _ptr(col_idx, torch.int32, "col_idx"),
        row_ptr.numel() - 1, col_idx.numel(), _ptr(seeds, torch.int32, "seeds"), n_seeds, M, m,
        _u64(rng_seed), _ptr(walks, torch.int32, "walks"), cap_rows,
        _ptr(rpe_off, torch.int64, "rpe_off"), _ptr(rpe_ids, torch.int32, "rpe_ids"),
        _ptr(rpe_cnt, torch.uint16, "rpe_cnt"), ctypes.byref(rows) if want_rows else None)
    return rc, (rows.value if want_rows else None)


def sample_walks_rpe(ctx: Context, row_ptr: torch.Tensor, col_idx: torch.Tensor,
                     seeds: torch.Tensor, M: int, m: int, rng_seed: int = 0):
    """(walks, rpe_off, rpe_ids, rpe_cnt) from the fused kernel; the table is allocated at the
    ``rpe_rows_bound`` size and returned as views of its first R rows."""
    n_seeds = seeds.numel()
    dev = row_ptr.device
    walks = torch.empty((n_seeds, M, m + 1), dtype=torch.int32, device=dev)
    cap_rows = rpe_rows_bound(n_seeds, M, m)
    off = torch.empty(n_seeds + 1, dtype=torch.int64, device=dev)
    ids = torch.empty(cap_rows, dtype=torch.int32, device=dev)
    cnt = torch.empty((cap_rows, m + 1), dtype=torch.uint16, device=dev)
    rc, rows = sample_walks_rpe_raw(ctx, row_ptr, col_idx, seeds, M, m, rng_seed, walks, cap_rows,
                                    off, ids, cnt)
    if rc != OK:
        raise SurelError(rc, "surel_sample_walks_rpe")
    return walks, off, ids[:rows], cnt[:rows]


def sample_walks_rpe_ids_raw(ctx: Context, row_ptr: torch.Tensor, col_idx: torch.Tensor,
                             seeds: torch.Tensor, M: int, m: int, rng_seed: int,
                             walks: torch.Tensor, cap_rows: int, rpe_off: torch.Tensor,
                             rpe_ids: torch.Tensor, rpe_cnt: torch.Tensor | None,
                             code: torch.Tensor, cap_T: int, T: torch.Tensor):
    """One call of surel_sample_walks_rpe_ids into caller buffers.  Returns (status, rows, n_T)."""
    n_seeds = seeds.numel()
    if walks.numel() != n_seeds * M * (m + 1):
        raise ValueError("walks has the wrong size")
    rows, n_T = _i64(-1), _i64(-1)
    rc = load().surel_sample_walks_rpe_ids(
        ctx.handle, _ptr(row_ptr, torch.int32, "row_ptr"), _ptr(col_idx, torch.int32, "col_idx"),
        row_ptr.numel() - 1, col_idx.numel(), _ptr(seeds, torch.int32, "seeds"), n_seeds, M, m,
        _u64(rng_seed), _ptr(walks, torch.int32, "walks"), cap_rows,
        _ptr(rpe_off, torch.int64, "rpe_off"), _ptr(rpe_ids, torch.int32, "rpe_ids"),
        _ptr(rpe_cnt, torch.uint16, "rpe_cnt"), _ptr(code, torch.int32, "code"), cap_T,
        _ptr(T, torch.uint16, "T"), ctypes.byref(rows), ctypes.byref(n_T))
    return rc, rows.value, n_T.value


def sample_walks_rpe_ids(ctx: Context, row_ptr: torch.Tensor, col_idx: torch.Tensor,
                         seeds: torch.Tensor, M: int, m: int, rng_seed: int = 0,
                         cap_T: int = 1 << 20, with_counts: bool = True):
    """(walks, rpe_off, rpe_ids, rpe_cnt or None, code, T): walks, RPE table and pruned array from
    one call (Algorithm 1 from end to end); rows carry T's index of their count vector."""
    n_seeds = seeds.numel()
    dev = row_ptr.device
    walks = torch.empty((n_seeds, M, m + 1), dtype=torch.int32, device=dev)
    cap_rows = rpe_rows_bound(n_seeds, M, m)
    off = torch.empty(n_seeds + 1, dtype=torch.int64, device=dev)
    ids = torch.empty(cap_rows, dtype=torch.int32, device=dev)
    cnt = torch.empty((cap_rows, m + 1), dtype=torch.uint16, device=dev) if with_counts else None
    code = torch.empty(cap_rows, dtype=torch.int32, device=dev)
    T = torch.empty((cap_T, m + 1), dtype=torch.uint16, device=dev)
    rc, rows, n_T = sample_walks_rpe_ids_raw(ctx, row_ptr, col_idx, seeds, M, m, rng_seed, walks,
                                             cap_rows, off, ids, cnt, code, cap_T, T)
    if rc != OK:
        raise SurelError(rc, "surel_sample_walks_rpe_ids")
    return walks, off, ids[:rows], (cnt[:rows] if with_counts else None), code[:rows], T[:n_T]


def join_queries_raw(ctx: Context, rpe_off: torch.Tensor, rpe_ids: torch.Tensor,
                     rpe_cnt: torch.Tensor, queries: torch.Tensor, max_set: int, cap_rows: int,
                     join_off: torch.Tensor, join_ids: torch.Tensor | None,
                     join_cnt: torch.Tensor | None, want_rows: bool = True, noalloc: bool = False):
    """One call of surel_join_queries (noalloc: of surel_join_queries_noalloc, which takes its
    device scratch from a static array inside the library) into caller buffers.  Returns
    (status, rows or None)."""
    n_q, k = queries.shape
    L = rpe_cnt.shape[1]
    rows = _i64(-1)
    fn = load().surel_join_queries_noalloc if noalloc else load().surel_join_queries
    rc = fn(
        ctx.handle, _ptr(rpe_off, torch.int64, "rpe_off"), _ptr(rpe_ids, torch.int32, "rpe_ids"),
        _ptr(rpe_cnt, torch.uint16, "rpe_cnt"), rpe_off.numel() - 1, L - 1, max_set,
        _ptr(queries, torch.int32, "queries"), n_q, k, cap_rows,
        _ptr(join_off, torch.int64, "join_off"), _ptr(join_ids, torch.int32, "join_ids"),
        _ptr(join_cnt, torch.uint16, "join_cnt"), ctypes.byref(rows) if want_rows else None)
    return rc, (rows.value if want_rows else None)


def join_queries(ctx: Context, rpe_off: torch.Tensor, rpe_ids: torch.Tensor,
                 rpe_cnt: torch.Tensor, queries: torch.Tensor, max_set: int,
                 cap_rows: int | None = None):
    """(join_off int64[n_q+1], join_ids int32[J], join_cnt uint16[J][k][m+1]) on the GPU."""
    n_q, k = queries.shape
    L = rpe_cnt.shape[1]
    dev = queries.device
    off = torch.empty(n_q + 1, dtype=torch.int64, device=dev)
    if cap_rows is None:
        rc, rows = join_queries_raw(ctx, rpe_off, rpe_ids, rpe_cnt, queries, max_set, 0, off,
                                    None, None)
        if rc != OK:
            raise SurelError(rc, "surel_join_queries (count)")
        cap_rows = rows
    ids = torch.empty(cap_rows, dtype=torch.int32, device=dev)
    cnt = torch.empty((cap_rows, k, L), dtype=torch.uint16, device=dev)
    rc, rows = join_queries_raw(ctx, rpe_off, rpe_ids, rpe_cnt, queries, max_set, cap_rows, off,
                                ids, cnt)
    if rc != OK:
        raise SurelError(rc, "surel_join_queries")
    return off, ids[:rows], cnt[:rows]


def join_count(ctx: Context, rpe_off: torch.Tensor, rpe_ids: torch.Tensor, queries: torch.Tensor,
               max_set: int, join_off: torch.Tensor, want_rows: bool = True):
    """surel_join_count: the join's layout only.  Returns (status, rows or None)."""
    n_q, k = queries.shape
    rows = _i64(-1)
    rc = load().surel_join_count(
        ctx.handle, _ptr(rpe_off, torch.int64, "rpe_off"), _ptr(rpe_ids, torch.int32, "rpe_ids"),
        rpe_off.numel() - 1, max_set, _ptr(queries, torch.int32, "queries"), n_q, k,
        _ptr(join_off, torch.int64, "join_off"), ctypes.byref(rows) if want_rows else None)
    return rc, (rows.value if want_rows else None)


def join_fill(ctx: Context, rpe_off: torch.Tensor, rpe_ids: torch.Tensor, rpe_cnt: torch.Tensor,
              queries: torch.Tensor, max_set: int, join_off: torch.Tensor, cap_rows: int,
              join_ids: torch.Tensor, join_cnt: torch.Tensor) -> int:
    """surel_join_fill: the joined rows only, at the offsets given.  Returns the status."""
    n_q, k = queries.shape
    L = rpe_cnt.shape[1]
    return load().surel_join_fill(
        ctx.handle, _ptr(rpe_off, torch.int64, "rpe_off"), _ptr(rpe_ids, torch.int32, "rpe_ids"),
        _ptr(rpe_cnt, torch.uint16, "rpe_cnt"), rpe_off.numel() - 1, L - 1, max_set,
        _ptr(queries, torch.int32, "queries"), n_q, k, _ptr(join_off, torch.int64, "join_off"),
        cap_rows, _ptr(join_ids, torch.int32, "join_ids"), _ptr(join_cnt, torch.uint16, "join_cnt"))


def join_query_ids_raw(ctx: Context, rpe_off: torch.Tensor, rpe_ids: torch.Tensor,
                       code: torch.Tensor, queries: torch.Tensor, max_set: int, cap_rows: int,
                       join_off: torch.Tensor, join_ids: torch.Tensor | None,
                       join_codes: torch.Tensor | None, want_rows: bool = True):
    """One call of surel_join_query_ids into caller buffers.  Returns (status, rows or None)."""
    n_q, k = queries.shape
    rows = _i64(-1)
    rc = load().surel_join_query_ids(
        ctx.handle, _ptr(rpe_off, torch.int64, "rpe_off"), _ptr(rpe_ids, torch.int32, "rpe_ids"),
        _ptr(code, torch.int32, "code"), rpe_off.numel() - 1, max_set,
        _ptr(queries, torch.int32, "queries"), n_q, k, cap_rows,
        _ptr(join_off, torch.int64, "join_off"), _ptr(join_ids, torch.int32, "join_ids"),
        _ptr(join_codes, torch.int32, "join_codes"), ctypes.byref(rows) if want_rows else None)
    return rc, (rows.value if want_rows else None)


def join_query_ids(ctx: Context, rpe_off: torch.Tensor, rpe_ids: torch.Tensor, code: torch.Tensor,
                   queries: torch.Tensor, max_set: int):
    """(join_off int64[n_q+1], join_ids int32[J], join_codes int32[J][k]) on the GPU: the union
    join with the rows' codes (indices into the pruned array T, -1 = absent) instead of counts."""
    n_q, k = queries.shape
    dev = queries.device
    off = torch.empty(n_q + 1, dtype=torch.int64, device=dev)
    rc, rows = join_query_ids_raw(ctx, rpe_off, rpe_ids, code, queries, max_set, 0, off, None, None)
    if rc != OK:
        raise SurelError(rc, "surel_join_query_ids")
    ids = torch.empty(rows, dtype=torch.int32, device=dev)
    codes = torch.empty((rows, k), dtype=torch.int32, device=dev)
    rc, rows2 = join_query_ids_raw(ctx, rpe_off, rpe_ids, code, queries, max_set, rows, off, ids,
                                   codes)
    if rc != OK:
        raise SurelError(rc, "surel_join_query_ids")
    return off, ids, codes


def query_rpe_ids(ctx: Context, walks: torch.Tensor, rpe_off: torch.Tensor, rpe_ids: torch.Tensor,
                  queries: torch.Tensor, max_set: int, out: torch.Tensor | None = None,
                  code: torch.Tensor | None = None):
    """int32[n_q][k][M][m+1][k] on the GPU: the query-level RPE-IDs of every walk position (table
    rows; with `code` from prune_rpe, the rows' codes, i.e. indices into the pruned array T)."""
    if code is not None and code.numel() != rpe_ids.numel():
        raise ValueError("code must have one entry per table row")
    n_blocks, M, L = walks.shape
    n_q, k = queries.shape
    if out is None:
        out = torch.empty((n_q, k, M, L, k), dtype=torch.int32, device=walks.device)
    elif out.numel() != n_q * k * M * L * k:
        raise ValueError("out has the wrong size")
    rc = load().surel_query_rpe_ids(
        ctx.handle, _ptr(walks, torch.int32, "walks"), _ptr(rpe_off, torch.int64, "rpe_off"),
        _ptr(rpe_ids, torch.int32, "rpe_ids"), _ptr(code, torch.int32, "code"), n_blocks,
        rpe_ids.numel(), M, L - 1, max_set, _ptr(queries, torch.int32, "queries"), n_q, k,
        _ptr(out, torch.int32, "out"))
    if rc != OK:
        raise SurelError(rc, "surel_query_rpe_ids")
    return out


def prune_rpe_raw(ctx: Context, rpe_cnt: torch.Tensor, cap_T: int, T: torch.Tensor,
                  code: torch.Tensor):
    """One call of surel_prune_rpe into caller buffers.  Returns (status, n_T)."""
    n_rows, L = rpe_cnt.shape
    n_T = _i64(-1)
    rc = load().surel_prune_rpe(ctx.handle, _ptr(rpe_cnt, torch.uint16, "rpe_cnt"), n_rows, L - 1,
                                cap_T, _ptr(T, torch.uint16, "T"), _ptr(code, torch.int32, "code"),
                                ctypes.byref(n_T))
    return rc, n_T.value


def prune_rpe(ctx: Context, rpe_cnt: torch.Tensor, cap_T: int = 1 << 20):
    """(T uint16[n_T][m+1], code int32[R]) on the GPU: the distinct count vectors, sorted, and
    every row's index among them."""
    n_rows, L = rpe_cnt.shape
    T = torch.empty((cap_T, L), dtype=torch.uint16, device=rpe_cnt.device)
    code = torch.empty(n_rows, dtype=torch.int32, device=rpe_cnt.device)
    rc, n_T = prune_rpe_raw(ctx, rpe_cnt, cap_T, T, code)
    if rc != OK:
        raise SurelError(rc, "surel_prune_rpe")
    return T[:n_T], code


def query_incidence(ctx: Context, queries: torch.Tensor, n_nodes: int):
    """(inc_off int64[n_nodes+1], inc_q int32[n_queries*k]) on the GPU: for every node the
    indices of the queries that name it, ascending (surel_query_incidence)."""
    n_queries, k = queries.shape
    inc_off = torch.empty(n_nodes + 1, dtype=torch.int64, device=queries.device)
    inc_q = torch.empty(n_queries * k, dtype=torch.int32, device=queries.device)
    rc = load().surel_query_incidence(ctx.handle, _ptr(queries, torch.int32, "queries"), n_queries,
                                      k, n_nodes, _ptr(inc_off, torch.int64, "inc_off"),
                                      _ptr(inc_q, torch.int32, "inc_q"))
    if rc != OK:
        raise SurelError(rc, "surel_query_incidence")
    return inc_off, inc_q


def bfs_batches_raw(ctx: Context, queries, n_nodes: int, inc_off, inc_q, start, B1: int, B2: int,
                    vbar, batch, tuples, counts) -> int:
    """One call of surel_bfs_batches into caller buffers.  Returns the status."""
    n_queries, k = queries.shape
    n_batches, n_start = start.shape
    return load().surel_bfs_batches(
        ctx.handle, _ptr(queries, torch.int32, "queries"), n_queries, k, n_nodes,
        _ptr(inc_off, torch.int64, "inc_off"), _ptr(inc_q, torch.int32, "inc_q"),
        _ptr(start, torch.int32, "start"), n_batches, n_start, B1, B2,
        _ptr(vbar, torch.int32, "vbar"), _ptr(batch, torch.int32, "batch"),
        None if tuples is None else _ptr(tuples, torch.int32, "tuples"),
        _ptr(counts, torch.int32, "counts"))


def bfs_batches(ctx: Context, queries: torch.Tensor, n_nodes: int, inc_off: torch.Tensor,
                inc_q: torch.Tensor, start: torch.Tensor, B1: int, B2: int, want_tuples=True):
    """(vbar int32[n_batches][B1], batch int32[n_batches][B2], tuples int32[n_batches][B2][k] or
    None, counts int32[n_batches][2]) on the GPU: one mini-batch per row of `start`
    (surel_bfs_batches).  Only the first counts[b] entries of a row are written."""
    n_batches = start.shape[0]
    k = queries.shape[1]
    dev = queries.device
    vbar = torch.empty((n_batches, B1), dtype=torch.int32, device=dev)
    batch = torch.empty((n_batches, B2), dtype=torch.int32, device=dev)
    tuples = torch.empty((n_batches, B2, k), dtype=torch.int32, device=dev) if want_tuples else None
    counts = torch.empty((n_batches, 2), dtype=torch.int32, device=dev)
    rc = bfs_batches_raw(ctx, queries, n_nodes, inc_off, inc_q, start, B1, B2, vbar, batch, tuples,
                         counts)
    if rc != OK:
        raise SurelError(rc, "surel_bfs_batches")
    return vbar, batch, tuples, counts


_TYPES = {torch.bfloat16: BF16, torch.float16: FP16}


def _rows(t: torch.Tensor, like: torch.Tensor, what: str):
    """(address, elements between rows, elements between heads) of a [rows][heads][dim] tensor, whose rows
    and heads may lie apart."""
    if t.dtype != like.dtype:
        raise TypeError(f"{what} must be {like.dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{what} must live on the GPU")
    if t.dim() != 3:
        raise ValueError(f"{what} must be [rows][heads][dim]")
    row, head, one = t.stride()
    if one != 1 and t.shape[2] > 1:
        raise ValueError(f"{what}'s last dimension must be contiguous")
    return t.data_ptr(), row, head


def _attention_args(q, k, v, q_off, k_off, causal, scale, bias, bucket) -> AttentionArgs:
    if q.dtype not in _TYPES:
        raise TypeError(f"q must be torch.bfloat16 or torch.float16, got {q.dtype}")
    q_ptr, q_row, q_head = _rows(q, q, "q")
    k_ptr, k_row, k_head = _rows(k, q, "k")
    v_ptr, v_row, v_head = _rows(v, q, "v")
    n_q, heads, dim = q.shape
    if k.shape != v.shape or k.shape[2] != dim:
        raise ValueError("k and v must have one shape, and q's last dimension")
    if k_off is None:
        k_off = q_off
    if q_off.numel() != k_off.numel() or q_off.numel() < 1:
        raise ValueError("q_off and k_off must have one entry more than there are sequences")
    if (bias is None) != (bucket is None):
        raise ValueError("bias and bucket go together")
    if bias is not None and (bias.dim() != 2 or bias.shape[1] != heads or bucket.numel() % 2 != 1):
        raise ValueError("bias must be [buckets][heads], bucket have 2 * reach + 1 entries")
    return AttentionArgs(
        q_ptr, k_ptr, v_ptr, q_row, q_head, k_row, k_head, v_row, v_head,
        _ptr(q_off, torch.int64, "q_off"), _ptr(k_off, torch.int64, "k_off"), q_off.numel() - 1, n_q,
        k.shape[0], _TYPES[q.dtype], heads, k.shape[1], dim, 1 if causal else 0,
        dim ** -0.5 if scale is None else scale, _ptr(bias, q.dtype, "bias"),
        _ptr(bucket, torch.int32, "bucket"), 0 if bias is None else bias.shape[0],
        0 if bucket is None else bucket.numel() // 2)


def attention(ctx: Context, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q_off: torch.Tensor,
              k_off: torch.Tensor | None = None, causal: bool = False, scale: float | None = None,
              bias: torch.Tensor | None = None, bucket: torch.Tensor | None = None):
    """(out [n_q][heads][dim], lse float32[n_q][heads]) on the GPU: attention of packed query rows
    q [n_q][heads][dim] to packed keys k, v [n_k][kv_heads][dim] (bfloat16 or float16; views of a larger
    tensor will do).  Sequence s has rows q_off[s] .. q_off[s+1]-1 and keys k_off[s] .. k_off[s+1]-1 (int64,
    like join_off and rpe_off; k_off None: the same as q_off).  causal: a sequence's last row stands at its
    last key, rows see keys up to their own.  scale None: 1 / sqrt(dim).  bias [buckets][heads] and bucket
    int32[2 * reach + 1] (see distance_buckets): a learned bias by the distance of key and row.

    Sequences that attend to themselves share one q_off (k_off None, or the same tensor): with a bias, two tensors of the
    same numbers are slower where sequences are short.  The result has no gradient of its own, whatever its inputs
    require: attention_grad computes them (examples/walk_model.py makes a torch.autograd.Function of both)."""
    args = _attention_args(q, k, v, q_off, k_off, causal, scale, bias, bucket)
    out = q.new_empty(q.shape)
    lse = q.new_empty(q.shape[:2], dtype=torch.float32)
    rc = load().surel_attention(ctx.handle, ctypes.byref(args), out.data_ptr(), lse.data_ptr())
    if rc != OK:
        raise SurelError(rc, "surel_attention")
    return out, lse


def attention_grad(ctx: Context, dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                   out: torch.Tensor, lse: torch.Tensor, q_off: torch.Tensor,
                   k_off: torch.Tensor | None = None, causal: bool = False, scale: float | None = None,
                   bias: torch.Tensor | None = None, bucket: torch.Tensor | None = None):
    """(dq, dk, dv, dbias or None) on the GPU for the gradient dout of attention's out; out and lse are what
    attention returned, everything else what it was given.  Gradients have the shapes and the type of what
    they belong to, and are dense."""
    args = _attention_args(q, k, v, q_off, k_off, causal, scale, bias, bucket)
    if dout.shape != q.shape or out.shape != q.shape or lse.shape != q.shape[:2]:
        raise ValueError("dout and out must have q's shape, lse its first two dimensions")
    dq = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    dk = torch.empty(k.shape, dtype=q.dtype, device=q.device)
    dv = torch.empty(k.shape, dtype=q.dtype, device=q.device)
    dbias = None if bias is None else torch.empty(bias.shape, dtype=q.dtype, device=q.device)
    rc = load().surel_attention_grad(
        ctx.handle, ctypes.byref(args), _ptr(dout, q.dtype, "dout"), _ptr(out, q.dtype, "out"),
        _ptr(lse, torch.float32, "lse"), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
        None if dbias is None else dbias.data_ptr())
    if rc != OK:
        raise SurelError(rc, "surel_attention_grad")
    return dq, dk, dv, dbias


def distance_buckets(reach: int, buckets: int, causal: bool = False) -> list[int]:
    """The bucket of every distance -reach .. reach: near distances have one each, farther ones share ever
    wider ones up to reach.  Where all distances count, keys ahead have the upper half of the buckets; a
    causal row sees none of them.  (torch.tensor(..., dtype=torch.int32) of it is a `bucket` for attention.)"""
    half = buckets if causal else buckets // 2
    if reach < 0 or half < 1:
        raise ValueError("reach must not be negative, and each direction needs a bucket")
    near = max(1, half // 2)
    out = []
    for d in range(-reach, reach + 1):
        b = abs(d)
        if b >= near:
            # bucket b starts at near * (reach / near) ** ((b - near) / (half - near)), whole numbers compared
            b, far = near, half - near
            while b + 1 < half and abs(d) ** far * near ** (b + 1 - near) >= \
                    reach ** (b + 1 - near) * near ** far:
                b += 1
            b = min(b, half - 1)
        out.append(b if d <= 0 or causal else half + b)
    return out


def _loss_shape(h: torch.Tensor, w: torch.Tensor, labels: torch.Tensor) -> tuple[int, int, int, int]:
    """(type, rows, classes, dim), checked."""
    if h.dtype not in _TYPES:
        raise TypeError(f"h must be torch.bfloat16 or torch.float16, got {h.dtype}")
    if h.dim() != 2 or w.dim() != 2 or h.shape[1] != w.shape[1]:
        raise ValueError("h must be [rows][dim], w [classes][dim]")
    if labels.shape != h.shape[:1]:
        raise ValueError("labels must have one entry a row")
    return _TYPES[h.dtype], h.shape[0], w.shape[0], h.shape[1]


def softmax_loss(ctx: Context, h: torch.Tensor, w: torch.Tensor, labels: torch.Tensor):
    """(loss float32[rows], lse float32[rows]) on the GPU: softmax cross entropy of rows h [rows][dim] against all
    classes w [classes][dim] (bfloat16 or float16, dense), of which labels int32[rows] names each row's; a
    negative label: the row does not count, its loss is 0.  Logits are not kept.  The result has no gradient of its own,
    whatever its inputs require: softmax_loss_grad computes them."""
    kind, n, classes, dim = _loss_shape(h, w, labels)
    loss = h.new_empty(n, dtype=torch.float32)
    lse = h.new_empty(n, dtype=torch.float32)
    rc = load().surel_softmax_loss(ctx.handle, kind, _ptr(h, h.dtype, "h"), _ptr(w, h.dtype, "w"),
                                   _ptr(labels, torch.int32, "labels"), n, classes, dim, loss.data_ptr(),
                                   lse.data_ptr())
    if rc != OK:
        raise SurelError(rc, "surel_softmax_loss")
    return loss, lse


def softmax_loss_grad(ctx: Context, dloss: torch.Tensor, h: torch.Tensor, w: torch.Tensor, labels: torch.Tensor,
                      lse: torch.Tensor):
    """(dh, dw) on the GPU, of the shapes and type of h and w, for the gradient dloss float32[rows] of
    softmax_loss's loss; lse is what it returned, everything else what it was given."""
    kind, n, classes, dim = _loss_shape(h, w, labels)
    if dloss.shape != labels.shape or lse.shape != labels.shape:
        raise ValueError("dloss and lse must have one entry a row")
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    rc = load().surel_softmax_loss_grad(
        ctx.handle, kind, _ptr(dloss, torch.float32, "dloss"), _ptr(h, h.dtype, "h"), _ptr(w, h.dtype, "w"),
        _ptr(labels, torch.int32, "labels"), _ptr(lse, torch.float32, "lse"), n, classes, dim, dh.data_ptr(),
        dw.data_ptr())
    if rc != OK:
        raise SurelError(rc, "surel_softmax_loss_grad")
    return dh, dw


def _beside(ctx: Context, tensors, *outputs):
    """Tensors that the context's stream may read and write: the given ones have to be on its device, and new ones, a (shape,
    dtype) each, are made there and returned.  Where torch works on another stream at the moment, the given ones are kept from
    being given away before the context's is done with them, and the new ones are that stream's own memory, kept likewise:
    memory of torch's present stream may be what its unfinished work still reads or writes."""
    index = ctx.device.index or 0
    for t in tensors:
        if t is not None and t.get_device() != index:   # (-1: not on a GPU)
            raise ValueError(f"every tensor must live on the context's cuda:{index}, got {t.device}")
    some = tensors[0]
    present = torch.cuda.current_stream(ctx.device)
    if present == ctx.stream:
        return [some.new_empty(shape, dtype=dtype) for shape, dtype in outputs]
    for t in tensors:
        if t is not None:
            t.record_stream(ctx.stream)
    with torch.cuda.stream(ctx.stream):
        made = [some.new_empty(shape, dtype=dtype) for shape, dtype in outputs]
    for t in made:
        t.record_stream(present)
    return made


def cache_plan(ctx: Context, length: torch.Tensor, added: torch.Tensor, pages: torch.Tensor, ring: torch.Tensor,
               turn: torch.Tensor, page_rows: int, n_rows: int):
    """(off int64[seqs+1], slots int32[n_rows], length int32[seqs], turn int64[2]) on the GPU: one step of a paged cache's
    bookkeeping (surel_cache_plan).  Sequence s has length[s] keys (int32) and adds added[s] rows, or ends and gives its
    pages back where that is negative.  pages int32[seqs][max_pages] gets its new pages' numbers, taken from ring
    int32[n_pages], whose free entries are those from turn[0] to turn[1] (int64; modulo n_pages); both are changed in place.
    Row i of sequence s, packed at off[s] + i, has the slot slots[off[s] + i], page * page_rows + row of the page; rows
    without a place, and those behind the last sequence's, have -1.  length and turn are what the next step starts from.

    A cache of all free pages: ring torch.arange(n_pages), turn (0, n_pages), lengths of zero."""
    if pages.dim() != 2 or length.shape != pages.shape[:1] or added.shape != length.shape:
        raise ValueError("pages must be [sequences][max_pages], length and added have an entry a sequence")
    if ring.dim() != 1 or turn.shape != (2,):
        raise ValueError("ring must have an entry a page, turn two")
    n, width = pages.shape
    off, slots, after, turn_after = _beside(ctx, (length, added, pages, ring, turn), (n + 1, torch.int64),
                                            (n_rows, torch.int32), (n, torch.int32), (2, torch.int64))
    rc = load().surel_cache_plan(
        ctx.handle, _ptr(length, torch.int32, "length"), _ptr(added, torch.int32, "added"), n, ring.shape[0], page_rows,
        width, n_rows, _ptr(pages, torch.int32, "pages"), _ptr(ring, torch.int32, "ring"),
        _ptr(turn, torch.int64, "turn"), off.data_ptr(), slots.data_ptr(), after.data_ptr(), turn_after.data_ptr())
    if rc != OK:
        raise SurelError(rc, "surel_cache_plan")
    return off, slots, after, turn_after


def _cache(k_pages: torch.Tensor, v_pages: torch.Tensor) -> Cache:
    if k_pages.dtype not in _TYPES:
        raise TypeError(f"k_pages must be torch.bfloat16 or torch.float16, got {k_pages.dtype}")
    if v_pages.dtype != k_pages.dtype:
        raise TypeError(f"v_pages must be {k_pages.dtype}, got {v_pages.dtype}")
    if not k_pages.is_cuda or not v_pages.is_cuda:
        raise ValueError("k_pages and v_pages must live on the GPU")
    if k_pages.dim() != 4 or k_pages.shape != v_pages.shape or k_pages.stride() != v_pages.stride():
        raise ValueError("k_pages and v_pages must be [pages][page_rows][kv_heads][dim], and lie alike")
    page, row, head, one = k_pages.stride()
    n_pages, page_rows, kv_heads, dim = k_pages.shape
    if one != 1 and dim > 1:
        raise ValueError("the last dimension of k_pages and v_pages must be contiguous")
    return Cache(k_pages.data_ptr(), v_pages.data_ptr(), page, row, head, n_pages, page_rows, _TYPES[k_pages.dtype], kv_heads,
                 dim)


def cache_store(ctx: Context, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, k_pages: torch.Tensor,
                v_pages: torch.Tensor) -> None:
    """Writes the rows k, v [rows][kv_heads][dim] (views of a larger tensor will do) into their slots (int32[rows], from
    cache_plan; -1: left out) of k_pages, v_pages [pages][page_rows][kv_heads][dim], bfloat16 or float16.  Pages whose
    heads lie outside their rows, as views of [pages][kv_heads][page_rows][dim], will do as well."""
    cache = _cache(k_pages, v_pages)
    k_ptr, k_row, k_head = _rows(k, k_pages, "k")
    v_ptr, v_row, v_head = _rows(v, k_pages, "v")
    if k.shape != v.shape or k.shape[1:] != k_pages.shape[2:] or slots.shape != k.shape[:1]:
        raise ValueError("k and v must be [rows][kv_heads][dim] of the pages' heads and dim, slots have an entry a row")
    _beside(ctx, (k, v, slots, k_pages, v_pages))
    rc = load().surel_cache_store(ctx.handle, ctypes.byref(cache), k_ptr, v_ptr, k_row, k_head, v_row, v_head,
                                  _ptr(slots, torch.int32, "slots"), k.shape[0])
    if rc != OK:
        raise SurelError(rc, "surel_cache_store")


def cache_attention(ctx: Context, q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, pages: torch.Tensor,
                    length: torch.Tensor, scale: float | None = None, bias: torch.Tensor | None = None,
                    bucket: torch.Tensor | None = None):
    """(out [seqs][heads][dim], lse float32[seqs][heads]) on the GPU: attention of one row a sequence, its newest,
    q [seqs][heads][dim], to the length[s] keys (int32, its own among them) that the sequence has in the pages
    pages[s] (int32[seqs][max_pages]) of k_pages, v_pages (see cache_store).  scale, bias and bucket as for attention; the
    row stands at its sequence's last key.  What attention(causal=True) gives for these rows over the same keys, packed."""
    cache = _cache(k_pages, v_pages)
    q_ptr, q_row, q_head = _rows(q, k_pages, "q")
    n, heads, dim = q.shape
    if dim != k_pages.shape[3] or pages.dim() != 2 or pages.shape[0] != n or length.shape != (n,):
        raise ValueError("q must have the pages' dim, pages and length a row and an entry a sequence")
    if (bias is None) != (bucket is None):
        raise ValueError("bias and bucket go together")
    if bias is not None and (bias.dim() != 2 or bias.shape[1] != heads or bucket.numel() % 2 != 1):
        raise ValueError("bias must be [buckets][heads], bucket have 2 * reach + 1 entries")
    args = CacheAttentionArgs(
        q_ptr, q_row, q_head, _ptr(pages, torch.int32, "pages"), _ptr(length, torch.int32, "length"), n, pages.shape[1],
        heads, dim ** -0.5 if scale is None else scale, _ptr(bias, q.dtype, "bias"), _ptr(bucket, torch.int32, "bucket"),
        0 if bias is None else bias.shape[0], 0 if bucket is None else bucket.numel() // 2)
    out, lse = _beside(ctx, (q, k_pages, v_pages, pages, length, bias, bucket), (q.shape, q.dtype), (q.shape[:2], torch.float32))
    rc = load().surel_cache_attention(ctx.handle, ctypes.byref(cache), ctypes.byref(args), out.data_ptr(), lse.data_ptr())
    if rc != OK:
        raise SurelError(rc, "surel_cache_attention")
    return out, lse


def sample_classes(ctx: Context, logits: torch.Tensor, u: torch.Tensor, temperature: torch.Tensor | None = None,
                   top_k: torch.Tensor | None = None, top_p: torch.Tensor | None = None, min_p: torch.Tensor | None = None):
    """(classes int32[rows], logp float32[rows]) on the GPU: a class for every row of logits [rows][classes] (bfloat16,
    float16 or float32; rows may lie apart), drawn with the uniform numbers u float32[rows] in [0, 1), and the logarithm of the
    probability that it had.  temperature float32[rows] (0: the largest logit's first class), top_k int32[rows] (below 1: not
    in use), top_p (1: not in use) and min_p float32[rows] (0: not in use); see surel_sample_classes for what they keep.
    A row without a class to draw has -1."""
    kinds = {**_TYPES, torch.float32: FP32}
    if logits.dtype not in kinds:
        raise TypeError(f"logits must be torch.bfloat16, torch.float16 or torch.float32, got {logits.dtype}")
    if not logits.is_cuda:
        raise ValueError("logits must live on the GPU")
    if logits.dim() != 2 or (logits.stride(1) != 1 and logits.shape[1] > 1):
        raise ValueError("logits must be [rows][classes], the classes of a row contiguous")
    n, classes = logits.shape
    if any(t is not None and t.shape != (n,) for t in (u, temperature, top_k, top_p, min_p)):
        raise ValueError("u, temperature, top_k, top_p and min_p must have one entry a row")
    chosen, logp = _beside(ctx, (logits, u, temperature, top_k, top_p, min_p), (n, torch.int32), (n, torch.float32))
    rc = load().surel_sample_classes(
        ctx.handle, kinds[logits.dtype], logits.data_ptr(), logits.stride(0), n, classes, _ptr(u, torch.float32, "u"),
        _ptr(temperature, torch.float32, "temperature"), _ptr(top_k, torch.int32, "top_k"),
        _ptr(top_p, torch.float32, "top_p"), _ptr(min_p, torch.float32, "min_p"), chosen.data_ptr(), logp.data_ptr())
    if rc != OK:
        raise SurelError(rc, "surel_sample_classes")
    return chosen, logp
