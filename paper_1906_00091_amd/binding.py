"""Thin ctypes binding of libdlrm_hot.so: same names as the C ABI, argument
marshalling only.  torch supplies device memory and the current HIP stream;
every step of the path runs in the library's kernels.  There is no fallback:
if the library is missing or a call fails, an exception is raised."""
from __future__ import annotations

import ctypes as C
import os
import struct
import threading
from typing import List, Optional, Sequence

import torch

from . import build as _build

F32, F16, BF16 = 0, 1, 2
I64, I32 = 0, 1
BWD_AUTO, BWD_SORT, BWD_ATOMIC, BWD_SORT_PREPARED, BWD_SORT_PREPARED_FLAT = 0, 1, 2, 3, 4
FWD_AUTO, FWD_FUSED, FWD_SPLIT = 0, 1, 2
ROPE_HALF, ROPE_INTERLEAVED = 0, 1
_TORCH_DTYPE = {F32: torch.float32, F16: torch.float16, BF16: torch.bfloat16}
_ELEM = {F32: 4, F16: 2, BF16: 2}


class DlrmError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        super().__init__("%s failed: status %d (%s)" % (fn, status, status_string(status)))


class _BwdTimingC(C.Structure):
    _fields_ = [("ev_start", C.c_void_p), ("ev_stop", C.c_void_p)]


class _SparseBatchC(C.Structure):
    _fields_ = [
        ("K", C.c_int32), ("B", C.c_int32), ("d", C.c_int32), ("table_dtype", C.c_int32),
        ("nnz_total", C.c_int64), ("max_rows", C.c_int64),
        ("tables", C.c_void_p), ("rows", C.c_void_p), ("indices", C.c_void_p),
        ("offsets", C.c_void_p), ("tbl_off", C.c_void_p), ("weights", C.c_void_p),
        ("index_dtype", C.c_int32),
    ]


class _QkRopeC(C.Structure):
    _fields_ = [
        ("T", C.c_int64), ("Hq", C.c_int32), ("Hk", C.c_int32), ("d", C.c_int32), ("dtype", C.c_int32),
        ("rot", C.c_int32), ("layout", C.c_int32), ("positions", C.c_void_p), ("inv_freq", C.c_void_p),
        ("wq", C.c_void_p), ("wk", C.c_void_p), ("eps", C.c_float), ("mscale", C.c_float),
    ]


class _KvCacheC(C.Structure):
    _fields_ = [
        ("k", C.c_void_p), ("v", C.c_void_p), ("table", C.c_void_p), ("B", C.c_int32), ("table_cols", C.c_int32),
        ("n_pages", C.c_int32), ("page", C.c_int32), ("Hk", C.c_int32), ("d", C.c_int32), ("dtype", C.c_int32),
    ]


class _SeqBatchC(C.Structure):
    _fields_ = [
        ("B", C.c_int32), ("causal", C.c_int32), ("Tq", C.c_int64), ("Tk", C.c_int64), ("max_q", C.c_int32),
        ("max_k", C.c_int32), ("q_off", C.c_void_p), ("k_off", C.c_void_p), ("prefix", C.c_void_p),
        ("slopes", C.c_void_p), ("scale", C.c_float), ("cap", C.c_float),
    ]


_lib = None


def lib() -> C.CDLL:
    """Loads the built library; builds it only if nothing is built."""
    global _lib
    if _lib is None:
        path = _build.LIB
        if not os.path.exists(path):
            _build.build(force=True)
        L = C.CDLL(path)
        vp, i32, i64, f32, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_size_t
        sb = C.POINTER(_SparseBatchC)
        L.dlrm_version.restype = i32
        L.dlrm_version.argtypes = []
        L.dlrm_status_string.restype = C.c_char_p
        L.dlrm_status_string.argtypes = [i32]
        L.dlrm_lengths_to_offsets.restype = i32
        L.dlrm_lengths_to_offsets.argtypes = [vp, i32, i32, vp, vp, vp]
        L.dlrm_validate_csr.restype = i32
        L.dlrm_validate_csr.argtypes = [sb, vp, vp]
        L.dlrm_emb_bag_fwd.restype = i32
        L.dlrm_emb_bag_fwd.argtypes = [sb, vp, i64, i64, vp]
        L.dlrm_place_dense.restype = i32
        L.dlrm_place_dense.argtypes = [vp, i32, i32, vp, i32, vp]
        L.dlrm_interact_dot_fwd.restype = i32
        L.dlrm_interact_dot_fwd.argtypes = [vp, i32, i32, i32, vp, vp]
        L.dlrm_emb_interact_fwd.restype = i32
        L.dlrm_emb_interact_fwd.argtypes = [sb, vp, vp, vp, i32, vp]
        L.dlrm_emb_interact_fwd_stamped.restype = i32
        L.dlrm_emb_interact_fwd_stamped.argtypes = [sb, vp, vp, vp, i32, vp, C.c_uint32, vp]
        L.dlrm_emb_interact_bwd.restype = i32
        L.dlrm_emb_interact_bwd.argtypes = [sb, vp, vp, vp, vp]
        L.dlrm_interact_dot_bwd.restype = i32
        L.dlrm_interact_dot_bwd.argtypes = [vp, vp, i32, i32, i32, vp, vp]
        L.dlrm_emb_bag_bwd_workspace_bytes.restype = sz
        L.dlrm_emb_bag_bwd_workspace_bytes.argtypes = [i32, i32, i32, i64, i64, i32]
        L.dlrm_emb_bag_bwd_sgd.restype = i32
        L.dlrm_emb_bag_bwd_sgd.argtypes = [sb, vp, i64, i64, f32, vp, sz, i32, vp]
        L.dlrm_emb_bag_bwd_sgd_noalloc.restype = i32
        L.dlrm_emb_bag_bwd_sgd_noalloc.argtypes = [sb, vp, i64, i64, f32, vp]
        L.dlrm_emb_bag_bwd_adagrad.restype = i32
        L.dlrm_emb_bag_bwd_adagrad.argtypes = [sb, vp, vp, i64, i64, f32, f32, vp, sz, i32, vp]
        L.dlrm_emb_bag_bwd_prepare.restype = i32
        L.dlrm_emb_bag_bwd_prepare.argtypes = [sb, vp, sz, vp]
        L.dlrm_emb_bag_bwd_prepared_oversized.restype = i32
        L.dlrm_emb_bag_bwd_prepared_oversized.argtypes = [sb, vp, sz, vp, vp]
        L.dlrm_emb_bag_bwd_route_counts.restype = i32
        L.dlrm_emb_bag_bwd_route_counts.argtypes = [sb, vp, sz, vp, vp]
        L.dlrm_emb_bag_bwd_export_groups.restype = i32
        L.dlrm_emb_bag_bwd_export_groups.argtypes = [sb, vp, sz, vp, vp, vp, vp, vp]
        L.dlrm_table_init_hash.restype = i32
        L.dlrm_table_init_hash.argtypes = [vp, i64, i32, i32, C.c_uint64, f32, vp]
        tm = C.POINTER(_BwdTimingC)
        L.dlrm_emb_bag_bwd_sgd_timed.restype = i32
        L.dlrm_emb_bag_bwd_sgd_timed.argtypes = [sb, vp, i64, i64, f32, vp, sz, i32, tm, vp]
        L.dlrm_emb_bag_bwd_adagrad_timed.restype = i32
        L.dlrm_emb_bag_bwd_adagrad_timed.argtypes = [sb, vp, vp, i64, i64, f32, f32, vp, sz, i32, tm, vp]
        rp, kc, sq = C.POINTER(_QkRopeC), C.POINTER(_KvCacheC), C.POINTER(_SeqBatchC)
        hd = vp  # dlrm_heads*
        L.dlrm_qk_rope_fwd.restype = i32
        L.dlrm_qk_rope_fwd.argtypes = [rp, hd, hd, hd, hd, vp]
        L.dlrm_qk_rope_bwd_workspace_bytes.restype = sz
        L.dlrm_qk_rope_bwd_workspace_bytes.argtypes = [rp]
        L.dlrm_qk_rope_bwd.restype = i32
        L.dlrm_qk_rope_bwd.argtypes = [rp, hd, hd, hd, hd, hd, hd, vp, vp, vp, sz, vp]
        L.dlrm_qk_rope_append.restype = i32
        L.dlrm_qk_rope_append.argtypes = [rp, hd, hd, hd, hd, kc, vp, vp]
        L.dlrm_seq_attn_fwd.restype = i32
        L.dlrm_seq_attn_fwd.argtypes = [sq, i32, i32, i32, i32, hd, hd, hd, hd, vp, vp]
        L.dlrm_seq_attn_bwd_workspace_bytes.restype = sz
        L.dlrm_seq_attn_bwd_workspace_bytes.argtypes = [sq, i32, i32, i32, i32]
        L.dlrm_seq_attn_bwd.restype = i32
        L.dlrm_seq_attn_bwd.argtypes = [sq, i32, i32, i32, i32, hd, hd, hd, hd, vp, hd, hd, hd, hd, vp, sz, vp]
        L.dlrm_cache_attn_workspace_bytes.restype = sz
        L.dlrm_cache_attn_workspace_bytes.argtypes = [kc, i32, i32]
        L.dlrm_cache_attn.restype = i32
        L.dlrm_cache_attn.argtypes = [kc, vp, i32, i32, hd, hd, vp, f32, f32, vp, sz, vp]
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().dlrm_status_string(int(status)).decode()


def version() -> int:
    return int(lib().dlrm_version())


def _check(fn: str, status: int) -> None:
    if status != 0:
        raise DlrmError(fn, status)


def _stream() -> int:
    """Handle of torch's current stream on the current device, what torch.cuda.current_stream().cuda_stream is.  That makes
    two Python objects on the way (2.8 us; 0.2 us here), more than a whole launch takes the host: a batch of 64 scored in one
    launch 6.7 / 4.4 us."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


class SparseBatch:
    """Device-side sparse batch: owns the pointer array and keeps the tensors alive."""

    def __init__(self, tables: Sequence[torch.Tensor], table_dtype: int, indices: torch.Tensor,
                 offsets: torch.Tensor, tbl_off: torch.Tensor, nnz_total: int,
                 max_rows: Optional[int] = None, weights: Optional[torch.Tensor] = None):
        self.tables = list(tables)
        K = len(self.tables)
        d = int(self.tables[0].shape[1])
        dev = indices.device if indices.numel() else offsets.device
        for t in self.tables:
            assert t.is_contiguous() and t.dtype == _TORCH_DTYPE[table_dtype] and t.shape[1] == d
        assert offsets.dtype == torch.int64 and offsets.is_contiguous() and offsets.shape[0] == K
        assert indices.dtype in (torch.int64, torch.int32) and tbl_off.dtype == torch.int64
        assert indices.is_contiguous()
        self.K, self.B, self.d = K, int(offsets.shape[1]) - 1, d
        self.table_dtype = table_dtype
        self.indices, self.offsets, self.tbl_off = indices, offsets, tbl_off
        if weights is not None:
            assert weights.dtype == torch.float32 and weights.is_contiguous() and weights.shape == indices.shape
        self.weights = weights
        rows_host = [int(t.shape[0]) for t in self.tables]
        self.rows = torch.tensor(rows_host, dtype=torch.int64, device=dev)
        self.table_ptrs = torch.tensor([t.data_ptr() for t in self.tables], dtype=torch.int64,
                                       device=dev)
        self.nnz_total = int(nnz_total)
        self.max_rows = int(max(rows_host) if max_rows is None else max_rows)
        self.c = _SparseBatchC(K, self.B, d, table_dtype, self.nnz_total, self.max_rows,
                               _ptr(self.table_ptrs), _ptr(self.rows),
                               _ptr(indices) if indices.numel() else None,
                               _ptr(offsets), _ptr(tbl_off),
                               _ptr(weights) if weights is not None and weights.numel() else None,
                               I32 if indices.dtype == torch.int32 else I64)

    def ref(self):
        return C.byref(self.c)


# ------------------------------------------------------------------ the C ABI, one to one
def dlrm_lengths_to_offsets(lengths: torch.Tensor, offsets: torch.Tensor, tbl_off: torch.Tensor):
    K, B = lengths.shape
    assert lengths.dtype == torch.int32 and lengths.is_contiguous()
    _check("dlrm_lengths_to_offsets",
           lib().dlrm_lengths_to_offsets(_ptr(lengths), K, B, _ptr(offsets), _ptr(tbl_off), _stream()))


def dlrm_validate_csr(batch: SparseBatch, n_bad: torch.Tensor):
    _check("dlrm_validate_csr", lib().dlrm_validate_csr(batch.ref(), _ptr(n_bad), _stream()))


def dlrm_emb_bag_fwd(batch: SparseBatch, out: torch.Tensor, stride_b: int, stride_k: int,
                     out_offset: int = 0):
    """out_offset: element offset into `out` (e.g. d, to write rows 1..K of T[B,F,d])."""
    _check("dlrm_emb_bag_fwd",
           lib().dlrm_emb_bag_fwd(batch.ref(), _ptr(out) + 4 * out_offset, stride_b, stride_k,
                                  _stream()))


def dlrm_place_dense(x: torch.Tensor, T: torch.Tensor):
    B, F, d = T.shape
    _check("dlrm_place_dense", lib().dlrm_place_dense(_ptr(x), B, d, _ptr(T), F, _stream()))


def dlrm_interact_dot_fwd(T: torch.Tensor, R: torch.Tensor):
    B, F, d = T.shape
    _check("dlrm_interact_dot_fwd", lib().dlrm_interact_dot_fwd(_ptr(T), B, F, d, _ptr(R), _stream()))


def dlrm_emb_interact_fwd(batch: SparseBatch, x: torch.Tensor, T: torch.Tensor, R: torch.Tensor,
                          algo: int = FWD_AUTO):
    _check("dlrm_emb_interact_fwd",
           lib().dlrm_emb_interact_fwd(batch.ref(), _ptr(x), _ptr(T), _ptr(R), algo, _stream()))


def dlrm_emb_interact_fwd_stamped(batch: SparseBatch, x: torch.Tensor, T: torch.Tensor, R: torch.Tensor,
                                  algo: int, stamp: torch.Tensor, stamp_value: int, index: int = 0):
    """stamp: int32 tensor the device can write (device memory, or host memory allocated pinned);
    element `index` receives stamp_value when the call's first kernel starts."""
    assert stamp.dtype == torch.int32 and (stamp.is_cuda or stamp.is_pinned()) and 0 <= index < stamp.numel()
    _check("dlrm_emb_interact_fwd_stamped",
           lib().dlrm_emb_interact_fwd_stamped(batch.ref(), _ptr(x), _ptr(T), _ptr(R), algo,
                                               _ptr(stamp) + 4 * index, stamp_value & 0xFFFFFFFF, _stream()))


def dlrm_emb_interact_bwd(batch: SparseBatch, x: torch.Tensor, dR: torch.Tensor, dT: torch.Tensor):
    """dT of the interaction with the pooled vectors formed again from the tables (no T)."""
    assert x.dtype == torch.float32 and x.is_contiguous() and x.shape == (batch.B, batch.d)
    F = batch.K + 1
    assert dR.dtype == torch.float32 and dR.is_contiguous() and dR.shape == (batch.B, batch.d + F * (F - 1) // 2)
    assert dT.dtype == torch.float32 and dT.is_contiguous() and dT.shape == (batch.B, F, batch.d)
    _check("dlrm_emb_interact_bwd", lib().dlrm_emb_interact_bwd(batch.ref(), _ptr(x), _ptr(dR), _ptr(dT), _stream()))


def dlrm_interact_dot_bwd(T: torch.Tensor, dR: torch.Tensor, dT: torch.Tensor):
    B, F, d = T.shape
    _check("dlrm_interact_dot_bwd",
           lib().dlrm_interact_dot_bwd(_ptr(T), _ptr(dR), B, F, d, _ptr(dT), _stream()))


def dlrm_emb_bag_bwd_workspace_bytes(K: int, B: int, d: int, nnz_total: int, max_rows: int,
                                     table_dtype: int) -> int:
    return int(lib().dlrm_emb_bag_bwd_workspace_bytes(K, B, d, nnz_total, max_rows, table_dtype))


def dlrm_emb_bag_bwd_sgd(batch: SparseBatch, dS: torch.Tensor, stride_b: int, stride_k: int,
                         lr: float, workspace: Optional[torch.Tensor], algo: int = BWD_AUTO,
                         dS_offset: int = 0):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check("dlrm_emb_bag_bwd_sgd",
           lib().dlrm_emb_bag_bwd_sgd(batch.ref(), _ptr(dS) + 4 * dS_offset, stride_b, stride_k,
                                      C.c_float(lr), _ptr(workspace), ws_bytes, algo, _stream()))


def _timing(ev_start, ev_stop):
    """ev_start / ev_stop: raw hipEvent_t handles (ints or c_void_p)."""
    val = lambda e: e.value if isinstance(e, C.c_void_p) else e
    return _BwdTimingC(val(ev_start), val(ev_stop))


def dlrm_emb_bag_bwd_sgd_timed(batch: SparseBatch, dS: torch.Tensor, stride_b: int, stride_k: int,
                               lr: float, workspace: Optional[torch.Tensor], ev_start, ev_stop,
                               algo: int = BWD_AUTO, dS_offset: int = 0):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    tm = _timing(ev_start, ev_stop)
    _check("dlrm_emb_bag_bwd_sgd_timed",
           lib().dlrm_emb_bag_bwd_sgd_timed(batch.ref(), _ptr(dS) + 4 * dS_offset, stride_b, stride_k,
                                            C.c_float(lr), _ptr(workspace), ws_bytes, algo, C.byref(tm), _stream()))


def dlrm_emb_bag_bwd_adagrad_timed(batch: SparseBatch, state_ptrs: torch.Tensor, dS: torch.Tensor, stride_b: int,
                                   stride_k: int, lr: float, eps: float, workspace: Optional[torch.Tensor],
                                   ev_start, ev_stop, algo: int = BWD_AUTO, dS_offset: int = 0):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    tm = _timing(ev_start, ev_stop)
    _check("dlrm_emb_bag_bwd_adagrad_timed",
           lib().dlrm_emb_bag_bwd_adagrad_timed(batch.ref(), _ptr(state_ptrs), _ptr(dS) + 4 * dS_offset, stride_b,
                                                stride_k, C.c_float(lr), C.c_float(eps), _ptr(workspace), ws_bytes,
                                                algo, C.byref(tm), _stream()))


NOALLOC_SCRATCH_BYTES = 64 << 20


def dlrm_emb_bag_bwd_sgd_noalloc(batch: SparseBatch, dS: torch.Tensor, stride_b: int, stride_k: int, lr: float,
                                 dS_offset: int = 0):
    """The update on the library's own per-GPU scratch array (no workspace argument, no allocation)."""
    _check("dlrm_emb_bag_bwd_sgd_noalloc",
           lib().dlrm_emb_bag_bwd_sgd_noalloc(batch.ref(), _ptr(dS) + 4 * dS_offset, stride_b, stride_k,
                                              C.c_float(lr), _stream()))


def dlrm_emb_bag_bwd_adagrad(batch: SparseBatch, state_ptrs: torch.Tensor, dS: torch.Tensor, stride_b: int,
                             stride_k: int, lr: float, eps: float, workspace: Optional[torch.Tensor],
                             algo: int = BWD_AUTO, dS_offset: int = 0):
    """state_ptrs: int64 device tensor [K] of the accumulators' addresses (see state_pointers)."""
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check("dlrm_emb_bag_bwd_adagrad",
           lib().dlrm_emb_bag_bwd_adagrad(batch.ref(), _ptr(state_ptrs), _ptr(dS) + 4 * dS_offset, stride_b,
                                          stride_k, C.c_float(lr), C.c_float(eps), _ptr(workspace), ws_bytes,
                                          algo, _stream()))


def state_pointers(state: Sequence[torch.Tensor]) -> torch.Tensor:
    """Device array of the K accumulators' base addresses; the caller keeps `state` alive."""
    for h in state:
        assert h.dtype == torch.float32 and h.is_contiguous()
    return torch.tensor([h.data_ptr() for h in state], dtype=torch.int64, device=state[0].device)


def dlrm_emb_bag_bwd_prepare(batch: SparseBatch, workspace: torch.Tensor,
                             stream: Optional[torch.cuda.Stream] = None):
    """Enqueued on `stream`, or like every other call on torch's current stream."""
    ws_bytes = workspace.numel() * workspace.element_size()
    _check("dlrm_emb_bag_bwd_prepare",
           lib().dlrm_emb_bag_bwd_prepare(batch.ref(), _ptr(workspace), ws_bytes,
                                          _stream() if stream is None else int(stream.cuda_stream)))


def dlrm_emb_bag_bwd_prepared_oversized(batch: SparseBatch, workspace: torch.Tensor, out: torch.Tensor,
                                        index: int = 0, stream: Optional[torch.cuda.Stream] = None):
    """out: int32 tensor the device can write (device memory, or host memory allocated pinned);
    element `index` receives the count once the stream has passed this call."""
    assert out.dtype == torch.int32 and (out.is_cuda or out.is_pinned()) and 0 <= index < out.numel()
    ws_bytes = workspace.numel() * workspace.element_size()
    _check("dlrm_emb_bag_bwd_prepared_oversized",
           lib().dlrm_emb_bag_bwd_prepared_oversized(batch.ref(), _ptr(workspace), ws_bytes,
                                                     _ptr(out) + 4 * index,
                                                     _stream() if stream is None else int(stream.cuda_stream)))


ROUTE_NAMES = ("heavy_ranges", "oversized_ranges", "segments", "segment_tiles", "dominant_row_splits",
               "global_sorts", "one_row_ranges", "huge_runs_in_place", "hot_rows", "dense_hot_tables")


def dlrm_emb_bag_bwd_route_counts(batch: SparseBatch, workspace: torch.Tensor, counts: torch.Tensor):
    """counts: int32 device tensor of >= 10 elements (see ROUTE_NAMES)."""
    assert counts.dtype == torch.int32 and counts.is_cuda and counts.numel() >= 10
    ws_bytes = workspace.numel() * workspace.element_size()
    _check("dlrm_emb_bag_bwd_route_counts",
           lib().dlrm_emb_bag_bwd_route_counts(batch.ref(), _ptr(workspace), ws_bytes, _ptr(counts), _stream()))


def dlrm_emb_bag_bwd_export_groups(batch: SparseBatch, workspace: torch.Tensor,
                                   uniq_rows: torch.Tensor, seg_start: torch.Tensor,
                                   sorted_bag: torch.Tensor, n_uniq: torch.Tensor):
    ws_bytes = workspace.numel() * workspace.element_size()
    _check("dlrm_emb_bag_bwd_export_groups",
           lib().dlrm_emb_bag_bwd_export_groups(batch.ref(), _ptr(workspace), ws_bytes,
                                                _ptr(uniq_rows), _ptr(seg_start), _ptr(sorted_bag),
                                                _ptr(n_uniq), _stream()))


def dlrm_table_init_hash(table: torch.Tensor, table_dtype: int, key: int, scale: float):
    rows, d = table.shape
    _check("dlrm_table_init_hash",
           lib().dlrm_table_init_hash(_ptr(table), rows, d, table_dtype, C.c_uint64(key),
                                      C.c_float(scale), _stream()))


def alloc_workspace(batch: SparseBatch) -> torch.Tensor:
    n = dlrm_emb_bag_bwd_workspace_bytes(batch.K, batch.B, batch.d, batch.nnz_total, batch.max_rows,
                                         batch.table_dtype)
    if n == 0:
        raise DlrmError("dlrm_emb_bag_bwd_workspace_bytes", -2)
    # torch's caching allocator returns 512-byte aligned blocks
    return torch.empty(n, dtype=torch.uint8, device=batch.offsets.device)


# ------------------------------------------------------------------ a history in order
_DTYPE_OF = {t: c for c, t in _TORCH_DTYPE.items()}


class _Scratch(threading.local):
    """The dlrm_heads of one call, 24 bytes each, which the library reads before it returns.  Written by one pack: an object
    per tensor costs the host 0.4 us more each, and a backward pass has eight."""

    def __init__(self):
        self.buf = bytearray(8 * 24)
        self.at = C.addressof((C.c_char * len(self.buf)).from_buffer(self.buf))


_scratch = _Scratch()
_PACK = [struct.Struct("%dq" % (3 * n)).pack_into for n in range(9)]


def _heads(fn: str, dtype: int, rows):
    """Addresses of the dlrm_heads of `rows`, pairs of a tensor [items, heads, d] (any item and head stride, columns next to each other)
    and the shape it has to have."""
    want = _TORCH_DTYPE[dtype]
    vals = []
    for x, shape in rows:
        if x.shape != shape:
            raise ValueError("%s: a tensor of shape %s where %s is wanted" % (fn, tuple(x.shape), shape))
        if x.dtype is not want:
            raise DlrmError(fn, -3)
        t, h, c = x.stride()
        if c != 1 != shape[2]:
            raise ValueError("%s: the columns of a head have to lie next to each other, got strides %s" % (fn, x.stride()))
        vals += (x.data_ptr(), t, h)
    s = _scratch
    _PACK[len(rows)](s.buf, 0, *vals)
    return range(s.at, s.at + 24 * len(rows), 24)


def _first(fn: str, x: torch.Tensor):
    """(shape, storage type) of the tensor that the others of a call go by."""
    if x.dim() != 3:
        raise ValueError("%s: rows of heads are [items, heads, d], got %s" % (fn, tuple(x.shape)))
    dt = _DTYPE_OF.get(x.dtype)
    if dt is None:
        raise DlrmError(fn, -3)
    return x.shape, dt


def _vector(fn: str, x: Optional[torch.Tensor], n: int, dtype: torch.dtype) -> Optional[int]:
    if x is None:
        return None
    if x.dtype != dtype or x.numel() != n or not x.is_contiguous():
        raise ValueError("%s: a contiguous %s array of %d elements is wanted, got %s %s" % (fn, dtype, n, x.dtype, tuple(x.shape)))
    return x.data_ptr()


def _workspace(x: Optional[torch.Tensor]):
    return (None, 0) if x is None else (x.data_ptr(), x.numel() * x.element_size())


class QkRope:
    """Norm and rotary position of Hq query and Hk key heads of d columns for the items at `positions` (dlrm_qk_rope).
    wq, wk: norm weights or None; inv_freq: radians per position of every rotated pair (see rope_frequencies)."""

    def __init__(self, positions: Optional[torch.Tensor], Hq: int, Hk: int, d: int, inv_freq: Optional[torch.Tensor] = None,
                 rot: Optional[int] = None, layout: int = ROPE_HALF, wq: Optional[torch.Tensor] = None,
                 wk: Optional[torch.Tensor] = None, eps: float = 1e-6, mscale: float = 1.0, T: Optional[int] = None):
        if rot is None:
            rot = 0 if inv_freq is None else 2 * inv_freq.numel()
        if T is None:
            if positions is None:
                raise ValueError("QkRope: positions or the number of items T is needed")
            T = positions.numel()
        self.T, self.Hq, self.Hk, self.d = int(T), Hq, Hk, d
        self.positions, self.inv_freq, self.wq, self.wk = positions, inv_freq, wq, wk
        self.fields = (rot, layout, _vector("QkRope", positions, self.T, torch.int32), _vector("QkRope", inv_freq, rot // 2, torch.float32),
                       _vector("QkRope", wq, d, torch.float32), _vector("QkRope", wk, d, torch.float32), eps, mscale)
        self.c = {}  # a struct for each storage type, written once: calls of several threads may use the plan at once

    def ref(self, dtype: int):
        c = self.c.get(dtype)
        if c is None:  # (as in SeqBatch.ref)
            c = self.c[dtype] = _QkRopeC(self.T, self.Hq, self.Hk, self.d, dtype, *self.fields)
        return C.byref(c)


def rope_frequencies(rot: int, base: float = 10000.0, stretch: float = 1.0, keep_turns: Optional[float] = None,
                     drop_turns: float = 1.0, trained_length: int = 0, device=None) -> torch.Tensor:
    """inv_freq of QkRope: base ** (-2 i / rot), positions divided by `stretch` for histories that long times the trained ones.  With
    keep_turns the division is by parts: a pair that turns at least keep_turns times over trained_length keeps its frequency, one
    that turns at most drop_turns times is divided, those between are blended linearly in their number of turns."""
    f = base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    if keep_turns is None:
        f = f / stretch
    else:
        if not (trained_length > 0 and keep_turns > drop_turns):
            raise ValueError("rope_frequencies: keep_turns > drop_turns and the trained length are needed for scaling by parts")
        turns = trained_length * f / 6.283185307179586
        keep = ((turns - drop_turns) / (keep_turns - drop_turns)).clamp(0, 1)
        f = f * (keep + (1 - keep) / stretch)
    return f.to(torch.float32).to(device)


def dlrm_qk_rope_fwd(rope: QkRope, q: torch.Tensor, k: Optional[torch.Tensor], q_out: torch.Tensor, k_out: Optional[torch.Tensor]):
    """q, q_out: [T, Hq, d]; k, k_out: [T, Hk, d] (None for Hk = 0).  An output may be its input."""
    fn = "dlrm_qk_rope_fwd"
    dt = _first(fn, q)[1]
    rq, rk = (rope.T, rope.Hq, rope.d), (rope.T, rope.Hk, rope.d)
    if rope.Hk:
        a, b, c, d = _heads(fn, dt, ((q, rq), (k, rk), (q_out, rq), (k_out, rk)))
    else:
        (a, c), b, d = _heads(fn, dt, ((q, rq), (q_out, rq))), None, None
    _check(fn, lib().dlrm_qk_rope_fwd(rope.ref(dt), a, b, c, d, _stream()))


def dlrm_qk_rope_bwd(rope: QkRope, q: torch.Tensor, k: Optional[torch.Tensor], dq_out: torch.Tensor, dk_out: Optional[torch.Tensor],
                     dq: torch.Tensor, dk: Optional[torch.Tensor], dwq: Optional[torch.Tensor], dwk: Optional[torch.Tensor],
                     workspace: Optional[torch.Tensor]):
    """Gradients dq, dk of the forward's inputs (may be dq_out, dk_out) and dwq, dwk (fp32 [d], written) of the norm weights."""
    fn = "dlrm_qk_rope_bwd"
    dt = _first(fn, q)[1]
    rq, rk = (rope.T, rope.Hq, rope.d), (rope.T, rope.Hk, rope.d)
    if rope.Hk:
        v = _heads(fn, dt, ((q, rq), (k, rk), (dq_out, rq), (dk_out, rk), (dq, rq), (dk, rk)))
    else:
        a, b, c = _heads(fn, dt, ((q, rq), (dq_out, rq), (dq, rq)))
        v = (a, None, b, None, c, None)
    ws, ws_bytes = _workspace(workspace)
    _check(fn, lib().dlrm_qk_rope_bwd(rope.ref(dt), *v, _vector(fn, dwq, rope.d, torch.float32), _vector(fn, dwk, rope.d, torch.float32), ws,
                                      ws_bytes, _stream()))


def alloc_qk_rope_workspace(rope: QkRope) -> torch.Tensor:
    # (sized for any storage type: the widest rows take the most groups)
    n = max(int(lib().dlrm_qk_rope_bwd_workspace_bytes(rope.ref(t))) for t in (F32, F16, BF16))
    if n == 0:
        raise DlrmError("dlrm_qk_rope_bwd_workspace_bytes", -2)
    device = next((x.device for x in (rope.positions, rope.wq, rope.wk) if x is not None), None)
    return torch.empty(n, dtype=torch.uint8, device=device)


class KvCache:
    """Pages of keys and values, k and v: [n_pages, Hk, page, d]; table: int32 [B, pages of a sequence] (dlrm_kv_cache)."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor):
        if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype or not (k.is_contiguous() and v.is_contiguous()):
            raise ValueError("KvCache: k and v are contiguous [pages, heads, items of a page, d] of one type")
        if table.dim() != 2 or table.dtype != torch.int32 or not table.is_contiguous():
            raise ValueError("KvCache: the table is a contiguous int32 [sequences, pages of a sequence]")
        if k.dtype not in _DTYPE_OF:
            raise DlrmError("KvCache", -3)
        self.k, self.v, self.table = k, v, table
        self.B = int(table.shape[0])
        self.n_pages, self.Hk, self.page, self.d = (int(x) for x in k.shape)
        self.dtype = _DTYPE_OF[k.dtype]
        self.c = _KvCacheC(k.data_ptr(), v.data_ptr(), table.data_ptr(), self.B, int(table.shape[1]), self.n_pages, self.page, self.Hk,
                           self.d, self.dtype)

    def ref(self):
        return C.byref(self.c)


def dlrm_qk_rope_append(rope: QkRope, q, k, v, q_out, cache: KvCache, seqs: torch.Tensor):
    """Queries to q_out, keys (normed and rotated) and values to the cache, item t as item positions[t] of sequence seqs[t]."""
    fn = "dlrm_qk_rope_append"
    dt = _first(fn, q)[1]
    if not rope.Hk:
        raise DlrmError(fn, -2)
    rq, rk = (rope.T, rope.Hq, rope.d), (rope.T, rope.Hk, rope.d)
    _check(fn, lib().dlrm_qk_rope_append(rope.ref(dt), *_heads(fn, dt, ((q, rq), (k, rk), (v, rk), (q_out, rq))), cache.ref(),
                                         _vector(fn, seqs, rope.T, torch.int32), _stream()))


class SeqBatch:
    """Sequences that attend (dlrm_seq_batch).  q_off, k_off: int64 [B + 1]; Tq, Tk: their last elements; max_q, max_k: bounds on a
    sequence's items; scale: of the products, 1 / sqrt(d) unless given."""

    def __init__(self, q_off: torch.Tensor, k_off: torch.Tensor, Tq: int, Tk: int, max_q: int, max_k: int, causal: bool = True,
                 prefix: Optional[torch.Tensor] = None, slopes: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                 cap: float = 0.0):
        self.B = int(q_off.numel()) - 1
        self.q_off, self.k_off, self.prefix, self.slopes, self.scale = q_off, k_off, prefix, slopes, scale
        if slopes is not None and (slopes.dtype != torch.float32 or not slopes.is_contiguous()):
            raise ValueError("SeqBatch: slopes are contiguous float32, one for each query head")
        self.Tq, self.Tk = int(Tq), int(Tk)
        self.fields = (self.B, int(causal), self.Tq, self.Tk, max_q, max_k, _vector("SeqBatch", q_off, self.B + 1, torch.int64),
                       _vector("SeqBatch", k_off, self.B + 1, torch.int64), _vector("SeqBatch", prefix, self.B, torch.int32), _ptr(slopes))
        self.cap = cap
        self.c = {}  # a struct for each width of the heads, written once: calls of several threads may use the plan at once

    def ref(self, Hq: int, d: int):
        if self.slopes is not None and self.slopes.numel() != Hq:
            raise ValueError("SeqBatch: %d slopes for %d query heads" % (self.slopes.numel(), Hq))
        c = self.c.get(d)
        if c is None:
            # (of two threads that come here at once one's struct is kept, and the other's, the same values, lives as long as its reference)
            c = self.c[d] = _SeqBatchC(*self.fields, d ** -0.5 if self.scale is None else self.scale, self.cap)
        return C.byref(c)


def dlrm_seq_attn_fwd(seq: SeqBatch, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, lse: Optional[torch.Tensor] = None):
    """q, out: [Tq, Hq, d]; k, v: [Tk, Hk, d]; lse: fp32 [Hq, Tq] for the backward, or None."""
    fn = "dlrm_seq_attn_fwd"
    (_, Hq, d), dt = _first(fn, q)
    Hk = _first(fn, k)[0][1]
    rq, rk = (seq.Tq, Hq, d), (seq.Tk, Hk, d)
    _check(fn, lib().dlrm_seq_attn_fwd(seq.ref(Hq, d), Hq, Hk, d, dt, *_heads(fn, dt, ((q, rq), (k, rk), (v, rk), (out, rq))),
                                       _vector(fn, lse, Hq * seq.Tq, torch.float32), _stream()))


def dlrm_seq_attn_bwd(seq: SeqBatch, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, lse: torch.Tensor, dout: torch.Tensor,
                      dq: torch.Tensor, dk: torch.Tensor, dv: torch.Tensor, workspace: torch.Tensor):
    """out, lse: the forward's; dout: gradient of out; dq, dk, dv: written."""
    fn = "dlrm_seq_attn_bwd"
    (_, Hq, d), dt = _first(fn, q)
    Hk = _first(fn, k)[0][1]
    rq, rk = (seq.Tq, Hq, d), (seq.Tk, Hk, d)
    h = _heads(fn, dt, ((q, rq), (k, rk), (v, rk), (out, rq), (dout, rq), (dq, rq), (dk, rk), (dv, rk)))
    ws, ws_bytes = _workspace(workspace)
    _check(fn, lib().dlrm_seq_attn_bwd(seq.ref(Hq, d), Hq, Hk, d, dt, h[0], h[1], h[2], h[3], _vector(fn, lse, Hq * seq.Tq, torch.float32),
                                       h[4], h[5], h[6], h[7], ws, ws_bytes, _stream()))


def alloc_seq_attn_workspace(seq: SeqBatch, Hq: int, Hk: int, d: int, dtype: Optional[int] = None) -> torch.Tensor:
    """For rows of one storage type, or of any."""
    n = max(int(lib().dlrm_seq_attn_bwd_workspace_bytes(seq.ref(Hq, d), Hq, Hk, d, t)) for t in ((F32, F16, BF16) if dtype is None else (dtype,)))
    if n == 0:
        raise DlrmError("dlrm_seq_attn_bwd_workspace_bytes", -2)
    return torch.empty(n, dtype=torch.uint8, device=seq.q_off.device)


def dlrm_cache_attn(cache: KvCache, lens: torch.Tensor, max_len: int, q: torch.Tensor, out: torch.Tensor, workspace: Optional[torch.Tensor],
                    slopes: Optional[torch.Tensor] = None, scale: Optional[float] = None, cap: float = 0.0):
    """q, out: [B, Hq, d]; lens: int32 [B], items of every sequence in the cache, its newest among them."""
    fn = "dlrm_cache_attn"
    Hq = _first(fn, q)[0][1]
    rows = (cache.B, Hq, cache.d)
    a, b = _heads(fn, cache.dtype, ((q, rows), (out, rows)))
    ws, ws_bytes = _workspace(workspace)
    _check(fn, lib().dlrm_cache_attn(cache.ref(), _vector(fn, lens, cache.B, torch.int32), max_len, Hq, a, b,
                                     _vector(fn, slopes, Hq, torch.float32), cache.d ** -0.5 if scale is None else scale, cap, ws, ws_bytes,
                                     _stream()))


def alloc_cache_attn_workspace(cache: KvCache, Hq: int, max_len: int) -> torch.Tensor:
    n = int(lib().dlrm_cache_attn_workspace_bytes(cache.ref(), Hq, max_len))
    if n == 0:
        raise DlrmError("dlrm_cache_attn_workspace_bytes", -2)
    return torch.empty(n, dtype=torch.uint8, device=cache.table.device)
