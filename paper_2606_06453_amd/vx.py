"""Thin ctypes binding of ``libvx.so`` (declared in ``include/vx.h``).

Argument marshalling only: every step of the decode path runs in the library's HIP
kernels.  torch supplies device memory and the current stream.  If the library is
missing the binding raises; there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libvx.so")

MEAN_DOT, QUEST, MAX_DOT = 0, 1, 2
QUEST_CONSENSUS, ENVELOPE_LOWER, QUEST_RECTIFIED = 3, 4, 5     # Appendix G envelope flows
MEAN_DOT_CONTENT, NSA, MEAN_DOT_SMOOTH = 6, 7, 8                 # rope-unaware, NSA, smoothing
NEEDS_MEAN = (MEAN_DOT, MEAN_DOT_CONTENT, NSA, MEAN_DOT_SMOOTH)
TWO_PASS_KINDS = (MEAN_DOT, MEAN_DOT_CONTENT)                    # may pass the bf16 Mean copy
NEEDS_MAX = (MAX_DOT, QUEST, QUEST_CONSENSUS, ENVELOPE_LOWER, QUEST_RECTIFIED)
NEEDS_MIN = (QUEST, QUEST_CONSENSUS, ENVELOPE_LOWER)
STAGE_SCORE_TOPK, STAGE_DECODE = 0, 1
KV_BF16, KV_FP8_E4M3, KV_FP8_E5M2, KV_MXFP4 = 0, 1, 2, 3


def kv_dtype_code(t: torch.Tensor) -> int:
    """vx_kv_dtype of a cache tensor: bfloat16, float8_e4m3fn (OCP E4M3), float8_e5m2, or uint8 for
    the slices of an mxfp4 cache (mxfp4_cache)."""
    code = _KV_CODES.get(t.dtype)
    if code is None:
        raise TypeError(f"KV cache dtype {t.dtype} is not bfloat16, float8_e4m3fn, float8_e5m2 or uint8 (mxfp4)")
    return code


_KV_CODES = {torch.bfloat16: KV_BF16, torch.float8_e4m3fn: KV_FP8_E4M3, torch.float8_e5m2: KV_FP8_E5M2,
             torch.uint8: KV_MXFP4}


def mxfp4_cache(num_pages: int, num_kv_heads: int, page_size: int, head_dim: int, device="cuda") -> torch.Tensor:
    """An mxfp4 K or V cache of zeros, uint8 [P][H][page_size][17 D / 32]: codes and scales of a
    (page, head) slice as include/vx.h lays them out."""
    return torch.zeros((num_pages, num_kv_heads, page_size, head_dim * 17 // 32), dtype=torch.uint8, device=device)
TWO_PASS_MAX_PAGES = 16384    # block-mean two-pass selection: blocks per request bound
# Below this many summary rows (batch x blocks per request x KV heads) the decoder scores the
# block mean in one pass: the bound pass saves half the summary bytes, but its re-scoring of the
# undecided pages adds a dependent round trip to the top-K kernel, which a short score stream does
# not pay back (MLA geometry, 16384 rows: score + top-K 22.9 us in one pass against 25.1 us in
# two; Llama-3-8B-shaped layer, 10^6 rows: 54.5 us in two passes against 72.8 us in one).
TWO_PASS_MIN_ROWS = 65536

_STATUS = {0: "VX_OK", 1: "VX_ERR_INVALID_ARG", 2: "VX_ERR_UNSUPPORTED", 3: "VX_ERR_WORKSPACE", 4: "VX_ERR_HIP"}


class VxError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{_STATUS.get(status, status)}: {msg}")
        self.status = status


class _Cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("num_phys_pages", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("head_dim_qk", ctypes.c_int32), ("head_dim_v", ctypes.c_int32), ("kv_dtype", ctypes.c_int32),
                ("k_scale", ctypes.c_float), ("v_scale", ctypes.c_float), ("block_size", ctypes.c_int32)]


class _Pool(ctypes.Structure):
    _fields_ = [("free_pages", ctypes.c_void_p), ("free_count", ctypes.c_void_p), ("table", ctypes.c_void_p),
                ("lens", ctypes.c_void_p), ("num_phys_pages", ctypes.c_int32), ("table_rows", ctypes.c_int32),
                ("table_stride", ctypes.c_int32), ("page_size", ctypes.c_int32), ("block_size", ctypes.c_int32)]


class _Rope(ctypes.Structure):
    _fields_ = [("inv_freq", ctypes.c_void_p), ("axis", ctypes.c_void_p), ("num_axes", ctypes.c_int32),
                ("first", ctypes.c_int32), ("dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("scale", ctypes.c_float)]


class _Chunk(ctypes.Structure):
    _fields_ = [("q_indptr", ctypes.c_void_p), ("q_lens", ctypes.c_void_p), ("num_rows", ctypes.c_int32)]


class _Batch(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("max_pages_per_seq", ctypes.c_int32),
                ("page_indptr", ctypes.c_void_p), ("page_indices", ctypes.c_void_p),
                ("seq_lens", ctypes.c_void_p)]


_lib = None


def lib():
    """Load libvx.so from the package directory (never a fallback)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
                               f"or python paper_2606_06453_amd/build.py")
        L = ctypes.CDLL(LIB_PATH)
        P, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        L.vx_version.restype = ctypes.c_uint32
        L.vx_last_error.restype = ctypes.c_char_p
        L.vx_workspace_size.argtypes = [i32, P, P, i32, i32, ctypes.POINTER(sz)]
        L.vx_page_summarize.argtypes = [P, P, P, P, P, P, P, P]
        L.vx_page_score_topk.argtypes = [P, i32, P, P, i32, P, P, P, P, P, i32, i32, i32, P, P, P, sz, P, P]
        L.vx_sparse_paged_decode.argtypes = [P, i32, P, P, P, P, i32, ctypes.c_float, P, P, sz, P]
        L.vx_page_score.argtypes = [P, i32, P, P, i32, P, P, P, P, i32, P]
        L.vx_topk_select.argtypes = [P, i32, i32, i32, P, P, i32, i32, i32, P, P, P, P]
        L.vx_score_flow.argtypes = [i32, P, P, i32, i32, i32, i32, P, P]
        L.vx_stream_read.argtypes = [P, sz, P, i32, P]
        L.vx_kv_append_summarize.argtypes = [P, P, P, P, P, P, P, P, P]
        L.vx_sparse_paged_decode_noalloc.argtypes = [P, i32, P, P, P, P, i32, ctypes.c_float, P, P]
        L.vx_append_score_topk.argtypes = [P, P, P, P, P, P, P, P, P, i32, i32, P, i32, i32, i32, P, P, P, sz, P, P]
        i64 = ctypes.c_int64
        L.vx_page_workspace_size.argtypes = [i32, ctypes.POINTER(sz)]
        L.vx_page_extend.argtypes = [P, i32, P, P, P, P, P, i32, P, P, i32, P, P, P, sz, P]
        L.vx_page_release.argtypes = [P, i32, P, P, P, sz, P]
        L.vx_kv_write.argtypes = [P, P, i64, i64, P, i64, i64, P, i32, P]
        L.vx_kv_read.argtypes = [P, P, i64, i64, P, i64, i64, P, i32, P]
        L.vx_rope_kv_write.argtypes = [P, P, P, i64, i64, i32, P, i64, i64, P, i64, i64, P, i64, i64, P, i64, P, i32, P]
        L.vx_chunk_workspace_size.argtypes = [i32, P, P, i32, i32, i32, ctypes.POINTER(sz)]
        L.vx_chunk_attention.argtypes = [P, i64, i64, i32, P, P, P, i32, i32, ctypes.c_float, P, P, P, sz, P]
        L.vx_chunk_score_topk.argtypes = [P, i64, i64, i32, P, P, P, i32, P, P, i32, i32, i32, P, P, P, sz, P]
        L.vx_sparse_chunk_attention.argtypes = [P, i64, i64, i32, P, P, P, P, P, i32, ctypes.c_float, P, P, P, sz, P]
        for f in (L.vx_rope_kv_write, L.vx_chunk_workspace_size, L.vx_chunk_attention, L.vx_chunk_score_topk,
                  L.vx_sparse_chunk_attention):
            f.restype = ctypes.c_int
        for f in (L.vx_page_workspace_size, L.vx_page_extend, L.vx_page_release, L.vx_kv_write, L.vx_kv_read):
            f.restype = ctypes.c_int
        for f in (L.vx_workspace_size, L.vx_page_summarize, L.vx_page_score_topk, L.vx_sparse_paged_decode,
                  L.vx_page_score, L.vx_topk_select, L.vx_score_flow, L.vx_kv_append_summarize,
                  L.vx_stream_read, L.vx_sparse_paged_decode_noalloc, L.vx_append_score_topk):
            f.restype = ctypes.c_int
        _lib = L
    return _lib


def version() -> int:
    return int(lib().vx_version())


def _check(status: int):
    if status != 0:
        raise VxError(status, lib().vx_last_error().decode())


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    assert t.is_contiguous(), "tensors passed to libvx must be contiguous"
    return t.data_ptr()


# The handle of the current stream, without the Stream object (2.7 us of a call's 10).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda device: torch.cuda.current_stream(device).cuda_stream)


# The current device, without the check that the runtime has started (a tensor on a GPU has seen to that).
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _stream(stream, device: Optional[int] = None) -> Optional[int]:
    if stream is None:
        return _raw_stream(torch.cuda.current_device() if device is None else device)
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


@dataclass
class PagedKV:
    """Paged KV cache: k [P][H][ps][Dqk], v [P][H][ps][Dv] or None (V = K[..., :Dv]); bf16,
    fp8 (float8_e4m3fn / float8_e5m2) codes whose values are k_scale * code and v_scale * code, or
    mxfp4 slices (uint8, mxfp4_cache)."""
    k: torch.Tensor
    v: Optional[torch.Tensor]
    head_dim_v: Optional[int] = None
    k_scale: float = 1.0
    v_scale: float = 1.0
    block_size: int = 0      # 0: one block per page; else 16 or 32 dividing the page size

    def struct(self) -> _Cache:
        k, v = self.k, self.v
        P, H, ps, Dqk = k.shape
        dt = kv_dtype_code(k)
        if v is None:
            Dv = self.head_dim_v or (self._mx_dim(Dqk) if dt == KV_MXFP4 else Dqk)
        else:
            Pv, Hv, psv, Dv = v.shape
            if v.dtype is not k.dtype:
                kv_dtype_code(v)
                raise TypeError("K and V caches must have the same dtype")
            d = k.get_device()
            if v.get_device() != d or (d < 0 and v.device != k.device):
                raise ValueError(f"K and V caches must be on one device (got {k.device} and {v.device})")
            if Hv != H or psv != ps or Pv < P:
                raise ValueError(f"the V cache must have K's pages, KV heads and page size (got {tuple(v.shape)} "
                                 f"beside {tuple(k.shape)})")
        if dt == KV_MXFP4:
            row, Dqk = Dqk, self._mx_dim(Dqk)
            if v is not None:
                Dv = Dqk if Dv == row else self._mx_dim(Dv)
        return _Cache(_ptr(k), _ptr(v), P, H, ps, Dqk, Dv, dt, float(self.k_scale), float(self.v_scale),
                      int(self.block_size))

    @staticmethod
    def _mx_dim(row_bytes: int) -> int:
        if row_bytes % 17:
            raise ValueError(f"an mxfp4 cache has 17 bytes per 32 channels of a token (got rows of {row_bytes} bytes)")
        return row_bytes // 17 * 32

    @property
    def head_dim_qk(self) -> int:
        return self._mx_dim(self.k.shape[3]) if kv_dtype_code(self.k) == KV_MXFP4 else self.k.shape[3]

    @property
    def row_dtype(self) -> torch.dtype:
        """Element type of new rows at a decode step: the cache's own, bf16 for an mxfp4 cache."""
        return torch.bfloat16 if kv_dtype_code(self.k) == KV_MXFP4 else self.k.dtype

    def __setattr__(self, name, value):
        self.__dict__[name] = value
        self.__dict__["_ref"] = None

    def ref(self):
        """A by-reference argument holding this geometry, built once for the fields' present values."""
        if self._ref is None:
            d = self.__dict__
            st = d["_st"] = self.struct()
            d["_dims"] = st.num_kv_heads, st.head_dim_qk, st.head_dim_v
            d["_seen"] = self._tensors()
            d["_ref"] = ctypes.byref(st)
        return self._ref

    def _tensors(self):
        k, v = self.k, self.v
        return (k.data_ptr(), k.dtype, k.shape, k.is_contiguous(),
                None if v is None else (v.data_ptr(), v.dtype, v.shape, v.is_contiguous()))

    def current(self):
        """ref(), built again where a tensor has taken other memory, another type or shape in place."""
        if self._ref is not None and self._seen != self._tensors():
            self.__dict__["_ref"] = None
        return self.ref()


@dataclass
class BatchSpec:
    """Ragged batch over the paged cache: int32 device tensors plus a host bound on P_i."""
    page_indptr: torch.Tensor
    page_indices: torch.Tensor
    seq_lens: torch.Tensor
    max_pages_per_seq: int

    def struct(self) -> _Batch:
        return _Batch(self.seq_lens.numel(), int(self.max_pages_per_seq), _ptr(self.page_indptr),
                      _ptr(self.page_indices), _ptr(self.seq_lens))

    def ref(self):
        """A by-reference argument holding this batch, built once (see PagedKV.ref)."""
        if getattr(self, "_ref", None) is None:
            self._st = self.struct()
            self._ref = ctypes.byref(self._st)
        return self._ref

    def current(self):
        """ref(), built again for the tensors and the bound as they are now."""
        self._ref = None
        return self.ref()

    def kept(self):
        """A by-reference argument holding this batch as it is now: built again where a tensor has other memory or
        another length, or the bound has changed, since."""
        lens = self.seq_lens
        at = (self.page_indptr.data_ptr(), self.page_indices.data_ptr(), lens.data_ptr(), lens.numel(), self.max_pages_per_seq)
        kept = self.__dict__.get("_kept")
        if kept is None or kept[0] != at:
            _counts(max_pages_per_seq=self.max_pages_per_seq)
            st = self.struct()
            kept = self.__dict__["_kept"] = (at, ctypes.byref(st))
        return kept[1]


@dataclass
class PagePool:
    """Pages, block table and lengths of growing requests (vx_page_pool): int32 device tensors
    free_pages [num_phys_pages], free_count [1], table [rows][stride] and lens [rows]."""
    free_pages: torch.Tensor
    free_count: torch.Tensor
    table: torch.Tensor
    lens: torch.Tensor
    page_size: int
    block_size: int = 0

    @classmethod
    def empty(cls, num_phys_pages: int, table_rows: int, table_stride: int, page_size: int, block_size: int = 0,
              device="cuda") -> "PagePool":
        """A pool whose pages are all free (page 0 is the first to go) and whose rows are empty."""
        i32 = dict(dtype=torch.int32, device=device)
        return cls(torch.arange(num_phys_pages - 1, -1, -1, **i32), torch.full((1,), num_phys_pages, **i32),
                   torch.zeros((table_rows, table_stride), **i32), torch.zeros(table_rows, **i32), page_size, block_size)

    def struct(self) -> _Pool:
        for n in ("free_pages", "free_count", "table", "lens"):
            t = getattr(self, n)
            if t.dtype != torch.int32 or t.device != self.table.device:
                raise TypeError(f"{n} must be int32 on {self.table.device} (got {t.dtype} on {t.device})")
        rows, stride = self.table.shape
        if self.lens.numel() != rows:
            raise ValueError(f"lens has {self.lens.numel()} entries for {rows} table rows")
        if self.free_count.numel() < 1:
            raise ValueError("free_count must have an entry")
        return _Pool(_ptr(self.free_pages), _ptr(self.free_count), _ptr(self.table), _ptr(self.lens),
                     self.free_pages.numel(), rows, stride, int(self.page_size), int(self.block_size))

    def __setattr__(self, name, value):
        self.__dict__[name] = value
        self.__dict__["_ref"] = None

    def current(self):
        """A by-reference argument holding this pool as it is now: built again where a field has been
        assigned, or a tensor has other memory, since."""
        at = (self.free_pages.data_ptr(), self.free_count.data_ptr(), self.table.data_ptr(), self.lens.data_ptr())
        kept = self.__dict__["_ref"]
        if kept is None or kept[0] != at:
            st = self.struct()
            kept = self.__dict__["_ref"] = (at, ctypes.byref(st))
        return kept[1]


_MOST = 2 ** 31 - 1      # what the calls' 32-bit counts hold


def _counts(**values) -> None:
    """Refuses what a call's 32-bit argument would hold the low bits of."""
    for name, x in values.items():
        if not -_MOST <= x <= _MOST:
            raise ValueError(f"{name} must fit 32 bits (got {x})")


def _gpu_of(t: torch.Tensor) -> int:
    """The current GPU, which t has to be on: the kernels take addresses, and another device's or the
    host's would fault it."""
    d = t.get_device()
    if d < 0 or d != _current_device():
        raise ValueError(f"tensors must be on the current GPU (got one on {t.device})")
    return d


def _refuse(t: torch.Tensor, dtype: torch.dtype, n: Optional[int], name: str) -> None:
    """Says what is wrong with an argument that a call's own checks have found unfit."""
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype} (got {t.dtype})")
    if n is not None and t.numel() != n:
        raise ValueError(f"{name} has {t.numel()} entries, {n} are needed")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    raise ValueError(f"tensors must be on the current GPU (got {name} on {t.device})")


def page_workspace_size(batch: int) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().vx_page_workspace_size(int(batch), ctypes.byref(out)))
    return int(out.value)


def page_extend(pool: PagePool, rows: torch.Tensor, new_lens: torch.Tensor, batch: BatchSpec,
                token_indptr: torch.Tensor, slots: torch.Tensor, granted: torch.Tensor, workspace: torch.Tensor,
                first_block: Optional[torch.Tensor] = None, stream=None) -> None:
    """Gives request i (row rows[i] of the pool) its new_lens[i] tokens: batch's page_indptr,
    page_indices and seq_lens are written for the lengths with them, and token_indptr, slots
    (int64), granted and first_block as include/vx.h says.  workspace: page_workspace_size bytes,
    zero-filled once."""
    B, i32, d = rows.numel(), torch.int32, _gpu_of(pool.table)
    seq_lens, page_indptr = batch.seq_lens, batch.page_indptr
    if not (rows.dtype is i32 and new_lens.dtype is i32 and seq_lens.dtype is i32 and page_indptr.dtype is i32
            and token_indptr.dtype is i32 and granted.dtype is i32
            and new_lens.numel() == B and seq_lens.numel() == B and page_indptr.numel() == B + 1
            and token_indptr.numel() == B + 1 and granted.numel() == B
            and rows.get_device() == d and new_lens.get_device() == d and seq_lens.get_device() == d
            and page_indptr.get_device() == d and token_indptr.get_device() == d and granted.get_device() == d
            and rows.is_contiguous() and new_lens.is_contiguous() and seq_lens.is_contiguous()
            and page_indptr.is_contiguous() and token_indptr.is_contiguous() and granted.is_contiguous()):
        for t, n, name in ((rows, B, "rows"), (new_lens, B, "new_lens"), (seq_lens, B, "seq_lens"),
                           (page_indptr, B + 1, "page_indptr"), (token_indptr, B + 1, "token_indptr"),
                           (granted, B, "granted")):
            if t.dtype is not i32 or t.numel() != n or t.get_device() != d or not t.is_contiguous():
                _refuse(t, i32, n, name)
    first = None
    if first_block is not None:
        if first_block.dtype is not i32 or first_block.numel() != B or first_block.get_device() != d:
            _refuse(first_block, i32, B, "first_block")
        first = _ptr(first_block)
    pages = batch.page_indices
    if pages.dtype is not i32 or pages.get_device() != d:
        _refuse(pages, i32, None, "page_indices")
    if slots.dtype is not torch.int64 or slots.get_device() != d:
        _refuse(slots, torch.int64, None, "slots")
    if workspace.get_device() != d:
        _refuse(workspace, workspace.dtype, None, "workspace")
    _check(lib().vx_page_extend(pool.current(), B, rows.data_ptr(), new_lens.data_ptr(), seq_lens.data_ptr(),
                                page_indptr.data_ptr(), _ptr(pages), min(pages.numel(), _MOST), token_indptr.data_ptr(),
                                _ptr(slots), min(slots.numel(), _MOST), granted.data_ptr(), first, _ptr(workspace),
                                workspace.numel() * workspace.element_size(), _stream(stream, d)))


def page_release(pool: PagePool, rows: torch.Tensor, keep_lens: Optional[torch.Tensor], workspace: torch.Tensor,
                 stream=None) -> None:
    """Row rows[i] keeps its first keep_lens[i] tokens (None: none) and gives its other pages back."""
    B, i32, d = rows.numel(), torch.int32, _gpu_of(pool.table)
    if rows.dtype is not i32 or rows.get_device() != d:
        _refuse(rows, i32, B, "rows")
    if keep_lens is not None and (keep_lens.dtype is not i32 or keep_lens.numel() != B or keep_lens.get_device() != d):
        _refuse(keep_lens, i32, B, "keep_lens")
    if workspace.get_device() != d:
        _refuse(workspace, workspace.dtype, None, "workspace")
    _check(lib().vx_page_release(pool.current(), B, _ptr(rows), _ptr(keep_lens), _ptr(workspace),
                                 workspace.numel() * workspace.element_size(), _stream(stream, d)))


def _row_args(t: Optional[torch.Tensor], n: int, heads: int, dim: int, d: int, name: str):
    """Address and strides of rows [n][heads][dim], bf16, channels side by side."""
    if t is None:
        return None, 0, 0
    if t.dtype is not torch.bfloat16 or t.get_device() != d:
        _refuse(t, torch.bfloat16, None, name)
    stride = t.stride()
    if t.shape != (n, heads, dim) or (n > 0 and stride[2] != 1):
        raise ValueError(f"{name} must be [{n}][{heads}][{dim}] with contiguous channels (got {tuple(t.shape)}, "
                         f"strides {stride})")
    return t.data_ptr(), stride[0], stride[1]


def _kv_rows(fn, kv: PagedKV, slots: torch.Tensor, k: torch.Tensor, v: Optional[torch.Tensor], names, stream) -> None:
    d, c = _gpu_of(kv.k), kv.current()
    if slots.dtype is not torch.int64 or slots.get_device() != d:
        _refuse(slots, torch.int64, None, "slots")
    n, (heads, dim_qk, dim_v) = slots.numel(), kv._dims
    if n > _MOST:
        raise ValueError(f"at most {_MOST} rows a call (got {n})")
    k_args = _row_args(k, n, heads, dim_qk, d, names[0])
    v_args = _row_args(v, n, heads, dim_v, d, names[1])
    _check(fn(c, *k_args, *v_args, _ptr(slots), n, _stream(stream, d)))


def kv_write(kv: PagedKV, k_new: torch.Tensor, v_new: Optional[torch.Tensor], slots: torch.Tensor, stream=None) -> None:
    """Rows k_new [n][H][Dqk] and v_new [n][H][Dv] (bf16, strided) into the cache, rounded to its
    type, at slots [n] (int64; negative: skipped)."""
    _kv_rows(lib().vx_kv_write, kv, slots, k_new, v_new, ("k_new", "v_new"), stream)


def kv_read(kv: PagedKV, slots: torch.Tensor, k_out: torch.Tensor, v_out: Optional[torch.Tensor], stream=None) -> None:
    """The cache's values at slots [n] as bf16 rows k_out [n][H][Dqk] and v_out [n][H][Dv] (zeros for a
    negative slot)."""
    _kv_rows(lib().vx_kv_read, kv, slots, k_out, v_out, ("k_out", "v_out"), stream)


@dataclass
class Rope:
    """The rotation of rows by their tokens' positions (vx_rope): inv_freq float32 [dim / 2] on the GPU
    turns channels first .. first + dim - 1, in pairs of halves or of neighbours (interleaved).  axis
    int32 [dim / 2]: the axis of each pair, of num_axes (None: one axis)."""
    inv_freq: torch.Tensor
    axis: Optional[torch.Tensor] = None
    num_axes: int = 1
    first: int = 0
    interleaved: bool = False
    scale: float = 1.0

    def current(self, d: int):
        """A by-reference argument holding this rotation as it is now, on GPU d."""
        f, ax = self.inv_freq, self.axis
        at = (f.data_ptr(), f.numel(), f.dtype, f.is_contiguous(), d,
              None if ax is None else (ax.data_ptr(), ax.numel(), ax.dtype, ax.is_contiguous()), self.num_axes, self.first,
              self.interleaved, self.scale)
        kept = self.__dict__.get("_kept")
        if kept is not None and kept[0] == at:
            return kept[1]
        if f.dtype is not torch.float32 or f.get_device() != d or not f.is_contiguous():
            _refuse(f, torch.float32, None, "inv_freq")
        if ax is not None and (ax.dtype is not torch.int32 or ax.numel() != f.numel() or ax.get_device() != d
                               or not ax.is_contiguous()):
            _refuse(ax, torch.int32, f.numel(), "axis")
        _counts(num_axes=self.num_axes, first=self.first)
        kept = self.__dict__["_kept"] = (at, ctypes.byref(
            _Rope(f.data_ptr(), None if ax is None else ax.data_ptr(), int(self.num_axes), int(self.first), 2 * f.numel(),
                  int(bool(self.interleaved)), float(self.scale))))
        return kept[1]


def rope_kv_write(kv: PagedKV, rope: Rope, q: Optional[torch.Tensor], k_new: torch.Tensor,
                  v_new: Optional[torch.Tensor], positions: torch.Tensor, slots: torch.Tensor,
                  q_out: Optional[torch.Tensor], stream=None) -> None:
    """Rows k_new [n][H][Dqk], rotated by positions [n] or [num_axes][n] (int64), and v_new [n][H][Dv] into
    the cache at slots [n] (int64; negative: skipped), rounded to its type; queries q [n][Hq][Dqk] rotated
    into q_out (which may be q).  All rows bf16, strided; q and q_out None: keys and values alone."""
    d, c = _gpu_of(kv.k), kv.current()
    if slots.dtype is not torch.int64 or slots.get_device() != d:
        _refuse(slots, torch.int64, None, "slots")
    n, (heads, dim_qk, dim_v) = slots.numel(), kv._dims
    if n > _MOST:
        raise ValueError(f"at most {_MOST} rows a call (got {n})")
    axes = int(rope.num_axes)
    if positions.dtype is not torch.int64 or positions.get_device() != d:
        _refuse(positions, torch.int64, None, "positions")
    if positions.shape != (axes, n) and not (axes == 1 and positions.shape == (n,)):
        raise ValueError(f"positions must be [{axes}][{n}] (got {tuple(positions.shape)})")
    if n > 1 and positions.stride(-1) != 1:
        raise ValueError("the positions along an axis must be contiguous")
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out must be given together")
    q_heads = 0 if q is None else q.shape[1]
    k_args = _row_args(k_new, n, heads, dim_qk, d, "k_new")
    v_args = _row_args(v_new, n, heads, dim_v, d, "v_new")
    q_args = _row_args(q, n, q_heads, dim_qk, d, "q")
    o_args = _row_args(q_out, n, q_heads, dim_qk, d, "q_out")
    _check(lib().vx_rope_kv_write(c, rope.current(d), *q_args, q_heads, *o_args, *k_args, *v_args, positions.data_ptr(),
                                  positions.stride(0) if positions.dim() == 2 else 0, _ptr(slots), n,
                                  _stream(stream, d)))


CHUNK_ATTENTION, CHUNK_SCORE_TOPK, CHUNK_SPARSE = 0, 1, 2


def chunk_workspace_size(stage: int, kv: PagedKV, batch: BatchSpec, num_rows: int, num_q_heads: int,
                         max_sel: int = 1) -> int:
    """Workspace bytes of chunk_attention, chunk_score_topk or sparse_chunk_attention (stage CHUNK_ATTENTION,
    CHUNK_SCORE_TOPK, CHUNK_SPARSE) for up to num_rows rows of queries, over up to as many requests and pages
    as the batch has and lists of up to max_sel blocks: one buffer serves all chunks of a prompt."""
    out = ctypes.c_size_t(0)
    _counts(stage=stage, num_rows=num_rows, num_q_heads=num_q_heads, max_sel=max_sel)
    _check(lib().vx_chunk_workspace_size(stage, kv.current(), batch.kept(), int(num_rows), int(num_q_heads), int(max_sel),
                                         ctypes.byref(out)))
    return int(out.value)


def _chunk_args(q: torch.Tensor, kv: PagedKV, batch: BatchSpec, q_indptr: torch.Tensor,
                q_lens: Optional[torch.Tensor], workspace: torch.Tensor):
    """What the chunk calls share: the device, the query's arguments, the cache, the batch and the chunk."""
    d, c, i32 = _gpu_of(kv.k), kv.current(), torch.int32
    lens, indptr, pages = batch.seq_lens, batch.page_indptr, batch.page_indices
    B = lens.numel()
    if not (lens.dtype is i32 and indptr.dtype is i32 and pages.dtype is i32 and q_indptr.dtype is i32
            and indptr.numel() == B + 1 and q_indptr.numel() == B + 1
            and lens.get_device() == d and indptr.get_device() == d and pages.get_device() == d and q_indptr.get_device() == d
            and lens.is_contiguous() and indptr.is_contiguous() and pages.is_contiguous() and q_indptr.is_contiguous()):
        for t, n, name in ((lens, B, "seq_lens"), (indptr, B + 1, "page_indptr"), (pages, None, "page_indices"),
                           (q_indptr, B + 1, "q_indptr")):
            if t.dtype is not i32 or (n is not None and t.numel() != n) or t.get_device() != d or not t.is_contiguous():
                _refuse(t, i32, n, name)
    if q_lens is not None and (q_lens.dtype is not i32 or q_lens.numel() != B or q_lens.get_device() != d
                               or not q_lens.is_contiguous()):
        _refuse(q_lens, i32, B, "q_lens")
    if workspace.get_device() != d or not workspace.is_contiguous():
        _refuse(workspace, workspace.dtype, None, "workspace")
    if q.dim() != 3:
        raise ValueError(f"q must be [rows][heads][dim] (got {tuple(q.shape)})")
    n, heads, dim = q.shape
    if n > _MOST:
        raise ValueError(f"at most {_MOST} rows a call (got {n})")
    address, row, head = _row_args(q, n, heads, kv._dims[1], d, "q")
    at = (q_indptr.data_ptr(), None if q_lens is None else q_lens.data_ptr(), n)
    kept = batch.__dict__.get("_chunk")
    if kept is None or kept[0] != at:
        kept = batch.__dict__["_chunk"] = (at, ctypes.byref(_Chunk(*at)))
    return d, (address, row, head, heads, c, batch.kept(), kept[1])


def _result(t: Optional[torch.Tensor], dtype: torch.dtype, shape, d: int, name: str):
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != d or not t.is_contiguous():
        _refuse(t, dtype, None, name)
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)} (got {list(t.shape)})")
    return t.data_ptr()


def _bytes(t: torch.Tensor) -> int:
    return t.numel() * t.element_size()


def chunk_attention(q: torch.Tensor, kv: PagedKV, batch: BatchSpec, q_indptr: torch.Tensor, sm_scale: float,
                    out: torch.Tensor, workspace: torch.Tensor, q_lens: Optional[torch.Tensor] = None,
                    window: int = 0, causal: bool = True, lse: Optional[torch.Tensor] = None, stream=None) -> None:
    """Attention of a chunk's tokens over the paged cache, which already holds their own rows: queries
    q [n][Hq][Dqk] (bf16, strided), rows q_indptr[i] .. of request i (int32 [batch+1]; q_lens int32 [batch]:
    how many of them are tokens), out [n][Hq][Dv] bf16, lse [n][Hq] float32 or None.  window: each token
    attends its last `window` tokens (0: all).  workspace: chunk_workspace_size(CHUNK_ATTENTION, ..) bytes."""
    d, args = _chunk_args(q, kv, batch, q_indptr, q_lens, workspace)
    n, heads = q.shape[:2]
    o = _result(out, torch.bfloat16, (n, heads, kv._dims[2]), d, "out")
    e = _result(lse, torch.float32, (n, heads), d, "lse")
    if window > _MOST:
        window = _MOST                                       # longer than any request
    elif window < -_MOST:
        _counts(window=window)
    _check(lib().vx_chunk_attention(*args, int(window), int(bool(causal)), float(sm_scale), o, e, workspace.data_ptr(),
                                    _bytes(workspace), _stream(stream, d)))


def chunk_score_topk(q: torch.Tensor, kv: PagedKV, batch: BatchSpec, q_indptr: torch.Tensor, kind: int,
                     mean: torch.Tensor, pages_budget: torch.Tensor, n_sink: int, n_local: int, max_sel: int,
                     sel_pages: torch.Tensor, sel_count: torch.Tensor, workspace: torch.Tensor,
                     q_lens: Optional[torch.Tensor] = None, stream=None) -> None:
    """The blocks that each token of a chunk attends: page_score_topk for every token by itself, into
    sel_pages [n][H][max_sel] and sel_count [n] (int32).  kind: MEAN_DOT; n_local >= 1."""
    d, args = _chunk_args(q, kv, batch, q_indptr, q_lens, workspace)
    n, H, D = q.shape[0], kv._dims[0], kv._dims[1]
    _counts(kind=kind, n_sink=n_sink, n_local=n_local)
    blocks = kv.k.shape[0] * (kv.k.shape[2] // kv.block_size if kv.block_size else 1)
    m = _result(mean, torch.float32, (blocks, H, D), d, "mean")
    budget = _result(pages_budget, torch.int32, (batch.seq_lens.numel(),), d, "pages_budget")
    sp = _result(sel_pages, torch.int32, (n, H, max_sel), d, "sel_pages")
    sc = _result(sel_count, torch.int32, (n,), d, "sel_count")
    _check(lib().vx_chunk_score_topk(*args, kind, m, budget, n_sink, n_local, max_sel, sp, sc, workspace.data_ptr(),
                                     _bytes(workspace), _stream(stream, d)))


def sparse_chunk_attention(q: torch.Tensor, kv: PagedKV, batch: BatchSpec, q_indptr: torch.Tensor,
                           sel_pages: torch.Tensor, sel_count: torch.Tensor, sm_scale: float, out: torch.Tensor,
                           workspace: torch.Tensor, q_lens: Optional[torch.Tensor] = None,
                           lse: Optional[torch.Tensor] = None, stream=None) -> None:
    """chunk_attention over the blocks listed for each row and KV head: sel_pages [n][H][max_sel] and
    sel_count [n] (int32), as chunk_score_topk writes them."""
    d, args = _chunk_args(q, kv, batch, q_indptr, q_lens, workspace)
    n, heads = q.shape[:2]
    if sel_pages.dim() != 3:
        raise ValueError(f"sel_pages must be [rows][KV heads][max_sel] (got {tuple(sel_pages.shape)})")
    max_sel = sel_pages.shape[2]
    sp = _result(sel_pages, torch.int32, (n, kv._dims[0], max_sel), d, "sel_pages")
    sc = _result(sel_count, torch.int32, (n,), d, "sel_count")
    o = _result(out, torch.bfloat16, (n, heads, kv._dims[2]), d, "out")
    e = _result(lse, torch.float32, (n, heads), d, "lse")
    _check(lib().vx_sparse_chunk_attention(*args, sp, sc, max_sel, float(sm_scale), o, e, workspace.data_ptr(),
                                           _bytes(workspace), _stream(stream, d)))


def workspace_size(stage: int, kv: PagedKV, batch: BatchSpec, num_q_heads: int, max_sel: int) -> int:
    out = ctypes.c_size_t(0)
    c, b = kv.struct(), batch.struct()
    _check(lib().vx_workspace_size(stage, ctypes.byref(c), ctypes.byref(b), num_q_heads, max_sel,
                                   ctypes.byref(out)))
    return int(out.value)


def page_summarize(kv: PagedKV, batch: BatchSpec, first_page: Optional[torch.Tensor] = None,
                   mean: Optional[torch.Tensor] = None, max: Optional[torch.Tensor] = None,
                   min: Optional[torch.Tensor] = None, stream=None,
                   mean_bf16: Optional[torch.Tensor] = None) -> None:
    c, b = kv.struct(), batch.struct()
    _check(lib().vx_page_summarize(ctypes.byref(c), ctypes.byref(b), _ptr(first_page), _ptr(mean),
                                   _ptr(mean_bf16), _ptr(max), _ptr(min), _stream(stream)))


def kv_append_summarize(kv: PagedKV, batch: BatchSpec, k_new: torch.Tensor, v_new: Optional[torch.Tensor],
                        mean: Optional[torch.Tensor] = None, max: Optional[torch.Tensor] = None,
                        min: Optional[torch.Tensor] = None, stream=None,
                        mean_bf16: Optional[torch.Tensor] = None) -> None:
    """Writes k_new [B][H][Dqk] / v_new [B][H][Dv] (the cache's dtype) at token seq_lens[i]-1 and
    refreshes that page's summaries, in one launch."""
    for t in (k_new, v_new):
        if t is not None and t.dtype != kv.row_dtype:
            raise TypeError(f"new rows must have the cache's dtype {kv.row_dtype} (got {t.dtype})")
    c, b = kv.struct(), batch.struct()
    _check(lib().vx_kv_append_summarize(ctypes.byref(c), ctypes.byref(b), _ptr(k_new), _ptr(v_new), _ptr(mean),
                                        _ptr(mean_bf16), _ptr(max), _ptr(min), _stream(stream)))


class _TopkOptions(ctypes.Structure):
    _fields_ = [("tolerate_ratio", ctypes.c_float), ("seed", ctypes.c_uint32), ("remap", ctypes.c_int32)]


REMAP_NONE, REMAP_AFFINE = 0, 1


def topk_options(tolerate_ratio: float = 0.0, seed: int = 0, remap: int = REMAP_NONE) -> _TopkOptions:
    return _TopkOptions(float(tolerate_ratio), int(seed) & 0xFFFFFFFF, int(remap))


def page_score_topk(q: torch.Tensor, kv: PagedKV, batch: BatchSpec, kind: int,
                    mean: Optional[torch.Tensor], max: Optional[torch.Tensor], min: Optional[torch.Tensor],
                    pages_budget: torch.Tensor, n_sink: int, n_local: int, max_sel: int,
                    sel_pages: torch.Tensor, sel_count: torch.Tensor, workspace: torch.Tensor,
                    stream=None, mean_bf16: Optional[torch.Tensor] = None,
                    options: Optional[_TopkOptions] = None) -> None:
    c, b = kv.struct(), batch.struct()
    _check(lib().vx_page_score_topk(_ptr(q), q.shape[1], ctypes.byref(c), ctypes.byref(b), kind, _ptr(mean),
                                    _ptr(mean_bf16), _ptr(max), _ptr(min), _ptr(pages_budget), n_sink, n_local,
                                    max_sel,
                                    _ptr(sel_pages), _ptr(sel_count), _ptr(workspace),
                                    workspace.numel() * workspace.element_size(),
                                    None if options is None else ctypes.byref(options), _stream(stream)))


def append_score_topk(kv: PagedKV, batch: BatchSpec, k_new: torch.Tensor, v_new: Optional[torch.Tensor],
                      mean: Optional[torch.Tensor], max: Optional[torch.Tensor], min: Optional[torch.Tensor],
                      q: torch.Tensor, kind: int, pages_budget: torch.Tensor, n_sink: int, n_local: int,
                      max_sel: int, sel_pages: torch.Tensor, sel_count: torch.Tensor, workspace: torch.Tensor,
                      stream=None, mean_bf16: Optional[torch.Tensor] = None,
                      options: Optional[_TopkOptions] = None) -> None:
    """kv_append_summarize followed by page_score_topk, the append inside the top-K launch."""
    for t in (k_new, v_new):
        if t is not None and t.dtype != kv.row_dtype:
            raise TypeError(f"new rows must have the cache's dtype {kv.row_dtype} (got {t.dtype})")
    c, b = kv.struct(), batch.struct()
    _check(lib().vx_append_score_topk(ctypes.byref(c), ctypes.byref(b), _ptr(k_new), _ptr(v_new), _ptr(mean),
                                      _ptr(mean_bf16), _ptr(max), _ptr(min), _ptr(q), q.shape[1], kind,
                                      _ptr(pages_budget), n_sink, n_local, max_sel, _ptr(sel_pages),
                                      _ptr(sel_count), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                      None if options is None else ctypes.byref(options), _stream(stream)))


def page_score(q: torch.Tensor, kv: PagedKV, batch: BatchSpec, kind: int, mean: Optional[torch.Tensor],
               max: Optional[torch.Tensor], min: Optional[torch.Tensor], scores: torch.Tensor, stream=None) -> None:
    """One-pass fp32 scores into scores [H][B][stride] (float32, contiguous)."""
    assert scores.dtype == torch.float32 and scores.dim() == 3
    c, b = kv.struct(), batch.struct()
    _check(lib().vx_page_score(_ptr(q), q.shape[1], ctypes.byref(c), ctypes.byref(b), kind, _ptr(mean), _ptr(max),
                               _ptr(min), _ptr(scores), scores.shape[2], _stream(stream)))


def score_flow(kind: int, scores_in: torch.Tensor, scores_out: torch.Tensor, num_kv_heads: int,
               num_items: torch.Tensor, stream=None) -> None:
    """Last steps of the NSA / smoothing flows: scores_in [rows][B][stride] (NSA: a row per query
    head) -> scores_out [H][B][stride] (float32)."""
    assert scores_in.dtype == torch.float32 and scores_out.dtype == torch.float32 and scores_out.dim() == 3
    H, B, stride = scores_out.shape
    assert H == num_kv_heads and scores_in.shape[1:] == (B, stride)
    rows = scores_in.shape[0]
    _check(lib().vx_score_flow(kind, _ptr(scores_in), _ptr(scores_out), stride, num_kv_heads,
                               rows if kind == NSA else num_kv_heads, B, _ptr(num_items), _stream(stream)))


def stream_read(buf: torch.Tensor, sink: torch.Tensor, stream=None) -> None:
    """The streaming-read measurement kernel over the bytes of buf (contiguous, 16-byte
    multiple); sink: int32 device tensor with one entry per workgroup."""
    _check(lib().vx_stream_read(_ptr(buf), buf.numel() * buf.element_size(), _ptr(sink), sink.numel(),
                                _stream(stream)))


def topk_select(scores: torch.Tensor, num_items: torch.Tensor, pages_budget: torch.Tensor, n_sink: int,
                n_local: int, max_sel: int, sel_pages: torch.Tensor, sel_count: torch.Tensor,
                tolerate_ratio: float = 0.0, seed: int = 0, remap: int = REMAP_NONE, stream=None) -> None:
    """Exact or approximate radix selection from scores [H][B][stride] (float32)."""
    assert scores.dtype == torch.float32 and scores.dim() == 3
    H, B, stride = scores.shape
    opt = topk_options(tolerate_ratio, seed, remap)
    _check(lib().vx_topk_select(_ptr(scores), stride, H, B, _ptr(num_items), _ptr(pages_budget), n_sink, n_local,
                                max_sel, ctypes.byref(opt), _ptr(sel_pages), _ptr(sel_count), _stream(stream)))


def sparse_paged_decode(q: torch.Tensor, kv: PagedKV, batch: BatchSpec, sel_pages: torch.Tensor,
                        sel_count: torch.Tensor, max_sel: int, sm_scale: float, out: torch.Tensor,
                        workspace: torch.Tensor, stream=None) -> None:
    c, b = kv.struct(), batch.struct()
    _check(lib().vx_sparse_paged_decode(_ptr(q), q.shape[1], ctypes.byref(c), ctypes.byref(b), _ptr(sel_pages),
                                        _ptr(sel_count), max_sel, float(sm_scale), _ptr(out), _ptr(workspace),
                                        workspace.numel() * workspace.element_size(), _stream(stream)))


def sparse_paged_decode_noalloc(q: torch.Tensor, kv: PagedKV, batch: BatchSpec, sel_pages: torch.Tensor,
                                sel_count: torch.Tensor, max_sel: int, sm_scale: float, out: torch.Tensor,
                                stream=None) -> None:
    """vx_sparse_paged_decode on the library's static per-GPU scratch (no workspace)."""
    c, b = kv.struct(), batch.struct()
    _check(lib().vx_sparse_paged_decode_noalloc(_ptr(q), q.shape[1], ctypes.byref(c), ctypes.byref(b),
                                                _ptr(sel_pages), _ptr(sel_count), max_sel, float(sm_scale),
                                                _ptr(out), _stream(stream)))


class BoundCall:
    """One entry point with every argument marshalled once; calling it only swaps in the
    stream.  For per-step loops whose buffers stay fixed (argument marshalling only, like the
    functions above)."""

    def __init__(self, fn, args: tuple, stream_index: int):
        self.fn, self.args, self.si = fn, list(args), stream_index

    def __call__(self, stream=None):
        self.args[self.si] = _stream(stream)
        _check(self.fn(*self.args))
