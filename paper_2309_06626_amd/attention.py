"""ctypes binding of the attention operators of libsparse_conv.so (include/sparse_attention.h): argument marshalling only.

Every function has the name and meaning of its C entry point.  Tensors are checked here, because the library cannot see their
sizes; all arithmetic runs in the HIP kernels.  There is no CPU fallback.  Row sets are those of the other block operators.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional, Sequence, Tuple

import torch

from . import binding as B
from . import block as K
from .block import (DTYPE_CODE, SC_BF16, SC_F16, SC_F32, SC_ROWS_COMPACT, SC_ROWS_DENSE, TORCH_DTYPE, RowSet, ScError,  # noqa: F401
                    sparse_rows_info, sparse_rows_plan, sparse_rows_set_mask)

_F32, _I8, _I64, _I32 = torch.float32, torch.int8, torch.int64, torch.int32
_current_device = K._current_device


class sc_attn_desc(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in ("heads", "kv_heads", "d", "dtype", "causal", "window")] + [("scale", ctypes.c_float)]


class sc_kv_desc(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in ("kv_heads", "d", "page_rows", "pages", "dtype", "bits")]


_declared = None


def lib() -> ctypes.CDLL:
    """The library, with the signatures of the attention operators."""
    global _declared
    L = B._lib or B.lib()
    if _declared is not L:
        vp, i32, i64, size = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        out = ctypes.POINTER
        pa, pk = out(sc_attn_desc), out(sc_kv_desc)
        matrix = [vp, i64]
        for name, args in {
            "sparse_attn_workspace_bytes": [pa, i64, i64, out(size)],
            "sparse_attn_plan": [pa, i64, out(i64), vp, vp, size, vp, out(vp)],
            "sparse_attn_info": [vp, out(i64), out(i64)],
            "sparse_attn_run": [vp, vp, i32] + 3 * matrix + [vp, vp, vp],
            "sparse_attn_backward_workspace_bytes": [vp, out(size)],
            "sparse_attn_backward": [vp, vp, i32] + 3 * matrix + [vp, vp, vp] + 3 * matrix + [vp, size, vp],
            "sparse_kv_row_entries": [pk, out(i32)],
            "sparse_kv_write": [pk, i64] + 2 * matrix + [vp] * 6,
            "sparse_kv_read": [pk, i64] + [vp] * 5 + 2 * matrix + [vp],
            "sparse_attn_decode_workspace_bytes": [pa, pk, i64, i64, out(size)],
            "sparse_attn_decode": [pa, pk, i64, vp, vp, i64] + [vp] * 7 + [size, vp],
        }.items():
            getattr(L, name).restype = ctypes.c_int
            getattr(L, name).argtypes = args
        L.sparse_attn_destroy.restype = None
        L.sparse_attn_destroy.argtypes = [vp]
        _declared = L
    return L


def make_attn_desc(heads, kv_heads, d, dtype=SC_BF16, causal=True, window=0, scale: Optional[float] = None) -> sc_attn_desc:
    """scale: None stands for 1 / sqrt(d)."""
    return sc_attn_desc(heads, kv_heads, d, dtype, int(causal), window, 1.0 / math.sqrt(max(d, 1)) if scale is None else scale)


def make_kv_desc(kv_heads, d, page_rows, pages, dtype=SC_BF16, bits=0) -> sc_kv_desc:
    return sc_kv_desc(kv_heads, d, page_rows, pages, dtype, bits)


def _matrix(t: torch.Tensor, what: str, rows: int, width: int, dtype: torch.dtype) -> Tuple[int, int]:
    """Address and stride of `rows` rows of `width` entries that lie together; a row may have several dimensions.  The calls for single tokens
    spend as long here as on the GPU: two cases that hold nearly always first, the reason looked for afterwards."""
    if t.dtype is dtype and t.is_cuda and t.get_device() == _current_device():
        shape = t.shape
        if shape and shape[0] == rows:
            if t.is_contiguous():
                if t.numel() == rows * width:
                    return t.data_ptr(), width
            elif len(shape) == 2 and shape[1] == width:
                stride, inner = t.stride()
                if inner == 1:
                    return t.data_ptr(), stride
    if t.dtype != dtype:
        raise ValueError(f"{what} must be {dtype}")
    if not t.is_cuda:
        raise ValueError(f"{what} must be a device tensor")
    if t.get_device() != _current_device():
        raise ValueError(f"{what} is on another device than the current one")
    if t.dim() < 2:
        raise ValueError(f"{what} must have rows")
    inner = 1
    for size, stride in zip(reversed(t.shape[1:]), reversed(t.stride()[1:])):
        if size != 1 and stride != inner:
            raise ValueError(f"the entries of a row of {what} must lie together")
        inner *= size
    if inner != width:
        raise ValueError(f"a row of {what} has {inner} entries, the call needs {width}")
    if t.shape[0] != rows:
        raise ValueError(f"{what} has {t.shape[0]} rows, the call needs {rows}")
    stride = t.stride(0) if t.shape[0] > 1 else max(t.stride(0), width)
    return t.data_ptr(), stride


def _same_device(*tensors: Optional[torch.Tensor]):
    """The library launches on the current device, whose kernels fault on another one's memory."""
    here = _current_device()
    for t in tensors:
        if t is not None and t.get_device() != here:
            raise ValueError("a tensor of the call is on another device than the current one")


# ---- attention over packed sequences -----------------------------------------------------------------------------------


class AttnPlan:
    """Owner of an sc_attn handle and of the workspace that its lists lie in.  end: rows of the sequences; kept: those that are kept."""

    def __init__(self, handle: int, desc: sc_attn_desc, workspace: torch.Tensor):
        self.handle = handle
        self.desc = sc_attn_desc.from_buffer_copy(desc)
        self.workspace = workspace
        end, kept = ctypes.c_int64(), ctypes.c_int64()
        B._check(lib().sparse_attn_info(handle, ctypes.byref(end), ctypes.byref(kept)), "sparse_attn_info")
        self.end, self.kept = end.value, kept.value

    def close(self):
        if self.handle:
            lib().sparse_attn_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _open(plan: AttnPlan) -> int:
    if not plan.handle:
        raise ValueError("the plan is closed")
    return plan.handle


def _open_both(plan: AttnPlan, rows: Optional[RowSet]):
    handles = _open(plan), K._handle(rows)
    _same_device(plan.workspace, None if rows is None else rows.workspace)
    return handles


def sparse_attn_workspace_bytes(desc: sc_attn_desc, seqs: int, rows: int) -> int:
    n = ctypes.c_size_t()
    B._check(lib().sparse_attn_workspace_bytes(ctypes.byref(desc), seqs, rows, ctypes.byref(n)), "sparse_attn_workspace_bytes")
    return n.value


def sparse_attn_plan(desc: sc_attn_desc, starts: Sequence[int], rows: Optional[RowSet] = None, workspace: Optional[torch.Tensor] = None,
                     stream=None, device="cuda") -> AttnPlan:
    """starts: first row of every sequence and the end of the last one (on the host); synchronises the stream."""
    starts = [int(v) for v in starts]
    if not starts:
        raise ValueError("starts ends with the end of the last sequence")
    seqs = len(starts) - 1
    if any(not 0 <= v < 1 << 62 for v in starts):
        raise ScError(B.SC_ERR_BAD_SHAPE, "sparse_attn_plan")
    nbytes = sparse_attn_workspace_bytes(desc, seqs, starts[-1])
    if workspace is None:
        workspace = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=device if rows is None else rows.workspace.device)
    at, size = K._workspace(workspace)
    set_handle = K._handle(rows)
    _same_device(workspace, None if rows is None else rows.workspace)
    out = ctypes.c_void_p()
    B._check(lib().sparse_attn_plan(ctypes.byref(desc), seqs, (ctypes.c_int64 * len(starts))(*starts), set_handle, at, size,
                                    K._stream_handle(stream), ctypes.byref(out)), "sparse_attn_plan")
    return AttnPlan(out.value, desc, workspace)


def _attn_rows(plan: AttnPlan, rows: Optional[RowSet], row_format: int, q: torch.Tensor) -> int:
    """Rows that every tensor of a call has: as many as q."""
    have = q.shape[0] if q.dim() else 0
    if rows is not None:
        want = rows.kept if row_format == SC_ROWS_COMPACT else rows.rows
        if have != want:
            raise ValueError(f"q has {have} rows, the call needs {want}")
    elif have < plan.end:
        raise ValueError(f"q has {have} rows, the sequences have {plan.end}")
    return have


def _flat(t: torch.Tensor, what: str, numel: int, dtype: torch.dtype) -> int:
    at = K._tensor(t, what, numel, dtype)
    _same_device(t)
    return at


def sparse_attn_run(plan: AttnPlan, q, k, v, o, lse=None, rows: Optional[RowSet] = None, row_format: int = SC_ROWS_DENSE, stream=None):
    """o = softmax(scale q k') v; q, k, v: [rows, ...] with rows of heads * d (kv_heads * d) entries that lie together, o contiguous;
    lse: float[plan.kept, heads], for the backward pass."""
    d, t = plan.desc, K._elem(plan.desc)
    n = _attn_rows(plan, rows, row_format, q)
    wide, narrow = d.heads * d.d, d.kv_heads * d.d
    status = lib().sparse_attn_run(
        *_open_both(plan, rows), row_format, *_matrix(q, "q", n, wide, t), *_matrix(k, "k", n, narrow, t), *_matrix(v, "v", n, narrow, t),
        _flat(o, "o", n * wide, t), None if lse is None else _flat(lse, "lse", plan.kept * d.heads, _F32), K._stream_handle(stream))
    if status:
        raise ScError(status, "sparse_attn_run")
    return o


def sparse_attn_backward_workspace_bytes(plan: AttnPlan) -> int:
    n = ctypes.c_size_t()
    B._check(lib().sparse_attn_backward_workspace_bytes(_open(plan), ctypes.byref(n)), "sparse_attn_backward_workspace_bytes")
    return n.value


def sparse_attn_backward(plan: AttnPlan, q, k, v, o, lse, do, dq, dk, dv, workspace, rows: Optional[RowSet] = None,
                         row_format: int = SC_ROWS_DENSE, stream=None):
    """Gradients into dq, dk, dv (formats of q, k, v, strides of their own); o and lse are those of the run."""
    d, t = plan.desc, K._elem(plan.desc)
    n = _attn_rows(plan, rows, row_format, q)
    wide, narrow = d.heads * d.d, d.kv_heads * d.d
    at, size = K._workspace(workspace)
    _same_device(workspace)
    B._check(lib().sparse_attn_backward(
        *_open_both(plan, rows), row_format, *_matrix(q, "q", n, wide, t), *_matrix(k, "k", n, narrow, t), *_matrix(v, "v", n, narrow, t),
        _flat(o, "o", n * wide, t), _flat(lse, "lse", plan.kept * d.heads, _F32), _flat(do, "do", n * wide, t),
        *_matrix(dq, "dq", n, wide, t), *_matrix(dk, "dk", n, narrow, t), *_matrix(dv, "dv", n, narrow, t), at, size,
        K._stream_handle(stream)), "sparse_attn_backward")


# ---- paged cache of keys and values ------------------------------------------------------------------------------------


def sparse_kv_row_entries(desc: sc_kv_desc) -> int:
    n = ctypes.c_int32()
    B._check(lib().sparse_kv_row_entries(ctypes.byref(desc), ctypes.byref(n)), "sparse_kv_row_entries")
    return n.value


class KvCache:
    """The tensors of a cache: k_pages and v_pages [pages, kv_heads, page_rows, row entries], of 8-bit caches int8 with float scales
    [pages, kv_heads, page_rows].  Those that are not given are made, with zeros.  They stay those of the object's making."""

    def __init__(self, desc: sc_kv_desc, k_pages: Optional[torch.Tensor] = None, v_pages: Optional[torch.Tensor] = None,
                 k_scales: Optional[torch.Tensor] = None, v_scales: Optional[torch.Tensor] = None, device="cuda"):
        shape, entries = (desc.pages, desc.kv_heads, desc.page_rows), sparse_kv_row_entries(desc)
        held = _I8 if desc.bits == 8 else K._elem(desc)

        def pages(t, what):
            t = torch.zeros(*shape, entries, dtype=held, device=device) if t is None else t
            return t, K._tensor(t, what, math.prod(shape) * entries, held)

        def scales(t, what):
            if desc.bits != 8:
                return None, None
            t = torch.zeros(shape, dtype=_F32, device=device) if t is None else t
            return t, K._tensor(t, what, math.prod(shape), _F32)

        self.desc, self.type = sc_kv_desc.from_buffer_copy(desc), K._elem(desc)
        self._reference, self._width = ctypes.byref(self.desc), desc.kv_heads * desc.d
        (self.k_pages, k), (self.v_pages, v) = pages(k_pages, "k_pages"), pages(v_pages, "v_pages")
        (self.k_scales, ks), (self.v_scales, vs) = scales(k_scales, "k_scales"), scales(v_scales, "v_scales")
        self._addresses, self._held = (k, v, ks, vs), (self.k_pages, self.v_pages, self.k_scales, self.v_scales)
        self.device_index = self.k_pages.get_device()
        if any(t is not None and t.get_device() != self.device_index for t in self._held):
            raise ValueError("the cache's tensors are on different devices")


def _elsewhere():
    raise ValueError("the cache or a tensor of the call is on another device than the current one")


def sparse_kv_write(cache: KvCache, k, v, slots, stream=None) -> KvCache:
    """k, v: [rows, ...] with rows of kv_heads * d entries that lie together; slots: int64[rows], places page * page_rows + row."""
    n, width, t = slots.numel(), cache._width, cache.type
    k_at, k_stride = _matrix(k, "k", n, width, t)
    v_at, v_stride = _matrix(v, "v", n, width, t)
    slots_at = K._tensor(slots, "slots", n, _I64)
    if not cache.device_index == _current_device() == slots.get_device():
        _elsewhere()
    status = lib().sparse_kv_write(cache._reference, n, k_at, k_stride, v_at, v_stride, slots_at, *cache._addresses,
                                   K._stream_handle(stream))
    if status:
        raise ScError(status, "sparse_kv_write")
    return cache


def sparse_kv_read(cache: KvCache, slots, k, v, stream=None):
    """Rows of the cache at slots into k and v; zeros where a slot is not in the cache."""
    n, width, t = slots.numel(), cache._width, cache.type
    k_at, k_stride = _matrix(k, "k", n, width, t)
    v_at, v_stride = _matrix(v, "v", n, width, t)
    slots_at = K._tensor(slots, "slots", n, _I64)
    if not cache.device_index == _current_device() == slots.get_device():
        _elsewhere()
    status = lib().sparse_kv_read(cache._reference, n, slots_at, *cache._addresses, k_at, k_stride, v_at, v_stride,
                                  K._stream_handle(stream))
    if status:
        raise ScError(status, "sparse_kv_read")
    return k, v


# ---- single tokens against the cache -----------------------------------------------------------------------------------


def sparse_attn_decode_workspace_bytes(desc: sc_attn_desc, cache: sc_kv_desc, rows: int, table_width: int) -> int:
    n = ctypes.c_size_t()
    B._check(lib().sparse_attn_decode_workspace_bytes(ctypes.byref(desc), ctypes.byref(cache), rows, table_width, ctypes.byref(n)),
             "sparse_attn_decode_workspace_bytes")
    return n.value


def sparse_attn_decode(desc: sc_attn_desc, cache: KvCache, q, table, lengths, o, workspace, stream=None):
    """o[r] = attention of q[r] over the first lengths[r] rows of the sequence whose pages table[r] lists; q, o: [rows, heads, d]."""
    t, n, wide = K._elem(desc), lengths.numel(), desc.heads * desc.d
    if t is not cache.type:
        raise ValueError("the descriptors' types differ")
    if table.dim() != 2 or table.shape[0] != n:
        raise ValueError(f"table must be [{n}, pages of a sequence]")
    tensor, width = K._tensor, table.shape[1]
    at, size = K._workspace(workspace)
    of = (_matrix(q, "q", n, wide, t)[0] if q.is_contiguous() else tensor(q, "q", n * wide, t), tensor(table, "table", n * width, _I32), width,
          tensor(lengths, "lengths", n, _I32), *cache._addresses, tensor(o, "o", n * wide, t), at, size)
    if not cache.device_index == _current_device() == table.get_device() == lengths.get_device() == o.get_device() == workspace.get_device():
        _elsewhere()
    status = lib().sparse_attn_decode(ctypes.byref(desc), cache._reference, n, *of, K._stream_handle(stream))
    if status:
        raise ScError(status, "sparse_attn_decode")
    return o
