"""ctypes binding of the block operators of libsparse_conv.so (include/sparse_block.h): argument marshalling only.

Every function has the name and meaning of its C entry point.  Tensors are checked here, because the library cannot see their
sizes; all arithmetic runs in the HIP kernels.  There is no CPU fallback.
"""
from __future__ import annotations

import ctypes
from typing import Dict, Optional, Tuple

import torch

from . import binding as B
from .binding import DTYPE_CODE, SC_BF16, SC_F16, SC_F32, SC_ROWS_COMPACT, SC_ROWS_DENSE, ScError, TORCH_DTYPE  # noqa: F401

SC_NORM_NONE, SC_NORM_RMS, SC_NORM_LAYER = 0, 1, 2
SC_ACT_SILU, SC_ACT_GELU, SC_ACT_GELU_TANH = 0, 1, 2
NORM_CODE = {"none": SC_NORM_NONE, "rms": SC_NORM_RMS, "layer": SC_NORM_LAYER}
ACT_CODE = {"silu": SC_ACT_SILU, "gelu": SC_ACT_GELU, "gelu_tanh": SC_ACT_GELU_TANH}
_F32 = torch.float32
_TORCH_OF_CODE = {code: TORCH_DTYPE[name] for name, code in DTYPE_CODE.items()}


class sc_norm_desc(ctypes.Structure):
    _fields_ = [("d", ctypes.c_int32), ("dtype", ctypes.c_int32), ("post", ctypes.c_int32), ("pre", ctypes.c_int32),
                ("eps", ctypes.c_float), ("residual_scale", ctypes.c_float), ("branch_scale", ctypes.c_float),
                ("rows_per_gate", ctypes.c_int32)]


class sc_ffn_desc(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in ("d_in", "d_hidden", "d_out", "dtype", "activation")]


class sc_q4_desc(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in ("k", "n", "group", "dtype")]


_declared = None


def lib() -> ctypes.CDLL:
    """The library, with the signatures of the block operators."""
    global _declared
    L = B._lib or B.lib()
    if _declared is not L:
        vp, i32, i64, size = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        out = ctypes.POINTER
        pn, pf, pq = out(sc_norm_desc), out(sc_ffn_desc), out(sc_q4_desc)
        for name, args in {
            "sparse_rows_workspace_bytes": [i64, out(size)],
            "sparse_rows_plan": [vp, i64, vp, size, vp, out(vp)],
            "sparse_rows_set_mask": [vp, vp, vp],
            "sparse_rows_info": [vp, out(i64), out(i64), out(vp), out(vp)],
            "sparse_norm_run": [pn, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp],
            "sparse_norm_workspace_bytes": [pn, i64, out(size)],
            "sparse_norm_backward": [pn, i64] + [vp] * 19 + [size, vp],
            "sparse_ffn_workspace_bytes": [pf, i64, i32, out(size)],
            "sparse_ffn_run": [pf, i64, vp, vp, i32, vp, vp, vp, vp, i32, vp, vp, size, vp],
            "sparse_ffn_backward": [pf, i64, vp, vp, i32, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp, vp, size, vp],
            "sparse_q4_workspace_bytes": [pq, i32, out(size)],
            "sparse_q4_plan": [pq, vp, vp, vp, vp, size, vp, out(vp)],
            "sparse_q4_plan_gated": [pq, i32] + [vp] * 7 + [size, vp, out(vp)],
            "sparse_q4_run": [vp, i64, vp, vp, vp],
        }.items():
            getattr(L, name).restype = ctypes.c_int
            getattr(L, name).argtypes = args
        for name in ("sparse_rows_destroy", "sparse_q4_destroy"):
            getattr(L, name).restype = None
            getattr(L, name).argtypes = [vp]
        _declared = L
    return L


def make_norm_desc(d, dtype=SC_BF16, post=SC_NORM_RMS, pre=SC_NORM_RMS, eps=1e-6, residual_scale=1.0, branch_scale=1.0,
                   rows_per_gate=0) -> sc_norm_desc:
    return sc_norm_desc(d, dtype, post, pre, eps, residual_scale, branch_scale, rows_per_gate)


def make_ffn_desc(d_in, d_hidden, d_out, dtype=SC_BF16, activation=SC_ACT_SILU) -> sc_ffn_desc:
    return sc_ffn_desc(d_in, d_hidden, d_out, dtype, activation)


def make_q4_desc(k, n, group=128, dtype=SC_BF16) -> sc_q4_desc:
    return sc_q4_desc(k, n, group, dtype)


def _tensor(t: Optional[torch.Tensor], what: str, numel: int, dtype: torch.dtype) -> Optional[int]:
    """Address of a tensor that must hold `numel` elements of `dtype` (None stays None).  The calls for single tokens spend as long
    here as on the GPU: one condition, the reason looked for afterwards."""
    if t is None:
        return None
    if t.dtype is dtype and t.numel() == numel and t.is_cuda and t.is_contiguous():
        return t.data_ptr()
    if t.dtype != dtype:
        raise ValueError(f"{what} must be {dtype}")
    if t.numel() != numel:
        raise ValueError(f"{what} holds {t.numel()} elements, the call needs {numel}")
    return B._dev_ptr(t, what)


_current_device, _current_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream


def _stream_handle(stream) -> int:
    """As binding._stream_handle; the current stream without the object around it (0.1 us instead of 2.8)."""
    return _current_stream(_current_device()) if stream is None else B._stream_handle(stream)


def _rows_of(t: torch.Tensor, d: int, what: str) -> int:
    if not t.dim() or t.shape[-1] != d:
        raise ValueError(f"the last extent of {what} must be {d}")
    return t.numel() // d


def _workspace(t: torch.Tensor) -> Tuple[int, int]:
    return B._dev_ptr(t, "workspace"), t.numel() * t.element_size()


# ---- kept rows of a mask -----------------------------------------------------------------------------------------------


class RowSet:
    """Owner of an sc_rows handle and of the workspace its lists lie in."""

    def __init__(self, handle: int, workspace: torch.Tensor):
        self.handle = handle
        self.workspace = workspace
        self.rows, self.kept = _row_counts(handle)

    def close(self):
        if self.handle:
            lib().sparse_rows_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _row_counts(handle: int) -> Tuple[int, int]:
    m, kept = ctypes.c_int64(), ctypes.c_int64()
    B._check(lib().sparse_rows_info(handle, ctypes.byref(m), ctypes.byref(kept), None, None), "sparse_rows_info")
    return m.value, kept.value


def _handle(rows: Optional[RowSet]) -> Optional[int]:
    """None stands for all rows, so a closed set must not turn into it: its tensors may hold fewer."""
    if rows is None:
        return None
    if not rows.handle:
        raise ValueError("the row set is closed")
    return rows.handle


def sparse_rows_workspace_bytes(rows: int) -> int:
    n = ctypes.c_size_t()
    B._check(lib().sparse_rows_workspace_bytes(rows, ctypes.byref(n)), "sparse_rows_workspace_bytes")
    return n.value


def sparse_rows_plan(mask: torch.Tensor, workspace: Optional[torch.Tensor] = None, stream=None) -> RowSet:
    """mask: uint8 device tensor, one byte a row; synchronises the stream."""
    if mask.dtype != torch.uint8:
        raise ValueError("mask must be uint8")
    nbytes = sparse_rows_workspace_bytes(mask.numel())
    if workspace is None:
        workspace = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=mask.device)
    at, size = _workspace(workspace)
    out = ctypes.c_void_p()
    B._check(lib().sparse_rows_plan(B._dev_ptr(mask, "mask"), mask.numel(), at, size, _stream_handle(stream), ctypes.byref(out)),
             "sparse_rows_plan")
    return RowSet(out.value, workspace)


def sparse_rows_set_mask(rows: RowSet, mask: torch.Tensor, stream=None) -> RowSet:
    """A new mask of as many rows (synchronises the stream); the number of kept rows may change."""
    try:
        B._check(lib().sparse_rows_set_mask(_handle(rows), _tensor(mask, "mask", rows.rows, torch.uint8), _stream_handle(stream)),
                 "sparse_rows_set_mask")
    finally:
        if rows.handle:
            rows.kept = _row_counts(rows.handle)[1]      # (after a failure the set keeps none)
    return rows


def sparse_rows_info(rows: RowSet) -> Tuple[int, int, torch.Tensor, torch.Tensor]:
    """(rows, kept, ascending list of the kept rows, slot of every row or -1); the lists are copies."""
    m, kept, idx, slot = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_void_p(), ctypes.c_void_p()
    B._check(lib().sparse_rows_info(_handle(rows), ctypes.byref(m), ctypes.byref(kept), ctypes.byref(idx), ctypes.byref(slot)),
             "sparse_rows_info")
    base = rows.workspace.data_ptr()
    flat = rows.workspace.view(torch.uint8).reshape(-1)

    def ints(address, count):
        at = (address or base) - base
        return flat[at: at + 4 * count].view(torch.int32).clone()

    return m.value, kept.value, ints(idx.value, kept.value), ints(slot.value, m.value)


# ---- norms around a block ----------------------------------------------------------------------------------------------


def sparse_norm_workspace_bytes(desc: sc_norm_desc, rows: int) -> int:
    n = ctypes.c_size_t()
    B._check(lib().sparse_norm_workspace_bytes(ctypes.byref(desc), rows, ctypes.byref(n)), "sparse_norm_workspace_bytes")
    return n.value


def _norm_shapes(desc, x, f_rows, h_rows):
    rows = _rows_of(x, desc.d, "x")
    f_kept = h_kept = rows
    if f_rows is not None or h_rows is not None:
        for r in (f_rows, h_rows):
            if r is not None and r.rows != rows:
                raise ValueError(f"the row set is of {r.rows} rows, x has {rows}")
        f_kept, h_kept = (rows if r is None else r.kept for r in (f_rows, h_rows))
    per = desc.rows_per_gate
    return rows, f_kept, h_kept, -(-rows // per) if per else min(rows, 1)


def _elem(desc) -> torch.dtype:
    t = _TORCH_OF_CODE.get(desc.dtype)
    if t is None:
        raise ScError(B.SC_ERR_UNSUPPORTED, "descriptor")
    return t


def sparse_norm_run(desc: sc_norm_desc, x, f, gate, w_post, b_post, w_pre, b_pre, x_new, h, f_rows: Optional[RowSet] = None,
                    h_rows: Optional[RowSet] = None, stats=None, stream=None):
    """(x_new, h): x_new = a x + b gate post(f), h = pre(x_new); tensors may be None where the C entry point allows NULL."""
    t, d, tensor = _elem(desc), desc.d, _tensor
    rows, f_kept, h_kept, gates = _norm_shapes(desc, x, f_rows, h_rows)
    all_of_x = rows * d
    status = lib().sparse_norm_run(
        ctypes.byref(desc), rows, tensor(x, "x", all_of_x, t), None if f is None else tensor(f, "f", f_kept * d, t),
        None if f_rows is None else _handle(f_rows), None if gate is None else tensor(gate, "gate", gates * d, t),
        None if w_post is None else tensor(w_post, "w_post", d, _F32), None if b_post is None else tensor(b_post, "b_post", d, _F32),
        None if w_pre is None else tensor(w_pre, "w_pre", d, _F32), None if b_pre is None else tensor(b_pre, "b_pre", d, _F32),
        None if x_new is None else tensor(x_new, "x_new", all_of_x, t), None if h is None else tensor(h, "h", h_kept * d, t),
        None if h_rows is None else _handle(h_rows), None if stats is None else tensor(stats, "stats", rows * 4, _F32),
        _stream_handle(stream))
    if status:
        raise ScError(status, "sparse_norm_run")
    return x_new, h


def sparse_norm_backward(desc: sc_norm_desc, x, f, gate, w_post, b_post, w_pre, stats, dx_new, dh, dx, df, dgate, dw_post, db_post,
                         dw_pre, db_pre, workspace, f_rows: Optional[RowSet] = None, h_rows: Optional[RowSet] = None, stream=None):
    """Gradients into dx .. db_pre; those that are None are not computed."""
    t, f32, d = _elem(desc), torch.float32, desc.d
    rows, f_kept, h_kept, gates = _norm_shapes(desc, x, f_rows, h_rows)
    at, size = _workspace(workspace)
    B._check(lib().sparse_norm_backward(
        ctypes.byref(desc), rows, _tensor(x, "x", rows * d, t), _tensor(f, "f", f_kept * d, t), _handle(f_rows),
        _tensor(gate, "gate", gates * d, t), _tensor(w_post, "w_post", d, f32), _tensor(b_post, "b_post", d, f32),
        _tensor(w_pre, "w_pre", d, f32), _tensor(stats, "stats", rows * 4, f32), _tensor(dx_new, "dx_new", rows * d, t),
        _tensor(dh, "dh", h_kept * d, t), _handle(h_rows), _tensor(dx, "dx", rows * d, t), _tensor(df, "df", f_kept * d, t),
        _tensor(dgate, "dgate", gates * d, t), _tensor(dw_post, "dw_post", d, f32), _tensor(db_post, "db_post", d, f32),
        _tensor(dw_pre, "dw_pre", d, f32), _tensor(db_pre, "db_pre", d, f32), at, size, _stream_handle(stream)),
        "sparse_norm_backward")


# ---- gated feed-forward block ------------------------------------------------------------------------------------------


def sparse_ffn_workspace_bytes(desc: sc_ffn_desc, kept: int, training: bool = False) -> int:
    n = ctypes.c_size_t()
    B._check(lib().sparse_ffn_workspace_bytes(ctypes.byref(desc), kept, int(training), ctypes.byref(n)), "sparse_ffn_workspace_bytes")
    return n.value


def _ffn_shapes(desc, rows, x, x_rows, y, y_rows, y_name):
    xn, yn = _rows_of(x, desc.d_in, "x"), _rows_of(y, desc.d_out, y_name)
    if rows is None:
        m = kept = xn
    else:
        m, kept = rows.rows, rows.kept
    for have, fmt, name in ((xn, x_rows, "x"), (yn, y_rows, y_name)):
        want = kept if fmt == SC_ROWS_COMPACT else m
        if have != want:
            raise ValueError(f"{name} has {have} rows, the call needs {want}")
    return m, kept


def sparse_ffn_run(desc: sc_ffn_desc, x, w_gate, w_up, w_down, y, workspace, rows: Optional[RowSet] = None,
                   x_rows: int = SC_ROWS_DENSE, y_rows: int = SC_ROWS_DENSE, saved=None, stream=None):
    """y = (act(x w_gate') * (x w_up')) w_down' over the kept rows; saved: [3, kept, d_hidden], what the backward pass
    needs of the two products (in its own layout)."""
    t = _elem(desc)
    m, kept = _ffn_shapes(desc, rows, x, x_rows, y, y_rows, "y")
    di, dh, do = desc.d_in, desc.d_hidden, desc.d_out
    at, size = _workspace(workspace)
    B._check(lib().sparse_ffn_run(
        ctypes.byref(desc), m, _handle(rows), _tensor(x, "x", x.numel(), t), x_rows, _tensor(w_gate, "w_gate", dh * di, t),
        _tensor(w_up, "w_up", dh * di, t), _tensor(w_down, "w_down", do * dh, t), _tensor(y, "y", y.numel(), t), y_rows,
        _tensor(saved, "saved", 3 * kept * dh, t), at, size, _stream_handle(stream)), "sparse_ffn_run")
    return y


def sparse_ffn_backward(desc: sc_ffn_desc, x, w_gate, w_up, w_down, saved, dy, dx, dw_gate, dw_up, dw_down, workspace,
                        rows: Optional[RowSet] = None, x_rows: int = SC_ROWS_DENSE, y_rows: int = SC_ROWS_DENSE, stream=None):
    """Gradients into dx (format of x; may be None) and the three weight gradients (may all be None)."""
    t = _elem(desc)
    m, kept = _ffn_shapes(desc, rows, x, x_rows, dy, y_rows, "dy")
    di, dh, do = desc.d_in, desc.d_hidden, desc.d_out
    at, size = _workspace(workspace)
    B._check(lib().sparse_ffn_backward(
        ctypes.byref(desc), m, _handle(rows), _tensor(x, "x", x.numel(), t), x_rows, _tensor(w_gate, "w_gate", dh * di, t),
        _tensor(w_up, "w_up", dh * di, t), _tensor(w_down, "w_down", do * dh, t), _tensor(saved, "saved", 3 * kept * dh, t),
        _tensor(dy, "dy", dy.numel(), t), y_rows, _tensor(dx, "dx", x.numel(), t), _tensor(dw_gate, "dw_gate", dh * di, t),
        _tensor(dw_up, "dw_up", dh * di, t), _tensor(dw_down, "dw_down", do * dh, t), at, size, _stream_handle(stream)),
        "sparse_ffn_backward")


# ---- products with 4-bit weights ---------------------------------------------------------------------------------------


class Q4Plan:
    """Owner of an sc_q4 handle and of the workspace that holds its weights."""

    def __init__(self, handle: int, desc: sc_q4_desc, workspace: torch.Tensor):
        self.handle = handle
        self.desc = desc
        self.workspace = workspace
        self.type, self.k, self.n = _elem(desc), desc.k, desc.n

    def close(self):
        if self.handle:
            lib().sparse_q4_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def sparse_q4_workspace_bytes(desc: sc_q4_desc, gated: bool = False) -> int:
    n = ctypes.c_size_t()
    B._check(lib().sparse_q4_workspace_bytes(ctypes.byref(desc), int(gated), ctypes.byref(n)), "sparse_q4_workspace_bytes")
    return n.value


def _q4_matrix(desc, codes, scales, zeros, what=""):
    groups = -(-desc.k // desc.group)
    t = _elem(desc)
    return (_tensor(codes, what + "codes", desc.n * (-(-desc.k // 2)), torch.uint8),
            _tensor(scales, what + "scales", desc.n * groups, t), _tensor(zeros, what + "zeros", desc.n * groups, t))


def sparse_q4_plan(desc: sc_q4_desc, codes, scales, zeros=None, workspace=None, stream=None) -> Q4Plan:
    """Lays out codes uint8[n, ceil(k / 2)], scales and zeros [n, ceil(k / group)]; they are not needed once the stream has passed."""
    nbytes = sparse_q4_workspace_bytes(desc)
    matrix = _q4_matrix(desc, codes, scales, zeros)
    if workspace is None:
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=codes.device)
    at, size = _workspace(workspace)
    out = ctypes.c_void_p()
    B._check(lib().sparse_q4_plan(ctypes.byref(desc), *matrix, at, size, _stream_handle(stream), ctypes.byref(out)), "sparse_q4_plan")
    return Q4Plan(out.value, desc, workspace)


def sparse_q4_plan_gated(desc: sc_q4_desc, gate: Dict[str, torch.Tensor], up: Dict[str, torch.Tensor], activation=SC_ACT_SILU,
                         workspace=None, stream=None) -> Q4Plan:
    """gate, up: {"codes", "scales"[, "zeros"]} as for sparse_q4_plan; the run is act(x gate') * (x up')."""
    nbytes = sparse_q4_workspace_bytes(desc, True)
    matrices = [_q4_matrix(desc, w["codes"], w["scales"], w.get("zeros"), name) for w, name in ((gate, "gate "), (up, "up "))]
    if workspace is None:
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=gate["codes"].device)
    at, size = _workspace(workspace)
    out = ctypes.c_void_p()
    B._check(lib().sparse_q4_plan_gated(ctypes.byref(desc), activation, *matrices[0], *matrices[1], at, size, _stream_handle(stream),
                                        ctypes.byref(out)), "sparse_q4_plan_gated")
    return Q4Plan(out.value, desc, workspace)


def sparse_q4_run(plan: Q4Plan, x, y, stream=None):
    t, k = plan.type, plan.k
    rows = x.numel() // k
    # (one condition for the call of a single token; what is wrong with it is said by the checks below)
    if not (x.dtype is t and y.dtype is t and x.dim() and x.shape[-1] == k and y.numel() == rows * plan.n and x.is_cuda and y.is_cuda
            and x.is_contiguous() and y.is_contiguous()):
        rows = _rows_of(x, k, "x")
        _tensor(x, "x", rows * k, t), _tensor(y, "y", rows * plan.n, t)
    status = lib().sparse_q4_run(plan.handle, rows, x.data_ptr(), y.data_ptr(), _stream_handle(stream))
    if status:
        raise ScError(status, "sparse_q4_run")
    return y
