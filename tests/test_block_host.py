"""Host-only checks of the block operators (include/sparse_block.h): symbols, the binding's signatures, refusals.  No call here
launches work."""
import ctypes
import os
import re

import pytest
import torch

from paper_2309_06626_amd import binding as B
from paper_2309_06626_amd import block as K

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x1000      # an address that no check dereferences
MIB = 1 << 20


def declarations():
    text = open(os.path.join(ROOT, "include", "sparse_block.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    found = re.findall(r"\b(?:sc_status|void)\s+(sparse_\w+)\s*\(([^;]*)\)\s*;", text)
    return {name: [a.strip() for a in args.split(",")] for name, args in found}


def test_every_entry_point_is_exported_and_declared_with_its_arguments():
    L = K.lib()
    names = declarations()
    assert len(names) == 16
    for name, args in names.items():
        kinds = getattr(L, name).argtypes
        assert len(kinds) == len(args), name
        for kind, arg in zip(kinds, args):
            if "*" in arg:
                assert kind is ctypes.c_void_p or issubclass(kind, ctypes._Pointer), (name, arg)
            elif arg.startswith("int32_t"):
                assert kind is ctypes.c_int32, (name, arg)
            elif arg.startswith("int64_t"):
                assert kind is ctypes.c_int64, (name, arg)
            else:
                assert arg.startswith("size_t") and kind is ctypes.c_size_t, (name, arg)


def test_row_sets_refuse():
    L, out, size = K.lib(), ctypes.c_void_p(7), ctypes.c_size_t()
    assert L.sparse_rows_workspace_bytes(100, ctypes.byref(size)) == B.SC_OK and size.value >= 808
    assert L.sparse_rows_workspace_bytes(100, None) == B.SC_ERR_NULL
    assert L.sparse_rows_workspace_bytes(-1, ctypes.byref(size)) == B.SC_ERR_BAD_SHAPE
    assert L.sparse_rows_workspace_bytes(1 << 31, ctypes.byref(size)) == B.SC_ERR_BAD_SHAPE
    plan = lambda *a: L.sparse_rows_plan(*a, None, ctypes.byref(out))  # noqa: E731
    assert plan(None, 100, FAKE, MIB) == B.SC_ERR_NULL and out.value is None
    assert plan(FAKE, 100, None, MIB) == B.SC_ERR_NULL
    assert plan(FAKE, -1, FAKE, MIB) == B.SC_ERR_BAD_SHAPE
    assert plan(FAKE, 100, FAKE, 800) == B.SC_ERR_WORKSPACE
    assert plan(FAKE, 100, FAKE + 4, MIB) == B.SC_ERR_ALIGN
    assert L.sparse_rows_plan(FAKE, 100, FAKE, MIB, None, None) == B.SC_ERR_NULL
    assert L.sparse_rows_set_mask(None, FAKE, None) == B.SC_ERR_NULL
    assert L.sparse_rows_info(None, None, None, None, None) == B.SC_ERR_NULL
    L.sparse_rows_destroy(None)


@pytest.mark.parametrize("field,value,status", [
    ("d", 0, B.SC_ERR_BAD_SHAPE), ("d", 8193, B.SC_ERR_BAD_SHAPE), ("dtype", 3, B.SC_ERR_UNSUPPORTED),
    ("post", 3, B.SC_ERR_UNSUPPORTED), ("pre", -1, B.SC_ERR_UNSUPPORTED), ("eps", -1.0, B.SC_ERR_BAD_SHAPE),
    ("eps", float("nan"), B.SC_ERR_BAD_SHAPE), ("rows_per_gate", -1, B.SC_ERR_BAD_SHAPE)])
def test_norm_descriptor_is_checked(field, value, status):
    L, size = K.lib(), ctypes.c_size_t(9)
    d = K.make_norm_desc(64)
    setattr(d, field, value)
    assert L.sparse_norm_workspace_bytes(ctypes.byref(d), 4, ctypes.byref(size)) == status and size.value == 0
    assert L.sparse_norm_run(ctypes.byref(d), 4, *[FAKE] * 2, None, *[FAKE] * 7, None, FAKE, None) == status
    assert L.sparse_norm_backward(ctypes.byref(d), 4, *[FAKE] * 2, None, *[FAKE] * 7, None, *[FAKE] * 8, MIB, None) == status


def test_norm_calls_refuse():
    L, d = K.lib(), K.make_norm_desc(64)
    names = ["x", "f", "f_rows", "gate", "w_post", "b_post", "w_pre", "b_pre", "x_new", "h", "h_rows", "stats"]

    def run(rows=4, **change):
        a = dict.fromkeys(names, FAKE)
        a.update(f_rows=None, h_rows=None)
        a.update(change)
        return L.sparse_norm_run(ctypes.byref(d), rows, *[a[n] for n in names], None)

    assert run(rows=-1) == B.SC_ERR_BAD_SHAPE
    assert run(rows=1 << 31) == B.SC_ERR_BAD_SHAPE
    assert run(x=None) == B.SC_ERR_NULL
    assert run(x_new=None, h=None) == B.SC_ERR_NULL
    assert run(h=FAKE + 8) == B.SC_ERR_ALIGN
    assert run(rows=0, x=None, f=None, h=None, x_new=None) == B.SC_OK
    assert L.sparse_norm_run(None, 4, *[FAKE] * 2, None, *[FAKE] * 7, None, FAKE, None) == B.SC_ERR_NULL
    names = ["x", "f", "f_rows", "gate", "w_post", "b_post", "w_pre", "stats", "dx_new", "dh", "h_rows", "dx", "df", "dgate",
             "dw_post", "db_post", "dw_pre", "db_pre", "workspace"]

    def backward(rows=4, size=MIB, **change):
        a = dict.fromkeys(names, FAKE)
        a.update(f_rows=None, h_rows=None)
        a.update(change)
        return L.sparse_norm_backward(ctypes.byref(d), rows, *[a[n] for n in names], size, None)

    assert backward(size=100) == B.SC_ERR_WORKSPACE
    assert backward(stats=None) == B.SC_ERR_NULL
    assert backward(dx_new=None, dh=None) == B.SC_ERR_NULL
    assert backward(f=None) == B.SC_ERR_NULL                 # df is wanted
    assert backward(gate=None) == B.SC_ERR_NULL              # dgate is wanted
    assert backward(dh=None) == B.SC_ERR_NULL                # dw_pre is wanted
    assert backward(workspace=None) == B.SC_ERR_NULL
    assert backward(dx=FAKE + 2) == B.SC_ERR_ALIGN


@pytest.mark.parametrize("field,value,status", [
    ("d_in", 0, B.SC_ERR_BAD_SHAPE), ("d_hidden", -8, B.SC_ERR_BAD_SHAPE), ("d_out", (1 << 20) + 1, B.SC_ERR_BAD_SHAPE),
    ("dtype", 7, B.SC_ERR_UNSUPPORTED), ("activation", 3, B.SC_ERR_UNSUPPORTED), ("activation", -1, B.SC_ERR_UNSUPPORTED)])
def test_ffn_descriptor_is_checked(field, value, status):
    L, size = K.lib(), ctypes.c_size_t(9)
    d = K.make_ffn_desc(64, 128, 64)
    setattr(d, field, value)
    assert L.sparse_ffn_workspace_bytes(ctypes.byref(d), 4, 1, ctypes.byref(size)) == status and size.value == 0
    assert L.sparse_ffn_run(ctypes.byref(d), 4, None, FAKE, 0, FAKE, FAKE, FAKE, FAKE, 0, None, FAKE, MIB, None) == status
    assert L.sparse_ffn_backward(ctypes.byref(d), 4, None, FAKE, 0, *[FAKE] * 5, 0, *[FAKE] * 5, MIB, None) == status


def test_ffn_calls_refuse():
    L, d = K.lib(), K.make_ffn_desc(64, 128, 64)
    names = ["rows", "x", "x_rows", "w_gate", "w_up", "w_down", "y", "y_rows", "saved", "workspace"]

    def run(m=4, size=MIB, **change):
        a = dict.fromkeys(names, FAKE)
        a.update(rows=None, x_rows=0, y_rows=0, saved=None)
        a.update(change)
        return L.sparse_ffn_run(ctypes.byref(d), m, *[a[n] for n in names], size, None)

    assert run(m=-1) == B.SC_ERR_BAD_SHAPE
    assert run(x_rows=2) == B.SC_ERR_UNSUPPORTED
    assert run(y_rows=-1) == B.SC_ERR_UNSUPPORTED
    for name in ("x", "w_gate", "w_up", "w_down", "y", "workspace"):
        assert run(**{name: None}) == B.SC_ERR_NULL
        assert run(**{name: FAKE + 8}) == B.SC_ERR_ALIGN
    assert run(size=4 * 128 * 2 - 1) == B.SC_ERR_WORKSPACE
    assert run(m=0, x=None, y=None) == B.SC_OK
    names = ["rows", "x", "x_rows", "w_gate", "w_up", "w_down", "saved", "dy", "y_rows", "dx", "dw_gate", "dw_up", "dw_down",
             "workspace"]

    def backward(m=4, size=MIB, **change):
        a = dict.fromkeys(names, FAKE)
        a.update(rows=None, x_rows=0, y_rows=0)
        a.update(change)
        return L.sparse_ffn_backward(ctypes.byref(d), m, *[a[n] for n in names], size, None)

    for name in ("x", "w_gate", "w_up", "w_down", "saved", "dy", "workspace", "dw_up"):
        assert backward(**{name: None}) == B.SC_ERR_NULL
    assert backward(dx=FAKE + 4) == B.SC_ERR_ALIGN
    assert backward(size=100) == B.SC_ERR_WORKSPACE


def test_q4_calls_refuse():
    L, size, out = K.lib(), ctypes.c_size_t(), ctypes.c_void_p(5)
    d = K.make_q4_desc(100, 33, 32)
    assert L.sparse_q4_workspace_bytes(ctypes.byref(d), 0, ctypes.byref(size)) == B.SC_OK and size.value >= 33 * 50
    one = size.value
    assert L.sparse_q4_workspace_bytes(ctypes.byref(d), 1, ctypes.byref(size)) == B.SC_OK and size.value == 2 * one
    for field, value, status in (("k", 0, B.SC_ERR_BAD_SHAPE), ("n", 0, B.SC_ERR_BAD_SHAPE), ("group", 48, B.SC_ERR_UNSUPPORTED),
                                 ("dtype", B.SC_F32, B.SC_ERR_UNSUPPORTED)):
        bad = K.make_q4_desc(100, 33, 32)
        setattr(bad, field, value)
        assert L.sparse_q4_workspace_bytes(ctypes.byref(bad), 0, ctypes.byref(size)) == status
        assert L.sparse_q4_plan(ctypes.byref(bad), FAKE, FAKE, None, FAKE, MIB, None, ctypes.byref(out)) == status
    plan = lambda c, s, z, w, n: L.sparse_q4_plan(ctypes.byref(d), c, s, z, w, n, None, ctypes.byref(out))  # noqa: E731
    assert plan(None, FAKE, None, FAKE, MIB) == B.SC_ERR_NULL and out.value is None
    assert plan(FAKE, None, None, FAKE, MIB) == B.SC_ERR_NULL
    assert plan(FAKE, FAKE, None, None, MIB) == B.SC_ERR_NULL
    assert plan(FAKE, FAKE, FAKE + 2, FAKE, MIB) == B.SC_ERR_ALIGN
    assert plan(FAKE, FAKE, None, FAKE, one - 1) == B.SC_ERR_WORKSPACE
    gated = lambda act, up, n: L.sparse_q4_plan_gated(ctypes.byref(d), act, FAKE, FAKE, None, up, FAKE, None, FAKE, n, None,  # noqa: E731
                                                      ctypes.byref(out))
    assert gated(9, FAKE, MIB) == B.SC_ERR_UNSUPPORTED
    assert gated(0, None, MIB) == B.SC_ERR_NULL
    assert gated(0, FAKE, 2 * one - 1) == B.SC_ERR_WORKSPACE
    assert L.sparse_q4_run(None, 1, FAKE, FAKE, None) == B.SC_ERR_NULL
    L.sparse_q4_destroy(None)


class Recorder:
    """Stands in for the library: takes every call, notes its name, launches nothing."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append(name) or 0


def test_a_closed_row_set_is_not_all_rows(monkeypatch):
    """The library takes NULL for all rows: with the kept rows alone in a tensor it would run over the end."""
    t = torch.zeros(3, 64, dtype=torch.bfloat16)
    x, w, stats = torch.zeros(8, 64, dtype=torch.bfloat16), torch.zeros(64, 64, dtype=torch.bfloat16), torch.zeros(8, 4)
    closed = K.RowSet.__new__(K.RowSet)
    closed.handle, closed.rows, closed.kept, closed.workspace = None, 8, 3, torch.zeros(512, dtype=torch.uint8)
    fake = Recorder()
    monkeypatch.setattr(K, "lib", lambda: fake)
    monkeypatch.setattr(K, "_tensor", lambda t, *_: None if t is None else t.data_ptr())
    monkeypatch.setattr(K, "_workspace", lambda t: (t.data_ptr(), t.numel()))
    monkeypatch.setattr(K, "_stream_handle", lambda stream: 0)
    norm, ffn, compact = K.make_norm_desc(64), K.make_ffn_desc(64, 64, 64), B.SC_ROWS_COMPACT
    none = [None] * 5
    for call in (lambda: K.sparse_ffn_run(ffn, t, w, w, w, t, x, closed, compact, compact),
                 lambda: K.sparse_ffn_backward(ffn, t, w, w, w, t, t, t, w, w, w, x, closed, compact, compact),
                 lambda: K.sparse_norm_run(norm, x, t, *none, x, x, f_rows=closed),
                 lambda: K.sparse_norm_run(norm, x, None, *none, x, t, h_rows=closed),
                 lambda: K.sparse_norm_backward(norm, x, t, None, None, None, None, stats, x, x, x, t, *none, x, f_rows=closed),
                 lambda: K.sparse_norm_backward(norm, x, None, None, None, None, None, stats, x, t, x, None, *none, x, h_rows=closed),
                 lambda: K.sparse_rows_set_mask(closed, torch.zeros(8, dtype=torch.uint8)),
                 lambda: K.sparse_rows_info(closed)):
        with pytest.raises(ValueError, match="closed"):
            call()
    assert not fake.calls


def test_a_mask_that_could_not_be_set_leaves_no_stale_count(monkeypatch):
    class Failing:
        """The library's set keeps nothing after a failure."""
        def sparse_rows_set_mask(self, *args):
            return B.SC_ERR_HIP

        def sparse_rows_info(self, handle, rows, kept, *lists):
            rows._obj.value, kept._obj.value = 8, 0
            return B.SC_OK

        def sparse_rows_destroy(self, handle):
            pass

    fake = Failing()
    rows = K.RowSet.__new__(K.RowSet)
    rows.handle, rows.rows, rows.kept = FAKE, 8, 3
    monkeypatch.setattr(K, "lib", lambda: fake)
    monkeypatch.setattr(K, "_tensor", lambda t, *_: t.data_ptr())
    monkeypatch.setattr(K, "_stream_handle", lambda stream: 0)
    with pytest.raises(K.ScError):
        K.sparse_rows_set_mask(rows, torch.zeros(8, dtype=torch.uint8))
    assert rows.kept == 0
    rows.handle = None      # (FAKE is no address to free)
