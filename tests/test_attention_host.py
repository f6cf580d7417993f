"""Host-only checks of the attention operators (include/sparse_attention.h): symbols, the binding's signatures, refusals, the oracle against
differentiation.  No call here launches work."""
import ctypes
import math
import os
import re

import pytest
import torch

import attention_oracle as O
from paper_2309_06626_amd import attention as A
from paper_2309_06626_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x1000      # an address that no check dereferences
MIB = 1 << 20


def declarations():
    text = open(os.path.join(ROOT, "include", "sparse_attention.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    found = re.findall(r"\b(?:sc_status|void)\s+(sparse_\w+)\s*\(([^;]*)\)\s*;", text)
    return {name: [a.strip() for a in args.split(",")] for name, args in found}


def test_every_entry_point_is_exported_and_declared_with_its_arguments():
    L = A.lib()
    names = declarations()
    assert len(names) == 12
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


BAD_ATTN = [("heads", 0, B.SC_ERR_BAD_SHAPE), ("kv_heads", 0, B.SC_ERR_BAD_SHAPE), ("kv_heads", 3, B.SC_ERR_BAD_SHAPE), ("heads", 513 * 2, B.SC_ERR_BAD_SHAPE),
            ("d", 0, B.SC_ERR_BAD_SHAPE), ("d", 129, B.SC_ERR_UNSUPPORTED), ("dtype", 3, B.SC_ERR_UNSUPPORTED), ("causal", 2, B.SC_ERR_UNSUPPORTED),
            ("window", -1, B.SC_ERR_BAD_SHAPE), ("scale", 0.0, B.SC_ERR_BAD_SHAPE), ("scale", -1.0, B.SC_ERR_BAD_SHAPE),
            ("scale", float("nan"), B.SC_ERR_BAD_SHAPE), ("scale", float("inf"), B.SC_ERR_BAD_SHAPE), ("scale", 2.0 ** 127 * 1.5, B.SC_ERR_BAD_SHAPE)]
BAD_KV = [("kv_heads", 0, B.SC_ERR_BAD_SHAPE), ("d", 0, B.SC_ERR_BAD_SHAPE), ("d", 129, B.SC_ERR_UNSUPPORTED), ("page_rows", 0, B.SC_ERR_BAD_SHAPE),
          ("page_rows", 24, B.SC_ERR_BAD_SHAPE), ("page_rows", 1 << 17, B.SC_ERR_BAD_SHAPE), ("pages", 0, B.SC_ERR_BAD_SHAPE),
          ("pages", 1 << 30, B.SC_ERR_BAD_SHAPE), ("dtype", -1, B.SC_ERR_UNSUPPORTED), ("bits", 4, B.SC_ERR_UNSUPPORTED)]


def changed(desc, field, value):
    setattr(desc, field, value)
    return desc


@pytest.mark.parametrize("field,value,status", BAD_ATTN)
def test_attention_descriptor_is_checked(field, value, status):
    L, size, out = A.lib(), ctypes.c_size_t(9), ctypes.c_void_p(5)
    d, kv = changed(A.make_attn_desc(4, 2, 64), field, value), A.make_kv_desc(2, 64, 16, 10)
    starts = (ctypes.c_int64 * 2)(0, 4)
    assert L.sparse_attn_workspace_bytes(ctypes.byref(d), 1, 4, ctypes.byref(size)) == status and size.value == 0
    assert L.sparse_attn_plan(ctypes.byref(d), 1, starts, None, FAKE, MIB, None, ctypes.byref(out)) == status and out.value is None
    assert L.sparse_attn_decode_workspace_bytes(ctypes.byref(d), ctypes.byref(kv), 1, 4, ctypes.byref(size)) == status
    assert L.sparse_attn_decode(ctypes.byref(d), ctypes.byref(kv), 1, FAKE, FAKE, 4, *[FAKE] * 7, MIB, None) == status


@pytest.mark.parametrize("field,value,status", BAD_KV)
def test_cache_descriptor_is_checked(field, value, status):
    L, size, entries = A.lib(), ctypes.c_size_t(9), ctypes.c_int32(9)
    d, kv = A.make_attn_desc(4, 2, 64), changed(A.make_kv_desc(2, 64, 16, 10), field, value)
    assert L.sparse_kv_row_entries(ctypes.byref(kv), ctypes.byref(entries)) == status and entries.value == 0
    assert L.sparse_kv_write(ctypes.byref(kv), 1, FAKE, 1 << 20, FAKE, 1 << 20, *[FAKE] * 5, None) == status
    assert L.sparse_kv_read(ctypes.byref(kv), 1, *[FAKE] * 6, 1 << 20, FAKE, 1 << 20, None) == status
    assert L.sparse_attn_decode_workspace_bytes(ctypes.byref(d), ctypes.byref(kv), 1, 4, ctypes.byref(size)) == status and size.value == 0
    assert L.sparse_attn_decode(ctypes.byref(d), ctypes.byref(kv), 1, FAKE, FAKE, 4, *[FAKE] * 7, MIB, None) == status


def test_cache_rows_are_whole_groups():
    for d, dtype, bits, want in ((41, A.SC_F32, 0, 44), (41, A.SC_BF16, 0, 48), (41, A.SC_BF16, 8, 48), (64, A.SC_F32, 8, 64), (1, A.SC_F16, 0, 8)):
        assert A.sparse_kv_row_entries(A.make_kv_desc(2, d, 16, 10, dtype, bits)) == want


def test_plans_refuse():
    L, size, out, d = A.lib(), ctypes.c_size_t(), ctypes.c_void_p(5), A.make_attn_desc(4, 2, 64)
    assert L.sparse_attn_workspace_bytes(ctypes.byref(d), 3, 1000, None) == B.SC_ERR_NULL
    for seqs, rows in ((-1, 5), (1, -1), (1, 1 << 31), (1 << 25, 5)):
        assert L.sparse_attn_workspace_bytes(ctypes.byref(d), seqs, rows, ctypes.byref(size)) == B.SC_ERR_BAD_SHAPE
    assert L.sparse_attn_workspace_bytes(ctypes.byref(A.make_attn_desc(512, 1, 64)), 1, 1 << 22, ctypes.byref(size)) == B.SC_ERR_BAD_SHAPE
    most = (1 << 23) - 512      # workgroups, of sequences of a row and of two key-value heads
    for seqs, status in ((most // 2 - 1, B.SC_OK), (most // 2, B.SC_ERR_BAD_SHAPE)):
        assert L.sparse_attn_workspace_bytes(ctypes.byref(d), seqs, 0, ctypes.byref(size)) == status
    assert L.sparse_attn_workspace_bytes(ctypes.byref(d), 3, 1000, ctypes.byref(size)) == B.SC_OK and size.value > 0
    need = size.value

    def plan(starts, rows=None, ws=FAKE, nbytes=MIB, desc=d):
        seqs = len(starts) - 1
        status = L.sparse_attn_plan(ctypes.byref(desc), seqs, (ctypes.c_int64 * len(starts))(*starts), rows, ws, nbytes, None, ctypes.byref(out))
        assert out.value is None
        return status

    assert plan([0, 10, 10, 1000], nbytes=need - 1) == B.SC_ERR_WORKSPACE
    assert plan([0, 10, 9]) == B.SC_ERR_BAD_SHAPE
    assert plan([1, 10]) == B.SC_ERR_BAD_SHAPE
    assert plan([0, -4]) == B.SC_ERR_BAD_SHAPE
    assert plan([0, 1 << 31]) == B.SC_ERR_BAD_SHAPE
    assert plan([0, 10], ws=None) == B.SC_ERR_NULL
    assert plan([0, 10], ws=FAKE + 4) == B.SC_ERR_ALIGN
    assert L.sparse_attn_plan(ctypes.byref(d), 1, None, None, FAKE, MIB, None, ctypes.byref(out)) == B.SC_ERR_NULL
    assert L.sparse_attn_plan(ctypes.byref(d), -1, (ctypes.c_int64 * 1)(0), None, FAKE, MIB, None, ctypes.byref(out)) == B.SC_ERR_BAD_SHAPE
    assert L.sparse_attn_plan(ctypes.byref(d), 0, (ctypes.c_int64 * 1)(0), None, FAKE, MIB, None, None) == B.SC_ERR_NULL
    assert L.sparse_attn_info(None, None, None) == B.SC_ERR_NULL
    assert L.sparse_attn_run(None, None, 0, *[FAKE, 512] * 3, FAKE, None, None) == B.SC_ERR_NULL
    assert L.sparse_attn_backward_workspace_bytes(None, ctypes.byref(size)) == B.SC_ERR_NULL
    assert L.sparse_attn_backward(None, None, 0, *[FAKE, 512] * 3, *[FAKE] * 3, *[FAKE, 512] * 3, FAKE, MIB, None) == B.SC_ERR_NULL
    L.sparse_attn_destroy(None)


def empty_plan(desc):
    """A plan of no rows needs no GPU."""
    L, out = A.lib(), ctypes.c_void_p()
    assert L.sparse_attn_plan(ctypes.byref(desc), 2, (ctypes.c_int64 * 3)(0, 0, 0), None, FAKE, MIB, None, ctypes.byref(out)) == B.SC_OK
    return out


def test_runs_refuse():
    L, d = A.lib(), A.make_attn_desc(4, 2, 64)
    plan = empty_plan(d)
    try:
        def run(fmt=0, rows=None, q=FAKE, qs=256, k=FAKE, ks=128, v=FAKE, vs=128, o=FAKE, lse=FAKE):
            return L.sparse_attn_run(plan, rows, fmt, q, qs, k, ks, v, vs, o, lse, None)

        assert run() == B.SC_OK and run(q=None, k=None, v=None, o=None, lse=None) == B.SC_OK
        assert run(fmt=2) == B.SC_ERR_UNSUPPORTED
        for bad in ({"qs": 255}, {"ks": 127}, {"vs": 0}, {"qs": -256}, {"qs": 1 << 41}):
            assert run(**bad) == B.SC_ERR_BAD_SHAPE
        assert run(q=FAKE + 1) == B.SC_ERR_ALIGN and run(q=FAKE + 2) == B.SC_OK
        assert run(o=FAKE + 8) == B.SC_ERR_ALIGN and run(lse=FAKE + 4) == B.SC_ERR_ALIGN

        def backward(size=MIB, ws=FAKE, dqs=256, dks=128, dvs=128, dq=FAKE, o=FAKE):
            return L.sparse_attn_backward(plan, None, 0, FAKE, 256, FAKE, 128, FAKE, 128, o, FAKE, FAKE, dq, dqs, FAKE, dks, FAKE, dvs, ws, size, None)

        assert backward() == B.SC_OK
        assert backward(size=10) == B.SC_ERR_WORKSPACE and backward(ws=None) == B.SC_ERR_NULL and backward(ws=FAKE + 8) == B.SC_ERR_ALIGN
        assert backward(dqs=255) == backward(dks=1) == backward(dvs=-1) == B.SC_ERR_BAD_SHAPE
        assert backward(dq=FAKE + 1) == B.SC_ERR_ALIGN and backward(o=FAKE + 2) == B.SC_ERR_ALIGN
    finally:
        L.sparse_attn_destroy(plan)


def test_cache_calls_refuse():
    L, d = A.lib(), A.make_kv_desc(2, 64, 16, 10, bits=8)

    def write(rows=3, k=FAKE, ks=128, v=FAKE, vs=128, slots=FAKE, kp=FAKE, vp=FAKE, kc=FAKE, vc=FAKE, desc=d):
        return L.sparse_kv_write(ctypes.byref(desc), rows, k, ks, v, vs, slots, kp, vp, kc, vc, None)

    def read(rows=3, k=FAKE, ks=128, v=FAKE, vs=128, slots=FAKE, kp=FAKE, vp=FAKE, kc=FAKE, vc=FAKE, desc=d):
        return L.sparse_kv_read(ctypes.byref(desc), rows, slots, kp, vp, kc, vc, k, ks, v, vs, None)

    plain = A.make_kv_desc(2, 64, 16, 10)
    for call in (write, read):
        assert call(rows=-1) == call(rows=1 << 31) == call(rows=1 << 28) == B.SC_ERR_BAD_SHAPE
        assert call(ks=127) == call(vs=-128) == B.SC_ERR_BAD_SHAPE
        for name in ("k", "v", "slots", "kp", "vp", "kc", "vc"):
            assert call(**{name: None}) == B.SC_ERR_NULL
        assert call(k=FAKE + 1) == call(slots=FAKE + 4) == call(kp=FAKE + 8) == call(vc=FAKE + 4) == B.SC_ERR_ALIGN
        assert call(rows=0) == call(rows=0, k=None, v=None, slots=None) == call(rows=0, kc=None, vc=None, desc=plain) == B.SC_OK
    assert L.sparse_kv_write(None, 1, FAKE, 1, FAKE, 1, *[FAKE] * 5, None) == B.SC_ERR_NULL


def test_decode_calls_refuse():
    L, d, kv, size = A.lib(), A.make_attn_desc(4, 2, 64), A.make_kv_desc(2, 64, 16, 10, bits=8), ctypes.c_size_t()
    nbytes = lambda rows=2, width=40, desc=d, cache=kv: L.sparse_attn_decode_workspace_bytes(ctypes.byref(desc), ctypes.byref(cache), rows, width, ctypes.byref(size))  # noqa: E731
    assert nbytes() == B.SC_OK
    need = size.value
    assert nbytes(rows=-1) == nbytes(width=-1) == nbytes(width=1 << 30) == nbytes(rows=1 << 25) == B.SC_ERR_BAD_SHAPE and size.value == 0
    ones = A.make_kv_desc(2, 64, 1, 10)      # stretches of 2 000 pages: a second launch has a workgroup for every head
    assert nbytes(rows=(1 << 22) - 1, width=1, cache=ones) == B.SC_OK and nbytes(rows=1 << 22, width=1, cache=ones) == B.SC_ERR_BAD_SHAPE
    for other in (A.make_kv_desc(1, 64, 16, 10), A.make_kv_desc(2, 32, 16, 10), A.make_kv_desc(2, 64, 16, 10, dtype=A.SC_F16)):
        assert nbytes(cache=other) == B.SC_ERR_BAD_SHAPE
    assert L.sparse_attn_decode_workspace_bytes(ctypes.byref(d), ctypes.byref(kv), 1, 1, None) == B.SC_ERR_NULL
    names = ["q", "table", "width", "lengths", "k_pages", "v_pages", "k_scales", "v_scales", "o", "workspace"]

    def decode(rows=2, nbytes=MIB, cache=kv, **change):
        a = dict.fromkeys(names, FAKE)
        a.update(width=40)
        a.update(change)
        return L.sparse_attn_decode(ctypes.byref(d), ctypes.byref(cache), rows, *[a[n] for n in names], nbytes, None)

    assert decode(nbytes=need - 1) == B.SC_ERR_WORKSPACE
    for name in names:
        if name != "width":
            assert decode(**{name: None}) == B.SC_ERR_NULL, name
            assert decode(**{name: FAKE + 8}) == B.SC_ERR_ALIGN, name
    assert decode(rows=0) == decode(rows=0, q=None, o=None, table=None, lengths=None) == B.SC_OK
    assert decode(rows=0, cache=A.make_kv_desc(2, 64, 16, 10), k_scales=None, v_scales=None) == B.SC_OK


class Recorder:
    """Stands in for the library: takes every call, notes its name, launches nothing."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append(name) or 0


class OnDevice(torch.Tensor):
    """A host tensor that says it is on the device."""
    is_cuda = True
    device_index = 0

    def get_device(self):
        return self.device_index


def fake(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice)


@pytest.fixture
def recorder(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(A, "lib", lambda: r)
    monkeypatch.setattr(A.K, "_stream_handle", lambda stream: 0)
    monkeypatch.setattr(A, "_current_device", lambda: 0)
    return r


def plan_of(desc, end, kept):
    p = A.AttnPlan.__new__(A.AttnPlan)
    p.handle, p.desc, p.workspace, p.end, p.kept = FAKE, desc, None, end, kept
    return p


def test_binding_looks_at_rows_types_and_strides(recorder):
    d = A.make_attn_desc(4, 2, 64)
    plan = plan_of(d, 10, 10)
    q, k, o, lse = fake(10, 4, 64), fake(10, 2, 64), fake(10, 4, 64), fake(10, 4, dtype=torch.float32)
    A.sparse_attn_run(plan, q, k, k, o, lse)
    wide = fake(12, 600)
    A.sparse_attn_run(plan, wide[:, :256], wide[:, 256:384], wide[:, 384:512], fake(12, 4, 64))      # two rows behind the last sequence
    assert recorder.calls == ["sparse_attn_run"] * 2
    for bad in (lambda: A.sparse_attn_run(plan, fake(9, 4, 64), k[:9], k[:9], fake(9, 4, 64)),               # rows missing
                lambda: A.sparse_attn_run(plan, q, fake(9, 2, 64), k, o),
                lambda: A.sparse_attn_run(plan, q, k, k, fake(9, 4, 64)),
                lambda: A.sparse_attn_run(plan, q, fake(10, 4, 64), k, o),                                      # heads
                lambda: A.sparse_attn_run(plan, q, k, k, o, fake(10, 2, dtype=torch.float32)),
                lambda: A.sparse_attn_run(plan, q, k, k, o, fake(10, 4)),
                lambda: A.sparse_attn_run(plan, fake(10, 4, 64, dtype=torch.float16), k, k, o),
                lambda: A.sparse_attn_run(plan, fake(10, 64, 4).transpose(1, 2), k, k, o),                      # entries apart
                lambda: A.sparse_attn_run(plan, torch.zeros(10, 4, 64, dtype=torch.bfloat16), k, k, o),         # on the host
                lambda: A.sparse_attn_run(plan, q[0], k, k, o)):
        with pytest.raises(ValueError):
            bad()
    elsewhere = fake(10, 2, 64)
    elsewhere.device_index = 1
    with pytest.raises(ValueError, match="another device"):
        A.sparse_attn_run(plan, q, elsewhere, k, o)
    plan.handle = None
    with pytest.raises(ValueError, match="closed"):
        A.sparse_attn_run(plan, q, k, k, o)
    closed = A.RowSet.__new__(A.RowSet)
    closed.handle, closed.rows, closed.kept = None, 10, 10
    plan.handle = FAKE
    with pytest.raises(ValueError, match="closed"):
        A.sparse_attn_run(plan, q, k, k, o, rows=closed)
    assert len(recorder.calls) == 2
    plan.handle = None


def test_binding_looks_at_devices(recorder, monkeypatch):
    """Of every tensor of a call, and of those that plans, row sets and caches hold."""
    def other(t):
        t.device_index = 1
        return t

    d, bf, f32, u8 = A.make_attn_desc(4, 2, 64), torch.bfloat16, torch.float32, torch.uint8
    plan, rows = plan_of(d, 10, 10), A.RowSet.__new__(A.RowSet)
    plan.workspace, rows.workspace, rows.handle, rows.rows, rows.kept = fake(64, dtype=u8), fake(64, dtype=u8), FAKE, 10, 10
    cache = A.KvCache.__new__(A.KvCache)
    cache.desc, cache.type, cache._width, cache._reference, cache._addresses, cache.device_index = A.make_kv_desc(2, 64, 16, 9), bf, 128, None, (0,) * 4, 0

    def calls():
        wide, narrow, ws = (10, 4, 64), (10, 2, 64), (64,)
        kept = (plan.workspace, rows.workspace)
        yield lambda *t: A.sparse_attn_run(plan, *t, rows=rows), [wide, narrow, narrow, wide], [bf] * 4, kept
        yield lambda *t: A.sparse_attn_run(plan, *t, rows=rows), [wide, narrow, narrow, wide, (10, 4)], [bf] * 4 + [f32], kept
        yield (lambda *t: A.sparse_attn_backward(plan, *t, rows=rows), [wide, narrow, narrow, wide, (10, 4), wide, wide, narrow, narrow, ws],
               [bf] * 4 + [f32] + [bf] * 4 + [u8], kept)
        yield lambda *t: A.sparse_kv_write(cache, *t), [narrow, narrow, (10,)], [bf, bf, torch.int64], (cache,)
        yield lambda s, k, v: A.sparse_kv_read(cache, s, k, v), [(10,), narrow, narrow], [torch.int64, bf, bf], (cache,)
        yield lambda *t: A.sparse_attn_decode(d, cache, *t), [wide, (10, 3), (10,), wide, ws], [bf, torch.int32, torch.int32, bf, u8], (cache,)

    for call, shapes, types, helds in calls():
        tensors = lambda: [fake(*s, dtype=t) for s, t in zip(shapes, types)]  # noqa: E731,B023
        call(*tensors())
        done = len(recorder.calls)
        for i in range(len(shapes)):
            with pytest.raises(ValueError, match="another device"):
                ts = tensors()
                other(ts[i])
                call(*ts)
        for held in helds:
            held.device_index = 1
            with pytest.raises(ValueError, match="another device"):
                call(*tensors())
            held.device_index = 0
        assert len(recorder.calls) == done
    with pytest.raises(ValueError, match="different devices"):
        A.KvCache(A.make_kv_desc(2, 64, 16, 9), fake(0), other(fake(0)))      # (the recorder has rows of no entries)
    plan.handle = rows.handle = None


def test_binding_looks_at_starts():
    d = A.make_attn_desc(4, 2, 64)
    with pytest.raises(ValueError):
        A.sparse_attn_plan(d, [])
    for starts in ([0, -1], [0, 1 << 63], [0, 1 << 40]):
        with pytest.raises(A.ScError):
            A.sparse_attn_plan(d, starts)


@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 5), (False, 4)])
def test_oracle_against_differentiation(causal, window):
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    starts, keep = [0, 12, 12, 28], torch.rand(30, generator=g) < 0.7
    x, do = [r(30, 4, 8), r(30, 2, 8), r(30, 2, 8)], r(30, 4, 8)
    c = (4, 2, 8, "f32", causal, window, 0.3)
    want, bound = O.packed(c, starts, keep, *x, do)
    leaves = [t.clone().requires_grad_(True) for t in x]
    out = O.packed(c, starts, keep, *leaves)[0]["o"]
    for got, n in zip(torch.autograd.grad(out, leaves, do), ("dq", "dk", "dv")):
        assert torch.allclose(got, want[n], atol=1e-12) and (bound[n] >= 0).all()
    # a row by hand
    at = torch.arange(12, 28)[keep[12:28]]
    i = len(at) // 2
    sees = [j for j in range(len(at)) if (j <= i or not causal) and (not window or abs(i - j) < window)]
    w = [math.exp(0.3 * float(x[0][at[i], 3] @ x[1][at[j], 1])) for j in sees]
    row = sum(a * x[2][at[j], 1] for a, j in zip(w, sees)) / sum(w)
    assert torch.allclose(out[at[i], 3], row)


def test_codes_of_the_oracle():
    x = torch.tensor([[127.0, 0.5, 1.5, -2.5], [0.0, 0, 0, 0], [1e-30, -1e30, 4e27, -4e27]], dtype=torch.float64)
    codes, scale = O.quantised(x)
    assert codes[0].tolist() == [127, 0, 2, -2] and codes[1].tolist() == [0] * 4 and codes[2].tolist() == [0, -127, 1, -1]
    assert scale.dtype == torch.float32 and scale[0] == 1
