"""Attention operators against the 64-bit oracle: types, heads, odd sizes, sequences from no row on, masks, windows, strides, pages."""
import math

import pytest
import torch

import attention_oracle as O
from paper_2309_06626_amd import attention as A
from paper_2309_06626_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def gen(seed):
    return torch.Generator().manual_seed(seed)


def normal(g, *shape, dtype="f32", std=1.0):
    """On the host, rounded to the type and widened to float64."""
    return (torch.randn(*shape, generator=g) * std).to(O.TORCH[dtype]).double()


def dev(t, dtype="f32"):
    return t.to(O.TORCH[dtype]).to(DEV)


def nans(*shape, dtype="f32"):
    return torch.full(shape, float("nan"), dtype=O.TORCH[dtype], device=DEV)


def same(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def inside(got, want, bound, what):
    got = got.double().cpu()
    assert got.shape == want.shape, what
    assert torch.isfinite(got).all(), what
    over = ((got - want).abs() / (bound + 1e-300)).max().item() if got.numel() else 0.0
    assert over <= 1.0, f"{what}: {over:.3g} times the bound"


def starts_of(lens):
    starts = [0]
    for n in lens:
        starts.append(starts[-1] + n)
    return starts


# ---- packed sequences --------------------------------------------------------------------------------------------------

CASES = [  # lengths, heads, kv heads, d, dtype, causal, window, share of rows kept, format, rows behind the last sequence
    ([1], 1, 1, 1, "f32", True, 0, 1.0, 0, 0),
    ([17], 32, 8, 128, "bf16", True, 0, 1.0, 0, 3),
    ([33, 0, 64, 1, 65], 4, 2, 64, "f16", True, 0, 1.0, 0, 0),
    ([129, 31, 0], 6, 6, 41, "f32", False, 0, 0.6, 0, 5),
    ([200, 7, 130], 3, 1, 72, "bf16", False, 0, 0.5, 1, 2),
    ([128, 300], 8, 8, 128, "bf16", True, 0, 1.0, 0, 0),
    ([260], 5, 1, 127, "f16", True, 33, 1.0, 0, 1),
    ([100, 100], 4, 4, 8, "bf16", False, 17, 0.7, 0, 0),
    ([257], 8, 2, 100, "f32", True, 64, 0.8, 1, 0),
    ([90, 5], 40, 1, 32, "bf16", True, 0, 1.0, 0, 0),
    ([70], 3, 3, 128, "f32", True, 0, 1.0, 0, 0),
    ([61, 64], 12, 4, 63, "bf16", True, 1, 0.9, 0, 0),
    ([190], 16, 2, 96, "f16", False, 0, 1.0, 0, 0),
    ([40, 0, 0, 24], 2, 2, 64, "bf16", True, 0, 0.0, 0, 4),
    ([513], 2, 1, 128, "bf16", False, 100, 1.0, 0, 0),
    ([3] * 50, 8, 8, 64, "f16", True, 0, 0.7, 0, 0),
    ([150, 40], 6, 3, 50, "bf16", True, 0, 0.8, 0, 2),
    ([150, 40], 4, 4, 110, "f16", False, 0, 1.0, 0, 0),
    ([600], 8, 2, 128, "bf16", True, 0, 1.0, 0, 0),
    ([600, 550], 4, 1, 64, "f16", True, 200, 0.9, 0, 0),
    ([550], 3, 1, 125, "bf16", True, 0, 1.0, 0, 0),
    ([700], 2, 1, 66, "bf16", False, 0, 1.0, 0, 0),
    ([5, 1, 9], 512, 1, 16, "f16", True, 0, 1.0, 0, 1),
    ([40], 48, 1, 64, "bf16", True, 7, 0.7, 0, 0),
    ([33, 70], 14, 2, 128, "bf16", False, 0, 1.0, 0, 0),
    ([70, 30], 64, 1, 128, "f32", True, 0, 1.0, 0, 0),
    ([900, 41], 3, 1, 41, "f32", True, 0, 0.6, 0, 2),
    ([700, 650], 4, 2, 63, "bf16", False, 0, 0.7, 0, 0),
    ([1100], 2, 2, 128, "f16", True, 300, 0.7, 1, 0),
]


def case_inputs(c, seed, strided=True):
    """One product's rows hold q, k and v, and so do their gradients, with a gap of `pad` entries behind every row."""
    lens, heads, kv, d, dtype, causal, window, share, fmt, tail = c
    g = gen(seed)
    starts = starts_of(lens)
    rows = starts[-1] + tail
    keep = torch.rand(rows, generator=g) < share
    x = {"q": normal(g, rows, heads, d, dtype=dtype, std=2.0), "k": normal(g, rows, kv, d, dtype=dtype), "v": normal(g, rows, kv, d, dtype=dtype),
         "do": normal(g, rows, heads, d, dtype=dtype)}
    return starts, rows, keep, x


def split(t, heads, kv, d):
    q, k, v = t[:, : (heads + 2 * kv) * d].split([heads * d, kv * d, kv * d], 1)
    return q, k, v


def packed_call(c, starts, keep, x, rows_set=None, pad=0, stream=None):
    """(o, lse, dq, dk, dv) of the rows that the format has; places that nothing is written to hold NaN."""
    lens, heads, kv, d, dtype, causal, window, share, fmt, tail = c
    desc = A.make_attn_desc(heads, kv, d, A.DTYPE_CODE[dtype], causal, window)
    rs = rows_set
    if rs is None and share < 1:
        rs = A.sparse_rows_plan(keep.to(torch.uint8).to(DEV))
    plan = A.sparse_attn_plan(desc, starts, rs)
    at = keep.nonzero()[:, 0] if fmt else torch.arange(len(keep))
    n, wide = len(at), (heads + 2 * kv) * d + pad
    qkv = torch.full((n, wide), float("nan"), dtype=O.TORCH[dtype])
    for part, name in zip(split(qkv, heads, kv, d), "qkv"):
        part.copy_(x[name][at].flatten(1))
    qkv = qkv.to(DEV)
    o, do, lse = nans(n, heads, d, dtype=dtype), dev(x["do"][at], dtype), nans(plan.kept, heads)
    A.sparse_attn_run(plan, *split(qkv, heads, kv, d), o, lse, rs, fmt)
    grads = nans(n, wide, dtype=dtype)
    ws = torch.empty(A.sparse_attn_backward_workspace_bytes(plan), dtype=torch.uint8, device=DEV)
    A.sparse_attn_backward(plan, *split(qkv, heads, kv, d), o, lse, do, *split(grads, heads, kv, d), ws, rs, fmt)
    dq, dk, dv = (t.reshape(n, -1, d) for t in split(grads, heads, kv, d))
    if pad:
        assert torch.isnan(grads[:, -pad:]).all()
    return plan, at, dict(o=o, lse=lse, dq=dq, dk=dk, dv=dv)


def packed_check(c, seed, pad=0, times=1):
    lens, heads, kv, d, dtype, causal, window, share, fmt, tail = c
    starts, rows, keep, x = case_inputs(c, seed)
    want, bound = O.packed((heads, kv, d, dtype, causal, window, 1 / math.sqrt(d)), starts, keep, x["q"], x["k"], x["v"], x["do"])
    if times > 1:      # the sequences again and again
        end = starts[-1]
        again = lambda t: torch.cat([t[:end]] * times + [t[end:]])  # noqa: E731
        keep, x, want, bound = again(keep), {n: again(t) for n, t in x.items()}, {n: again(t) for n, t in want.items()}, {n: again(t) for n, t in bound.items()}
        starts = starts_of(lens * times)
        c = (lens * times, *c[1:])
    plan, at, got = packed_call(c, starts, keep, x, pad=pad)
    inside_rows = at < starts[-1]
    kept_rows = keep.nonzero()[:, 0]
    kept_rows = kept_rows[kept_rows < starts[-1]]
    assert plan.end == starts[-1] and plan.kept == len(kept_rows)
    inside(got["lse"], want["lse"][kept_rows], bound["lse"][kept_rows], "lse")
    for name in ("o", "dq", "dk", "dv"):
        t = got[name].cpu()
        inside(t[inside_rows], want[name][at][inside_rows], bound[name][at][inside_rows], name)
        dropped = inside_rows & ~keep[at]
        assert (t[dropped].view(torch.int32 if dtype == "f32" else torch.int16) == 0).all(), "zeros of dropped rows"
        assert torch.isnan(t[~inside_rows]).all(), "rows behind the last sequence"
    return got


@pytest.mark.parametrize("c", CASES, ids=lambda c: "-".join(map(str, [sum(c[0]), len(c[0]), *c[1:]])))
def test_packed_forward_and_gradients(c):
    packed_check(c, 7 * sum(c[0]) + c[3])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("pad", [1, 2, 8])
def test_rows_with_gaps(dtype, pad):
    packed_check(([70, 33], 4, 2, 64, dtype, True, 0, 0.8, 0, 1), 3, pad)


@pytest.mark.parametrize("c", [c for c in CASES if c[0] != [700, 650]], ids=lambda c: "-".join(map(str, [sum(c[0]), len(c[0]), *c[1:]])))
def test_many_of_them(c):
    """Few rows are cut into smaller tiles than many: more than 2 048 tiles of 32, kept rows counted."""
    tiles = sum(-(-int(n * c[7] * 0.8) * c[1] // c[2] // 32) for n in c[0]) * c[2]
    packed_check(c, sum(c[0]) + c[3], times=2049 // max(tiles, 1) + 1 if c[7] else 2)


@pytest.mark.parametrize("pad", [1, 2, 8])
@pytest.mark.parametrize("d", [64, 128])
def test_long_rows_with_gaps(d, pad):
    packed_check(([600], 4, 2, d, "bf16", True, 0, 1.0, 0, 0), 5, pad)


@pytest.mark.parametrize("pad", [1, 2, 8])
@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "f16"), (96, "f32")])
def test_many_long_rows_with_gaps(d, dtype, pad):
    packed_check(([600], 4, 2, d, dtype, True, 0, 1.0, 0, 0), 5, pad, times=28)


def test_keys_and_values_of_different_strides_and_far_apart():
    """Queries follow each other, keys and values lie at other distances, the values' beyond what the offsets of plain rows span."""
    n, d = 90, 64
    g = gen(31)
    x = {"q": normal(g, n, 2, d, dtype="bf16"), "k": normal(g, n, 1, d, dtype="bf16"), "v": normal(g, n, 1, d, dtype="bf16"), "do": normal(g, n, 2, d, dtype="bf16")}
    want, bound = O.packed((2, 1, d, "bf16", True, 0, 0.125), [0, n], torch.ones(n, dtype=torch.bool), x["q"], x["k"], x["v"], x["do"])
    plan = A.sparse_attn_plan(A.make_attn_desc(2, 1, d), [0, n])
    ws = torch.empty(A.sparse_attn_backward_workspace_bytes(plan), dtype=torch.uint8, device=DEV)
    q, do = dev(x["q"], "bf16"), dev(x["do"], "bf16")
    for k_wide, v_wide in ((64, 200), (72, 64), (64, (1 << 22) + 8), ((1 << 22) + 8, (1 << 22) + 8)):
        k, v, dk, dv = (torch.empty(n, w, dtype=torch.bfloat16, device=DEV)[:, :d] for w in (k_wide, v_wide, k_wide, v_wide))
        k.copy_(x["k"][:, 0])
        v.copy_(x["v"][:, 0])
        o, lse, dq = nans(n, 2, d, dtype="bf16"), nans(n, 2), nans(n, 2, d, dtype="bf16")
        A.sparse_attn_run(plan, q, k, v, o, lse)
        A.sparse_attn_backward(plan, q, k, v, o, lse, do, dq, dk, dv, ws)
        for name, t in (("o", o), ("dq", dq), ("dk", dk), ("dv", dv)):
            inside(t.reshape(want[name].shape), want[name], bound[name], name)


def test_many_tiles_with_offsets_beyond_32_bits():
    n, heads, kv, d, stride = 1100, 32, 16, 64, (1 << 21) + 8
    g = gen(32)
    x = {name: normal(g, n, h, d, dtype="bf16") for name, h in (("q", heads), ("k", kv), ("v", kv), ("do", heads))}
    want, bound = O.packed((heads, kv, d, "bf16", True, 0, 0.125), [0, n], torch.ones(n, dtype=torch.bool), x["q"], x["k"], x["v"], x["do"])
    plan = A.sparse_attn_plan(A.make_attn_desc(heads, kv, d), [0, n])
    ws = torch.empty(A.sparse_attn_backward_workspace_bytes(plan), dtype=torch.uint8, device=DEV)
    q, k, v, dq, dk, dv = (torch.empty(n, stride, dtype=torch.bfloat16, device=DEV)[:, :h * d] for h in (heads, kv, kv) * 2)
    for t, name in ((q, "q"), (k, "k"), (v, "v")):
        t.copy_(dev(x[name], "bf16").flatten(1))
    o, lse = nans(n, heads, d, dtype="bf16"), nans(n, heads)
    A.sparse_attn_run(plan, q, k, v, o, lse)
    A.sparse_attn_backward(plan, q, k, v, o, lse, dev(x["do"], "bf16"), dq, dk, dv, ws)
    for name, t in (("o", o), ("dq", dq), ("dk", dk), ("dv", dv)):
        inside(t.reshape(want[name].shape), want[name], bound[name], name)


def test_no_sequences_and_empty_ones():
    x, o = nans(3, 2, 64, dtype="bf16"), nans(3, 2, 64, dtype="bf16")
    for starts in ([0], [0, 0, 0]):
        plan = A.sparse_attn_plan(A.make_attn_desc(2, 2, 64), starts)
        assert (plan.end, plan.kept) == (0, 0)
        ws = torch.empty(A.sparse_attn_backward_workspace_bytes(plan), dtype=torch.uint8, device=DEV)
        lse, grads = torch.empty(0, 2, device=DEV), [nans(3, 2, 64, dtype="bf16") for _ in range(3)]
        A.sparse_attn_run(plan, x, x, x, o, lse)
        A.sparse_attn_backward(plan, x, x, x, o, lse, x, *grads, ws)
        torch.cuda.synchronize()
        assert all(torch.isnan(t).all() for t in (o, *grads))


def test_many_short_sequences():
    """Whole numbers: every row of a sequence of equal keys is the mean of the values so far."""
    lens = [i % 4 for i in range(30000)]
    starts = starts_of(lens)
    n = starts[-1]
    q = torch.zeros(n, 2, 64, dtype=torch.bfloat16, device=DEV)
    v = torch.randint(-8, 9, (n, 1, 64), device=DEV, generator=torch.Generator(DEV).manual_seed(1)).to(torch.bfloat16)
    plan = A.sparse_attn_plan(A.make_attn_desc(2, 1, 64), starts)
    o = nans(n, 2, 64, dtype="bf16")
    A.sparse_attn_run(plan, q, torch.zeros_like(v), v, o)
    first = torch.tensor(starts[:-1], device=DEV).repeat_interleave(torch.tensor(lens, device=DEV))
    at = torch.arange(n, device=DEV)
    total = v[:, 0].double().cumsum(0)
    before = torch.where((first > 0)[:, None], total[(first - 1).clamp_min(0)], torch.zeros_like(total))
    want = ((total - before) / (at - first + 1)[:, None]).cpu()
    inside(o[:, 0], want, 2.0 ** -8 * want.abs() + 2.0 ** -20, "o")
    assert same(o[:, 0], o[:, 1])


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 95, 96, 127, 128, 129, 191, 192, 193, 255, 256, 257])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_end_of_a_tile(n, dtype):
    packed_check(([n, n], 2, 1, 64, dtype, n % 2 == 0, 0, 1.0, 0, 0), n)


@pytest.mark.parametrize("window", [1, 2, 31, 32, 33, 64, 65, 200, 1 << 30])
@pytest.mark.parametrize("causal", [True, False])
def test_windows(window, causal):
    packed_check(([150], 3, 1, 64, "bf16", causal, window, 1.0, 0, 0), window % 97)


def test_same_bits_again_and_in_both_formats():
    c = ([90, 61, 8], 6, 2, 64, "bf16", True, 0, 0.6, 0, 3)
    starts, rows, keep, x = case_inputs(c, 5)
    _, _, a = packed_call(c, starts, keep, x)
    _, _, b = packed_call(c, starts, keep, x)
    assert all(same(a[n], b[n]) for n in a)
    _, at, compact = packed_call(c[:8] + (1, 3), starts, keep, x)
    assert same(a["lse"], compact["lse"])
    for n in ("o", "dq", "dk", "dv"):
        assert same(a[n][at.to(DEV)], compact[n])


def test_rows_that_do_not_count_are_not_looked_at():
    """NaN in dropped rows, behind the last sequence and in the other sequence change nothing."""
    c = ([90, 61, 40], 6, 2, 64, "f16", False, 0, 0.6, 0, 3)
    starts, rows, keep, x = case_inputs(c, 6)
    _, _, clean = packed_call(c, starts, keep, x)
    for t in x.values():
        t[~keep] = float("nan")
        t[starts[-1]:] = float("nan")
    _, _, got = packed_call(c, starts, keep, x)
    assert all(same(clean[n], got[n]) for n in ("o", "dq", "dk", "dv", "lse"))
    for t in x.values():
        t[starts[1]:starts[2]] = float("inf")
    _, _, got = packed_call(c, starts, keep, x)
    for n in ("o", "dq", "dk", "dv"):
        for a, b in ((starts[0], starts[1]), (starts[2], starts[3])):
            assert same(clean[n][a:b], got[n][a:b])


@pytest.mark.parametrize("dtype,times", [("f32", 1), ("f32", 30), ("bf16", 30)])
@pytest.mark.parametrize("d", [64, 41])
def test_rows_that_do_not_count_of_few_and_many(dtype, times, d):
    """The same where tiles are those of few rows and of many: bits again, in both formats, with NaN in rows that do not count."""
    c = ([90, 61, 40] * times, 6, 2, d, dtype, True, 0, 0.7, 0, 3)
    starts, rows, keep, x = case_inputs(c, 6)
    _, _, clean = packed_call(c, starts, keep, x)
    _, at, compact = packed_call(c[:8] + (1, 3), starts, keep, x)
    inside_rows = at < starts[-1]
    for t in x.values():
        t[~keep] = float("nan")
        t[starts[-1]:] = float("nan")
    _, _, got = packed_call(c, starts, keep, x)
    assert all(same(clean[n], got[n]) for n in clean) and same(clean["lse"], compact["lse"])
    assert all(same(clean[n][at[inside_rows].to(DEV)], compact[n][inside_rows.to(DEV)]) for n in ("o", "dq", "dk", "dv"))
    assert all(torch.isfinite(clean[n][:starts[-1]]).all() for n in ("o", "dq", "dk", "dv"))
    for t in x.values():
        t[starts[-2]:starts[-1]] = float("inf")
    _, _, got = packed_call(c, starts, keep, x)
    assert all(same(clean[n][:starts[-2]], got[n][:starts[-2]]) for n in ("o", "dq", "dk", "dv"))


def test_a_query_that_is_not_finite_is_lost_alone():
    c = ([90], 4, 2, 64, "bf16", True, 0, 1.0, 0, 0)
    starts, rows, keep, x = case_inputs(c, 8)
    _, _, clean = packed_call(c, starts, keep, x)
    x["q"][40, 1] = float("nan")
    _, _, got = packed_call(c, starts, keep, x)
    ok = torch.ones(90, 4, dtype=torch.bool)
    ok[40, 1] = False
    assert same(clean["o"][ok.to(DEV)], got["o"][ok.to(DEV)]) and torch.isnan(got["o"][40, 1]).all()


def test_large_scores_do_not_overflow():
    """Scores of up to 39 000: softmax is a choice of one key, and lse the score: scale log2(e) and the score's product with it are rounded, and
    so are the constant and lse itself, 2^-24 each."""
    n, d = 40, 64
    q = torch.zeros(n, 1, d, dtype=torch.float64)
    k = torch.zeros(n, 1, d, dtype=torch.float64)
    q[:, 0, 0], k[:, 0, 0] = 1000, torch.arange(n).double()
    v = torch.randn(n, 1, d, generator=gen(1)).to(torch.bfloat16).double()
    plan = A.sparse_attn_plan(A.make_attn_desc(1, 1, d, scale=1.0), [0, n])
    o, lse = nans(n, 1, d, dtype="bf16"), nans(n, 1)
    A.sparse_attn_run(plan, dev(q, "bf16"), dev(k, "bf16"), dev(v, "bf16"), o, lse)
    assert torch.equal(o.double().cpu(), v)
    scores = 1000.0 * torch.arange(n).double()
    assert ((lse.double().cpu()[:, 0] - scores).abs() <= 4 * O.E * scores).all()


def test_gradients_against_differences():
    c = ([9, 14], 4, 2, 10, "f32", True, 0, 0.8, 0, 0)
    starts, rows, keep, x = case_inputs(c, 2)
    _, _, got = packed_call(c, starts, keep, x)

    def loss(v):
        want, _ = O.packed((4, 2, 10, "f32", True, 0, 1 / math.sqrt(10)), starts, keep, v["q"], v["k"], v["v"])
        return float((want["o"] * x["do"])[keep].sum())

    for n in "qkv":
        way, step = normal(gen(9), *x[n].shape), 1e-5
        slope = (loss({**x, n: x[n] + step * way}) - loss({**x, n: x[n] - step * way})) / (2 * step)
        terms = got["d" + n].double().cpu() * way
        assert abs(float(terms.sum()) - slope) <= 1e-5 * (1 + float(terms.abs().sum())), n


def test_long_rows_with_offsets_beyond_32_bits():
    """Rows 2^17 entries apart: the last ones lie beyond 2^32 entries."""
    n, heads, d, stride = 40000, 1, 64, 1 << 17
    lens = [20000, 19935, 65]
    big = torch.empty(n, stride, dtype=torch.bfloat16, device=DEV)
    g = torch.Generator(DEV).manual_seed(3)
    q, k, v = (big[:, i * 64: i * 64 + 64] for i in range(3))
    for t in (q, k, v):
        t.copy_(torch.randn(n, 64, generator=g, device=DEV))
    plan = A.sparse_attn_plan(A.make_attn_desc(heads, 1, d, window=64), starts_of(lens))
    o, lse = nans(n, heads, d, dtype="bf16"), nans(n, heads)
    A.sparse_attn_run(plan, q, k, v, o, lse)
    do = torch.randn(n, heads, d, generator=g, device=DEV).to(torch.bfloat16)
    ws = torch.empty(A.sparse_attn_backward_workspace_bytes(plan), dtype=torch.uint8, device=DEV)
    dq, dk, dv = (big[:, i * 64: i * 64 + 64] for i in range(3, 6))
    A.sparse_attn_backward(plan, q, k, v, o, lse, do, dq, dk, dv, ws)
    at = slice(n - 65, n)
    host = {name: t[at].double().cpu().view(65, 1, 64) for name, t in (("q", q), ("k", k), ("v", v), ("do", do))}
    want, bound = O.packed((1, 1, 64, "bf16", True, 64, 0.125), [0, 65], torch.ones(65, dtype=torch.bool), host["q"], host["k"], host["v"], host["do"])
    for name, t in (("o", o), ("dq", dq), ("dk", dk), ("dv", dv)):
        inside(t[at].reshape(65, 1, 64), want[name], bound[name], name)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n,heads,kv,d", [(300, 4, 4, 64), (300, 8, 2, 128), (190, 4, 4, 40)])
def test_results_are_as_near_as_their_operands_allow(dtype, n, heads, kv, d):
    """Probabilities and gradients of scores are rounded once, as operands of products, and results once more.  In a forward pass probabilities
    are rounded where the maximum so far is 1, in another binade than here: signs of errors change, not their size.  dq's scores have a delta from
    o as it is stored; dk's have not."""
    c = ([n], heads, kv, d, dtype, True, 0, 1.0, 0, 0)
    starts, rows, keep, x = case_inputs(c, 23)
    _, _, got = packed_call(c, starts, keep, x)
    want, _ = O.packed((heads, kv, d, dtype, True, 0, 1 / math.sqrt(d)), starts, keep, x["q"], x["k"], x["v"], x["do"])
    once = lambda v: v.to(O.TORCH[dtype]).double()  # noqa: E731
    near = {name: torch.zeros_like(want[name]) for name in ("o", "dq", "dk", "dv")}
    visible = O.seen(n, True, 0)
    for h in range(heads):
        j, scale = h * kv // heads, 1 / math.sqrt(d)
        q, k, v, do = x["q"][:, h], x["k"][:, j], x["v"][:, j], x["do"][:, h]
        o, _, p = O.attend(q, k, v, scale, visible)
        near["o"][:, h] = once(p) @ v
        dp = do @ v.T
        near["dq"][:, h] = once(p * (dp - (do * once(once(p) @ v)).sum(1, keepdim=True))) @ k * scale
        near["dk"][:, j] += once(p * (dp - (do * o).sum(1, keepdim=True))).T @ q * scale
        near["dv"][:, j] += once(p).T @ do
    for name in near:
        off, ideal = (got[name].double().cpu() - want[name]).norm(), (once(near[name]) - want[name]).norm()
        assert off <= 1.1 * ideal, f"{name}: {off / ideal:.3f}"


def test_a_new_mask_needs_a_new_plan():
    keep = torch.arange(64) % 3 != 0
    rs = A.sparse_rows_plan(keep.to(torch.uint8).to(DEV))
    plan = A.sparse_attn_plan(A.make_attn_desc(2, 2, 64), [0, 64], rs)
    x = nans(64, 2, 64, dtype="bf16")
    A.sparse_rows_set_mask(rs, keep.to(torch.uint8).to(DEV))
    with pytest.raises(A.ScError) as e:
        A.sparse_attn_run(plan, x, x, x, torch.empty_like(x), rows=rs)
    assert e.value.status == B.SC_ERR_MASK_COUNT
    with pytest.raises(A.ScError):
        A.sparse_attn_run(plan, x, x, x, torch.empty_like(x))
    plan = A.sparse_attn_plan(A.make_attn_desc(2, 2, 64), [0, 64], rs, workspace=plan.workspace)
    A.sparse_attn_run(plan, torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(x), x, rows=rs)
    assert (x == 0).all()


# ---- cache -------------------------------------------------------------------------------------------------------------


def cache_of(kv, d, page, pages, dtype, bits):
    return A.KvCache(A.make_kv_desc(kv, d, page, pages, A.DTYPE_CODE[dtype], bits), device=DEV)


@pytest.mark.parametrize("bits", [0, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,kv,d,page,pad", [(1, 1, 1, 1, 0), (5, 3, 41, 8, 1), (200, 8, 128, 64, 0), (77, 2, 64, 16, 8), (33, 5, 100, 32, 3)])
def test_cache_rows_come_back(rows, kv, d, page, pad, dtype, bits):
    g = gen(rows + d)
    pages = rows // page + 3
    cache = cache_of(kv, d, page, pages, dtype, bits)
    for t in (cache.k_pages, cache.v_pages):
        t.fill_(7)
    slots = torch.randperm(pages * page, generator=g)[:rows]
    slots[3::4] = -1
    if rows > 8:
        slots[2], slots[5], slots[6] = pages * page, 1 << 40, -(1 << 40)
    there = (slots >= 0) & (slots < pages * page)
    x = torch.full((rows, 2 * kv * d + pad), float("nan"), dtype=torch.float64)
    x[:, : 2 * kv * d] = normal(g, rows, 2 * kv * d, dtype=dtype) * 2.0 ** torch.randint(-8, 8, (rows, 1), generator=g)
    x = x.to(O.TORCH[dtype])
    k, v = (t.reshape(rows, kv, d).double() for t in x[:, : 2 * kv * d].split(kv * d, 1))
    on = x.to(DEV)
    A.sparse_kv_write(cache, *on[:, : 2 * kv * d].split(kv * d, 1), slots.to(DEV))
    out = nans(rows, 2 * kv * d + pad, dtype=dtype)
    A.sparse_kv_read(cache, slots.to(DEV), *out[:, : 2 * kv * d].split(kv * d, 1))
    if pad:
        assert torch.isnan(out[:, -pad:]).all()
    at = slots[there]
    for got, want, held, scales in zip(out[:, : 2 * kv * d].split(kv * d, 1), (k, v), (cache.k_pages, cache.v_pages), (cache.k_scales, cache.v_scales)):
        got, held = got.reshape(rows, kv, d).cpu(), held.cpu()
        assert (got[~there] == 0).all()
        mine = held[at // page, :, at % page]
        assert (mine[..., d:] == 0).all()
        others = torch.ones(pages * page, dtype=torch.bool)
        others[at] = False
        left = others.nonzero()[:, 0]
        assert (held[left // page, :, left % page] == 7).all()
        if bits:
            codes, scale = O.quantised(want[there])
            assert torch.equal(mine[..., :d].double(), codes) and torch.equal(scales.cpu()[at // page, :, at % page], scale)
            want = torch.zeros_like(want)
            want[there] = (codes.float() * scale[..., None]).double()
            want = want.to(O.TORCH[dtype]).double()
        else:
            assert torch.equal(mine[..., :d].double(), want[there])
        assert torch.equal(got[there].double(), want[there])


def test_codes_of_halves_zeros_small_and_lost_rows():
    d = 64
    x = torch.zeros(9, 1, d)
    x[0, 0, :6] = torch.tensor([127.0, 0.5, 1.5, -2.5, -0.5, 126.5])      # scale 1: ties to even
    x[2] = 2.0 ** -140                                                     # below the smallest scale: halves of one unit and less
    x[3] = 2.0 ** -127
    x[4, 0, 3] = float("nan")
    x[5, 0, 3] = float("-inf")
    x[6] = 3e38
    x[7, 0, :2] = torch.tensor([1e-30, -1e30])
    x[8] = -5.0
    cache = cache_of(1, d, 16, 1, "f32", 8)
    slots = torch.arange(9, device=DEV)
    A.sparse_kv_write(cache, x.to(DEV), x.to(DEV), slots)
    k, v = nans(9, 1, d), nans(9, 1, d)
    A.sparse_kv_read(cache, slots, k, v)
    assert same(k, v)
    codes = cache.k_pages[0, 0, :9].cpu()
    assert codes[0, :6].tolist() == [127, 0, 2, -2, 0, 126]
    k = k.cpu()
    assert (k[1] == 0).all() and (k[2] == 0).all() and (codes[3] == 0).all()
    assert torch.isnan(k[4:6]).all()
    assert torch.allclose(k[6], x[6], rtol=1e-6) and torch.equal(k[8], x[8])
    assert codes[7, :3].tolist() == [0, -127, 0] and (codes[6] == 127).all()
    assert (codes.abs() <= 127).all()


# ---- single tokens -----------------------------------------------------------------------------------------------------

DECODES = [  # lengths, heads, kv heads, d, page rows, dtype, bits, window, spare columns of the table
    ([1], 1, 1, 1, 1, "f32", 0, 0, 0),
    ([0, 5, 1], 8, 2, 64, 4, "bf16", 0, 0, 1),
    ([500], 32, 8, 128, 64, "bf16", 0, 0, 0),
    ([31, 32, 33, 64, 127, 128, 129, 0, 300], 6, 6, 41, 16, "f16", 0, 0, 0),
    ([700, 3, 260], 40, 1, 72, 32, "bf16", 0, 0, 2),
    ([513, 90], 4, 4, 128, 8, "f32", 0, 0, 0),
    ([513, 90], 4, 2, 127, 128, "f32", 8, 0, 0),
    ([1000, 1, 999], 16, 4, 128, 16, "f16", 8, 0, 0),
    ([640, 77], 8, 8, 100, 64, "bf16", 8, 0, 1),
    ([400, 20, 65], 6, 2, 64, 16, "bf16", 0, 50, 0),
    ([400, 20, 65], 6, 2, 64, 1, "f16", 8, 64, 0),
    ([5000], 9, 3, 96, 2, "bf16", 0, 0, 0),
    ([70] * 40, 8, 8, 64, 32, "f16", 0, 0, 0),
    ([3000, 2999], 70, 2, 128, 256, "bf16", 8, 1000, 0),
    ([37, 20], 512, 1, 32, 16, "f16", 0, 0, 0),
    ([37, 20], 512, 1, 32, 16, "bf16", 8, 0, 0),
    ([1500], 4, 4, 16, 65536, "bf16", 0, 0, 0),
    ([9000], 2, 1, 64, 1, "f32", 8, 0, 3),
    ([6000, 11], 8, 1, 128, 64, "f32", 0, 4000, 0),
]


def decode_inputs(c, seed):
    """A cache whose pages hold NaN where no sequence has a row; 64-bit keys and values as it holds them."""
    lens, heads, kv, d, page, dtype, bits, window, spare = c
    g = gen(seed)
    n, width = len(lens), max(max(-(-x // page) for x in lens), 1) + spare
    need = [-(-x // page) for x in lens]
    pages = sum(need) + 2
    cache = cache_of(kv, d, page, pages, dtype, bits)
    order = torch.randperm(pages, generator=g).to(torch.int32)
    table = torch.full((n, width), -1, dtype=torch.int32)
    if bits:
        for t in (cache.k_pages, cache.v_pages):
            t.fill_(99)
        for t in (cache.k_scales, cache.v_scales):
            t.fill_(float("nan"))
    else:
        for t in (cache.k_pages, cache.v_pages):
            t.fill_(float("nan"))
    keys, values, at = [], [], 0
    for i, length in enumerate(lens):
        table[i, : need[i]] = order[at: at + need[i]]
        at += need[i]
        j = torch.arange(length)
        slots = (table[i, j // page].long() * page + j % page).to(DEV)
        k, v = normal(g, length, kv, d, dtype=dtype), normal(g, length, kv, d, dtype=dtype)
        A.sparse_kv_write(cache, dev(k, dtype), dev(v, dtype), slots)
        if bits:
            k, v = (codes * scale.double()[..., None] for codes, scale in map(O.quantised, (k, v)))
        keys.append(k)
        values.append(v)
    return cache, table, normal(g, n, heads, d, dtype=dtype, std=2.0), keys, values


def decode_oracle(c, q, keys, values):
    lens, heads, kv, d, page, dtype, bits, window, spare = c
    want, bound = torch.zeros(len(lens), heads, d, dtype=torch.float64), torch.zeros(len(lens), heads, d, dtype=torch.float64)
    for i, n in enumerate(lens):
        first = max(0, n - window) if window else 0
        if n == 0:
            continue
        visible = torch.ones(1, n - first, dtype=torch.bool)
        for h in range(heads):
            one = q[i, h][None], keys[i][first:, h * kv // heads], values[i][first:, h * kv // heads]
            want[i, h] = O.attend(*one, 1 / math.sqrt(d), visible)[0][0]
            bound[i, h] = O.attend_bounds(*one, 1 / math.sqrt(d), visible, dtype)[0][0]
    return want, bound


def decode_call(c, cache, table, lens, q):
    heads, kv, d, dtype, window = c[1], c[2], c[3], c[5], c[7]
    desc = A.make_attn_desc(heads, kv, d, A.DTYPE_CODE[dtype], window=window)
    ws = torch.empty(A.sparse_attn_decode_workspace_bytes(desc, cache.desc, len(lens), table.shape[1]), dtype=torch.uint8, device=DEV)
    o = nans(len(lens), heads, d, dtype=dtype)
    return A.sparse_attn_decode(desc, cache, dev(q, dtype), table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), o, ws)


@pytest.mark.parametrize("c", DECODES, ids=lambda c: "-".join(map(str, [sum(c[0]), len(c[0]), *c[1:]])))
def test_decode(c):
    cache, table, q, keys, values = decode_inputs(c, sum(c[0]) + c[3])
    got = decode_call(c, cache, table, c[0], q)
    want, bound = decode_oracle(c, q, keys, values)
    inside(got, want, bound, "o")
    assert same(got, decode_call(c, cache, table, c[0], q))


def test_decode_of_pages_that_are_not_there_and_lengths_beyond_the_table():
    """Bad numbers in the table are rows that are not there; lengths below zero and beyond the table stand for none and for all it holds."""
    c = ([64, 64, 64, 64], 4, 2, 64, 16, "bf16", 0, 0, 0)
    cache, table, q, keys, values = decode_inputs(c, 4)
    table[0, 1], table[1, 0], table[1, 3], table[2] = -7, cache.desc.pages, 2 ** 31 - 1, -1
    got = decode_call(c, cache, table, [64, 60, 64, 1000], q)
    keep = [[(0, 16), (32, 64)], [(16, 48)], [], [(0, 64)]]
    pick = lambda t, spans: torch.cat([t[a:b] for a, b in spans]) if spans else t[:0]  # noqa: E731
    c = ([48, 32, 0, 64],) + c[1:]
    want, bound = decode_oracle(c, q, [pick(t, s) for t, s in zip(keys, keep)], [pick(t, s) for t, s in zip(values, keep)])
    inside(got, want, bound, "o")
    got = decode_call(c, cache, table, [-1, -(2 ** 31), 0, 2 ** 31 - 1], q)
    assert (got[:3] == 0).all()
    inside(got[3:], want[3:], bound[3:], "o")


def test_decode_without_pages_and_of_many_rows():
    cache = cache_of(1, 64, 16, 2, "bf16", 0)
    desc = A.make_attn_desc(2, 1, 64)
    rows = 70000
    q, o = torch.randn(rows, 2, 64, device=DEV).to(torch.bfloat16), nans(rows, 2, 64, dtype="bf16")
    ws = torch.empty(A.sparse_attn_decode_workspace_bytes(desc, cache.desc, rows, 1), dtype=torch.uint8, device=DEV)
    lengths = torch.full((rows,), 5, dtype=torch.int32, device=DEV)
    A.sparse_attn_decode(desc, cache, q, torch.empty(rows, 0, dtype=torch.int32, device=DEV), lengths, o, ws)
    assert (o == 0).all()
    v = torch.randint(-8, 9, (5, 1, 64), device=DEV).to(torch.bfloat16)      # equal keys: the values' mean
    A.sparse_kv_write(cache, torch.zeros_like(v), v, torch.arange(16, 21, device=DEV))
    table = torch.full((rows, 1), 1, dtype=torch.int32, device=DEV)
    A.sparse_attn_decode(desc, cache, q, table, lengths, o, ws)
    want = (v[:, 0].double().mean(0)).cpu().expand(rows, 2, 64)
    inside(o, want, 2.0 ** -8 * want.abs() + 2.0 ** -20, "o")


@pytest.mark.parametrize("bits", [0, 8])
def test_a_key_or_value_that_is_not_finite_loses_its_heads_alone(bits):
    c = ([100, 70], 4, 2, 64, 16, "bf16", bits, 0, 0)
    cache, table, q, keys, values = decode_inputs(c, 4)
    clean = decode_call(c, cache, table, c[0], q)
    if bits:
        cache.k_scales[table[0, 2].item(), 1, 3] = float("nan")
    else:
        cache.k_pages[table[0, 2].item(), 1, 3, 5] = float("nan")
    got = decode_call(c, cache, table, c[0], q)
    assert torch.isnan(got[0, 2:]).all()
    assert same(got[0, :2], clean[0, :2]) and same(got[1], clean[1])


def test_one_key_that_is_not_finite_is_not_an_empty_row():
    c = ([1], 2, 1, 64, 16, "bf16", 0, 0, 0)
    cache, table, q, keys, values = decode_inputs(c, 4)
    cache.k_pages[table[0, 0].item(), 0, 0, 5] = float("nan")
    assert torch.isnan(decode_call(c, cache, table, c[0], q)).all()


@pytest.mark.parametrize("small", [1e-3, 1.0, 300.0])
def test_8_bit_values_of_all_sizes_in_f16(small):
    """Values of one sequence differ by four decades in size: weights of the codes keep their digits."""
    c = ([300], 8, 2, 64, 16, "f16", 8, 0, 0)
    g = gen(12)
    cache = cache_of(2, 64, 16, 21, "f16", 8)
    table, j = torch.arange(20, dtype=torch.int32)[None], torch.arange(300)
    k, v = normal(g, 300, 2, 64, dtype="f16"), (normal(g, 300, 2, 64) * (10.0 ** (torch.arange(300) % 5 - 4))[:, None, None] * small).half().double()
    A.sparse_kv_write(cache, dev(k, "f16"), dev(v, "f16"), j.to(DEV))
    k, v = (codes * scale.double()[..., None] for codes, scale in map(O.quantised, (k, v)))
    q = normal(g, 1, 8, 64, dtype="f16", std=2.0)
    got = decode_call(c, cache, table, c[0], q)
    want, bound = decode_oracle(c, q, [k], [v])
    # weights are taken in units of a power of two near the largest scale: below 2^-14 of it they lose digits, 2^-25 units each, times codes up to 127
    inside(got, want, bound + 300 * 2.0 ** -25 * 127 * float(cache.v_scales.max()), "o")


def test_cache_beyond_32_bits():
    """5 GiB of pages: the last ones lie beyond 2^32 bytes."""
    kv, d, page, pages = 8, 128, 64, 40000
    cache = A.KvCache(A.make_kv_desc(kv, d, page, pages), device=DEV)
    g = gen(2)
    n = 150
    table = torch.tensor([[pages - 1, 3, pages - 2]], dtype=torch.int32)
    j = torch.arange(n)
    slots = (table[0, j // page].long() * page + j % page).to(DEV)
    k, v = normal(g, n, kv, d, dtype="bf16"), normal(g, n, kv, d, dtype="bf16")
    A.sparse_kv_write(cache, dev(k, "bf16"), dev(v, "bf16"), slots)
    k2, v2 = nans(n, kv, d, dtype="bf16"), nans(n, kv, d, dtype="bf16")
    A.sparse_kv_read(cache, slots, k2, v2)
    assert torch.equal(k2.double().cpu(), k) and torch.equal(v2.double().cpu(), v)
    c = ([n], 16, kv, d, page, "bf16", 0, 0, 0)
    q = normal(g, 1, 16, d, dtype="bf16", std=2.0)
    inside(decode_call(c, cache, table, [n], q), *decode_oracle(c, q, [k], [v]), "o")


# ---- together ----------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype,bits", [("bf16", 0), ("f16", 8), ("f32", 0)])
def test_a_prompt_and_the_tokens_behind_it(dtype, bits):
    """A prompt's attention, its rows into the cache, then token by token: as the attention over the whole sequence; in a graph too."""
    heads, kv, d, page, prompt, new = 8, 2, 64, 16, 37, 20
    g = gen(3)
    total = prompt + new
    x = {"q": normal(g, total, heads, d, dtype=dtype, std=2.0), "k": normal(g, total, kv, d, dtype=dtype), "v": normal(g, total, kv, d, dtype=dtype)}
    desc = A.make_attn_desc(heads, kv, d, A.DTYPE_CODE[dtype])
    held = [x["k"], x["v"]]
    if bits:
        held = [codes * scale.double()[..., None] for codes, scale in map(O.quantised, held)]
    want, bound = O.packed((heads, kv, d, dtype, True, 0, 1 / math.sqrt(d)), [0, total], torch.ones(total, dtype=torch.bool), x["q"], *held)
    on = {n: dev(t, dtype) for n, t in x.items()}
    plan = A.sparse_attn_plan(desc, [0, prompt])
    first = nans(prompt, heads, d, dtype=dtype)
    A.sparse_attn_run(plan, *(on[n][:prompt] for n in "qkv"), first)
    if not bits:
        inside(first, want["o"][:prompt], bound["o"][:prompt], "prompt")
    cache = cache_of(kv, d, page, 5, dtype, bits)
    table = torch.tensor([[4, 0, 3, 1]], dtype=torch.int32, device=DEV)
    slot = lambda j: table[0, j // page].long() * page + j % page  # noqa: E731
    A.sparse_kv_write(cache, on["k"][:prompt], on["v"][:prompt], slot(torch.arange(prompt, device=DEV)))
    ws = torch.empty(A.sparse_attn_decode_workspace_bytes(desc, cache.desc, 1, 4), dtype=torch.uint8, device=DEV)
    now = {n: torch.empty_like(t[:1]) for n, t in on.items()}
    slots, lengths, o = torch.empty(1, dtype=torch.int64, device=DEV), torch.empty(1, dtype=torch.int32, device=DEV), nans(1, heads, d, dtype=dtype)

    def step():
        A.sparse_kv_write(cache, now["k"], now["v"], slots)
        A.sparse_attn_decode(desc, cache, now["q"], table, lengths, o, ws)

    graph = None
    for j in range(prompt, total):
        for n in now:
            now[n].copy_(on[n][j: j + 1])
        slots.copy_(slot(torch.tensor([j], device=DEV)))
        lengths.fill_(j + 1)
        if j == prompt + 5:
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        if graph is not None:
            graph.replay()
        else:
            step()
        inside(o, want["o"][j: j + 1], bound["o"][j: j + 1], f"token {j}")


@pytest.mark.parametrize("d", [64, 128])
def test_training_step_in_a_graph(d):
    """Forward and backward, captured once and replayed on other inputs, with eager work of the program between: the bits of eager calls.  Two
    graphs share the workspace."""
    c = ([90, 61, 8], 6, 2, d, "bf16", True, 0, 0.6, 0, 3)
    starts, rows, keep, _ = case_inputs(c, 5)
    rs = A.sparse_rows_plan(keep.to(torch.uint8).to(DEV))
    plan = A.sparse_attn_plan(A.make_attn_desc(6, 2, d), starts, rs)
    ws = torch.empty(A.sparse_attn_backward_workspace_bytes(plan), dtype=torch.uint8, device=DEV)

    def buffers():
        b = {n: torch.zeros(rows, h, d, dtype=torch.bfloat16, device=DEV) for n, h in (("q", 6), ("k", 2), ("v", 2), ("o", 6), ("do", 6), ("dq", 6), ("dk", 2), ("dv", 2))}
        b["lse"] = torch.zeros(plan.kept, 6, device=DEV)
        return b

    def step(b):
        A.sparse_attn_run(plan, b["q"], b["k"], b["v"], b["o"], b["lse"], rs)
        A.sparse_attn_backward(plan, b["q"], b["k"], b["v"], b["o"], b["lse"], b["do"], b["dq"], b["dk"], b["dv"], ws, rs)

    sets, graphs = [buffers(), buffers()], []
    eager = buffers()
    for b in sets:
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            step(b)
    for turn in range(4):
        for which in (0, 1):
            x = case_inputs(c, 10 * turn + which)[3]
            for n, t in x.items():
                sets[which][n].copy_(dev(t, "bf16"))
                eager[n].copy_(sets[which][n])
            graphs[which].replay()
            step(eager)
            torch.cuda.synchronize()
            inside_rows = slice(0, starts[-1])
            assert all(same(sets[which][n][inside_rows], eager[n][inside_rows]) for n in ("o", "dq", "dk", "dv"))
            assert same(sets[which]["lse"], eager["lse"])


@pytest.mark.parametrize("dtype,times", [("f32", 1), ("f32", 30), ("bf16", 30)])
def test_graphs_of_few_and_many(dtype, times):
    c = ([90, 61, 8] * times, 6, 2, 72, dtype, True, 0, 1.0, 0, 0)
    starts, rows, _, x = case_inputs(c, 5)
    plan = A.sparse_attn_plan(A.make_attn_desc(6, 2, 72, A.DTYPE_CODE[dtype]), starts)
    ws = torch.empty(A.sparse_attn_backward_workspace_bytes(plan), dtype=torch.uint8, device=DEV)

    def buffers():
        b = {n: torch.zeros(rows, h, 72, dtype=O.TORCH[dtype], device=DEV) for n, h in (("q", 6), ("k", 2), ("v", 2), ("o", 6), ("do", 6), ("dq", 6), ("dk", 2), ("dv", 2))}
        b["lse"] = torch.zeros(rows, 6, device=DEV)
        return b

    def step(b):
        A.sparse_attn_run(plan, b["q"], b["k"], b["v"], b["o"], b["lse"])
        A.sparse_attn_backward(plan, b["q"], b["k"], b["v"], b["o"], b["lse"], b["do"], b["dq"], b["dk"], b["dv"], ws)

    captured, eager, graph = buffers(), buffers(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(captured)
    for turn in range(3):
        for n, t in x.items():
            eager[n].copy_(dev(t.roll(turn, 0), dtype))
            captured[n].copy_(eager[n])
        graph.replay()
        step(eager)
        torch.cuda.synchronize()
        assert all(same(captured[n], eager[n]) for n in ("o", "lse", "dq", "dk", "dv"))


def test_on_another_stream():
    c = ([90, 61], 6, 2, 64, "f16", True, 0, 1.0, 0, 0)
    starts, rows, keep, x = case_inputs(c, 5)
    _, _, want = packed_call(c, starts, keep, x)
    plan = A.sparse_attn_plan(A.make_attn_desc(6, 2, 64, A.SC_F16), starts)
    q, k, v = (dev(x[n], "f16") for n in "qkv")
    o = nans(rows, 6, 64, dtype="f16")
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    A.sparse_attn_run(plan, q, k, v, o, stream=stream)
    stream.synchronize()
    assert same(o, want["o"])


def test_two_calls_at_once():
    """One plan and one cache on two streams, with outputs and workspaces of their own."""
    c = ([900, 30, 1100], 8, 2, 128, "bf16", True, 0, 1.0, 0, 0)
    starts, rows, keep, x = case_inputs(c, 6)
    plan = A.sparse_attn_plan(A.make_attn_desc(8, 2, 128), starts)
    sets = [{n: dev(t if s == 0 else t.flip(0), "bf16").reshape(rows, -1, 128) for n, t in x.items() if n in ("q", "k", "v", "do")} for s in range(2)]
    dc = ([700, 1900, 64], 8, 2, 128, 16, "bf16", 8, 0, 0)
    cache, table, dq, _, _ = decode_inputs(dc, 7)
    table, desc, lens = table.to(DEV), A.make_attn_desc(8, 2, 128), torch.tensor(dc[0], dtype=torch.int32, device=DEV)
    ask, size = [dev(dq, "bf16"), dev(dq.flip(0), "bf16")], A.sparse_attn_decode_workspace_bytes(desc, cache.desc, 3, table.shape[1])

    def buffers():
        b = {"o": nans(rows, 8, 128, dtype="bf16"), "lse": nans(rows, 8), "dq": nans(rows, 8, 128, dtype="bf16"), "dk": nans(rows, 2, 128, dtype="bf16"),
             "dv": nans(rows, 2, 128, dtype="bf16"), "token": nans(3, 8, 128, dtype="bf16")}
        return b, [torch.empty(max(n, 16), dtype=torch.uint8, device=DEV) for n in (A.sparse_attn_backward_workspace_bytes(plan), size)]

    def go(i, b, ws, stream=None):
        s = sets[i]
        A.sparse_attn_run(plan, s["q"], s["k"], s["v"], b["o"], b["lse"], stream=stream)
        A.sparse_attn_backward(plan, s["q"], s["k"], s["v"], b["o"], b["lse"], s["do"], b["dq"], b["dk"], b["dv"], ws[0], stream=stream)
        A.sparse_attn_decode(desc, cache, ask[i], table, lens, b["token"], ws[1], stream=stream)

    want = []
    for i in range(2):
        b, ws = buffers()
        go(i, b, ws)
        want.append(b)
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [buffers(), buffers()]
    torch.cuda.synchronize()
    for _ in range(5):
        for i in range(2):
            go(i, *got[i], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        for name, t in want[i].items():
            assert same(got[i][0][name], t), (i, name)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_scores_of_minus_infinity(dtype):
    """A key whose score is -infinity has no weight; a row of such scores alone gives zeros, and so does a token."""
    n, d = 70, 64
    q, k = torch.ones(n, 1, d), torch.zeros(n, 1, d)
    v = torch.arange(n).float().reshape(n, 1, 1).expand(n, 1, d).contiguous()
    lost = torch.tensor([0, 1, 5, 64])
    k[lost, 0, 3] = -float("inf")
    plan = A.sparse_attn_plan(A.make_attn_desc(1, 1, d, A.DTYPE_CODE[dtype]), [0, n])
    o, lse = nans(n, 1, d, dtype=dtype), nans(n, 1)
    A.sparse_attn_run(plan, dev(q, dtype), dev(k, dtype), dev(v, dtype), o, lse)
    some = torch.ones(n).index_fill(0, lost, 0)
    count = some.cumsum(0)
    want = ((some * torch.arange(n)).double().cumsum(0) / count.clamp_min(1)).reshape(n, 1, 1).expand(n, 1, d)
    step = torch.finfo(O.TORCH[dtype]).eps / 2 + 4 * O.E      # weights are 1; of the result, of 1 / sum, of the product and of the shares' join
    inside(o, want, step * want.abs(), "o")
    assert (lse.cpu()[count == 0] == -float("inf")).all()
    inside(lse[2:], count[2:].double().log()[:, None], 8 * O.E * count[2:].double().log()[:, None] + 2.0 ** -22, "lse")
    cache = cache_of(1, d, 16, 5, dtype, 0)
    A.sparse_kv_write(cache, dev(k, dtype), dev(v, dtype), torch.arange(n, device=DEV))
    desc = A.make_attn_desc(1, 1, d, plan.desc.dtype)
    lengths = torch.tensor([1, 2, 3, 6, 70, 0], dtype=torch.int32, device=DEV)
    table = torch.arange(5, dtype=torch.int32, device=DEV).repeat(6, 1)
    ws = torch.empty(A.sparse_attn_decode_workspace_bytes(desc, cache.desc, 6, 5), dtype=torch.uint8, device=DEV)
    token = nans(6, 1, d, dtype=dtype)
    A.sparse_attn_decode(desc, cache, dev(q[:6], dtype), table, lengths, token, ws)
    want = torch.stack([want[i - 1] if i else torch.zeros_like(want[0]) for i in lengths.tolist()])
    inside(token, want, step * want.abs(), "token")
