"""Attention operators at the limits of their numbers: scores that leave a float's range, small weights beside a large one, values of very different
sizes in 8 bits, rows that are not finite; and the kernels of few and of many rows and of long sequences at the same tests."""
import math

import pytest
import torch

import attention_oracle as O
from paper_2309_06626_amd import attention as A
from test_gpu_attention import DEV, cache_of, case_inputs, decode_call, decode_oracle, dev, gen, inside, nans, normal, packed_call, packed_check, same, starts_of

pytestmark = pytest.mark.gpu


def train(desc, dtype, starts, x):
    """One training step of whole sequences: o, lse, dq, dk, dv."""
    plan = A.sparse_attn_plan(desc, starts)
    on = {n: dev(t, dtype) for n, t in x.items()}
    got = {"o": torch.empty_like(on["q"]), "lse": nans(plan.kept, desc.heads)}
    got.update({"d" + n: torch.full_like(on[n], float("nan")) for n in "qkv"})
    ws = torch.empty(A.sparse_attn_backward_workspace_bytes(plan), dtype=torch.uint8, device=DEV)
    A.sparse_attn_run(plan, on["q"], on["k"], on["v"], got["o"], got["lse"])
    A.sparse_attn_backward(plan, on["q"], on["k"], on["v"], got["o"], got["lse"], on["do"], got["dq"], got["dk"], got["dv"], ws)
    return got


# ---- scores beyond a float's range -------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("times", [1, 80])
@pytest.mark.parametrize("d", [64, 72, 128])
def test_gradients_of_rows_whose_scores_are_minus_infinity(dtype, times, d):
    """The first rows' products with all keys that they see leave a float's range: o is 0, and so are dq and what they add to dk and dv.  Other rows see
    these keys as any other.  (The oracle takes a row's contributions away with its gradient.)"""
    c = ([70, 33], 4, 2, d, dtype, True, 0, 1.0, 0, 0)
    starts, rows, keep, x = case_inputs(c, 41)
    lost = torch.tensor([0, 1, 2, 70, 71])
    x["q"][..., 0] = x["k"][..., 0] = 0
    x["q"][lost, :, 0], x["k"][lost, :, 0] = 2.0 ** 100, -(2.0 ** 100)
    without = x["do"].clone()
    without[lost] = 0
    want, bound = O.packed((4, 2, d, dtype, True, 0, 1 / math.sqrt(d)), starts, keep, x["q"], x["k"], x["v"], without)
    again = lambda t: torch.cat([t] * times)  # noqa: E731
    got = train(A.make_attn_desc(4, 2, d, A.DTYPE_CODE[dtype]), dtype, starts_of([70, 33] * times), {n: again(t) for n, t in x.items()})
    kept = torch.ones(rows, dtype=torch.bool).index_fill(0, lost, False).repeat(times)
    for n in ("o", "dq", "dk", "dv"):
        mine = kept if n in ("o", "dq") else torch.ones_like(kept)
        inside(got[n][mine.to(DEV)], again(want[n])[mine], again(bound[n])[mine], n)
    for n in ("o", "dq"):
        assert (got[n][~kept.to(DEV)] == 0).all(), n
    assert (got["lse"][~kept.to(DEV)] == -math.inf).all()


@pytest.mark.parametrize("times", [1, 400])
def test_gradients_of_rows_whose_scores_are_minus_infinity_in_f16(times):
    """The same by the scale; rows see themselves alone, so that nothing else is multiplied by it."""
    n, d = 70, 64
    g = gen(7)
    x = {name: torch.zeros(n, 1, d, dtype=torch.float64) for name in "qk"}
    x["v"], x["do"] = normal(g, n, 1, d, dtype="f16"), normal(g, n, 1, d, dtype="f16")
    lost = torch.tensor([0, 5, 31, 32, 69])
    x["q"][lost, 0, 0], x["k"][lost, 0, 0] = 2.0 ** 15, -(2.0 ** 15)
    x = {name: torch.cat([t] * times) for name, t in x.items()}
    got = train(A.make_attn_desc(1, 1, d, A.SC_F16, window=1, scale=2.0 ** 100), "f16", starts_of([n] * times), x)
    some = torch.ones(n).index_fill(0, lost, 0).repeat(times)[:, None, None].double()
    assert torch.equal(got["o"].double().cpu(), x["v"] * some) and torch.equal(got["dv"].double().cpu(), x["do"] * some)
    assert (got["dq"] == 0).all() and (got["dk"] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,times", [(70, 1), (70, 600), (2100, 1)])
def test_a_score_beyond_a_floats_range_is_not_an_empty_row(dtype, n, times):
    """A score that is +infinity once it is scaled makes its row NaN, and no other; it is not a row without weights."""
    d = 64
    x = {name: torch.zeros(n, 2, d, dtype=torch.float64) for name in "qk"}
    v = (torch.arange(n) % 7).double().reshape(n, 1, 1).expand(n, 2, d)
    lost = torch.tensor([3, 64])
    x["q"][lost, 0, 0], x["k"][5, :, 0] = 2.0 ** 15, 2.0 ** 15
    desc = A.make_attn_desc(2, 2, d, A.DTYPE_CODE[dtype], causal=False, scale=2.0 ** 100)
    plan = A.sparse_attn_plan(desc, starts_of([n] * times))
    q, k, w = (dev(t.repeat(times, 1, 1), dtype) for t in (x["q"], x["k"], v))
    o, lse = torch.zeros_like(q), torch.zeros(plan.kept, 2, device=DEV)
    A.sparse_attn_run(plan, q, k, w, o, lse)
    ok = torch.ones(n, 2, dtype=torch.bool)
    ok[lost, 0] = False
    ok = ok.repeat(times, 1).to(DEV)
    mean = v[:, 0].mean(0)
    # weights are 1: the sums are exact, the quotient's three roundings are floats', the result's the type's
    step = torch.finfo(O.TORCH[dtype]).eps / 2 + 4 * O.E
    inside(o[ok], mean.expand(int(ok.sum()), d), step * mean.expand(int(ok.sum()), d), "o")
    inside(lse[ok], torch.full((int(ok.sum()),), math.log(n), dtype=torch.float64), torch.full((int(ok.sum()),), 8 * O.E * (1 + math.log(n))), "lse")
    assert torch.isnan(o[~ok]).all() and torch.isnan(lse[~ok]).all()


@pytest.mark.parametrize("dtype,bits", [("bf16", 0), ("f16", 0), ("f32", 0), ("bf16", 8), ("f16", 8), ("f32", 8)])
@pytest.mark.parametrize("n,requests", [(1, 3), (300, 2), (3000, 2), (300, 900)])
def test_a_tokens_score_beyond_a_floats_range_is_not_an_empty_row(dtype, bits, n, requests):
    """The same of single tokens, whose shares of wavefronts and stretches are joined; with 900 requests there is one stretch."""
    d = 64
    cache = cache_of(1, d, 16, -(-n // 16), dtype, bits)
    k = torch.zeros(n, 1, d, dtype=torch.float64)
    k[n // 2, 0, 0] = 2.0 ** 15
    v = (torch.arange(n) % 7 + 1.0).reshape(n, 1, 1).expand(n, 1, d)
    A.sparse_kv_write(cache, dev(k, dtype), dev(v, dtype), torch.arange(n, device=DEV))
    q = torch.zeros(requests, 2, d)
    q[1::2, 0, 0] = 2.0 ** 15
    desc = A.make_attn_desc(2, 1, d, A.DTYPE_CODE[dtype], scale=2.0 ** 100)
    table = torch.arange(-(-n // 16), dtype=torch.int32, device=DEV).repeat(requests, 1)
    ws = torch.empty(A.sparse_attn_decode_workspace_bytes(desc, cache.desc, requests, table.shape[1]), dtype=torch.uint8, device=DEV)
    o = torch.zeros(requests, 2, d, dtype=O.TORCH[dtype], device=DEV)
    A.sparse_attn_decode(desc, cache, dev(q, dtype), table, torch.full((requests,), n, dtype=torch.int32, device=DEV), o, ws)
    assert torch.isnan(o[1::2, 0]).all()
    held = v[:, 0, 0].double()
    if bits:
        codes, scale = O.quantised(v[:, 0].double())
        held = codes[:, 0] * scale.double()
    # weights are 1; in 8 bits they are products with a scale, rounded to the type
    step = torch.finfo(O.TORCH[dtype]).eps / 2 + (O.U["f16" if dtype == "bf16" else dtype] if bits else 0) + O.acc(n)
    for got in (o[::2, 0], o[:, 1]):
        inside(got, held.mean().expand(got.shape), step * held.mean().expand(got.shape), "o")


# ---- small weights beside a large one ----------------------------------------------------------------------------------

SCORE = 17.359375      # beside it, a score of 0 has 2^-25.04 of the weight: below half of f16's smallest number


def one_large_weight(n, d=64):
    x = {"q": torch.zeros(n, 1, d), "k": torch.zeros(n, 1, d), "v": torch.ones(n, 1, d), "do": torch.full((n, 1, d), 2.0 ** -4)}
    x["q"][:, 0, 0], x["k"][0, 0, 0] = 1, SCORE
    return train(A.make_attn_desc(1, 1, d, A.SC_F16, causal=False, scale=1.0), "f16", [0, n], x)


@pytest.mark.parametrize("n", [65536, 100000])
def test_many_small_weights_beside_a_large_one_in_f16(n):
    """One key has most of the weight, the others the rest, 0.3 % of it: o is 1 as all values are."""
    got = one_large_weight(n)
    # The result's rounding; weights below f16's normal numbers, half of 2^-24 in units of 2^-6; the numerator is n / 16 additions to a float and the sum
    # n / 32 to another, half a step each
    off = O.U["f16"] + n * 2.0 ** -31 + (n / 16 + n / 32) * O.E
    inside(got["o"], torch.ones(n, 1, 64, dtype=torch.float64), torch.full((n, 1, 64), off), "o")
    lse = torch.full((n, 1), SCORE + math.log1p((n - 1) * math.exp(-SCORE)), dtype=torch.float64)
    inside(got["lse"], lse, 8 * O.E * (1 + lse) + n / 32 * O.E, "lse")


def test_many_small_weights_beside_a_large_one_in_f16_of_single_tokens():
    """The same of 800 000 rows of a cache, whose wavefronts have one large weight each."""
    n, d, page, requests = 800000, 64, 4096, 768
    cache = cache_of(1, d, page, -(-n // page), "f16", 0)
    k, v = torch.zeros(n, 1, d, dtype=torch.float16, device=DEV), torch.ones(n, 1, d, dtype=torch.float16, device=DEV)
    k[torch.tensor([0, 32, 64, 96], device=DEV), 0, 0] = SCORE
    A.sparse_kv_write(cache, k, v, torch.arange(n, device=DEV))
    q = torch.zeros(requests, 1, d, dtype=torch.float16, device=DEV)
    q[:, 0, 0] = 1
    desc = A.make_attn_desc(1, 1, d, A.SC_F16, scale=1.0)
    table = torch.arange(-(-n // page), dtype=torch.int32, device=DEV).repeat(requests, 1)
    ws = torch.empty(A.sparse_attn_decode_workspace_bytes(desc, cache.desc, requests, table.shape[1]), dtype=torch.uint8, device=DEV)
    o = nans(requests, 1, d, dtype="f16")
    A.sparse_attn_decode(desc, cache, q, table, torch.full((requests,), n, dtype=torch.int32, device=DEV), o, ws)
    # as above; a wavefront adds up a quarter of the rows
    off = O.U["f16"] + n / 4 * 2.0 ** -31 + (n / 64 + n / 128) * O.E
    inside(o, torch.ones(requests, 1, d, dtype=torch.float64), torch.full((requests, 1, d), off), "o")


@pytest.mark.parametrize("n", [65536, 100000])
def test_many_small_probabilities_of_a_key_in_f16(n):
    """The gradients of the other values: many rows' probabilities of 2^-25.  65 536 rows go by the small tiles of the gradients, 100 000 by the large ones."""
    got = one_large_weight(n)["dv"][1:]
    small = math.exp(-SCORE)
    dv = torch.full(got.shape, n * small / (1 + (n - 1) * small) * 2.0 ** -4, dtype=torch.float64)
    # a probability's and the result's rounding; what makes a probability: lse and the score, twice each, and lse's sum; n / 16 additions of n equal terms
    inside(got, dv, dv * (2 * O.U["f16"] + 4 * 8 * O.E * (1 + SCORE) + (n / 32 + n / 16) * O.E), "dv")


# ---- values of very different sizes in 8 bits --------------------------------------------------------------------------


@pytest.mark.parametrize("dtype,small", [("bf16", 1e-4), ("bf16", 1e-5), ("bf16", 1e-30), ("f16", 1e-3), ("f16", 1e-4), ("f32", 1e-5)])
@pytest.mark.parametrize("requests", [1, 400])
@pytest.mark.parametrize("large", [(0, 1), (150, 151), (290, 291), (0, 128), (100, 164)])
def test_8_bit_values_beside_larger_ones_that_have_no_weight(dtype, small, large, requests, monkeypatch):
    """Rows of large values that the token hardly sees take no digits from those that it sees.  Of 400 tokens one stretch is made, whose wavefronts have three
    tiles each, a first one of large values alone among them."""
    monkeypatch.setitem(O.SUB, "f16", 0.0)      # (weights keep their digits: the loss that is left is in the bound below)
    n, d = 300, 64
    c = ([n], 8, 2, d, 16, dtype, 8, 0, 0)
    g = gen(12)
    cache = cache_of(2, d, 16, 21, dtype, 8)
    table, j = torch.arange(20, dtype=torch.int32)[None], torch.arange(n)
    k, v = normal(g, n, 2, d, dtype=dtype), (normal(g, n, 2, d) * small).to(O.TORCH[dtype]).double()
    k[..., 0] = 0
    k[slice(*large), :, 0] = -60
    v[slice(*large)] = normal(g, large[1] - large[0], 2, d, dtype=dtype) * 1024
    A.sparse_kv_write(cache, dev(k, dtype), dev(v, dtype), j.to(DEV))
    (k, _), (v, scales) = ((codes * scale.double()[..., None], scale.double()) for codes, scale in map(O.quantised, (k, v)))
    q = normal(g, 1, 8, d, dtype=dtype)
    q[..., 0] = 16      # scores of -120 and less
    got = decode_call(c, cache, table.repeat(requests, 1), [n] * requests, q.repeat(requests, 1, 1))
    want, bound = decode_oracle(c, q, [k], [v])
    # f16's half steps below its normal numbers, 2^-25, in units of 2^-6 of the largest weight and scale, times codes up to 127
    for h in range(8):
        p = O.attend(q[0, h][None], k[:, h // 4], v[:, h // 4], 1 / 8, torch.ones(1, n, dtype=torch.bool))[2][0]
        bound[0, h] += n * 2.0 ** -31 * 127 * (p * scales[:, h // 4]).max()
    inside(got[:1], want, bound, "o")
    assert same(got, got[:1].expand_as(got))


# ---- rows that are not finite ------------------------------------------------------------------------------------------


@pytest.mark.parametrize("which", ["q", "do"])
@pytest.mark.parametrize("dtype,times", [("bf16", 1), ("bf16", 40), ("f32", 1), ("f32", 40)])
def test_a_row_that_is_not_finite_loses_its_keys_gradients(which, dtype, times):
    """A NaN row of q or of do loses its own o (q) and dq, and dk and dv of its sequence's key-value head; all else keeps its bits."""
    c = ([90, 61, 40] * times, 4, 2, 64, dtype, True, 0, 1.0, 0, 0)
    starts, rows, keep, x = case_inputs(c, 8)
    _, _, clean = packed_call(c, starts, keep, x)
    x[which][40, 1] = float("nan")                       # key-value head 0
    _, _, got = packed_call(c, starts, keep, x)
    own = torch.zeros(rows, 4, dtype=torch.bool, device=DEV)
    own[40, 1] = True
    for n in ("o", "lse", "dq"):
        mine = own if n == "dq" or which == "q" else torch.zeros_like(own)
        assert same(clean[n][~mine], got[n][~mine]) and torch.isnan(got[n][mine]).all(), n
    for n in ("dk", "dv"):
        assert same(clean[n][90:], got[n][90:]) and same(clean[n][:90, 1], got[n][:90, 1]), n
        assert torch.isnan(got[n][:41, 0]).all(), n


# ---- every kernel, below and above the limits of the small tiles ---------------------------------------------------------

LONG = [  # tiles that see 2 048 keys or more on average
    ([2100], 2, 1, 64, "bf16", False, 0, 1.0, 0, 0),
    ([2100], 2, 2, 128, "f16", False, 0, 1.0, 0, 3),
    ([2600, 40, 0, 300], 2, 1, 128, "bf16", False, 0, 1.0, 0, 0),
    ([2400], 3, 1, 64, "f16", False, 0, 0.9, 0, 1),
    ([2500, 70], 2, 1, 128, "bf16", False, 0, 0.9, 1, 2),
    ([4500], 2, 1, 64, "bf16", True, 0, 1.0, 0, 0),
    ([3100], 1, 1, 128, "f16", False, 2200, 1.0, 0, 0),
    ([2200], 2, 1, 40, "f16", False, 0, 1.0, 0, 0),
    ([2200], 2, 1, 66, "bf16", False, 0, 1.0, 0, 0),
    ([2111], 3, 1, 41, "bf16", False, 0, 0.98, 0, 0),
    ([2111], 1, 1, 127, "f16", False, 0, 1.0, 0, 0),
]


@pytest.mark.parametrize("c", LONG, ids=lambda c: "-".join(map(str, [sum(c[0]), len(c[0]), *c[1:]])))
def test_tiles_that_see_many_keys(c):
    packed_check(c, 3 * sum(c[0]) + c[3])


@pytest.mark.parametrize("pad", [1, 2, 8])
@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "f16")])
def test_tiles_that_see_many_keys_of_rows_with_gaps(d, dtype, pad):
    packed_check(([2100], 2, 1, d, dtype, False, 0, 1.0, 0, 0), 5, pad)


def many(c):
    """How often the sequences have to come for more than 2 048 tiles of 32."""
    return 2049 // (sum(-(-n * c[1] // c[2] // 32) for n in c[0]) * c[2]) + 1


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 95, 96, 127, 128, 129, 191, 192, 193, 255, 256, 257])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_end_of_a_tile_of_many(n, dtype):
    c = ([n, n], 2, 1, 64, dtype, n % 2 == 0, 0, 1.0, 0, 0)
    packed_check(c, n, times=many(c))


@pytest.mark.parametrize("window", [1, 2, 31, 32, 33, 64, 65, 200, 1 << 30])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_windows_of_many(window, causal, dtype):
    c = ([150], 3, 1, 64, dtype, causal, window, 1.0, 0, 0)
    packed_check(c, window % 97, times=many(c))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n,heads,kv,d,causal", [(300, 4, 4, 64, True), (300, 8, 2, 128, True), (190, 4, 4, 40, True), (190, 6, 2, 41, True), (2100, 1, 1, 128, False)])
@pytest.mark.parametrize("of_many", [False, True])
def test_results_are_as_near_as_their_operands_allow_of_few_and_many(dtype, n, heads, kv, d, causal, of_many):
    """Probabilities and gradients of scores are rounded once, as operands of products, and results once more, whichever tiles form them.  dq's scores have
    a delta from o as it is stored; dk's have not: with that delta dk would be off by as much more as dq is."""
    c = ([n], heads, kv, d, dtype, causal, 0, 1.0, 0, 0)
    times = many(c) if of_many else 1
    starts, rows, keep, x = case_inputs(c, 23)
    _, _, got = packed_call(([n] * times, *c[1:]), starts_of([n] * times), keep.repeat(times), {name: t.repeat(times, 1, 1) for name, t in x.items()})
    want, _ = O.packed((heads, kv, d, dtype, causal, 0, 1 / math.sqrt(d)), starts, keep, x["q"], x["k"], x["v"], x["do"])
    once = lambda v: v.to(O.TORCH[dtype]).double()  # noqa: E731
    near = {name: torch.zeros_like(want[name]) for name in ("o", "dq", "dk", "dv")}
    visible = O.seen(n, causal, 0)
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
        ideal = (once(near[name]) - want[name]).norm()
        off = (got[name].double().cpu().view(times, *want[name].shape) - want[name]).flatten(1).norm(dim=1)
        assert (off <= 1.1 * ideal).all(), f"{name}: {(off.max() / ideal):.3f}"


def test_training_steps_of_many_rows_at_once():
    """One plan on two streams, more than 2 048 tiles of 32: the gradients' large tiles, too, keep to their own workspaces."""
    c = ([900, 30, 1100] * 5, 8, 2, 128, "bf16", True, 0, 1.0, 0, 0)
    starts, rows, keep, x = case_inputs(c, 6)
    plan = A.sparse_attn_plan(A.make_attn_desc(8, 2, 128), starts)
    sets = [{n: dev(t if s == 0 else t.flip(0), "bf16") for n, t in x.items()} for s in range(2)]

    def buffers():
        b = {"o": nans(rows, 8, 128, dtype="bf16"), "lse": nans(rows, 8), "dq": nans(rows, 8, 128, dtype="bf16"), "dk": nans(rows, 2, 128, dtype="bf16"),
             "dv": nans(rows, 2, 128, dtype="bf16")}
        return b, torch.empty(A.sparse_attn_backward_workspace_bytes(plan), dtype=torch.uint8, device=DEV)

    def go(s, b, ws, stream=None):
        A.sparse_attn_run(plan, s["q"], s["k"], s["v"], b["o"], b["lse"], stream=stream)
        A.sparse_attn_backward(plan, s["q"], s["k"], s["v"], b["o"], b["lse"], s["do"], b["dq"], b["dk"], b["dv"], ws, stream=stream)

    want, got = [buffers(), buffers()], [buffers(), buffers()]
    for s, (b, ws) in zip(sets, want):
        go(s, b, ws)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, (b, ws), stream in zip(sets, got, streams):
            go(s, b, ws, stream)
    torch.cuda.synchronize()
    for (a, _), (b, _) in zip(want, got):
        assert all(same(a[n], b[n]) for n in a)
