"""Block operators against the 64-bit oracle: types, odd sizes, masks from nothing to everything, gradients also against differences."""
import math

import pytest
import torch

import block_oracle as O
from paper_2309_06626_amd import binding as B
from paper_2309_06626_amd import block as K

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def gen(seed):
    return torch.Generator().manual_seed(seed)


def normal(g, *shape, dtype="f32", std=1.0, mean=0.0):
    """On the host, rounded to the type and widened to float64."""
    return (torch.randn(*shape, generator=g) * std + mean).to(O.TORCH[dtype]).double()


def dev(t, dtype="f32"):
    return None if t is None else t.to(O.TORCH[dtype]).to(DEV)


def nan_like(*shape, dtype="f32"):
    return torch.full(shape, float("nan"), dtype=O.TORCH[dtype], device=DEV)


def inside(got, want, bound, what):
    got = got.double().cpu()
    assert got.shape == want.shape, what
    assert torch.isfinite(got).all(), what
    over = ((got - want).abs() / bound).max().item() if got.numel() else 0.0
    assert over <= 1.0, f"{what}: {over:.3g} times the bound"


def mask_of(kind, rows, g):
    m = torch.ones(rows, dtype=torch.uint8)
    if kind == "half":
        m[torch.randperm(rows, generator=g)[: rows // 2]] = 0
    elif kind == "nothing":
        m.zero_()
    elif kind == "ends":
        m[1:-1] = 0
    elif kind == "block":
        m[rows // 4: rows // 4 + rows // 2] = 0
    return m


# ---- row sets ----------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("rows", [0, 1, 63, 64, 4095, 4096, 4097, 70001])
@pytest.mark.parametrize("kind", ["half", "nothing", "all", "ends"])
def test_row_lists(rows, kind):
    g = gen(rows)
    mask = mask_of(kind, rows, g) * 5      # any byte but 0 keeps
    rs = K.sparse_rows_plan(mask.to(DEV))
    for m in (mask, mask_of("half", rows, g)):
        K.sparse_rows_set_mask(rs, m.to(DEV))
        want = m.nonzero()[:, 0]
        got = K.sparse_rows_info(rs)
        assert got[0] == rows and got[1] == rs.kept == len(want)
        assert torch.equal(got[2].cpu().long(), want)
        slot = torch.full((rows,), -1, dtype=torch.int64)
        slot[want] = torch.arange(len(want))
        assert torch.equal(got[3].cpu().long(), slot)


# ---- norms -------------------------------------------------------------------------------------------------------------

NORMS = [  # rows, d, dtype, post, pre, rows_per_gate (None: no gate), masks of f and h, a, b
    (1, 1, "f32", "rms", "rms", None, "all", "all", 1.0, 1.0),
    (1, 2048, "bf16", "rms", "rms", None, "all", "all", 1.0, 1.0),
    (3, 7, "bf16", "layer", "layer", 2, "all", "all", 1.0, 1.0),
    (70, 64, "f16", "layer", "rms", 9, "half", "half", 0.5, 2.0),
    (33, 410, "f32", "layer", "layer", 0, "half", "block", 1.0, 1.0),
    (1100, 513, "bf16", "rms", "layer", 196, "block", "half", 1.0, 1.0),
    (600, 1000, "f16", "none", "layer", 1, "half", "half", 1.0, -1.0),
    (40, 1028, "f32", "rms", "none", 7, "nothing", "half", 1.0, 1.0),
    (40, 2056, "bf16", "rms", "rms", 5, "half", "nothing", 0.7, 1.0),
    (1030, 96, "bf16", "layer", "rms", 600, "ends", "ends", 1.0, 1.0),
    (21, 4099, "bf16", "layer", "layer", 4, "half", "half", 1.0, 1.0),
    (530, 4100, "f32", "rms", "layer", 530, "half", "half", 1.0, 1.0),
    (13, 8191, "f16", "layer", "rms", 3, "half", "all", 1.0, 1.0),
    (520, 8192, "bf16", "rms", "rms", 2, "all", "half", 1.0, 1.0),
]


def norm_inputs(rows, d, dtype, post, pre, per, f_mask, h_mask, seed):
    g = gen(seed)
    fm, hm = mask_of(f_mask, rows, g), mask_of(h_mask, rows, g)
    t = dict(x=normal(g, rows, d, dtype=dtype), f=normal(g, int(fm.sum()), d, dtype=dtype, std=0.5, mean=0.2))
    t["gate"] = None if per is None else normal(g, -(-rows // (per or rows)), d, dtype=dtype, std=0.5, mean=0.5)
    t["w_post"], t["w_pre"] = normal(g, d, std=0.1, mean=1.0), normal(g, d, std=0.1, mean=1.0)
    t["b_post"] = normal(g, d, std=0.1) if post == "layer" else None
    t["b_pre"] = normal(g, d, std=0.1) if pre == "layer" else None
    return g, t, fm, hm


def norm_call(c, t, fm, hm, **over):
    rows, d, dtype, post, pre, per, _, _, a, b = c
    desc = K.make_norm_desc(d, K.DTYPE_CODE[dtype], K.NORM_CODE[post], K.NORM_CODE[pre], 1e-5, a, b, per or 0)
    dt = {n: dev(v, dtype if n in ("x", "f", "gate") else "f32") for n, v in t.items()}
    fr = None if fm.all() else K.sparse_rows_plan(fm.to(DEV))
    hr = None if hm.all() else K.sparse_rows_plan(hm.to(DEV))
    out = dict(x_new=nan_like(rows, d, dtype=dtype), h=nan_like(int(hm.sum()), d, dtype=dtype), stats=nan_like(rows, 4))
    K.sparse_norm_run(desc, *[dt[n] for n in ("x", "f", "gate", "w_post", "b_post", "w_pre", "b_pre")], out["x_new"], out["h"],
                      f_rows=fr, h_rows=hr, stats=out["stats"])
    return desc, dt, fr, hr, out


def norm_oracle(c, t, fm, hm):
    rows, d, dtype, post, pre, per, _, _, a, b = c
    return O.norm_forward(t["x"], t["f"], t["gate"], t["w_post"], t["b_post"], t["w_pre"], t["b_pre"], post, pre, 1e-5, a, b,
                          per or max(rows, 1), fm.bool(), hm.bool())


def rowwise(want, d, u):
    """A normalised row's float error is a few units of its largest terms, the sums over d included."""
    return u * want.abs() + O.acc(d) * (want.abs().amax(-1, keepdim=True) + 1) * 4 + 1e-37


@pytest.mark.parametrize("c", NORMS, ids=lambda c: "-".join(map(str, c[:8])))
def test_norm_forward_and_gradients(c):
    rows, d, dtype, post, pre, per, f_mask, h_mask, a, b = c
    g, t, fm, hm = norm_inputs(rows, d, dtype, post, pre, per, f_mask, h_mask, 11 * rows + d)
    desc, dt, fr, hr, out = norm_call(c, t, fm, hm)
    x_new, h = norm_oracle(c, t, fm, hm)
    u = O.U[dtype] + (2.0 ** -24 if dtype == "f16" else 0)
    inside(out["x_new"], x_new, rowwise(x_new, d, u) + O.TINY[dtype], "x_new")
    inside(out["h"], h, rowwise(h, d, u) + O.TINY[dtype], "h")

    dx_new, dh = normal(g, rows, d, dtype=dtype), normal(g, int(hm.sum()), d, dtype=dtype)
    names = [n for n in ("x", "f", "gate", "w_post", "b_post", "w_pre", "b_pre") if t[n] is not None]
    leaves = {n: (t[n].clone().requires_grad_(True) if n in names else None) for n in t}
    want = torch.autograd.grad(norm_oracle(c, leaves, fm, hm), [leaves[n] for n in names], [dx_new, dh], allow_unused=True)
    want = {n: torch.zeros_like(t[n]) if w is None else w for n, w in zip(names, want)}
    got = {n: torch.full_like(dt[n], float("nan")) for n in names}
    ws = torch.empty(K.sparse_norm_workspace_bytes(desc, rows), dtype=torch.uint8, device=DEV)
    args = [dt[n] for n in ("x", "f", "gate", "w_post", "b_post", "w_pre")] + [out["stats"], dev(dx_new, dtype), dev(dh, dtype)]
    grads = lambda into: [into.get(n) for n in ("x", "f", "gate", "w_post", "b_post", "w_pre", "b_pre")]  # noqa: E731
    K.sparse_norm_backward(desc, *args, *grads(got), ws, f_rows=fr, h_rows=hr)
    # magnitudes that enter: gradients of a row scale with 1 / spread
    spread = lambda v, kind: 1.0 if kind == "none" or not v.numel() else float(  # noqa: E731
        (1 / torch.sqrt(((v - (v.mean(-1, keepdim=True) if kind == "layer" else 0)) ** 2).mean(-1) + 1e-5)).max())
    big = (1 + abs(a) + abs(b)) * (1 + spread(x_new, pre)) * (1 + spread(t["f"], post)) * 8
    for n in names:
        w = want[n]
        terms = rows if n.startswith(("w_", "b_")) else (per or rows) if n == "gate" else 1
        scale = (w.abs().amax() if w.numel() else 0.0) + 1 + math.sqrt(terms)
        uu = u if n in ("x", "f", "gate") else O.E
        inside(got[n], w, uu * w.abs() + O.acc(d) * big * scale + O.TINY[dtype], "d" + n)
    # the same bits again, into other buffers, with only some of the gradients wanted
    again = {n: torch.full_like(dt[n], float("nan")) for n in names}
    K.sparse_norm_backward(desc, *args, *grads(again), ws, f_rows=fr, h_rows=hr)
    assert all(torch.equal(got[n].view(torch.uint8), again[n].view(torch.uint8)) for n in names)
    some = {"x": torch.full_like(dt["x"], float("nan"))}
    K.sparse_norm_backward(desc, *args, *grads(some), ws, f_rows=fr, h_rows=hr)
    assert torch.equal(some["x"], got["x"])


def test_norm_before_a_block_alone_and_in_place():
    c = (50, 200, "bf16", "rms", "rms", None, "all", "all", 1.0, 1.0)
    g, t, fm, hm = norm_inputs(*c[:8], 5)
    desc = K.make_norm_desc(200, B.SC_BF16)
    x, h = dev(t["x"], "bf16"), nan_like(50, 200, dtype="bf16")
    K.sparse_norm_run(desc, x, None, None, None, None, dev(t["w_pre"]), None, None, h)
    want = O.normed(t["x"], "rms", 1e-6) * t["w_pre"]
    inside(h, want, rowwise(want, 200, O.U["bf16"]), "h")
    _, dt, _, _, out = norm_call(c, t, fm, hm)
    K.sparse_norm_run(K.make_norm_desc(200, B.SC_BF16, eps=1e-5), dt["x"], dt["f"], None, dt["w_post"], None, dt["w_pre"], None,
                      dt["x"], h)
    assert torch.equal(dt["x"], out["x_new"]) and torch.equal(h, out["h"])


def test_norm_gradient_against_differences():
    c = (6, 20, "f32", "layer", "rms", 4, "half", "all", 0.5, 2.0)
    g, t, fm, hm = norm_inputs(*c[:8], 3)
    desc, dt, fr, hr, out = norm_call(c, t, fm, hm)
    dx_new, dh = normal(g, 6, 20), normal(g, 6, 20)
    got = {n: torch.empty_like(v) for n, v in dt.items() if v is not None}
    ws = torch.empty(K.sparse_norm_workspace_bytes(desc, 6), dtype=torch.uint8, device=DEV)
    K.sparse_norm_backward(desc, *[dt[n] for n in ("x", "f", "gate", "w_post", "b_post", "w_pre")], out["stats"], dev(dx_new), dev(dh),
                           *[got.get(n) for n in ("x", "f", "gate", "w_post", "b_post", "w_pre", "b_pre")], ws, f_rows=fr, h_rows=hr)

    def loss(v):
        x_new, h = norm_oracle(c, v, fm, hm)
        return float((x_new * dx_new).sum() + (h * dh).sum())

    for n in got:
        way = normal(g, *t[n].shape)
        step = 1e-5
        slope = (loss({**t, n: t[n] + step * way}) - loss({**t, n: t[n] - step * way})) / (2 * step)
        have = float((got[n].double().cpu() * way).sum())
        assert abs(have - slope) <= 1e-5 * (1 + float((got[n].double().cpu() * way).abs().sum())), n


def test_rows_that_the_mask_drops_are_not_looked_at():
    """f and h hold kept rows only; what lies in x's other rows stays in its own row."""
    c = (64, 96, "bf16", "rms", "rms", 8, "half", "half", 1.0, 1.0)
    g, t, fm, hm = norm_inputs(*c[:8], 9)
    _, _, _, _, clean = norm_call(c, t, fm, hm)
    lost = (hm == 0).nonzero()[:, 0]
    t["x"][lost] = float("nan")
    _, _, _, _, out = norm_call(c, t, fm, hm)
    assert torch.equal(out["h"], clean["h"])
    assert torch.equal(out["x_new"][hm.bool().to(DEV)], clean["x_new"][hm.bool().to(DEV)])


@pytest.mark.parametrize("rows,d,per", [(6151, 64, 2), (6151, 64, 3), (6151, 64, 5), (20001, 40, 3), (20001, 40, 9), (20001, 40, 10),
                                        (4100, 1000, 2), (4100, 1000, 3), (1300, 4104, 2), (1300, 4104, 5), (777, 2100, 2)])
def test_norm_gradients_of_thousands_of_gates(rows, d, per):
    # rows of a team: 4, 10, 5, 6 and 4; gates of fewer rows, that the teams' stretches hold whole or not, of as many, and of more
    test_norm_forward_and_gradients((rows, d, "bf16", "layer", "rms", per, "half", "half", 0.5, 2.0))


def test_norm_gradients_of_millions_of_gates():
    """A gate for every two of 33 million rows, some across the borders of the teams' 16 385 rows: whole numbers, so sums are exact."""
    rows, d = (1 << 25) + 7, 8
    desc = K.make_norm_desc(d, B.SC_BF16, K.SC_NORM_NONE, K.SC_NORM_NONE, rows_per_gate=2)
    whole = lambda n: torch.randint(-3, 4, (n, d), device=DEV, generator=torch.Generator(DEV).manual_seed(n)).to(torch.bfloat16)  # noqa: E731
    x, f, dx_new, gate = whole(rows), whole(rows), whole(rows), whole((rows + 1) // 2)
    stats = torch.empty(rows, 4, dtype=torch.float32, device=DEV)
    K.sparse_norm_run(desc, x, f, gate, None, None, None, None, x, None, stats=stats)
    dgate, df = torch.full_like(gate, float("nan")), torch.full_like(f, float("nan"))
    ws = torch.empty(K.sparse_norm_workspace_bytes(desc, rows), dtype=torch.uint8, device=DEV)
    K.sparse_norm_backward(desc, x, f, gate, None, None, None, stats, dx_new, None, None, df, dgate, None, None, None, None, ws)
    terms = dx_new * f
    assert torch.equal(dgate[:-1], terms[:-1].view(-1, 2, d).sum(1)) and torch.equal(dgate[-1], terms[-1])
    assert torch.equal(df, dx_new * gate.repeat_interleave(2, 0)[:rows])


def test_norm_gradients_where_no_row_is_kept_and_none_comes_from_elsewhere():
    """dh is empty, and an empty tensor has no address: gradients are zero, the call is not refused."""
    c = (40, 96, "bf16", "rms", "rms", 7, "nothing", "nothing", 1.0, 1.0)
    g, t, fm, hm = norm_inputs(*c[:8], 4)
    desc, dt, fr, hr, out = norm_call(c, t, fm, hm)
    empty = torch.empty(0, 96, dtype=torch.bfloat16, device=DEV)
    dx, dgate = nan_like(40, 96, dtype="bf16"), nan_like(6, 96, dtype="bf16")
    dw = [nan_like(96) for _ in range(2)]
    ws = torch.empty(K.sparse_norm_workspace_bytes(desc, 40), dtype=torch.uint8, device=DEV)
    for gradient in (empty, None):
        K.sparse_norm_backward(desc, dt["x"], dt["f"], dt["gate"], dt["w_post"], None, dt["w_pre"], out["stats"], None, gradient, dx, empty,
                               dgate, dw[0], None, dw[1], None, ws, f_rows=fr, h_rows=hr)
        for v in (dx, dgate, *dw):
            assert (v == 0).all()
            v.fill_(float("nan"))


# ---- feed-forward block ------------------------------------------------------------------------------------------------

FFNS = [  # rows, d_in, d_hidden, d_out, dtype, activation, mask, x_rows, y_rows
    (1, 1, 1, 1, "f32", "silu", "all", 0, 0),
    (1, 64, 128, 64, "bf16", "silu", "all", 0, 0),
    (2, 200, 88, 72, "f16", "gelu", "all", 0, 0),
    (5, 51, 102, 205, "bf16", "gelu_tanh", "half", 0, 0),
    (16, 256, 520, 256, "bf16", "silu", "all", 0, 0),
    (17, 264, 136, 8, "f16", "silu", "half", 1, 0),
    (33, 65, 129, 63, "f32", "gelu", "half", 0, 1),
    (64, 512, 96, 512, "bf16", "gelu", "ends", 0, 0),
    (100, 128, 256, 128, "f32", "silu", "half", 0, 0),
    (130, 96, 160, 224, "f16", "gelu_tanh", "block", 1, 1),
    (257, 264, 392, 264, "bf16", "silu", "half", 0, 0),
    (300, 320, 640, 192, "bf16", "gelu", "nothing", 0, 0),
    (700, 136, 328, 136, "f32", "gelu_tanh", "half", 0, 0),
    (1030, 72, 1160, 2056, "f16", "silu", "half", 0, 0),
    (2000, 410, 300, 410, "bf16", "silu", "block", 0, 0),
]


def ffn_case(c, seed):
    rows, di, dh, do, dtype, kind, mask, x_rows, y_rows = c
    g = gen(seed)
    m = mask_of(mask, rows, g)
    keep = m.bool()
    full = dict(x=normal(g, rows, di, dtype=dtype), wg=normal(g, dh, di, dtype=dtype, std=di ** -0.5),
                wu=normal(g, dh, di, dtype=dtype, std=di ** -0.5), wd=normal(g, do, dh, dtype=dtype, std=dh ** -0.5),
                dy=normal(g, rows, do, dtype=dtype))
    return m, keep, full


def ffn_call(c, m, keep, full, backward=True):
    rows, di, dh, do, dtype, kind, mask, x_rows, y_rows = c
    kept = int(keep.sum())
    rs = None if mask == "all" else K.sparse_rows_plan(m.to(DEV))
    desc = K.make_ffn_desc(di, dh, do, K.DTYPE_CODE[dtype], K.ACT_CODE[kind])
    t = {n: dev(v, dtype) for n, v in full.items()}
    if rs is not None:      # what dropped rows hold must not matter
        t["x"][~keep.to(DEV)] = float("nan")
        t["dy"][~keep.to(DEV)] = float("nan")
    x = t["x"][keep.to(DEV)].contiguous() if x_rows else t["x"]
    dy = t["dy"][keep.to(DEV)].contiguous() if y_rows else t["dy"]
    y, saved = nan_like(kept if y_rows else rows, do, dtype=dtype), nan_like(3, kept, dh, dtype=dtype)
    ws = torch.empty(K.sparse_ffn_workspace_bytes(desc, kept, True), dtype=torch.uint8, device=DEV)
    K.sparse_ffn_run(desc, x, t["wg"], t["wu"], t["wd"], y, ws, rows=rs, x_rows=x_rows, y_rows=y_rows, saved=saved)
    plain = nan_like(*y.shape, dtype=dtype)
    K.sparse_ffn_run(desc, x, t["wg"], t["wu"], t["wd"], plain, ws, rows=rs, x_rows=x_rows, y_rows=y_rows)
    assert torch.equal(plain, y)
    if not backward:
        return y
    grads = [nan_like(*s.shape, dtype=dtype) for s in (x, t["wg"], t["wu"], t["wd"])]
    K.sparse_ffn_backward(desc, x, t["wg"], t["wu"], t["wd"], saved, dy, *grads, ws, rows=rs, x_rows=x_rows, y_rows=y_rows)
    again = [nan_like(*s.shape, dtype=dtype) for s in grads]
    K.sparse_ffn_backward(desc, x, t["wg"], t["wu"], t["wd"], saved, dy, *again, ws, rows=rs, x_rows=x_rows, y_rows=y_rows)
    assert all(torch.equal(p, q) for p, q in zip(grads, again))
    only = nan_like(*x.shape, dtype=dtype)
    K.sparse_ffn_backward(desc, x, t["wg"], t["wu"], t["wd"], saved, dy, only, None, None, None, ws, rows=rs, x_rows=x_rows, y_rows=y_rows)
    assert torch.equal(only, grads[0])
    return [y] + grads


@pytest.mark.parametrize("c", FFNS, ids=lambda c: "-".join(map(str, c)))
def test_ffn_forward_and_gradients(c):
    rows, di, dh, do, dtype, kind, mask, x_rows, y_rows = c
    m, keep, full = ffn_case(c, 7 * rows + dh)
    got = ffn_call(c, m, keep, full)
    x, dy = full["x"][keep], full["dy"][keep]
    leaves = [v.clone().requires_grad_(True) for v in (x, full["wg"], full["wu"], full["wd"])]
    y = O.ffn_forward(*leaves, kind)
    want = [y.detach(), *torch.autograd.grad(y, leaves, dy)]
    bounds = O.ffn_bounds(x, full["wg"], full["wu"], full["wd"], kind, dtype, dy)
    for name, v, w, b in zip(("y", "dx", "dw_gate", "dw_up", "dw_down"), got, want, bounds):
        if name in ("y", "dx") and not (y_rows if name == "y" else x_rows):
            dropped = v[~keep.to(DEV)]
            assert (dropped.view(torch.int32 if dtype == "f32" else torch.int16) == 0).all(), name
            v = v[keep.to(DEV)]
        inside(v, w, b, name)


@pytest.mark.parametrize("c", [(6000, 768, 384, 768, "bf16", "gelu", "all", 0, 0), (8192, 256, 520, 776, "f16", "silu", "half", 1, 0),
                               (9000, 505, 771, 258, "bf16", "gelu_tanh", "half", 0, 1),
                               (8200, 1040, 2072, 1032, "bf16", "gelu", "half", 0, 0), (8200, 1037, 2071, 1030, "f16", "silu", "half", 0, 0),
                               (5200, 1288, 3080, 1544, "f16", "gelu", "half", 0, 1)], ids=lambda c: "-".join(map(str, c)))
def test_ffn_in_larger_tiles(c):
    test_ffn_forward_and_gradients(c)


# Weight gradients of dense rows go through the list of kept rows, 4 096 entries at a time: kept rows beyond a stretch, or three, in one
# piece (gate's and up's of the first, fourth and last, down's of the first) and in parts longer than a stretch (down's of the second, third
# and last, gate's and up's of the third)
@pytest.mark.parametrize("rows,di,dh,do,dtype", [(9200, 1040, 2072, 2056, "bf16"), (26000, 264, 1544, 1032, "f16"),
                                                 (16800, 1032, 1672, 1032, "bf16"), (9000, 1928, 1288, 264, "f32"),
                                                 (26000, 1544, 1800, 1160, "f32")])
def test_ffn_weight_gradients_through_long_row_lists(rows, di, dh, do, dtype):
    """The same sums in the same order as with the kept rows alone in memory; these against products in 64 bits."""
    g, t = torch.Generator(DEV).manual_seed(rows), O.TORCH[dtype]
    draw = lambda *s, std=1.0: (torch.randn(*s, generator=g, device=DEV) * std).to(t)  # noqa: E731
    keep = torch.rand(rows, generator=g, device=DEV) < 0.5
    rs = K.sparse_rows_plan(keep.to(torch.uint8))
    x, dy, w = draw(rows, di), draw(rows, do), [draw(dh, di, std=di ** -0.5), draw(dh, di, std=di ** -0.5), draw(do, dh, std=dh ** -0.5)]
    x[~keep], dy[~keep] = float("nan"), float("nan")
    desc = K.make_ffn_desc(di, dh, do, K.DTYPE_CODE[dtype])
    ws = torch.empty(K.sparse_ffn_workspace_bytes(desc, rs.kept, True), dtype=torch.uint8, device=DEV)
    results = []
    for a, b, fmt in ((x, dy, B.SC_ROWS_DENSE), (x[keep], dy[keep], B.SC_ROWS_COMPACT)):
        y, saved = torch.empty_like(b), torch.empty(3, rs.kept, dh, dtype=t, device=DEV)
        K.sparse_ffn_run(desc, a, *w, y, ws, rows=rs, x_rows=fmt, y_rows=fmt, saved=saved)
        dw = [torch.full_like(v, float("nan")) for v in w]
        K.sparse_ffn_backward(desc, a, *w, saved, b, None, *dw, ws, rows=rs, x_rows=fmt, y_rows=fmt)
        results.append(dw)
    assert all(torch.equal(p, q) for p, q in zip(*results))
    gate, up = (x[keep].double() @ v.double().t().contiguous() for v in w[:2])
    hidden, left = O.act(gate, "silu") * up, dy[keep].double()
    want, size = left.t().contiguous() @ hidden, left.abs().t().contiguous() @ hidden.abs()
    # of hidden: half a unit, and its float sums and activation, which are far below that of 16 bits and 16 acc(d_in) of a float's terms
    rounding = O.U[dtype] if dtype != "f32" else 0.0
    off = rounding * hidden.abs() + 16 * O.acc(di) * (1 + gate.abs()) * (1 + up.abs())
    bound = O.U[dtype] * want.abs() + O.acc(rs.kept) * size + left.abs().t().contiguous() @ off
    inside(results[0][2], want.cpu(), 1.05 * bound.cpu() + O.TINY[dtype], "dw_down")


FEW = [(rows, di, dh, do, dtype, "silu", mask, 0, 0)
       for dtype, di, dh, do in (("bf16", 520, 1037, 264), ("f16", 1048, 264, 5), ("f32", 333, 68, 130), ("f16", 77, 1030, 1031))
       for rows, mask in ((3, "all"), (4, "all"), (8, "half"), (8, "all"), (9, "all"), (15, "half"))]
FEW += [(64, 1024, 5632, 1024, "bf16", "gelu", "all", 0, 0), (70, 2048, 5632, 1024, "f16", "silu", "half", 0, 0),
        (40, 1024, 4096, 2048, "f32", "silu", "half", 0, 0)]


@pytest.mark.parametrize("c", FEW, ids=lambda c: "-".join(map(str, c)))
def test_ffn_of_a_few_rows(c):
    rows, di, dh, do, dtype, kind, mask, _, _ = c
    m, keep, full = ffn_case(c, 11 * rows + di)
    got = ffn_call(c, m, keep, full, backward=False)
    x = full["x"][keep]
    want = O.ffn_forward(x, full["wg"], full["wu"], full["wd"], kind)
    assert (got[~keep.to(DEV)] == 0).all()
    inside(got[keep.to(DEV)], want, O.ffn_bounds(x, full["wg"], full["wu"], full["wd"], kind, dtype), "y")


@pytest.mark.parametrize("size", [2.0 ** -40, 2.0 ** 40])
def test_float_rows_of_any_size(size):
    # parts of 16 bits have a float's range: rows far from 1, weights that bring them back
    c = (150, 96, 72, 80, "f32", "gelu_tanh", "half", 0, 0)
    m, keep, full = ffn_case(c, 31)
    full["x"], full["wg"], full["wu"] = full["x"] * size, full["wg"] / size, full["wu"] / size
    got = ffn_call(c, m, keep, full)
    x, dy = full["x"][keep], full["dy"][keep]
    leaves = [v.clone().requires_grad_(True) for v in (x, full["wg"], full["wu"], full["wd"])]
    y = O.ffn_forward(*leaves, "gelu_tanh")
    want = [y.detach(), *torch.autograd.grad(y, leaves, dy)]
    bounds = O.ffn_bounds(x, full["wg"], full["wu"], full["wd"], "gelu_tanh", "f32", dy)
    for name, v, w, b in zip(("y", "dx", "dw_gate", "dw_up", "dw_down"), got, want, bounds):
        inside(v[keep.to(DEV)] if name in ("y", "dx") else v, w, b, name)


@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh"])
def test_ffn_gradient_against_differences(kind):
    c = (9, 12, 20, 8, "f32", kind, "half", 0, 0)
    m, keep, full = ffn_case(c, 21)
    got = ffn_call(c, m, keep, full)
    g = gen(4)

    def loss(v):
        return float((O.ffn_forward(v["x"][keep], v["wg"], v["wu"], v["wd"], kind) * full["dy"][keep]).sum())

    for n, have in zip(("x", "wg", "wu", "wd"), got[1:]):
        way, step = normal(g, *full[n].shape), 1e-5
        slope = (loss({**full, n: full[n] + step * way}) - loss({**full, n: full[n] - step * way})) / (2 * step)
        terms = have.double().cpu() * way
        assert abs(float(terms.sum()) - slope) <= 1e-5 * (1 + float(terms.abs().sum())), n


def test_ffn_far_out_activations():
    """Products of +-100: the activations saturate, nothing overflows."""
    full = dict(x=torch.tensor([[100.0] * 8, [-100.0] * 8]).double(), wg=torch.eye(8).double(), wu=torch.ones(8, 8).double() / 8,
                wd=torch.eye(8).double(), dy=torch.ones(2, 8).double())
    for kind in ("silu", "gelu", "gelu_tanh"):
        c = (2, 8, 8, 8, "f32", kind, "all", 0, 0)
        got = ffn_call(c, torch.ones(2, dtype=torch.uint8), torch.ones(2, dtype=torch.bool), full)
        y = got[0].double().cpu()
        assert torch.allclose(y[0], torch.full((8,), 10000.0, dtype=torch.float64), rtol=1e-6)
        assert y[1].abs().max() <= 1e-30 and torch.isfinite(got[1]).all()


def activations(v, dtype, kind, rows):
    """act(v) and act'(v) of the values v as the block has them: gate products v, up products and the rest 1; `rows` rows alike."""
    n = len(v)
    first = torch.zeros(n, 8, dtype=torch.float64)
    gate = first.clone()
    gate[:, 0], first[:, 0] = v, 1
    full = dict(x=first[:1].repeat(rows, 1), wg=gate, wu=first, wd=torch.eye(n, dtype=torch.float64), dy=torch.zeros(rows, n).double())
    full["dy"][-1] = 1      # one row's gradients alone, so that the weights' are the row's
    y, _, dwg, _, _ = ffn_call((rows, 8, n, n, dtype, kind, "all", 0, 0), torch.ones(rows, dtype=torch.uint8),
                               torch.ones(rows, dtype=torch.bool), full)
    assert torch.equal(y, y[:1].expand_as(y))
    return y[-1].double().cpu(), dwg[:, 0].double().cpu()


def all_values(dtype, low, high):
    v = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(O.TORCH[dtype]).double()
    v = v[(v >= low) & (v <= high) & (v.abs() >= 1e-3)].unique()
    return v[:: -(-len(v) // 1536)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows", [1, 130])
def test_gelu_keeps_its_small_results(dtype, rows):
    """Far below zero v Phi(v) is small and still a number of 16 bits: it is rounded, not lost.  The products with 1 are exact, so the error
    is half a unit and that of Phi and the exponential in float: below 2^-13 of the terms of v Phi(v), and of Phi(v) + v phi(v)."""
    v = all_values(dtype, -12.5 if dtype == "bf16" else -5.5, 6.0)
    y, slope = activations(v, dtype, "gelu", rows)
    small = 0.0 if dtype == "bf16" else 2.0 ** -25      # half of f16's smallest
    phi, density = 0.5 * torch.special.erfc(-v / math.sqrt(2)), torch.exp(-0.5 * v * v) / math.sqrt(2 * math.pi)
    inside(y, v * phi, (O.U[dtype] + 2.0 ** -13) * (v * phi).abs() + small, "gelu")
    inside(slope, phi + v * density, O.U[dtype] * (phi + v * density).abs() + 2.0 ** -13 * (phi + (v * density).abs()) + small, "its slope")


def test_silu_of_floats_has_a_floats_digits():
    """v / (1 + exp(-v)): the exponential within 3 units of 2^-24, the sum, quotient and product within one each, as the slope's further
    terms: no more than 16.  A row's products with 1 are exact."""
    v = torch.linspace(-85.0, 20.0, 1401, dtype=torch.float32).double()
    y, slope = activations(v, "f32", "silu", 1)
    s = torch.sigmoid(v)
    inside(y, v * s, 16 * O.E * (v * s).abs(), "silu")
    inside(slope, s * (1 + v * (1 - s)), 16 * O.E * s * (1 + (v * (1 - s)).abs()) + O.TINY["f32"], "its slope")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 130])
@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh"])
def test_activations_of_the_largest_numbers(dtype, rows, kind):
    """v and 0 with slopes 1 and 0, exactly: the squares and cubes on the way are infinite."""
    v = torch.tensor([1e10, 2e19, 1e30, 2e38, -1e10, -2e19, -1e30, -2e38]).to(O.TORCH[dtype]).double()
    y, slope = activations(v, dtype, kind, rows)
    assert torch.equal(y, v.clamp_min(0)) and torch.equal(slope, (v > 0).double())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows,di,dh,do", [(3, 256, 512, 256), (60, 264, 520, 200), (900, 256, 512, 320), (900, 201, 403, 255)])
@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh"])
def test_ffn_gradients_are_as_near_as_their_operands_allow(dtype, rows, di, dh, do, kind):
    """hidden, dg and du are rounded once, as operands of products, and nothing else is on the way: a gradient is as far from the exact one as a
    product in 64 bits of operands rounded once.  g and u in 24 bits turn the rounding of up to 6 % of the operands, which lie half way between
    two numbers, to the other side: signs of errors change, not their size."""
    c = (rows, di, dh, do, dtype, kind, "all", 0, 0)
    m, keep, full = ffn_case(c, 17)
    got = ffn_call(c, m, keep, full)
    x, wg, wu, wd, dy = (full[n] for n in ("x", "wg", "wu", "wd", "dy"))
    once = lambda v: v.to(O.TORCH[dtype]).double()  # noqa: E731
    g, u, dhidden = x @ wg.T, x @ wu.T, dy @ wd
    a = O.act(g, kind)
    dg, du, hidden = once(dhidden * u * O.act_grad(g, kind)), once(dhidden * a), once(a * u)
    leaves = [v.clone().requires_grad_(True) for v in (x, wg, wu, wd)]
    exact = torch.autograd.grad(O.ffn_forward(*leaves, kind), leaves, dy)
    for name, have, want, near in zip(("dx", "dw_gate", "dw_up", "dw_down"), got[1:], exact, (dg @ wg + du @ wu, dg.T @ x, du.T @ x, dy.T @ hidden)):
        off, ideal = (have.double().cpu() - want).norm(), (once(near) - want).norm()
        assert off <= 1.1 * ideal, f"{name}: {off / ideal:.3f}"


@pytest.mark.parametrize("rows", [1, 130])
def test_f16_products_beyond_its_range(rows):
    """g of 90 000 with u of 0.01: hidden and every gradient are within f16, and so are the results."""
    full = dict(x=torch.zeros(rows, 8).double(), wg=torch.zeros(16, 8).double(), wu=torch.zeros(16, 8).double(), wd=torch.eye(16).double(),
                dy=torch.full((rows, 16), 0.0625).double())
    full["x"][:, 0], full["x"][:, 1], full["wg"][:, 0], full["wu"][:, 1] = 300, 1, 300, 0.0078125
    c = (rows, 8, 16, 16, "f16", "silu", "all", 0, 0)
    y, dx, dwg, dwu, dwd = (v.double().cpu() for v in ffn_call(c, torch.ones(rows, dtype=torch.uint8), torch.ones(rows, dtype=torch.bool), full))
    within = lambda have, want: ((have - want).abs() <= 2.0 ** -9 * abs(want)).all()  # noqa: E731
    assert within(y, 90000 / 128)
    assert within(dx[:, 0], 16 * 300 / 2048) and within(dx[:, 1], 16 * 5625 / 128) and (dx[:, 2:] == 0).all()
    if rows == 1:      # (a sum over 130 rows of 5 625 is beyond f16)
        assert within(dwg[:, 0], 300 / 2048) and within(dwu[:, 1], 5625) and within(dwd, 90000 / 2048)


def test_floats_in_parts_lose_what_lies_below_the_smallest_normal_number():
    """u of 2^-90 to 2^-124 in 130 rows: two of the three parts of u, and of the hidden row, may fall below 2^-126."""
    small = torch.logspace(-90, -124, 700, base=2.0, dtype=torch.float32).double()
    first, gate = torch.zeros(700, 8, dtype=torch.float64), torch.zeros(700, 8, dtype=torch.float64)
    first[:, 0], gate[:, 0] = small, 20
    full = dict(x=torch.tensor([1.0] + [0.0] * 7).double().repeat(130, 1), wg=gate, wu=first, wd=torch.eye(700).double(), dy=torch.zeros(130, 700))
    y = ffn_call((130, 8, 700, 700, "f32", "silu", "all", 0, 0), torch.ones(130, dtype=torch.uint8), torch.ones(130, dtype=torch.bool), full,
                 backward=False)
    act = 20 / (1 + math.exp(-20))
    inside(y, (act * small).expand(130, -1), (16 * O.E * act * small + (act + 1) * 2 * 2.0 ** -126).expand(130, -1), "y")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows", [4, 40, 200])
def test_ffn_of_infinities_and_of_rows_too_large(dtype, rows):
    """A row with an infinity, or with hidden values beyond f16, has no finite result; every other row is as it would be without."""
    c = (rows, 96, 136, 80, dtype, "silu", "all", 0, 0)
    m, keep, full = ffn_case(c, 13)
    want = ffn_call(c, m, keep, full)
    for lost, value in ((0, float("inf")), (rows // 2, -float("inf")), (rows - 1, float("nan")), (1, 3e4 if dtype == "f16" else float("inf"))):
        bad = {n: v.clone() for n, v in full.items()}
        bad["x"][lost, ::3] = value
        t = {n: dev(v, dtype) for n, v in bad.items()}
        desc = K.make_ffn_desc(96, 136, 80, K.DTYPE_CODE[dtype])
        ws = torch.empty(K.sparse_ffn_workspace_bytes(desc, rows, True), dtype=torch.uint8, device=DEV)
        y, saved = torch.empty_like(want[0]), nan_like(3, rows, 136, dtype=dtype)
        K.sparse_ffn_run(desc, t["x"], t["wg"], t["wu"], t["wd"], y, ws, saved=saved)
        grads = [torch.empty_like(v) for v in want[1:]]
        K.sparse_ffn_backward(desc, t["x"], t["wg"], t["wu"], t["wd"], saved, t["dy"], *grads, ws)
        others = torch.arange(rows) != lost
        for have, clean in ((y, want[0]), (grads[0], want[1])):
            assert torch.equal(have[others.to(DEV)], clean[others.to(DEV)])
        assert not torch.isfinite(y[lost]).any()


def test_ffn_on_another_stream_and_in_a_graph():
    c = (96, 128, 256, 128, "bf16", "silu", "half", 0, 0)
    m, keep, full = ffn_case(c, 2)
    want = ffn_call(c, m, keep, full, backward=False)
    t = {n: dev(v, "bf16") for n, v in full.items()}
    rs = K.sparse_rows_plan(m.to(DEV))
    desc = K.make_ffn_desc(128, 256, 128)
    ws = torch.empty(K.sparse_ffn_workspace_bytes(desc, rs.kept), dtype=torch.uint8, device=DEV)
    y = nan_like(96, 128, dtype="bf16")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        K.sparse_ffn_run(desc, t["x"], t["wg"], t["wu"], t["wd"], y, ws, rows=rs)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(y, want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        K.sparse_ffn_run(desc, t["x"], t["wg"], t["wu"], t["wd"], y, ws, rows=rs)
    for _ in range(3):
        y.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)


@pytest.mark.parametrize("rows,d_out", [((1 << 26) + 9, 8), ((1 << 26) + 9, 3)])
def test_zeros_in_millions_of_dropped_rows(rows, d_out):
    mask = torch.zeros(rows, dtype=torch.uint8, device=DEV)
    at = torch.tensor([0, 12345, (1 << 24) + 3, rows - 2], device=DEV)
    mask[at] = 1
    rs = K.sparse_rows_plan(mask)
    w = [torch.ones(*s, dtype=torch.bfloat16, device=DEV) for s in ((8, 8), (8, 8), (d_out, 8))]
    desc = K.make_ffn_desc(8, 8, d_out)
    ws = torch.empty(K.sparse_ffn_workspace_bytes(desc, 4), dtype=torch.uint8, device=DEV)
    y = nan_like(rows, d_out, dtype="bf16")
    K.sparse_ffn_run(desc, torch.ones(4, 8, dtype=torch.bfloat16, device=DEV), *w, y, ws, rows=rs, x_rows=B.SC_ROWS_COMPACT)
    assert (y[at] > 400).all()                                  # 8 silu(8) 8 = 511.8
    y[at] = 0
    assert int(torch.count_nonzero(y.view(torch.int16))) == 0   # (NaN and -0.0 count)


def test_backward_passes_in_a_graph():
    """Norm and block forward and backward: parts of gradients, copies of odd rows and zeros are launches of their own."""
    rows, d, hidden = 700, 410, 300
    g = torch.Generator(DEV).manual_seed(6)
    draw = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    rs = K.sparse_rows_plan((draw(rows) < 0).to(torch.uint8))
    nd, fd = K.make_norm_desc(d, B.SC_F32, rows_per_gate=3), K.make_ffn_desc(d, hidden, d, B.SC_F32)
    x, f, gate, dx_new, dh = draw(rows, d), draw(rs.kept, d), draw(-(-rows // 3), d), draw(rows, d), draw(rs.kept, d)
    w, wn = [draw(hidden, d) * d ** -0.5, draw(hidden, d) * d ** -0.5, draw(d, hidden) * hidden ** -0.5], [draw(d), draw(d)]
    new = torch.empty_like
    x_new, h, y, saved, stats = new(x), new(f), new(x), draw(3, rs.kept, hidden), draw(rows, 4)
    out = [new(t) for t in (x, f, gate, wn[0], wn[1], f, *w)]
    ws = torch.empty(max(K.sparse_norm_workspace_bytes(nd, rows), K.sparse_ffn_workspace_bytes(fd, rs.kept, True)), dtype=torch.uint8, device=DEV)

    def run():
        K.sparse_norm_run(nd, x, f, gate, wn[0], None, wn[1], None, x_new, h, f_rows=rs, h_rows=rs, stats=stats)
        K.sparse_ffn_run(fd, h, *w, y, ws, rows=rs, x_rows=B.SC_ROWS_COMPACT, saved=saved)
        K.sparse_ffn_backward(fd, h, *w, saved, dx_new, out[5], *out[6:], ws, rows=rs, x_rows=B.SC_ROWS_COMPACT)
        K.sparse_norm_backward(nd, x, f, gate, wn[0], None, wn[1], stats, dx_new, out[5], *out[:4], None, out[4], None, ws, f_rows=rs, h_rows=rs)

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    results = [x_new, h, y, *out]
    for _ in range(3):
        x.copy_(draw(rows, d))
        for t in (*results, saved, stats, ws):
            t.fill_(77)
        run()
        want = [t.clone() for t in results]
        for t in (*results, saved, stats, ws):
            t.fill_(99)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) and torch.isfinite(a).all() for a, b in zip(results, want))


@pytest.mark.parametrize("d", [4096, 4098])
def test_tensors_beyond_32_bits(d):
    """1 100 000 rows, 4.5e9 entries, of which a few hundred at both ends and around 2^31 and 2^32 entries are kept."""
    rows, hidden, t = 1_100_000, 40, torch.bfloat16
    g = torch.Generator(DEV).manual_seed(d)
    at = torch.cat([torch.arange(a, a + 70, device=DEV) for a in (0, (1 << 31) // d - 35, (1 << 32) // d - 35, rows - 70)])
    mask = torch.zeros(rows, dtype=torch.uint8, device=DEV)
    mask[at] = 1
    rs = K.sparse_rows_plan(mask)
    draw = lambda *s, std=1.0: (torch.randn(*s, generator=g, device=DEV) * std).to(t)  # noqa: E731
    w = [draw(hidden, d, std=d ** -0.5), draw(hidden, d, std=d ** -0.5), draw(d, hidden, std=hidden ** -0.5)]
    x, y = torch.zeros(rows, d, dtype=t, device=DEV), torch.empty(rows, d, dtype=t, device=DEV)
    x[at] = draw(280, d)
    fd, nd = K.make_ffn_desc(d, hidden, d), K.make_norm_desc(d, rows_per_gate=100)
    ws = torch.empty(K.sparse_ffn_workspace_bytes(fd, 280, True) + K.sparse_norm_workspace_bytes(nd, rows), dtype=torch.uint8, device=DEV)

    def block(x, y, rows, fmt):      # y of the block, then gradients for y = dy
        saved, dx, dw = torch.empty(3, 280, hidden, dtype=t, device=DEV), torch.empty_like(x), [torch.empty_like(v) for v in w]
        K.sparse_ffn_run(fd, x, *w, y, ws, rows=rows, x_rows=fmt, y_rows=fmt, saved=saved)
        K.sparse_ffn_backward(fd, x, *w, saved, y, dx, *dw, ws, rows=rows, x_rows=fmt, y_rows=fmt)
        return dx, dw

    small_x, small_y = x[at], torch.empty(280, d, dtype=t, device=DEV)
    dx, dw = block(x, y, rs, B.SC_ROWS_DENSE)
    want_dx, want_dw = block(small_x, small_y, None, B.SC_ROWS_COMPACT)
    assert torch.equal(y[at], small_y) and torch.equal(dx[at], want_dx) and all(torch.equal(p, q) for p, q in zip(dw, want_dw))
    for v in (y, dx):      # (a sum over all would be in 16 bits)
        v[at] = 0
        assert not any(bool(piece.any()) for piece in v.split(1 << 17))

    f, gate, ones, stats = draw(280, d), draw(rows // 100, d), torch.ones(d, device=DEV), torch.empty(rows, 4, device=DEV)
    x_new, h, df = y, torch.empty_like(f), torch.empty_like(f)
    K.sparse_norm_run(nd, x, f, gate, ones, None, ones, None, x_new, h, f_rows=rs, h_rows=rs, stats=stats)
    K.sparse_norm_backward(nd, x, f, gate, ones, None, ones, stats, None, small_x, dx, df, None, None, None, None, None, ws, f_rows=rs, h_rows=rs)
    one, small = K.make_norm_desc(d, rows_per_gate=1), (gate[at // 100], torch.empty_like(f), torch.empty_like(f), torch.empty(280, 4, device=DEV))
    K.sparse_norm_run(one, x[at], f, small[0], ones, None, ones, None, small[1], small[2], stats=small[3])
    assert torch.equal(x_new[at], small[1]) and torch.equal(h, small[2])
    grads = torch.empty_like(f), torch.empty_like(f)
    K.sparse_norm_backward(one, x[at], f, small[0], ones, None, ones, small[3], None, small_x, *grads, None, None, None, None, None, ws)
    assert torch.equal(dx[at], grads[0]) and torch.equal(df, grads[1])


# ---- 4-bit weights -----------------------------------------------------------------------------------------------------

Q4S = [  # rows, n, k, group, dtype, zeros
    (1, 1, 1, 32, "bf16", True), (1, 16, 128, 128, "bf16", True), (1, 100, 260, 64, "f16", True), (2, 33, 127, 32, "f16", False),
    (5, 17, 1000, 128, "bf16", False), (16, 64, 1024, 64, "bf16", True), (17, 48, 515, 32, "bf16", True),
    (33, 130, 640, 128, "f16", True), (64, 96, 2049, 64, "bf16", True), (65, 40, 300, 128, "f16", True), (150, 24, 96, 32, "bf16", True)]


def q4_matrix(g, n, k, group, dtype, zeros):
    groups = -(-k // group)
    codes = torch.randint(0, 256, (n, -(-k // 2)), generator=g, dtype=torch.uint8)
    scales = (torch.rand(n, groups, generator=g) * 0.02 + 0.001).to(O.TORCH[dtype])
    z = torch.randint(0, 16, (n, groups), generator=g).to(O.TORCH[dtype]) if zeros else None
    return codes, scales, z


@pytest.mark.parametrize("c", Q4S, ids=lambda c: "-".join(map(str, c)))
def test_q4_products(c):
    rows, n, k, group, dtype, zeros = c
    g = gen(n + k)
    x = normal(g, rows, k, dtype=dtype)
    codes, scales, z = q4_matrix(g, n, k, group, dtype, zeros)
    desc = K.make_q4_desc(k, n, group, K.DTYPE_CODE[dtype])
    held = [v.to(DEV) if v is not None else None for v in (codes, scales, z)]
    plan = K.sparse_q4_plan(desc, *held)
    torch.cuda.synchronize()
    for v in held:      # not needed any more
        if v is not None:
            v.zero_()
    y = nan_like(rows, n, dtype=dtype)
    K.sparse_q4_run(plan, dev(x, dtype), y)
    want, bound = O.q4_bound(x, codes, scales, z, k, group, dtype)
    inside(y, want, bound, "y")
    again = nan_like(rows, n, dtype=dtype)
    K.sparse_q4_run(plan, dev(x, dtype), again)
    assert torch.equal(y, again)


@pytest.mark.parametrize("rows,n,k,group,dtype,kind", [(1, 40, 192, 64, "bf16", "silu"), (3, 33, 100, 32, "f16", "gelu"),
                                                       (20, 80, 512, 128, "bf16", "gelu_tanh"), (70, 16, 140, 64, "f16", "silu")])
def test_q4_gated_products(rows, n, k, group, dtype, kind):
    g = gen(rows)
    x = normal(g, rows, k, dtype=dtype)
    mats = [q4_matrix(g, n, k, group, dtype, True) for _ in range(2)]
    desc = K.make_q4_desc(k, n, group, K.DTYPE_CODE[dtype])
    sides = [dict(codes=c.to(DEV), scales=s.to(DEV), zeros=z.to(DEV)) for c, s, z in mats]
    plan = K.sparse_q4_plan_gated(desc, *sides, activation=K.ACT_CODE[kind])
    y = K.sparse_q4_run(plan, dev(x, dtype), nan_like(rows, n, dtype=dtype))
    (a, ea), (p, ep) = (O.q4_bound(x, *mt, k, group, dtype) for mt in mats)
    ea, ep = ea - O.U[dtype] * a.abs(), ep - O.U[dtype] * p.abs()      # the two products are not rounded
    want = O.act(a, kind) * p
    bound = O.U[dtype] * want.abs() + 1.2 * ea * p.abs() + O.act(a, kind).abs() * ep + 1.2 * ea * ep + O.TINY[dtype]
    bound = bound + 64 * O.E * (1 + a.abs()) * a.abs().clamp_max(8) * p.abs()
    inside(y, want, bound, "y")


# columns beyond a round of the wavefronts, so that they take second and third blocks, and outputs beyond those that sixteen are used for
@pytest.mark.parametrize("c", [(1, 40, 4100, 128, "bf16", True), (3, 24, 2177, 32, "f16", True), (16, 33, 6000, 64, "bf16", False),
                               (2, 8209, 2200, 128, "bf16", True), (16, 8209, 2177, 32, "f16", True), (1, 8200, 130, 64, "bf16", True),
                               (20, 8209, 1300, 64, "f16", True), (40, 20, 2300, 32, "bf16", True)], ids=lambda c: "-".join(map(str, c)))
def test_q4_products_of_long_rows_and_many_outputs(c):
    test_q4_products(c)


@pytest.mark.parametrize("rows,n,k,group,dtype,kind", [(1, 40, 2200, 128, "bf16", "silu"), (16, 33, 4500, 32, "f16", "gelu"),
                                                       (2, 8209, 2200, 64, "bf16", "silu"), (16, 8201, 2177, 128, "f16", "silu"),
                                                       (40, 40, 1300, 64, "bf16", "gelu")])
def test_q4_gated_products_of_long_rows_and_many_outputs(rows, n, k, group, dtype, kind):
    test_q4_gated_products(rows, n, k, group, dtype, kind)


@pytest.mark.parametrize("rows", [3, 40])
def test_q4_rows_that_are_not_finite_stay_alone(rows):
    g = gen(rows)
    x = normal(g, rows, 300, dtype="bf16")
    plan = K.sparse_q4_plan(K.make_q4_desc(300, 70, 64), *[v.to(DEV) for v in q4_matrix(g, 70, 300, 64, "bf16", True)])
    want = K.sparse_q4_run(plan, dev(x, "bf16"), nan_like(rows, 70, dtype="bf16"))
    x[1, 5] = float("inf")
    y = K.sparse_q4_run(plan, dev(x, "bf16"), nan_like(rows, 70, dtype="bf16"))
    others = torch.arange(rows, device=DEV) != 1
    assert torch.equal(y[others], want[others]) and not torch.isfinite(y[1]).any()


# ---- refusals of the binding -------------------------------------------------------------------------------------------


def test_wrong_tensors_are_refused():
    desc = K.make_ffn_desc(64, 128, 64)
    w, wd = torch.zeros(128, 64, dtype=torch.bfloat16, device=DEV), torch.zeros(64, 128, dtype=torch.bfloat16, device=DEV)
    x, y = torch.zeros(4, 64, dtype=torch.bfloat16, device=DEV), torch.zeros(4, 64, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    K.sparse_ffn_run(desc, x, w, w, wd, y, ws)
    for bad in (dict(x=x.float()), dict(x=x[:, :32]), dict(w_gate=w[:64]), dict(w_gate=w.t()), dict(y=y[:3]), dict(x=x.cpu()),
                dict(y_rows=B.SC_ROWS_COMPACT, rows=K.sparse_rows_plan(torch.tensor([1, 0, 0, 1], dtype=torch.uint8, device=DEV)))):
        a = dict(x=x, w_gate=w, w_up=w, w_down=wd, y=y, workspace=ws)
        a.update(bad)
        with pytest.raises(ValueError):
            K.sparse_ffn_run(desc, **a)
    with pytest.raises(K.ScError):
        K.sparse_ffn_run(desc, x, w, w, wd, y, ws[:100])
    with pytest.raises(ValueError):
        K.sparse_rows_plan(torch.zeros(4, device=DEV))
    nd = K.make_norm_desc(64)
    with pytest.raises(ValueError):
        K.sparse_norm_run(nd, x, y[:2], None, None, None, None, None, y, y)
    q = K.sparse_q4_plan(K.make_q4_desc(64, 32, 32), torch.zeros(32, 32, dtype=torch.uint8, device=DEV),
                         torch.zeros(32, 2, dtype=torch.bfloat16, device=DEV))
    with pytest.raises(ValueError):
        K.sparse_q4_run(q, x, y)


def test_empty_calls():
    desc = K.make_ffn_desc(64, 128, 64)
    e = lambda *s, dtype="bf16": torch.empty(*s, dtype=O.TORCH[dtype], device=DEV)  # noqa: E731
    w, wd = nan_like(128, 64, dtype="bf16"), nan_like(64, 128, dtype="bf16")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    K.sparse_ffn_run(desc, e(0, 64), w, w, wd, e(0, 64), ws)
    grads = [nan_like(128, 64, dtype="bf16"), nan_like(128, 64, dtype="bf16"), nan_like(64, 128, dtype="bf16")]
    K.sparse_ffn_backward(desc, e(0, 64), w, w, wd, e(3, 0, 128), e(0, 64), e(0, 64), *grads, ws)
    assert all((g == 0).all() for g in grads)
    nd = K.make_norm_desc(64)
    K.sparse_norm_run(nd, e(0, 64), e(0, 64), None, None, None, None, None, e(0, 64), e(0, 64))
    dw = [nan_like(64) for _ in range(2)]
    K.sparse_norm_backward(nd, e(0, 64), e(0, 64), None, None, None, None, e(0, 4, dtype="f32"), e(0, 64), e(0, 64), e(0, 64), e(0, 64),
                           None, dw[0], None, dw[1], None, ws)
    assert all((v == 0).all() for v in dw)
    plan = K.sparse_q4_plan(K.make_q4_desc(64, 32, 32), torch.zeros(32, 32, dtype=torch.uint8, device=DEV),
                            torch.zeros(32, 2, dtype=torch.bfloat16, device=DEV))
    K.sparse_q4_run(plan, e(0, 64), e(0, 32))
