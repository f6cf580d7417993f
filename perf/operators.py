"""The operators of the feed-forward half of a transformer block over kept rows, as a user's program calls them.

A row is a token, or a position of a feature map; a mask keeps some rows and drops the others, as it does in the masked
convolutions.  Three operators:

    norm    x' = a x + b gate * post(f),  h = pre(x'): the norm behind one block, its gate, the residual sum and the norm before
            the next block; "norm_train" is that with its gradients
    ffn     y = (act(x Wg') * (x Wu')) Wd' over the kept rows; "ffn_train" is that with its gradients
    q4      y = x W' with W in 4 bits, a scale and a zero point per group of columns; "q4_ffn" is the ffn on such weights

    listed()             the cases
    draw(rng)            one more case of the same ranges
    prepare(case, seed)  inputs, plans and buffers as a user's program holds them before the call
    run(state)           one pass; returns its outputs: the plain form, or with `own` this package's kernels
    work(case)           bytes and operations that a pass cannot do without
    exact(case, seed)    the outputs in 64 bits
"""
import math

import torch

own = False

DEVICE = "cuda:0"
TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}


# ---- the cases ---------------------------------------------------------------------------------------------------------


def norm(kind="norm", rows=1, d=64, dtype="bf16", post="rms", pre="rms", gate_rows=0, s=0.0, a=1.0, b=1.0, **more):
    """gate_rows: consecutive rows that share a gate vector, 0 for none.  s: share of the rows that the block left out."""
    return dict(kind=kind, rows=rows, d=d, dtype=dtype, post=post, pre=pre, gate_rows=gate_rows, s=s, a=a, b=b, **more)


def ffn(kind="ffn", rows=1, d=64, hidden=64, dtype="bf16", act="silu", s=0.0, **more):
    return dict(kind=kind, rows=rows, d=d, hidden=hidden, dtype=dtype, act=act, s=s, **more)


def q4(rows=1, n=64, k=64, group=128, dtype="bf16", **more):
    return dict(kind="q4", rows=rows, n=n, k=k, group=group, dtype=dtype, **more)


def q4_ffn(rows=1, d=64, hidden=64, group=128, dtype="bf16", act="silu", **more):
    return dict(kind="q4_ffn", rows=rows, d=d, hidden=hidden, group=group, dtype=dtype, act=act, **more)


def listed():
    return [
        # one token of a decoder: the time of a launch
        norm(name="norm_1x2048_bf16", rows=1, d=2048),
        # a long prompt, or a training batch's forward pass
        norm(name="norm_8192x4096_bf16", rows=8192, d=4096),
        # 64 images of 14 x 14 tokens, half of them kept by the mask; layer norms, a gate per image
        norm(name="norm_12544x768_f16_s50", rows=12544, d=768, dtype="f16", post="layer", pre="layer", gate_rows=196, s=0.5),
        # one training step of the pair of norms, a gate per sequence of 1 024
        norm("norm_train", name="norm_train_4096x4096_bf16", rows=4096, d=4096, gate_rows=1024),
        # the same in 32 bits with the channels of a pruned network, no 16-byte rows
        norm("norm_train", name="norm_train_3137x410_f32_s30", rows=3137, d=410, dtype="f32", post="layer", pre="layer", gate_rows=196,
             s=0.3, a=0.5, b=2.0),
        # one token of a decoder: the weights are read once
        ffn(name="ffn_1x2048x5632_bf16", rows=1, d=2048, hidden=5632),
        # the tokens of 64 images, half of them kept, from and into the dense layout
        ffn(name="ffn_12544x768x2048_f16_s50", rows=12544, d=768, hidden=2048, dtype="f16", act="gelu", s=0.5),
        # one training step, the largest case
        ffn("ffn_train", name="ffn_train_8192x2048x5632_bf16", rows=8192, d=2048, hidden=5632),
        # one training step in 32 bits, sizes of a pruned network
        ffn("ffn_train", name="ffn_train_1568x410x1093_f32_s30", rows=1568, d=410, hidden=1093, dtype="f32", act="gelu_tanh", s=0.3),
        # one token times a square projection
        q4(name="q4_1x4096x4096_bf16", rows=1, n=4096, k=4096),
        # a few requests at once, odd sizes, small groups
        q4(name="q4_24x4100x1000_f16", rows=24, n=4100, k=1000, group=32, dtype="f16"),
        # one token through a whole feed-forward block in 4 bits
        q4_ffn(name="q4_ffn_1x4096x11264_bf16", rows=1, d=4096, hidden=11264, group=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size of lo .. hi: usually whole tiles, sometimes whole 16-byte groups only, sometimes odd."""
    v, kind = _log(rng, lo, hi), rng.random()
    v = max(64, v // 64 * 64) if kind < 0.6 else max(8, v // 8 * 8) if kind < 0.85 else v | 1
    return v if v != 3072 else 3136


def draw(rng):
    kind = rng.choice(["norm", "norm_train", "ffn", "ffn_train", "q4", "q4_ffn"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    s = rng.choice([0.0, 0.25, 0.5, 0.7])
    if kind in ("norm", "norm_train"):
        c = norm(kind, rows=_log(rng, 1, 16384), d=_size(rng, 32, 8192), dtype=dtype, post=rng.choice(["none", "rms", "layer"]),
                 pre=rng.choice(["rms", "layer"]), s=s, a=rng.choice([1.0, 1.0, 0.5]), b=rng.choice([1.0, 1.0, 2.0]))
        c["gate_rows"] = rng.choice([0, 1, _log(rng, 2, 2048)])
        most = {"norm": 8192 * 4096 * 4 * 2, "norm_train": 4096 * 4096 * 10 * 2}[kind]
        while work(c)["bytes"] > most:
            c["rows"] = c["rows"] * 2 // 3
        return c
    if kind in ("ffn", "ffn_train"):
        c = ffn(kind, rows=_log(rng, 1, 16384), d=_size(rng, 64, 4096), hidden=_size(rng, 64, 11264), dtype=dtype, s=s,
                act=rng.choice(["silu", "gelu", "gelu_tanh"]))
        most = 18 * 8192 * 2048 * 5632 if dtype != "f32" else 18 * 2048 * 2048 * 2048
        while work(c)["flops"] > most:
            c["rows"] = c["rows"] * 2 // 3
        return c
    dtype, group = rng.choice(["bf16", "f16"]), rng.choice([32, 64, 128])
    if kind == "q4":
        return q4(rows=_log(rng, 1, 64), n=_size(rng, 64, 11264), k=_size(rng, 64, 8192), group=group, dtype=dtype)
    return q4_ffn(rows=_log(rng, 1, 64), d=_size(rng, 64, 4096), hidden=_size(rng, 64, 11264), group=group, dtype=dtype,
                  act=rng.choice(["silu", "gelu", "gelu_tanh"]))


# ---- inputs ------------------------------------------------------------------------------------------------------------


def _kept(c):
    return int(math.floor((1.0 - c["s"]) * c["rows"] + 0.5))


def _inputs(c, seed):
    """All tensors of a case, from the seed alone."""
    g = torch.Generator(device=DEVICE).manual_seed(2309 + 7919 * int(seed))
    t = TORCH[c["dtype"]]

    def normal(*shape, std=1.0, mean=0.0, dtype=t):
        return (torch.randn(*shape, generator=g, device=DEVICE) * std + mean).to(dtype)

    def mask():
        m = torch.zeros(c["rows"], dtype=torch.uint8, device=DEVICE)
        m[torch.randperm(c["rows"], generator=g, device=DEVICE)[: _kept(c)]] = 1
        return m

    def weights4(n, k):
        """A trained matrix's 4-bit form: per row and group the codes span the group's range."""
        groups = -(-k // c["group"])
        w = torch.zeros(n, groups * c["group"], device=DEVICE)
        w[:, :k] = torch.randn(n, k, generator=g, device=DEVICE) / math.sqrt(k)
        w = w.view(n, groups, c["group"])
        lo, hi = w.amin(2, keepdim=True), w.amax(2, keepdim=True)
        scale = ((hi - lo) / 15).clamp_min(1e-6).to(t).float()
        zero = (-lo / scale).round().clamp(0, 15)
        code = ((w / scale).round() + zero).clamp(0, 15).to(torch.uint8).view(n, -1)[:, :k]
        code = torch.nn.functional.pad(code, (0, k % 2))
        return {"codes": (code[:, 0::2] | (code[:, 1::2] << 4)).contiguous(), "scales": scale[..., 0].to(t).contiguous(),
                "zeros": zero[..., 0].to(t).contiguous()}

    kind, rows = c["kind"], c["rows"]
    if kind in ("norm", "norm_train"):
        d, kept = c["d"], _kept(c)
        v = {"mask": mask() if c["s"] else None, "x": normal(rows, d), "f": normal(kept, d, std=0.5)}
        v["gate"] = normal(-(-rows // c["gate_rows"]), d, std=0.5, mean=0.5) if c["gate_rows"] else None
        f32 = torch.float32
        v["w_post"], v["w_pre"] = normal(d, std=0.1, mean=1.0, dtype=f32), normal(d, std=0.1, mean=1.0, dtype=f32)
        v["b_post"] = normal(d, std=0.1, dtype=f32) if c["post"] == "layer" else None
        v["b_pre"] = normal(d, std=0.1, dtype=f32) if c["pre"] == "layer" else None
        if kind == "norm_train":
            v["dx_new"], v["dh"] = normal(rows, d), normal(kept, d)
        return v
    if kind in ("ffn", "ffn_train"):
        d, hidden = c["d"], c["hidden"]
        v = {"mask": mask() if c["s"] else None, "x": normal(rows, d), "w_gate": normal(hidden, d, std=d ** -0.5),
             "w_up": normal(hidden, d, std=d ** -0.5), "w_down": normal(d, hidden, std=hidden ** -0.5)}
        if kind == "ffn_train":
            v["dy"] = normal(rows, d)
        return v
    if kind == "q4":
        return {"x": normal(rows, c["k"]), "w": weights4(c["n"], c["k"])}
    return {"x": normal(rows, c["d"]), "gate": weights4(c["hidden"], c["d"]), "up": weights4(c["hidden"], c["d"]),
            "down": weights4(c["d"], c["hidden"])}


def prepare(case, seed):
    c = case
    v = _inputs(c, seed)
    state = dict(v, case=c)
    if "mask" in v:
        state["kept_rows"] = v["mask"].nonzero()[:, 0] if v["mask"] is not None else None
    if own:
        _prepare_own(c, state)
    return state


def _prepare_own(c, st):
    """Row sets, plans, outputs and workspaces, as a user's program keeps them."""
    from paper_2309_06626_amd import block as K

    t, x, kind = TORCH[c["dtype"]], st["x"], c["kind"]
    empty = lambda *shape, dtype=t: torch.empty(*shape, dtype=dtype, device=DEVICE)  # noqa: E731
    if st.get("mask") is not None:
        st["row_set"] = K.sparse_rows_plan(st["mask"])
    rows = st.setdefault("row_set", None)
    if kind in ("norm", "norm_train"):
        st["desc"] = K.make_norm_desc(c["d"], dtype=K.DTYPE_CODE[c["dtype"]], post=K.NORM_CODE[c["post"]], pre=K.NORM_CODE[c["pre"]],
                                      residual_scale=c["a"], branch_scale=c["b"], rows_per_gate=c["gate_rows"])
        st["x_new"], st["h"] = empty(x.shape), empty(st["f"].shape)
        st["stats"] = empty(c["rows"], 4, dtype=torch.float32) if kind == "norm_train" else None
        if kind == "norm_train":
            grads = {n: torch.empty_like(st[n]) for n in ("x", "f", "gate", "w_post", "b_post", "w_pre", "b_pre") if st[n] is not None}
            st["grads"] = grads
            st["workspace"] = empty(K.sparse_norm_workspace_bytes(st["desc"], c["rows"]), dtype=torch.uint8)
    elif kind in ("ffn", "ffn_train"):
        st["desc"] = K.make_ffn_desc(c["d"], c["hidden"], c["d"], dtype=K.DTYPE_CODE[c["dtype"]], activation=K.ACT_CODE[c["act"]])
        train = kind == "ffn_train"
        st["y"] = empty(x.shape)
        st["saved"] = empty(3, _kept(c), c["hidden"]) if train else None
        st["workspace"] = empty(K.sparse_ffn_workspace_bytes(st["desc"], _kept(c), train), dtype=torch.uint8)
        if train:
            st["grads"] = {n: torch.empty_like(st[n]) for n in ("x", "w_gate", "w_up", "w_down")}
    elif kind == "q4":
        st["plan"] = K.sparse_q4_plan(K.make_q4_desc(c["k"], c["n"], c["group"], K.DTYPE_CODE[c["dtype"]]), **st["w"])
        st["y"] = empty(c["rows"], c["n"])
    else:
        dt = K.DTYPE_CODE[c["dtype"]]
        st["up_plan"] = K.sparse_q4_plan_gated(K.make_q4_desc(c["d"], c["hidden"], c["group"], dt), st["gate"], st["up"],
                                               activation=K.ACT_CODE[c["act"]])
        st["down_plan"] = K.sparse_q4_plan(K.make_q4_desc(c["hidden"], c["d"], c["group"], dt), **st["down"])
        st["hidden"], st["y"] = empty(c["rows"], c["hidden"]), empty(c["rows"], c["d"])


# ---- one pass, with the framework's operators --------------------------------------------------------------------------


def _run_own(st):
    from paper_2309_06626_amd import block as K

    kind = st["case"]["kind"]
    if kind in ("norm", "norm_train"):
        K.sparse_norm_run(st["desc"], st["x"], st["f"], st["gate"], st["w_post"], st["b_post"], st["w_pre"], st["b_pre"], st["x_new"],
                          st["h"], f_rows=st["row_set"], h_rows=st["row_set"], stats=st["stats"])
        out = {"x_new": st["x_new"], "h": st["h"]}
        if kind == "norm_train":
            g = st["grads"]
            K.sparse_norm_backward(st["desc"], st["x"], st["f"], st["gate"], st["w_post"], st["b_post"], st["w_pre"], st["stats"],
                                   st["dx_new"], st["dh"], g["x"], g["f"], g.get("gate"), g["w_post"], g.get("b_post"), g["w_pre"],
                                   g.get("b_pre"), st["workspace"], f_rows=st["row_set"], h_rows=st["row_set"])
            out["grads"] = g
        return out
    if kind in ("ffn", "ffn_train"):
        K.sparse_ffn_run(st["desc"], st["x"], st["w_gate"], st["w_up"], st["w_down"], st["y"], st["workspace"], rows=st["row_set"],
                         saved=st["saved"])
        out = {"y": st["y"]}
        if kind == "ffn_train":
            g = st["grads"]
            K.sparse_ffn_backward(st["desc"], st["x"], st["w_gate"], st["w_up"], st["w_down"], st["saved"], st["dy"], g["x"], g["w_gate"],
                                  g["w_up"], g["w_down"], st["workspace"], rows=st["row_set"])
            out["grads"] = g
        return out
    if kind == "q4":
        return {"y": K.sparse_q4_run(st["plan"], st["x"], st["y"])}
    K.sparse_q4_run(st["up_plan"], st["x"], st["hidden"])
    return {"y": K.sparse_q4_run(st["down_plan"], st["hidden"], st["y"])}


# ---- one pass, plain: elementary operations in 32 bits, rounded once at the end ----------------------------------------


EPS = 1e-6


def _normed(v, kind):
    """(normalised rows, 1 / their spread)"""
    if kind == "none":
        return v, None
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    r = torch.rsqrt((v * v).mean(1, keepdim=True) + EPS)
    return v * r, r


def _normed_backward(g, n, r, kind):
    if kind == "none":
        return g
    out = g - n * (g * n).mean(1, keepdim=True)
    if kind == "layer":
        out = out - g.mean(1, keepdim=True)
    return out * r


def _run_norm(st):
    c = st["case"]
    t, kept, d = st["x"].dtype, st["kept_rows"], c["d"]
    x, f = st["x"].float(), st["f"].float()
    nf, rf = _normed(f, c["post"])
    n = nf * st["w_post"]
    if st["b_post"] is not None:
        n = n + st["b_post"]
    group = None
    if st["gate"] is not None:
        group = torch.arange(c["rows"], device=x.device) // c["gate_rows"]
        group = group if kept is None else group[kept]
        gated = n * st["gate"].float()[group]
    else:
        gated = n
    x_new = c["a"] * x
    if kept is None:
        x_new = x_new + c["b"] * gated
    else:
        x_new[kept] += c["b"] * gated
    z = x_new if kept is None else x_new[kept]
    nz, rz = _normed(z, c["pre"])
    h = nz * st["w_pre"]
    if st["b_pre"] is not None:
        h = h + st["b_pre"]
    out = {"x_new": x_new.to(t), "h": h.to(t)}
    if c["kind"] == "norm":
        return out
    dh, total = st["dh"].float(), st["dx_new"].float()
    dz = _normed_backward(dh * st["w_pre"], nz, rz, c["pre"])
    grads = {"w_pre": (dh * nz).sum(0)}
    if st["b_pre"] is not None:
        grads["b_pre"] = dh.sum(0)
    if kept is None:
        total = total + dz
        branch = c["b"] * total
    else:
        total = total.clone()
        total[kept] += dz
        branch = c["b"] * total[kept]
    grads["x"] = (c["a"] * total).to(t)
    if group is not None:
        gate = st["gate"]
        grads["gate"] = torch.zeros(gate.shape, device=x.device).index_add_(0, group, branch * n).to(t)
        branch = branch * gate.float()[group]
    grads["w_post"] = (branch * nf).sum(0)
    if st["b_post"] is not None:
        grads["b_post"] = branch.sum(0)
    grads["f"] = _normed_backward(branch * st["w_post"], nf, rf, c["post"]).to(t)
    out["grads"] = grads
    return out


def _act(v, kind):
    """(act(v), its derivative)"""
    if kind == "silu":
        s = torch.sigmoid(v)
        return v * s, s * (1 + v * (1 - s))
    if kind == "gelu":
        p = 0.5 * (1 + torch.erf(v * math.sqrt(0.5)))
        return v * p, p + v * torch.exp(-0.5 * v * v) / math.sqrt(2 * math.pi)
    k = math.sqrt(2 / math.pi)
    th = torch.tanh(k * (v + 0.044715 * v * v * v))
    return 0.5 * v * (1 + th), 0.5 * (1 + th) + 0.5 * v * (1 - th * th) * k * (1 + 3 * 0.044715 * v * v)


def _whole(v, kept, like):
    """Kept rows back in the dense layout, zeros between them."""
    if kept is None:
        return v.to(like.dtype)
    out = torch.zeros(like.shape, dtype=like.dtype, device=like.device)
    out[kept] = v.to(like.dtype)
    return out


def _run_ffn(st):
    c = st["case"]
    t, kept = st["x"].dtype, st["kept_rows"]
    x = st["x"].float() if kept is None else st["x"][kept].float()
    wg, wu, wd = st["w_gate"].float(), st["w_up"].float(), st["w_down"].float()
    g, u = x @ wg.t(), x @ wu.t()
    a, da = _act(g, c["act"])
    h = a * u
    out = {"y": _whole(h @ wd.t(), kept, st["x"])}
    if c["kind"] == "ffn":
        return out
    dy = st["dy"].float() if kept is None else st["dy"][kept].float()
    dh = dy @ wd
    dg, du = dh * u * da, dh * a
    out["grads"] = {"w_down": (dy.t() @ h).to(t), "w_gate": (dg.t() @ x).to(t), "w_up": (du.t() @ x).to(t),
                    "x": _whole(dg @ wg + du @ wu, kept, st["x"])}
    return out


def _widened(w, k, group):
    """The matrix that 4-bit codes stand for."""
    code = torch.stack((w["codes"] & 15, w["codes"] >> 4), 2).flatten(1)[:, :k].float()
    at = torch.arange(k, device=code.device) // group
    return (code - w["zeros"].float()[:, at]) * w["scales"].float()[:, at]


def _run_q4(st):
    c = st["case"]
    x = st["x"].float()
    if c["kind"] == "q4":
        return {"y": (x @ _widened(st["w"], c["k"], c["group"]).t()).to(st["x"].dtype)}
    g = x @ _widened(st["gate"], c["d"], c["group"]).t()
    h = _act(g, c["act"])[0] * (x @ _widened(st["up"], c["d"], c["group"]).t())
    return {"y": (h @ _widened(st["down"], c["hidden"], c["group"]).t()).to(st["x"].dtype)}


def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    return _run_norm(state) if kind.startswith("norm") else _run_ffn(state) if kind.startswith("ffn") else _run_q4(state)


# ---- what a pass cannot do without -------------------------------------------------------------------------------------


def work(case):
    c, e = case, BYTES[case["dtype"]]
    kind, rows = c["kind"], c["rows"]
    if kind in ("norm", "norm_train"):
        kept, d = _kept(c), c["d"]
        gates = -(-rows // c["gate_rows"]) if c["gate_rows"] else 0
        vectors = 2 + (c["post"] == "layer") + (c["pre"] == "layer")
        # x, f, gate and the weights in, x' and h out
        nbytes = e * d * (2 * rows + 2 * kept + gates) + 4 * d * vectors
        flops = 14 * rows * d
        if kind == "norm_train":
            # behind the forward pass the gradients of x' and h in, those of x, f, gate and the weights out
            nbytes += e * d * (2 * rows + 2 * kept + gates) + 4 * d * vectors
            flops += 30 * rows * d
        return {"bytes": nbytes, "flops": flops}
    if kind in ("ffn", "ffn_train"):
        kept, d, hidden = _kept(c), c["d"], c["hidden"]
        nbytes = e * ((kept + rows) * d + 3 * d * hidden)
        if kind == "ffn_train":
            nbytes += e * ((kept + rows) * d + 3 * d * hidden)
        return {"bytes": nbytes, "flops": (18 if kind == "ffn_train" else 6) * kept * d * hidden}

    def matrix(n, k):
        return n * (-(-k // 2) + 2 * e * -(-k // c["group"]))

    if kind == "q4":
        return {"bytes": matrix(c["n"], c["k"]) + e * rows * (c["k"] + c["n"]), "flops": 2 * rows * c["n"] * c["k"]}
    d, hidden = c["d"], c["hidden"]
    return {"bytes": 2 * matrix(hidden, d) + matrix(d, hidden) + 2 * e * rows * d, "flops": 6 * rows * d * hidden}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------------


def _functions64():
    norms = {
        "none": lambda v: v,
        "rms": lambda v: v / (v.pow(2).sum(-1, keepdim=True) / v.shape[-1] + EPS).sqrt(),
        "layer": lambda v: (v - v.sum(-1, keepdim=True) / v.shape[-1])
        / (v.var(-1, unbiased=False, keepdim=True) + EPS).sqrt(),
    }
    acts = {
        "silu": lambda v: v / (1 + torch.exp(-v)),
        "gelu": lambda v: v * torch.special.erfc(-v / math.sqrt(2)) / 2,
        "gelu_tanh": lambda v: v * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)),
    }
    return norms, acts


def exact(case, seed):
    """From the definition, with a selection matrix's meaning spelled out per row; gradients by differentiating the 64-bit forward pass."""
    c, v = case, _inputs(case, seed)
    norms, acts = _functions64()
    wide = {n: (t.double() if isinstance(t, torch.Tensor) and t.is_floating_point() else t) for n, t in v.items()}
    kind = c["kind"]
    if kind.startswith("q4"):
        def matrix(w, k):
            low, high = w["codes"].long() % 16, w["codes"].long() // 16
            code = torch.empty(low.shape[0], 2 * low.shape[1], dtype=torch.float64, device=DEVICE)
            code[:, 0::2], code[:, 1::2] = low.double(), high.double()
            wide_of = lambda p: p.double().repeat_interleave(c["group"], 1)[:, :k]  # noqa: E731
            return wide_of(w["scales"]) * (code[:, :k] - wide_of(w["zeros"]))

        if kind == "q4":
            return {"y": torch.matmul(matrix(v["w"], c["k"]), wide["x"].t().contiguous()).t().contiguous()}
        xt = wide["x"].t().contiguous()
        h = acts[c["act"]](torch.matmul(matrix(v["gate"], c["d"]), xt)) * torch.matmul(matrix(v["up"], c["d"]), xt)
        return {"y": torch.matmul(matrix(v["down"], c["hidden"]), h).t().contiguous()}

    keep = torch.ones(c["rows"], dtype=torch.bool, device=DEVICE) if v["mask"] is None else v["mask"].bool()
    train = kind.endswith("_train")
    if train:
        for n in ("x", "f", "gate", "w_post", "b_post", "w_pre", "b_pre", "w_gate", "w_up", "w_down"):
            if wide.get(n) is not None:
                wide[n].requires_grad_(True)
    if kind.startswith("ffn"):
        h = acts[c["act"]](wide["x"] @ wide["w_gate"].t()) * (wide["x"] @ wide["w_up"].t())
        y = (h @ wide["w_down"].t()) * keep[:, None]
        if not train:
            return {"y": y}
        names = ["x", "w_gate", "w_up", "w_down"]
        grads = torch.autograd.grad(y, [wide[n] for n in names], wide["dy"])
        return {"y": y.detach(), "grads": dict(zip(names, grads))}
    n = norms[c["post"]](wide["f"]) * wide["w_post"]
    if wide["b_post"] is not None:
        n = n + wide["b_post"]
    branch = torch.zeros_like(wide["x"]).masked_scatter(keep[:, None].expand(-1, c["d"]), n)
    if wide["gate"] is not None:
        branch = branch * wide["gate"].repeat_interleave(c["gate_rows"], 0)[: c["rows"]]
    x_new = c["a"] * wide["x"] + c["b"] * branch
    h = norms[c["pre"]](x_new) * wide["w_pre"]
    if wide["b_pre"] is not None:
        h = h + wide["b_pre"]
    h = h[keep]
    if not train:
        return {"x_new": x_new, "h": h}
    names = [k for k in ("x", "f", "gate", "w_post", "b_post", "w_pre", "b_pre") if wide[k] is not None]
    grads = torch.autograd.grad([x_new, h], [wide[k] for k in names], [wide["dx_new"], wide["dh"]])
    return {"x_new": x_new.detach(), "h": h.detach(), "grads": dict(zip(names, grads))}
