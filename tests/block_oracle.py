"""Oracle of the block operators: plain torch in 64 bits on the CPU, and how far a correct kernel may be from it.

Bounds are per element and follow from how the operators round (include/sparse_block.h), with u the half unit in the last place of the
tensor's type and e = 2^-24 that of float:
  * a result is rounded once: u |result|;
  * a float sum of n products whose absolute values sum to S is off by at most (n + 4) e S, in whatever order; the bounds use
    ACC = 32 + 2 sqrt(n) in place of n + 4 (roundings of random signs; the 32 covers the exponential's few units);
  * rounded intermediates (hidden rows, g, u, and the gradients dg, du) carry u of themselves into the sums that they enter.
"""
import math

import torch

U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 1e-37, "f16": 2.0 ** -24, "bf16": 1e-37}      # f16: results below the normal range
E = 2.0 ** -24
TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def acc(n):
    return (32 + 2 * math.sqrt(n)) * E


# ---- norms -------------------------------------------------------------------------------------------------------------


def normed(v, kind, eps):
    if kind == "none":
        return v
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    return v / torch.sqrt((v * v).mean(-1, keepdim=True) + eps)


def norm_forward(x, f, gate, w_post, b_post, w_pre, b_pre, post, pre, eps, a, b, per, f_keep, h_keep):
    """x [rows, d], f [kept, d] or None, gate [groups, d] or None, all float64; keeps: bool[rows]."""
    x_new = a * x
    if f is not None and f.shape[0]:
        n = normed(f, post, eps)
        n = n if w_post is None else n * w_post
        n = n if b_post is None else n + b_post
        rows = f_keep.nonzero()[:, 0]
        if gate is not None:
            n = n * gate[rows // per]
        x_new = x_new.index_add(0, rows, b * n)
    h = normed(x_new[h_keep], pre, eps)
    h = h if w_pre is None else h * w_pre
    h = h if b_pre is None else h + b_pre
    return x_new, h


# ---- feed-forward block ------------------------------------------------------------------------------------------------


def act(v, kind):
    if kind == "silu":
        return v * torch.sigmoid(v)
    if kind == "gelu":
        return 0.5 * v * torch.special.erfc(-v / math.sqrt(2))
    return v * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))


def act_grad(v, kind):
    v = v.detach().clone().requires_grad_(True)
    return torch.autograd.grad(act(v, kind).sum(), v)[0]


def ffn_forward(x, wg, wu, wd, kind):
    return (act(x @ wg.T, kind) * (x @ wu.T)) @ wd.T


def ffn_bounds(x, wg, wu, wd, kind, dtype, dy=None):
    """Allowed error of y, or with dy of (y, dx, dwg, dwu, dwd)."""
    u, d, hid, m = U[dtype], x.shape[1], wg.shape[0], x.shape[0]
    ax = x.abs()
    g, p = x @ wg.T, x @ wu.T
    eg, ep = acc(d) * (ax @ wg.abs().T), acc(d) * (ax @ wu.abs().T)          # of the float products
    a, da = act(g, kind), act_grad(g, kind)
    h = a * p
    slope = 1.2                                                              # |act'| and |act''| stay below it
    # the activation's own float error: a few units of its argument in the exponent, then relative ones
    ea = slope * eg + 32 * E * (1 + g.abs()) * g.abs().clamp_max(8) + 32 * E * a.abs()
    eh = ea * p.abs() + a.abs() * ep + u * h.abs()
    y = h @ wd.T
    ey = u * y.abs() + eh @ wd.abs().T + acc(hid) * (h.abs() @ wd.abs().T)
    if dy is None:
        return ey + TINY[dtype]
    eg, ep = eg + u * g.abs(), ep + u * p.abs()                              # as saved
    dh = dy @ wd
    edh = acc(wd.shape[0]) * (dy.abs() @ wd.abs())
    eda = slope * eg + 64 * E * (1 + g.abs())
    ea = slope * eg + 32 * E * (1 + g.abs()) * g.abs().clamp_max(8) + 32 * E * a.abs()
    dg, dp = dh * p * da, dh * a
    edg = edh * (p * da).abs() + dh.abs() * (ep * da.abs() + p.abs() * eda) + u * dg.abs() + TINY[dtype]
    edp = edh * a.abs() + dh.abs() * ea + u * dp.abs() + TINY[dtype]
    dx = dg @ wg + dp @ wu
    edx = u * dx.abs() + edg @ wg.abs() + edp @ wu.abs() + acc(2 * hid) * (dg.abs() @ wg.abs() + dp.abs() @ wu.abs())

    def weight(left, eleft, right, eright):
        v = left.T @ right
        return u * v.abs() + eleft.T @ right.abs() + left.abs().T @ eright + acc(m) * (left.abs().T @ right.abs())

    zero_x, zero_dy = torch.zeros_like(x), torch.zeros_like(dy)
    bounds = [ey, edx, weight(dg, edg, x, zero_x), weight(dp, edp, x, zero_x), weight(dy, zero_dy, h, eh)]
    # second order of the errors above
    return [1.05 * b + TINY[dtype] for b in bounds]


# ---- 4-bit weights -----------------------------------------------------------------------------------------------------


def widen4(codes, scales, zeros, k, group):
    low, high = (codes & 15).double(), (codes >> 4).double()
    code = torch.stack((low, high), 2).flatten(1)[:, :k]
    wide = lambda p: p.double().repeat_interleave(group, 1)[:, :k]  # noqa: E731
    return (code - (wide(zeros) if zeros is not None else 8.0)) * wide(scales), code


def q4_bound(x, codes, scales, zeros, k, group, dtype):
    """The kernel sums x (B + code) and (B + zero) x per group, B = 128 (bf16) or 1024 (f16)."""
    w, code = widen4(codes, scales, zeros, k, group)
    base = {"bf16": 128.0, "f16": 1024.0}[dtype]
    s = scales.double().abs().repeat_interleave(group, 1)[:, :k]
    z = zeros.double().abs().repeat_interleave(group, 1)[:, :k] if zeros is not None else 8.0
    total = x.abs() @ (s * (2 * base + code + z)).T
    y = x @ w.T
    return y, U[dtype] * y.abs() + acc(group) * total + TINY[dtype]
