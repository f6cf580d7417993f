"""Oracle of the attention operators: plain torch in 64 bits on the CPU, and how far a correct kernel may be from it.

Bounds are per element and follow from how the operators round (include/sparse_attention.h), with u the half unit in the last place of the
tensors' type, e = 2^-24 that of float and ACC(n) = (32 + 2 sqrt(n)) e the relative error of a float sum of n products:
  * a score is a float sum over d: off by es = scale ACC(d) sum |q k|; its exponential's argument is rounded where it is formed and where the
    maximum or lse is taken off: 8 e (1 + |s| + |max|), and so is a probability, relatively;
  * probabilities and gradients of scores are rounded to the type as operands: u relatively, and in f16 half of its smallest number,
    2^-25, at least;
  * sums over keys or rows add ACC(n) of the sum of absolute values, and a result is rounded once.
"""
import math

import torch

from block_oracle import E, TINY, TORCH, U, acc  # noqa: F401

SUB = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}


def seen(n, causal, window):
    i = torch.arange(n)
    m = torch.ones(n, n, dtype=torch.bool)
    if causal:
        m &= i[None] <= i[:, None]
    if window:
        m &= (i[None] - i[:, None]).abs() < window
    return m


def attend(q, k, v, scale, visible):
    """One head of one sequence: (o, lse, p); rows that see nothing are zero, their lse -inf."""
    s = (q @ k.T * scale).masked_fill(~visible, -math.inf)
    lse = torch.logsumexp(s, 1)
    p = torch.exp(s - torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)[:, None])
    return p @ v, lse, p


def attend_bounds(q, k, v, scale, visible, dtype, do=None):
    """Allowed errors of o and lse, and with do of (dq, dk, dv) of this head."""
    u, sub, d, n = U[dtype], SUB[dtype], q.shape[1], k.shape[0]
    o, lse, p = attend(q, k, v, scale, visible)
    s = (q @ k.T * scale).masked_fill(~visible, 0.0)
    top = s.abs().amax(1, keepdim=True) if n else torch.zeros(q.shape[0], 1)
    es = acc(d) * scale * (q.abs() @ k.abs().T) + 8 * E * (1 + s.abs() + top)
    mean = (p * es).sum(1, keepdim=True)
    ep = es + mean + acc(n)                                  # relative error of a probability, its sum's included
    eo = u * o.abs() + (p * (u + ep)) @ v.abs() + acc(n) * (p @ v.abs()) + sub * visible.double() @ v.abs() + TINY[dtype]
    elogsum = (mean[:, 0] + acc(n) + 8 * E * (1 + torch.where(torch.isinf(lse), torch.zeros_like(lse), lse).abs()))
    if do is None:
        return eo, elogsum
    ep = ep + 8 * E * (1 + top)
    delta, edelta = (do * o).sum(1, keepdim=True), (do.abs() * eo).sum(1, keepdim=True) + acc(d) * (do * o).abs().sum(1, keepdim=True)
    dp = do @ v.T
    ds = p * (dp - delta)
    eds = p * (acc(d) * (do.abs() @ v.abs().T) + edelta) + ds.abs() * (ep + u + 4 * E) + sub * visible.double()
    dq, dk, dv = ds @ k * scale, ds.T @ q * scale, p.T @ do
    rows = q.shape[0]
    edq = u * dq.abs() + scale * (eds @ k.abs() + acc(n) * (ds.abs() @ k.abs())) + TINY[dtype]
    edk = scale * (eds.T @ q.abs() + acc(rows) * (ds.abs().T @ q.abs())), dk
    edv = (p * (u + ep)).T @ do.abs() + acc(rows) * (p.T @ do.abs()) + sub * visible.double().T @ do.abs(), dv
    return eo, elogsum, edq, edk, edv


def packed(c, starts, keep, q, k, v, do=None):
    """Attention of packed sequences, all heads, in 64 bits, and the bounds: dicts by name; rows that no sequence has or the mask drops are 0.
    c: (heads, kv, d, dtype, causal, window, scale)."""
    heads, kv, d, dtype, causal, window, scale = c
    group, rows = heads // kv, q.shape[0]
    names = ["o", "lse"] + (["dq", "dk", "dv"] if do is not None else [])
    shape = {"o": (rows, heads, d), "lse": (rows, heads), "dq": (rows, heads, d), "dk": (rows, kv, d), "dv": (rows, kv, d)}
    want = {n: torch.zeros(shape[n], dtype=torch.float64) for n in names}
    bound = {n: torch.zeros(shape[n], dtype=torch.float64) for n in names}
    for a, b in zip(starts, starts[1:]):
        at = torch.arange(a, b)
        at = at[keep[a:b]]
        if not len(at):
            continue
        visible = seen(len(at), causal, window)
        for h in range(heads):
            j = h // group
            one = q[at, h], k[at, j], v[at, j]
            o, lse, p = attend(*one, scale, visible)
            want["o"][at, h], want["lse"][at, h] = o, lse
            if do is None:
                bound["o"][at, h], bound["lse"][at, h] = attend_bounds(*one, scale, visible, dtype)
                continue
            g = do[at, h]
            delta = (g * o).sum(1, keepdim=True)
            ds = p * (g @ one[2].T - delta)
            want["dq"][at, h] = ds @ one[1] * scale
            eo, elogsum, edq, (edk, dk), (edv, dv) = attend_bounds(*one, scale, visible, dtype, g)
            bound["o"][at, h], bound["lse"][at, h], bound["dq"][at, h] = eo, elogsum, edq
            want["dk"][at, j] += dk
            want["dv"][at, j] += dv
            bound["dk"][at, j] += edk
            bound["dv"][at, j] += edv
    for n in ("dk", "dv"):
        if n in want:
            bound[n] += U[dtype] * want[n].abs() + group * acc(rows) * want[n].abs() + TINY[dtype]
    return want, bound


def quantised(x):
    """8-bit codes of rows (last dimension) of floats in 64 bits, and the float scales: code = x / scale to the nearest, ties to even."""
    scale = (x.abs().amax(-1) / 127).float().clamp_min(2.0 ** -126)
    return torch.round(x / scale.double()[..., None]), scale
