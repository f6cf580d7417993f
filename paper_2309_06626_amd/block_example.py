"""The block operators together: a stack of feed-forward halves over the kept tokens of a mask, trained, then served from 4-bit weights.

    python -m paper_2309_06626_amd.block_example

A half is norm -> gated feed-forward block -> norm, gate and residual sum; the norm behind one half and the norm before the next are
one call, so a stack of L halves takes 1 + 2 L calls:

    h_0 = norm(x_0);   f_l = ffn_l(h_l);   x_{l+1} = x_l + gate_l * norm(f_l) on kept tokens, x_l on dropped ones;   h_{l+1} = norm(x_{l+1})

h and f hold the kept tokens only.  Serving runs the same calls for single tokens, with the products from 4-bit weights, in one HIP graph.
"""
from __future__ import annotations

import argparse
from typing import Dict, List, Optional

import torch

from . import block as K

EPS = 1e-6


class FeedForwardStack:
    """Weights of `layers` halves of width d and hidden width d_hidden, random-init, and the buffers of one pass."""

    def __init__(self, d: int, d_hidden: int, layers: int, dtype: str = "bf16", activation: str = "silu", seed: int = 0,
                 device="cuda:0"):
        self.d, self.d_hidden, self.layers = d, d_hidden, layers
        self.code, self.type = K.DTYPE_CODE[dtype], K.TORCH_DTYPE[dtype]
        self.activation = K.ACT_CODE[activation]
        gen = torch.Generator().manual_seed(seed)

        def weight(n, k):
            return (torch.randn(n, k, generator=gen) * k ** -0.5).to(device=device, dtype=self.type)

        self.w: List[Dict[str, torch.Tensor]] = [
            {"gate": weight(d_hidden, d), "up": weight(d_hidden, d), "down": weight(d, d_hidden)} for _ in range(layers)]
        ones = lambda: torch.ones(d, dtype=torch.float32, device=device)
        self.pre = [ones() for _ in range(layers + 1)]          # of h_0 .. h_L
        self.post = [ones() for _ in range(layers)]
        self.gate = [torch.full((1, d), 0.5, dtype=self.type, device=device) for _ in range(layers)]
        self.first = K.make_norm_desc(d, self.code, K.SC_NORM_NONE, K.SC_NORM_RMS, EPS)
        self.between = K.make_norm_desc(d, self.code, K.SC_NORM_RMS, K.SC_NORM_RMS, EPS)
        self.ffn = K.make_ffn_desc(d, d_hidden, d, self.code, self.activation)

    def _rows_buffer(self, rows: int, like: torch.Tensor) -> torch.Tensor:
        return torch.empty(rows, self.d, dtype=self.type, device=like.device)

    def forward(self, x: torch.Tensor, rows: Optional[K.RowSet] = None, training: bool = True) -> torch.Tensor:
        """h_L of the kept tokens; x_L of all tokens is self.x[-1].  What backward needs stays in the object until the next forward."""
        kept = x.size(0) if rows is None else rows.kept
        compact = K.SC_ROWS_COMPACT
        stats = lambda: torch.empty(x.size(0), 4, dtype=torch.float32, device=x.device) if training else None
        self.rows, self.x, self.f, self.saved = rows, [x], [], []
        self.h, self.stats = [self._rows_buffer(kept, x)], [stats()]
        self.workspace = torch.empty(
            max(K.sparse_ffn_workspace_bytes(self.ffn, kept, training),
                *(K.sparse_norm_workspace_bytes(desc, x.size(0)) for desc in (self.first, self.between))),
            dtype=torch.uint8, device=x.device)
        K.sparse_norm_run(self.first, x, None, None, None, None, self.pre[0], None, None, self.h[0], h_rows=rows, stats=self.stats[0])
        for l, w in enumerate(self.w):
            self.f.append(self._rows_buffer(kept, x))
            self.saved.append(torch.empty(3, kept, self.d_hidden, dtype=self.type, device=x.device) if training else None)
            K.sparse_ffn_run(self.ffn, self.h[l], w["gate"], w["up"], w["down"], self.f[l], self.workspace, rows, compact, compact,
                             self.saved[l])
            self.x.append(torch.empty_like(x))
            self.h.append(self._rows_buffer(kept, x))
            self.stats.append(stats())
            K.sparse_norm_run(self.between, self.x[l], self.f[l], self.gate[l], self.post[l], None, self.pre[l + 1], None,
                              self.x[l + 1], self.h[l + 1], f_rows=rows, h_rows=rows, stats=self.stats[l + 1])
        return self.h[-1]

    def backward(self, dh: torch.Tensor, dx: Optional[torch.Tensor] = None):
        """Gradients for that of h_L (and of x_L): (of x_0, [of layer l's parameters by name], of pre[0]).  After forward(training=True)."""
        rows, compact = self.rows, K.SC_ROWS_COMPACT
        grads: List[Dict[str, torch.Tensor]] = []
        for l in reversed(range(self.layers)):
            w, into = self.w[l], torch.empty_like(self.x[l])
            g = {name: torch.empty_like(t) for name, t in w.items()}
            g.update(post=torch.empty_like(self.post[l]), pre=torch.empty_like(self.pre[l + 1]),
                     branch=torch.empty_like(self.gate[l]))
            df = torch.empty_like(self.f[l])
            K.sparse_norm_backward(self.between, self.x[l], self.f[l], self.gate[l], self.post[l], None, self.pre[l + 1],
                                   self.stats[l + 1], dx, dh, into, df, g["branch"], g["post"], None, g["pre"], None, self.workspace,
                                   f_rows=rows, h_rows=rows)
            dh = torch.empty_like(df)
            K.sparse_ffn_backward(self.ffn, self.h[l], w["gate"], w["up"], w["down"], self.saved[l], df, dh, g["gate"], g["up"],
                                  g["down"], self.workspace, rows, compact, compact)
            dx = into
            grads.insert(0, g)
        first = torch.empty_like(self.pre[0])
        K.sparse_norm_backward(self.first, self.x[0], None, None, None, None, self.pre[0], self.stats[0], dx, dh, dx, None, None, None,
                               None, first, None, self.workspace, h_rows=rows)
        return dx, grads, first

    def step(self, grads, first, rate: float):
        """Plain gradient descent."""
        for l, g in enumerate(grads):
            for name, t in {**self.w[l], "post": self.post[l], "pre": self.pre[l + 1], "branch": self.gate[l]}.items():
                t.sub_(g[name], alpha=rate)
        self.pre[0].sub_(first, alpha=rate)


def quantise(w: torch.Tensor, group: int) -> Dict[str, torch.Tensor]:
    """4-bit codes with a scale and a zero point for every `group` columns of a row (rounded to the nearest of 16 steps)."""
    n, k = w.shape
    groups = -(-k // group)
    v = torch.nn.functional.pad(w.float(), (0, groups * group - k)).view(n, groups, group)
    low, high = v.amin(2).clamp(max=0), v.amax(2).clamp(min=0)
    scale = ((high - low) / 15).clamp(min=2.0 ** -14).to(w.dtype)       # (a normal number in 16 bits; all-zero groups)
    zero = (-low / scale.float()).to(w.dtype)
    code = (v / scale.float()[..., None] + zero.float()[..., None]).round().clamp(0, 15).to(torch.uint8).view(n, -1)[:, :k]
    code = torch.nn.functional.pad(code, (0, k % 2))
    return {"codes": (code[:, 0::2] | (code[:, 1::2] << 4)).contiguous(), "scales": scale, "zeros": zero}


class FeedForwardServer:
    """The same stack for a few tokens at a time, products from 4-bit weights laid out once; fixed buffers, so it can be captured."""

    def __init__(self, stack: FeedForwardStack, tokens: int, group: int = 128):
        if stack.type == torch.float32:
            raise ValueError("4-bit products take f16 or bf16")
        self.stack = stack
        desc_up = K.make_q4_desc(stack.d, stack.d_hidden, group, stack.code)
        desc_down = K.make_q4_desc(stack.d_hidden, stack.d, group, stack.code)
        self.matrices = [{name: quantise(t, group) for name, t in w.items()} for w in stack.w]
        self.up = [K.sparse_q4_plan_gated(desc_up, m["gate"], m["up"], stack.activation) for m in self.matrices]
        self.down = [K.sparse_q4_plan(desc_down, **m["down"]) for m in self.matrices]
        like = stack.w[0]["gate"]
        self.x = torch.zeros(tokens, stack.d, dtype=like.dtype, device=like.device)      # in
        self.h = torch.empty_like(self.x)                                                # out
        self._x, self._f = torch.empty_like(self.x), torch.empty_like(self.x)
        self._hidden = torch.empty(tokens, stack.d_hidden, dtype=like.dtype, device=like.device)

    def run(self) -> torch.Tensor:
        s = self.stack
        K.sparse_norm_run(s.first, self.x, None, None, None, None, s.pre[0], None, None, self.h)
        x = self.x
        for l in range(s.layers):
            K.sparse_q4_run(self.up[l], self.h, self._hidden)
            K.sparse_q4_run(self.down[l], self._hidden, self._f)
            K.sparse_norm_run(s.between, x, self._f, s.gate[l], s.post[l], None, s.pre[l + 1], None, self._x, self.h)
            x = self._x
        return self.h

    def capture(self) -> torch.cuda.CUDAGraph:
        self.run()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            self.run()
        return graph


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--tokens", type=int, default=64 * 196)
    ap.add_argument("--width", type=int, default=768)
    ap.add_argument("--hidden", type=int, default=2048)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--sparsity", type=float, default=0.5)
    ap.add_argument("--dtype", choices=("bf16", "f16", "f32"), default="bf16")
    ap.add_argument("--steps", type=int, default=8)
    a = ap.parse_args()
    gen = torch.Generator().manual_seed(1)
    stack = FeedForwardStack(a.width, a.hidden, a.layers, a.dtype)
    x = torch.randn(a.tokens, a.width, generator=gen).to("cuda:0", stack.type)
    mask = (torch.rand(a.tokens, generator=gen) >= a.sparsity).to(torch.uint8).to("cuda:0")
    rows = K.sparse_rows_plan(mask)
    listed = K.sparse_rows_info(rows)[2].long()
    want = torch.tanh(2.0 * x[listed].float())                  # synthetic target: a function of the token
    print(f"{a.layers} halves {a.width} -> {a.hidden} -> {a.width}, {a.dtype}, {rows.kept} of {rows.rows} tokens kept")
    for step in range(a.steps):
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        error = stack.forward(x, rows).float() - want
        grads = stack.backward((error * (2.0 / rows.kept)).to(stack.type))[1:]
        end.record()
        stack.step(*grads, rate=0.05)
        end.synchronize()
        print(f"step {step}: loss {error.square().sum(1).mean().item():.4f}, forward and backward {begin.elapsed_time(end) * 1e3:.0f} us")
    if stack.type == torch.float32:
        return
    server = FeedForwardServer(stack, 1)
    graph = server.capture()
    server.x.copy_(x[:1])
    graph.replay()
    full = stack.forward(server.x, training=False)
    rel = ((server.h.float() - full.float()).norm() / full.float().norm()).item()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(200):
        graph.replay()
    end.record()
    end.synchronize()
    print(f"one token from 4-bit weights: {begin.elapsed_time(end) * 5:.1f} us, {rel:.3f} away from the full weights")


if __name__ == "__main__":
    main()
