"""The stack of feed-forward halves of the example: against plain torch in 64 bits, and its 4-bit form."""
import pytest
import torch

import block_oracle as O
from paper_2309_06626_amd import block as K
from paper_2309_06626_amd import block_example as X


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("shape,group", [((5, 256), 128), ((3, 100), 64), ((4, 33), 32)])
def test_codes_are_the_nearest_steps(shape, group, dtype):
    w = torch.randn(*shape, generator=torch.Generator().manual_seed(3)).to(O.TORCH[dtype])
    w[0, :group] = 0                                            # a group of zeros
    w[1] = w[1].abs()                                           # rows of one sign keep zero among their steps
    q = X.quantise(w, group)
    codes = torch.stack((q["codes"] & 15, q["codes"] >> 4), 2).view(shape[0], -1)[:, :shape[1]].double()
    of = torch.arange(shape[1]) // group
    scale, zero = q["scales"].double()[:, of], q["zeros"].double()[:, of]
    # half a step; the ends of a range lie within 15 * 2^-8 steps for the scale's rounding and as much for the zero point's
    assert (((codes - zero) * scale - w.double()).abs() <= 0.501 * scale).all()


def plain(x, keep, w, pre, post, gate, kind):
    """h_L and x_L in the type of the inputs; w: [(gate, up, down)]."""
    rows = keep.nonzero()[:, 0]
    norm = lambda v, g: v / torch.sqrt((v * v).mean(-1, keepdim=True) + X.EPS) * g
    h = norm(x[rows], pre[0])
    for (wg, wu, wd), post_l, gate_l, pre_l in zip(w, post, gate, pre[1:]):
        x = x.index_add(0, rows, gate_l * norm(O.ffn_forward(h, wg, wu, wd, kind), post_l))
        h = norm(x[rows], pre_l)
    return h, x


@pytest.mark.gpu
def test_stack_and_its_gradients():
    # float: 12 passes through a product of up to n = 200, each off by at most acc(n) of the sum of absolute values, which is about
    # 0.8 sqrt(n) times the result for random signs: 12 * 3.6e-6 * 11 = 4.8e-4 of a tensor's norm
    stack = X.FeedForwardStack(72, 200, 2, "f32", "gelu", seed=5)
    gen = torch.Generator().manual_seed(7)
    x, keep = torch.randn(301, 72, generator=gen), torch.rand(301, generator=gen) < 0.6
    for t in (*stack.pre, *stack.post):
        t.copy_(1 + 0.3 * torch.randn(72, generator=gen))
    rows = K.sparse_rows_plan(keep.to(torch.uint8).cuda())
    h = stack.forward(x.cuda(), rows)
    dh, dx = torch.randn(rows.kept, 72, generator=gen), torch.randn(301, 72, generator=gen)
    got_dx, grads, first = stack.backward(dh.cuda(), dx.cuda())

    leaf = lambda t: t.detach().double().cpu().requires_grad_(True)
    w = [tuple(leaf(m[name]) for name in ("gate", "up", "down")) for m in stack.w]
    pre, post, gate, x64 = [leaf(t) for t in stack.pre], [leaf(t) for t in stack.post], [leaf(t) for t in stack.gate], leaf(x)
    want, x_last = plain(x64, keep, w, pre, post, gate, "gelu")
    ((want * dh.double()).sum() + (x_last * dx.double()).sum()).backward()
    pairs = {"h": (h, want.detach()), "x": (stack.x[-1], x_last.detach()), "dx": (got_dx, x64.grad), "pre 0": (first, pre[0].grad)}
    for l, g in enumerate(grads):
        pairs.update({f"{name} {l}": (g[name], w[l][i].grad) for i, name in enumerate(("gate", "up", "down"))})
        pairs.update({f"post {l}": (g["post"], post[l].grad), f"pre {l + 1}": (g["pre"], pre[l + 1].grad),
                      f"branch {l}": (g["branch"], gate[l].grad)})
    for name, (a, b) in pairs.items():
        assert (a.double().cpu() - b).norm() <= 4.8e-4 * b.norm(), name


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [1, 3])
def test_server_against_its_own_weights_and_in_a_graph(tokens):
    # f16: h, hidden rows, f and x are rounded in each of two halves, and hidden rows are of second degree in h:
    # 2 * 5 * 2^-11 = 5e-3 of the result's norm, twice that for the norms' and activations' slopes
    stack = X.FeedForwardStack(160, 320, 2, "f16", "silu", seed=9)
    server = X.FeedForwardServer(stack, tokens, 32)
    graph = server.capture()

    def full(m):
        codes = torch.stack((m["codes"] & 15, m["codes"] >> 4), 2).flatten(1).double()
        wide = lambda t: t.double().repeat_interleave(32, 1)
        return ((codes - wide(m["zeros"])) * wide(m["scales"])).cpu()

    w = [tuple(full(m[name]) for name in ("gate", "up", "down")) for m in server.matrices]
    wide = lambda ts: [t.double().cpu() for t in ts]
    for seed in range(3):
        x = torch.randn(tokens, 160, generator=torch.Generator().manual_seed(seed))
        server.x.copy_(x)
        eager = server.run().clone()
        torch.cuda.synchronize()
        server.h.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(server.h, eager)
        want = plain(server.x.double().cpu(), torch.ones(tokens, dtype=torch.bool), w, wide(stack.pre), wide(stack.post),
                     wide(stack.gate), "silu")[0]
        assert (eager.double().cpu() - want).norm() <= 1e-2 * want.norm()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_training_reduces_the_loss(dtype):
    stack = X.FeedForwardStack(64, 128, 2, dtype, seed=1)
    x = torch.randn(500, 64, generator=torch.Generator().manual_seed(2)).to("cuda", stack.type)
    rows = K.sparse_rows_plan((torch.arange(500, device="cuda") % 3 != 0).to(torch.uint8))
    target = torch.tanh(2 * x[K.sparse_rows_info(rows)[2].long()].float())
    losses = []
    for _ in range(6):
        error = stack.forward(x, rows).float() - target
        losses.append(error.square().sum(1).mean().item())
        stack.step(*stack.backward((error * (2 / rows.kept)).to(stack.type))[1:], rate=0.05)
    assert all(b < a for a, b in zip(losses, losses[1:]))


@pytest.mark.gpu
def test_a_mask_that_keeps_nothing_trains_nothing():
    stack = X.FeedForwardStack(64, 128, 2, "bf16", seed=1)
    x = torch.randn(50, 64, generator=torch.Generator().manual_seed(2)).to("cuda", stack.type)
    rows = K.sparse_rows_plan(torch.zeros(50, dtype=torch.uint8, device="cuda"))
    h = stack.forward(x, rows)
    assert h.shape == (0, 64) and torch.equal(stack.x[-1], x)
    dx, grads, first = stack.backward(torch.empty_like(h))
    for t in (dx, first, *(t for g in grads for t in g.values())):
        assert (t == 0).all()
