"""The operators run together, as a program that tunes the norms of a frozen stack runs them: loss and gradients against the same model in 64 bits
(8-bit blocks by their definition, their rounding the identity for gradients).

Tolerance.  bf16 keeps 9 significand bits, e4m3 has 4: a value that bf16 moves by 2^-9 crosses a boundary of the 8-bit grid, whose cells are 2^-4 .. 2^-3 wide, in 2 - 3 % of
all cases and is then off by up to 6 %, 1 % in the root mean square of a tensor.  Ten such tensors lie behind one another here (two blocks and the head, there
and back): 3 % in quadrature, held to twice that in the 2-norm of every gradient.  The loss is a mean over rows of such errors: 2 %."""
import numpy as np
import pytest

from reference8 import blocks8

pytestmark = pytest.mark.gpu


def test_step_against_64_bits_and_a_falling_loss():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device")
    from paper_2405_10951_amd.norm_tuning import EPS, FrozenStack
    g = torch.Generator().manual_seed(0)
    rows, width, hidden, classes, depth, top, T, a = 70, 256, 384, 200, 2, 9, 2.0, 0.25

    def normal(*shape, scale=1.0):
        return (scale * torch.randn(*shape, generator=g)).bfloat16().float()

    blocks = [(normal(width, hidden, scale=width ** -0.5), normal(hidden, scale=0.1), normal(hidden, width, scale=hidden ** -0.5), normal(width, scale=0.1))
              for _ in range(depth)]
    head = (normal(width, classes, scale=2 * width ** -0.5), normal(classes, scale=0.1))
    stack = FrozenStack([tuple(t.cuda() for t in b) for b in blocks], tuple(t.cuda() for t in head))
    for gamma, beta in stack.norms:
        gamma += (0.1 * torch.randn(width, generator=g)).cuda()
        beta += (0.1 * torch.randn(width, generator=g)).cuda()
    x = normal(rows, width)
    index = torch.stack([torch.randperm(classes, generator=g)[:top] for _ in range(rows)]).int()
    t = 2 * torch.randn(rows, top, generator=g)
    labels = torch.randint(classes, (rows,), generator=g, dtype=torch.int32)
    labels[3] = -1
    index[5, 4:] = -1

    def eight(v, br):                                    # straight through
        q, _ = blocks8(v.detach().numpy(), br, 128)
        return v + (torch.from_numpy(np.ascontiguousarray(q)) - v).detach()

    norms = [[p.double().cpu().requires_grad_() for p in n] for n in stack.norms]

    def back(fwd):                                       # gradients pass a frozen layer in 8 bits as well
        class Layer(torch.autograd.Function):
            @staticmethod
            def forward(ctx, v):
                return v @ fwd

            @staticmethod
            def backward(ctx, d):
                return torch.from_numpy(blocks8(d.numpy(), 1, 128)[0]) @ fwd.t()
        return Layer.apply

    def norm(v, n):
        return torch.nn.functional.layer_norm(v, (width,), n[0], n[1], EPS)

    h = x.double()
    for (w1, b1, w2, b2), n in zip(blocks, norms):
        w1q, w2q = (torch.from_numpy(blocks8(w.double().numpy(), 128, 128)[0]) for w in (w1, w2))
        u = back(w1q)(eight(norm(h, n), 1)) + b1.double()
        h = h + back(w2q)(eight(torch.nn.functional.gelu(u), 1)) + b2.double()
    z = back(torch.from_numpy(blocks8(head[0].double().numpy(), 128, 128)[0]))(eight(norm(h, norms[-1]), 1)) + head[1].double()
    there = index >= 0
    p = torch.softmax((t.double() / T).masked_fill(~there, -np.inf), 1)
    lq = torch.log_softmax(z / T, 1).gather(1, index.clamp_min(0).long())
    loss = (1 - a) * T * T * (torch.special.xlogy(p, p) - p * lq).masked_fill(~there, 0).sum(1)
    loss = loss + a * torch.nn.functional.cross_entropy(z, labels.long(), ignore_index=-1, reduction="none")
    flat = [q for n in norms for q in n]
    want = torch.autograd.grad(loss.mean(), flat)

    args = (x.bfloat16().cuda(), index.cuda(), t.cuda(), labels.cuda())
    got_loss, grads = stack.step(*args, temperature=T, hard_weight=a)
    assert abs(got_loss.mean().item() / loss.mean().item() - 1) < 2e-2
    for i, (got, ref) in enumerate(zip([q for n in grads for q in n], want)):
        err = (got.double().cpu() - ref).norm() / ref.norm()
        assert err < 6e-2, (i, float(err))
    losses = [stack.step(*args, temperature=T, hard_weight=a, lr=0.5)[0].mean().item() for _ in range(20)]
    assert losses[-1] < losses[0] and all(np.isfinite(losses))


def test_a_step_in_a_graph():
    """the calls of a step recorded once and replayed, with other work between: the eager results each time"""
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device")
    from paper_2405_10951_amd.norm_tuning import random_stack
    stack = random_stack(384, 512, 2, 300)
    x = torch.randn(197, 384, device="cuda").bfloat16()
    index = torch.randint(300, (197, 8), device="cuda", dtype=torch.int32)
    t = torch.randn(197, 8, device="cuda")
    stack.step(x, index, t)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s), torch.cuda.graph(graph, stream=s):
        loss, grads = stack.step(x, index, t)
    torch.cuda.synchronize()
    for i in range(4):
        x.copy_(torch.randn(197, 384, device="cuda").bfloat16())
        graph.replay()
        torch.cuda.synchronize()
        ref_loss, ref = stack.step(x, index, t)
        torch.cuda.synchronize()
        assert torch.equal(loss, ref_loss) and all(torch.equal(p, q) for a, b in zip(grads, ref) for p, q in zip(a, b))
