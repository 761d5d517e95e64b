"""RMSNorm, the 8-bit layers, the cross-entropy of the head and the clipping run together, as a program that tunes a head runs them: loss and gradients against the same model in 64 bits
(8-bit blocks by their definition, their rounding the identity for gradients).

Tolerance: as for the norms of a frozen stack (tests/test_gpu_norm_tuning.py).  A value that bf16 moves by 2^-9 crosses a boundary of the 8-bit grid in 2 - 3 % of all cases and is then off by up to
6 %, 1 % in the root mean square of a tensor; eight such tensors lie behind one another here: 3 % in quadrature, held to twice that in the 2-norm of every gradient, and 2 % for the loss."""
import numpy as np
import pytest

from reference8 import blocks8

pytestmark = pytest.mark.gpu


def model_and_inputs(torch, rows, width, hidden, classes, depth, seed=0):
    from paper_2405_10951_amd.head_tuning import TunedHead
    g = torch.Generator().manual_seed(seed)

    def normal(*shape, scale=1.0):
        return (scale * torch.randn(*shape, generator=g)).bfloat16().float()

    blocks = [(normal(width, hidden, scale=width ** -0.5), normal(hidden, scale=0.1), normal(hidden, width, scale=hidden ** -0.5), normal(width, scale=0.1)) for _ in range(depth)]
    head = (normal(classes, width, scale=2 * width ** -0.5), normal(classes, scale=0.1))
    model = TunedHead([tuple(t.cuda() for t in b) for b in blocks], tuple(t.cuda() for t in head))
    for gain in model.gains:
        gain += (0.1 * torch.randn(width, generator=g)).cuda()
    labels = torch.randint(classes, (rows,), generator=g, dtype=torch.int32)
    labels[3] = -1
    return model, blocks, head, normal(rows, width), labels


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device")
    return torch


@pytest.mark.parametrize("rows,width,hidden,classes,depth", [(70, 256, 384, 200, 2), (20, 130, 100, 1001, 1)])
def test_step_against_64_bits(torch, rows, width, hidden, classes, depth):
    from paper_2405_10951_amd.head_tuning import EPS
    model, blocks, head, x, labels = model_and_inputs(torch, rows, width, hidden, classes, depth)

    def eight(v):                                        # straight through
        return v + (torch.from_numpy(np.ascontiguousarray(blocks8(v.detach().numpy(), 1, 128)[0])) - v).detach()

    def frozen(w):                                       # gradients pass a frozen layer in 8 bits as well
        wq = torch.from_numpy(blocks8(w.double().numpy(), 128, 128)[0])

        class Layer(torch.autograd.Function):
            @staticmethod
            def forward(ctx, v):
                return v @ wq

            @staticmethod
            def backward(ctx, d):
                return torch.from_numpy(blocks8(d.numpy(), 1, 128)[0]) @ wq.t()
        return Layer.apply

    def norm(v, gain):
        return v / torch.sqrt(v.pow(2).mean(1, keepdim=True) + EPS) * gain

    gains = [p.double().cpu().requires_grad_() for p in model.gains]
    weight, bias = (t.double().requires_grad_() for t in head)
    h = x.double()
    for (w1, b1, w2, b2), gain in zip(blocks, gains):
        h = h + frozen(w2)(eight(torch.nn.functional.gelu(frozen(w1)(eight(norm(h, gain))) + b1.double()))) + b2.double()
    loss = torch.nn.functional.cross_entropy(norm(h, gains[-1]) @ weight.t() + bias, labels.long(), ignore_index=-1, reduction="none")
    want = torch.autograd.grad(loss.sum() / rows, gains + [weight, bias])
    got_loss, grads, _ = model.step(x.bfloat16().cuda(), labels.cuda())
    assert abs(got_loss.mean().item() / (loss.sum() / rows).item() - 1) < 2e-2 and got_loss[3] == 0
    for i, (got, ref) in enumerate(zip(grads, want)):
        err = (got.double().cpu() - ref).norm() / ref.norm()
        assert err < 6e-2, (i, float(err))
    # clipped: the same direction, of the length asked for, and the weights follow it
    before = [p.clone() for p in model.gains + [model.weight, model.bias]]
    length = np.sqrt(sum(float(g.double().pow(2).sum()) for g in grads))
    _, clipped, norm_ = model.step(x.bfloat16().cuda(), labels.cuda(), lr=0.5, max_norm=0.5 * length)
    assert abs(float(norm_) / length - 1) < 2.0 ** -23
    for g, c, p, b in zip(grads, clipped, model.gains + [model.weight, model.bias], before):
        assert torch.allclose(c, 0.5 * g, rtol=2.0 ** -21, atol=1e-38) and torch.equal(p, b.add(c, alpha=-0.5))


@pytest.mark.parametrize("rows,classes", [(197, 3000), (12, 300)])
def test_a_step_in_a_graph(torch, rows, classes):
    """the calls of a step recorded once and replayed on new inputs, with other work between: the eager results each time"""
    from paper_2405_10951_amd.head_tuning import random_model
    model = random_model(384, 512, 2, classes)
    x = torch.randn(rows, 384, device="cuda").bfloat16()
    labels = torch.randint(classes, (rows,), device="cuda", dtype=torch.int32)
    model.step(x, labels, max_norm=0.1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s), torch.cuda.graph(graph, stream=s):
        loss, grads, norm = model.step(x, labels, max_norm=0.1)
    torch.cuda.synchronize()
    for i in range(4):
        x.copy_(torch.randn(rows, 384, device="cuda").bfloat16())
        labels.copy_(torch.randint(classes, (rows,), device="cuda", dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        ref_loss, ref, ref_norm = model.step(x, labels, max_norm=0.1)
        torch.cuda.synchronize()
        assert torch.equal(loss, ref_loss) and torch.equal(norm, ref_norm) and all(torch.equal(p, q) for p, q in zip(grads, ref))


def test_the_norm_tuning_clips(torch):
    from paper_2405_10951_amd.norm_tuning import random_stack
    x = torch.randn(64, 128, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    index = torch.arange(64 * 3, dtype=torch.int32, device="cuda").view(64, 3) % 50
    t = torch.randn(64, 3, generator=torch.Generator().manual_seed(2)).cuda()
    stack = random_stack(128, 128, 1, 50)
    _, grads = stack.step(x, index, t)
    length = float(torch.sqrt(sum(g.double().pow(2).sum() for pair in grads for g in pair)))
    _, clipped = stack.step(x, index, t, max_norm=0.25 * length)
    for a, b in zip(grads, clipped):
        assert all(torch.allclose(q, 0.25 * p, rtol=2.0 ** -21, atol=1e-38) for p, q in zip(a, b))
