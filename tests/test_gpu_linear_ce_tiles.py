"""The cross-entropy of a linear layer in every tile of its kernels, and in several pieces of the classes with packed operands, against 64 bits on the GPU.

Tolerances as in test_gpu_linear_ce.py, with what a sum is made of: a workgroup's share of the contraction, n terms in chains of n / 16, then the shares and the pieces one after another.  G in one fp16 term is
off by half a step, 2^-11 of itself (11 bits: fp16's eps is 2^-10), or by 2^-39 (two terms: by 2^-22), and so is x times a weight.  Half of every row's probability lies in the first and the last classes, so that a piece's, a tile's or a row's end that goes missing
misses by far more."""
import math

import pytest

import paper_2405_10951_amd as P
from linear_ce_sizes import PIECES, TILES

pytestmark = pytest.mark.gpu
HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device")
    return torch


def make(torch, N, D, V, dtype, aligned):
    g = torch.Generator(device="cuda").manual_seed(N + 131 * D + 17 * V)
    kind = {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]
    ld, first = ((D + 63) // 64 * 64, 0) if aligned else (D + 5, 3)

    def rows(n, scale):
        t = torch.empty(n, ld, dtype=kind, device="cuda")
        for part in t.split(1 << 20):
            part.copy_(scale * torch.randn(part.shape, generator=g, device="cuda"))
        return t[:, first:first + D]
    x, w = rows(N, 1.0), rows(V, 2 / D ** 0.5)
    labels = torch.randint(V, (N,), generator=g, device="cuda", dtype=torch.int32)
    labels[2::7] = V - 1 - labels[2::7] % min(V, 100)
    if N > 4:
        labels[4::9] = -1
    bias = 0.5 * torch.randn(V, generator=g, device="cuda")
    if V > 1000:
        bias[:100] += math.log(V / 200)
        bias[-100:] += math.log(V / 200)
    return x, w, labels, bias


class Reference:
    """loss and G in 64 bits, and what they may be off by"""

    def __init__(self, torch, x, w, labels, bias, weight, f32, fine):
        self.torch, self.x, self.w = torch, x.double(), w.double()
        N, D = x.shape
        V = len(w)
        z = self.x @ self.w.t() + bias.double()
        some = (labels >= 0) & (labels < V)
        at = torch.where(some, labels, 0).long()
        most = z.amax(1, keepdim=True)
        ez = (D / 16 + 20) * 2.0 ** -24 * (self.x.abs() @ self.w.abs().t())
        if f32:
            ez += 2.0 ** -39 * (self.x.abs().amax(1)[:, None] * self.w.abs().sum(1) + self.x.abs().sum(1)[:, None] * self.w.abs().amax(1))
        self.loss = torch.where(some, torch.logsumexp(z, 1) - z.gather(1, at[:, None])[:, 0], 0.0)
        self.loss_off = 2 * ez.amax(1) + 2.0 ** -20 + 2.0 ** -22 * z.abs().amax(1)
        G = torch.softmax(z, 1)
        flat = G * (2 * ez + 2.0 ** -20 * (1 + most - z))
        del ez, z
        G[torch.arange(N, device="cuda"), at] -= 1
        by = torch.where(some, weight.double(), 0.0)[:, None]
        size, rest = G.abs(), 2.0 ** -39
        self.off = {"dx": by.abs() * (flat + (2.0 ** -22 if f32 else 2.0 ** -11) * size + rest), "dw": by.abs() * (flat + (2.0 ** -22 if f32 or fine else 2.0 ** -11) * size + rest),
                    "db": by.abs() * (flat + 40 * 2.0 ** -24 * size)}
        self.G = G * by


def close(torch, got, want, bound, what):
    err = (got.double() - want).abs()
    assert (err <= bound + 1e-38).all(), f"{what}: {float((err / (bound + 1e-38)).max()):.3g} times the bound"


@pytest.mark.parametrize("size,want", TILES + PIECES)
def test_against_64_bits(torch, size, want):
    N, D, V, dtype, dw_type, aligned = size
    t = P.bsr_linear_ce_tiles(N, D, V, dtype, aligned, dw_type)
    f32, fine = dtype == "fp32", dtype == "bf16" and dw_type == "fp32"
    x, w, labels, bias = make(torch, N, D, V, dtype, aligned)
    weight = 0.5 + torch.rand(N, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    ref = Reference(torch, x, w, labels, bias, weight, f32, fine)
    scale = 2.0 ** -8
    new = lambda: torch.empty(V, D, dtype={"bf16": torch.bfloat16, "fp32": torch.float32}[dw_type], device="cuda")      # noqa: E731
    loss, stats = P.bsr_linear_ce_forward(x, w, labels, bias=bias)
    apart = P.bsr_linear_ce_backward(x, w, labels, stats, bias=bias, row_grad=weight, grad_scale=scale, dw=new())
    both = P.bsr_linear_ce_forward_backward(x, w, labels, bias=bias, row_grad=weight, grad_scale=scale, dw=new())
    plain = P.bsr_linear_ce_backward(x, w, labels, stats, bias=bias, row_grad=weight, grad_scale=scale, dw=new(), need_db=False)
    for got in (loss, both[0]):
        close(torch, got, ref.loss, ref.loss_off, "loss")
    assert torch.equal(plain[0], apart[0]) and torch.equal(plain[1], apart[1])
    # (the operand beside G: exact in bf16, but for weights; two terms and the product left out in fp32, and of a weighted x)
    chain = V / max(t.pieces * t.splits_x, 1) / 16 + 60 + t.pieces + t.splits_x
    size_ = ref.G.abs() @ ref.w.abs()
    exact = ref.G @ ref.w
    bound = ref.off["dx"] @ ref.w.abs() + ((2.0 ** -21 if f32 else 0) + chain * 2.0 ** -24) * size_ + 2.0 ** -39 * ref.G.abs().sum(1, keepdim=True) * ref.w.abs().amax(0) + HALF[dtype] * exact.abs()
    for got in (apart[0], both[1]):
        close(torch, got, scale * exact, scale * bound, "dx")
    del size_, exact, bound
    chain = (3 if fine else 1) * N / max(t.splits_w, 1) / 16 + 60 + t.splits_w
    size_ = ref.G.t().abs() @ ref.x.abs()
    exact = ref.G.t() @ ref.x
    beside = 2.0 ** -21 if f32 or fine else 2.0 ** -11
    some = ref.G.abs().sum(1) > 0
    bound = ref.off["dw"].t() @ ref.x.abs() + (beside + chain * 2.0 ** -24) * size_ + 2.0 ** -38 * ref.G.abs().sum(0)[:, None] * (ref.x.abs() * some[:, None]).amax(0) + HALF[dw_type] * exact.abs()
    for got in (apart[1], both[2]):
        close(torch, got, scale * exact, scale * bound, "dw")
    exact, bound = ref.G.sum(0), ref.off["db"].sum(0)
    for got in (apart[2], both[3]):
        close(torch, got, scale * exact, scale * bound, "db")
