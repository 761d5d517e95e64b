"""The cross-entropy of a linear layer on both sides of every number at which it goes another way, against 64 bits (tolerances: test_gpu_linear_ce.py)."""
import pytest

from test_gpu_linear_ce import check, make

pytestmark = pytest.mark.gpu

# (rows, width, classes): classes whose gradients take two launches; those whose rows have 1024 threads, and that a launch of its own turns; those from which workgroups take two times 16 of them, beside rows of up to 256 bytes
# and longer ones; rows in tiles of 16, 32 and 64; little work by products, and by tiles; logits that are kept between the passes; tiles of rows that one thread or several add up for db
SIZES = [(20, 100, 128), (20, 100, 129), (20, 100, 256), (20, 100, 257), (20, 70, 4096), (20, 70, 4097), (20, 70, 32768), (20, 70, 32769), (17, 64, 8191), (17, 64, 8192), (17, 65, 8192), (40, 128, 8192), (40, 129, 8192), (33, 64, 8200),
         (32, 130, 8200), (1, 63, 8192), (16, 300, 8193), (500, 40, 8192), (65, 100, 8193), (64, 200, 700), (65, 200, 700), (300, 200, 2000), (300, 448, 2000), (256, 1024, 512), (256, 1024, 1030), (512, 576, 1024),
         (500, 512, 8384), (500, 512, 8392), (600, 448, 3000), (960, 64, 2200), (1025, 64, 2200)]


@pytest.fixture(scope="module")
def env():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device")
    import paper_2405_10951_amd as P
    return torch, P


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,D,V", SIZES)
def test_against_64_bits(env, N, D, V, dtype):
    torch, P = env
    for extra, first in ((-D % 64, 0), (3, 1)):
        x, w, labels, b = make(torch, N, D, V, dtype, 80, extra, first)
        weight = (0.5 + torch.rand(N, generator=torch.Generator().manual_seed(81))).cuda()
        loss, _, dx, dw, db = check(torch, P, x, w, labels, b, dtype, row_grad=weight, grad_scale=0.5)
        both = P.bsr_linear_ce_forward_backward(x, w, labels, bias=b, row_grad=weight, grad_scale=0.5)
        # in one call logits may be added in another order, and the results rounded the other way
        half = {"bf16": 2.0 ** -8, "f32": 2.0 ** -13}[dtype]
        assert (both[0] - loss).abs().max() <= 2.0 ** -13
        for got, want in zip(both[1:], (dx, dw, db)):
            assert (got.double() - want.double()).norm() <= half * want.double().norm()
