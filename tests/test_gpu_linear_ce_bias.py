"""The bias's gradient of the cross-entropy of a linear layer over many rows: a sum over rows whose error does not grow with their number.

Tolerances, from the arithmetic.  A logit is off by e_z = (D / 16 + 20) 2^-24 of the sum of its terms' sizes (fp32 operands: and the bounds of their two terms), a probability by a factor
1 + 2 e_z + 2^-20 (1 + the distance to the maximum).  A tile's rows are added up in fp32, 256 at most in chains of 16 and a tree: 24 additions at most.  What follows is 15 further ones in fp32, or a
sum in fp64 rounded once: 40 2^-24 of the terms' sizes in all."""
import pytest

from test_gpu_linear_ce import make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device")
    import paper_2405_10951_amd as P
    return torch, P


def check(torch, x, w, labels, bias, weight, got, rows=1):
    """rows: how many times each row counts"""
    N, D = x.shape
    V = len(w)
    want, bound = torch.zeros(V, dtype=torch.float64, device="cuda"), torch.zeros(V, dtype=torch.float64, device="cuda")
    wd = w.double()
    for at in range(0, N, 1 << 15):
        part = slice(at, min(N, at + (1 << 15)))
        xd, ld = x[part].double(), labels[part]
        z = xd @ wd.t() + bias.double()
        some = (ld >= 0) & (ld < V)
        by = torch.where(some, 1.0 if weight is None else weight[part].double(), 0.0)[:, None]
        p = torch.softmax(z, 1)
        G = p.clone()
        G[torch.arange(len(xd), device="cuda"), torch.where(some, ld, 0).long()] -= 1
        ez = (D / 16 + 20) * 2.0 ** -24 * (xd.abs() @ wd.abs().t())
        if x.dtype is torch.float32:
            ez = ez + 2.0 ** -39 * (xd.abs().amax(1)[:, None] * wd.abs().sum(1) + xd.abs().sum(1)[:, None] * wd.abs().amax(1))
        off = p * (2 * ez + 2.0 ** -20 * (1 + z.amax(1, keepdim=True) - z)) + 40 * 2.0 ** -24 * G.abs()
        want += rows * (by * G).sum(0)
        bound += rows * (by.abs() * off).sum(0)
    err = (got.double() - want).abs()
    assert (err <= bound).all(), f"{float((err / bound).max()):.3g} times the bound"


@pytest.mark.parametrize("dtype,N", [("bf16", 1 << 22), ("bf16", (1 << 21) + 77), ("f32", 1 << 21)])
def test_rows_all_alike(env, dtype, N):
    """so that every addition to a long sum in fp32 would be rounded the same way"""
    torch, P = env
    x, w, _, b = make(torch, 1, 8, 12, dtype, 70)
    labels = torch.zeros(N, device="cuda", dtype=torch.int32)
    rows = x.expand(N, 8).contiguous()
    _, stats = P.bsr_linear_ce_forward(rows, w, labels, bias=b)
    _, _, db = P.bsr_linear_ce_backward(rows, w, labels, stats, bias=b, need_dx=False, need_dw=False)
    check(torch, x, w, labels[:1], b, None, db, rows=N)


# around the numbers of tiles of rows from which several threads share the sum
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,D,V", [(900, 64, 9000), (960, 300, 2000), (1025, 64, 21), (1920, 64, 4001), (2049, 100, 4002), (4097, 64, 3), (32700, 64, 70), (65537, 8, 130), (131073, 16, 9)])
def test_numbers_of_rows(env, N, D, V, dtype):
    torch, P = env
    x, w, labels, b = make(torch, N, D, V, dtype, 71)
    weight = (0.5 + torch.rand(N, generator=torch.Generator().manual_seed(72))).cuda()
    _, dx, dw, db = P.bsr_linear_ce_forward_backward(x, w, labels, bias=b, row_grad=weight)
    check(torch, x, w, labels, b, weight, db)
    _, _, _, plain = P.bsr_linear_ce_forward_backward(x, w, labels, bias=b, need_dx=False, need_dw=False)
    check(torch, x, w, labels, b, None, plain)
