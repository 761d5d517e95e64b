"""The gains' gradient of RMSNorm where only a few rows of many count: the rows at a launch's, a workgroup's and the tensor's ends are in the sum, once each.

Tolerance: the kernel forms dy (x rstd) in fp32, off by two roundings, 2 x 2^-24 of the term, and adds n terms (and zeros): (n + 2) 2^-24 of the terms' sizes.  Each row counts for 1 / 8 n of that sum or
more in every column, which for up to 40 rows is more than 2^10 times as much."""
import pytest

pytestmark = pytest.mark.gpu
LAUNCH = 1 << 21


@pytest.fixture(scope="module")
def env():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device")
    import paper_2405_10951_amd as P
    return torch, P


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,D", [(LAUNCH + 3, 16), (LAUNCH + 3, 5), (LAUNCH, 5), (LAUNCH + 1, 16), (2 * LAUNCH + 2, 8), (2 * LAUNCH + 2, 3), (2049, 768), (2047, 1777), (513, 8192), (1025, 20000), (4097, 7)])
def test_the_rows_at_the_ends(env, M, D, dtype):
    torch, P = env
    kind = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    g = torch.Generator(device="cuda").manual_seed(M + D)
    rows = sorted({r for c in (0, 64, 512, 1024, 2048, M // 64, LAUNCH, 2 * LAUNCH, M) for r in (c - 2, c - 1, c, c + 1) if 0 <= r < M})

    def between(*shape):                                  # 1/2 .. 1, of either sign
        v = 0.5 + 0.5 * torch.rand(*shape, generator=g, device="cuda")
        return torch.where(torch.rand(*shape, generator=g, device="cuda") < 0.5, -v, v)
    x = between(1, D).expand(M, D).to(kind).contiguous()
    at = torch.tensor(rows, device="cuda")
    x[at] = between(len(rows), D).to(kind)
    dy = torch.zeros(M, D, dtype=kind, device="cuda")
    dy[at] = between(len(rows), D).to(kind)
    gamma = 1 + 0.1 * torch.randn(D, generator=g, device="cuda")
    rstd = torch.rsqrt(x.float().square().mean(1) + 1e-6)
    terms = dy[at].double() * x[at].double() * rstd[at].double()[:, None]
    size, n = terms.abs().sum(0), len(rows)
    assert n <= 40 and (terms.abs() >= size / (8 * n)).all()
    for need_dx in (True, False):
        dx, dgamma = P.bsr_rmsnorm_backward(dy, x, rstd, gamma, need_dx=need_dx)
        assert ((dgamma.double() - terms.sum(0)).abs() <= (n + 2) * 2.0 ** -24 * size).all()
    dx, _ = P.bsr_rmsnorm_backward(dy, x, rstd, gamma, need_params=False)
    rest = torch.ones(M, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert not dx[rest].any() and (dx[at].abs().sum(1) > 0).all()
