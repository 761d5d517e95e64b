"""GELU and its derivative behind a frozen linear layer in 8 bits, at chosen points: the product is nothing but the bias, or 1.

Bounds.  To fp32: u / sqrt(2) is rounded, which moves erfc(x) by 2 x^2 2^-24 = u^2 2^-24 of itself at most, with the product's own rounding twice that; erfc may be 16 units off in its
last place (2^-23), exp 3, and a handful of roundings: |u| Phi (u^2 + 20) 2^-23, and |u| phi (u^2 + 12) 2^-23 for the Gaussian; below 1e-37 nothing is promised.  To bf16: Phi within 5e-7,
2^-8 of the result for its rounding."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def points(torch):
    return torch.cat([torch.linspace(-13, 13, 4001), torch.tensor([0.0, -0.0, 1e-20, -1e-20, 30.0, -30.0, 1e4, -1e4])])


def phi(u):
    from scipy.special import erfc
    return 0.5 * erfc(-u / np.sqrt(2))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M", [3, 20, 64, 300])
def test_gelu_and_its_derivative(M, dtype):
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device")
    import paper_2405_10951_amd as P
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    at = points(torch).to(dt)
    N = len(at)
    layer = P.bsr_quantize8_weight(torch.randn(128, N, device="cuda"))
    u = torch.empty(M, N, dtype=dt, device="cuda")
    y = P.bsr_linear8_forward(torch.zeros(M, 128, device="cuda"), layer, bias=at.float().cuda(), act=1, u_out=u, out_dtype=dt)
    assert torch.equal(u, at.cuda().expand(M, N))
    ones = torch.zeros(N, 128)
    ones[:, 0] = 1
    dy = torch.zeros(M, 128, device="cuda")
    dy[:, 0] = 1
    dx = P.bsr_linear8_dgrad(dy, P.bsr_quantize8_weight(ones.cuda()), u=u, out_dtype=dt)
    assert torch.equal(y, y[:1].expand(M, N)) and torch.equal(dx, dx[:1].expand(M, N))
    v = at.double().numpy()
    p, gauss = phi(v), np.exp(-v * v / 2) / np.sqrt(2 * np.pi)
    sizes = np.abs(p), np.abs(v * gauss)
    if dtype == "f32":
        bounds = np.abs(v) * p * (v * v + 20) * 2.0 ** -23 + 1e-37, (sizes[0] * (v * v + 20) + sizes[1] * (v * v + 12)) * 2.0 ** -23 + 1e-37
    else:
        bounds = (5e-7 * np.abs(v) + 2.0 ** -8 * np.abs(v * p) + 1e-37), (1e-6 + 1e-6 * np.abs(v * gauss) + 2.0 ** -8 * np.abs(p + v * gauss))
    for got, want, bound in ((y, v * p, bounds[0]), (dx, p + v * gauss, bounds[1])):
        err = np.abs(got[0].double().cpu().numpy() - want)
        assert (err <= bound).all(), f"{(err / bound).max():.3g} times the bound at {v[np.argmax(err / bound)]}"
