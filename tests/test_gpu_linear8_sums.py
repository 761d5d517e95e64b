"""How the products of 8-bit blocks are added, on operands with outliers: pairs of the largest products that cancel, among products of 7.5, just under 2^-13 of the largest's power of two, 2^16.

Bound of the exact sums, from the arithmetic: the matrix instructions take at least eight products at a time and add them to 24 bits of the largest, and those sums
one after the other in fp32, as do the wavefronts that share a sum (at most eight): (K / 8 + 32) 2^-23 sum|a w|, plus 2^-8 of the result where that is bf16 (twice half an ulp).
Of the cut sums: each product is off by less than 2^-13 of the largest of its block of 128, and the blocks are added in fp32."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device")
    import paper_2405_10951_amd as P
    return torch, P


def operands(torch, M, K, N, cancel):
    """x [M,K], w [K,N], all of them e4m3 values at scale 1: 448 x (+-448) once or twice in every eight columns, 3 x 2.5 = 7.5 elsewhere, the signs of rows and
    columns at random"""
    x, w = torch.full((M, K), 3.0), torch.full((K, N), 2.5)
    x[:, ::8], w[::8] = 448.0, 448.0
    if cancel:
        x[:, 1::8], w[1::8] = 448.0, -448.0
    g = torch.Generator().manual_seed(M + K + N)
    x *= torch.randint(0, 2, (M, 1), generator=g) * 2 - 1
    w *= torch.randint(0, 2, (1, N), generator=g) * 2 - 1
    return x, w


# few rows (one and two tiles of 16), few tiles whose sums are shared, many tiles, sums that end inside a block
CASES = [(5, 768, 64), (20, 4096, 100), (33, 1024, 64), (100, 4096, 128), (70, 768, 96), (300, 776, 1030), (2100, 1024, 1100), (1000, 384, 640)]


@pytest.mark.parametrize("cancel", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N", CASES)
def test_outliers_take_nothing_with_them(env, M, K, N, dtype, cancel):
    torch, P = env
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    x, w = operands(torch, M, K, N, cancel)
    ref = x.double().numpy() @ w.double().numpy()
    bound = (K / 8 + 32) * 2.0 ** -23 * (np.abs(x.double().numpy()) @ np.abs(w.double().numpy())) + (2.0 ** -8 * np.abs(ref) if dtype == "bf16" else 0.0)
    layer = P.bsr_quantize8_weight(w.cuda())
    for rows in (x.to(dt).cuda(), P.bsr_quantize8_rows(x.cuda())):
        y = P.bsr_linear8_forward(rows, layer, out_dtype=dt).double().cpu().numpy()
        assert (np.abs(y - ref) <= bound).all(), f"{(np.abs(y - ref) / bound).max():.3g} times the bound"
    back = P.bsr_quantize8_weight(w.t().contiguous().cuda())
    dx = P.bsr_linear8_dgrad(x.to(dt).cuda(), back).double().cpu().numpy()
    assert (np.abs(dx - ref) <= bound).all()


@pytest.mark.parametrize("M,K,N", CASES + [(100, 100, 70), (4160, 1536, 2100)])
def test_cut_sums_keep_their_bound(env, M, K, N):
    """asked for by the caller, bf16 results; and what else the product does is as ever"""
    torch, P = env
    g = torch.Generator().manual_seed(M)
    for x, w in (operands(torch, M, K, N, True), (torch.randn(M, K, generator=g), torch.randn(K, N, generator=g) / K ** 0.5)):
        rows, layer = P.bsr_quantize8_rows(x.cuda()), P.bsr_quantize8_weight(w.cuda())
        bias, res = torch.randn(N, generator=g).cuda(), torch.randn(M, N, generator=g).bfloat16().cuda()
        # the fp32 results are the exact sums (the test above), and good to 1 / 8 of the cut
        exact = P.bsr_linear8_forward(rows, layer, bias, out_dtype=torch.float32).double()
        v, e = rows.values.view(torch.float8_e4m3fn).double(), torch.exp2(rows.scales.double() - 127).repeat_interleave(128, 1)
        a = (v * e[:, :v.shape[1]]).abs()
        v, e = layer.values.view(torch.float8_e4m3fn).double(), torch.exp2(layer.scales.double() - 127).repeat_interleave(128, 1).repeat_interleave(128, 0)
        b = (v * e[:N, :v.shape[1]]).abs()
        size = sum(a[:, k:k + 128].amax(1)[:, None] * b[:, k:k + 128].amax(1)[None] for k in range(0, K, 128))
        bound = 1.125 * 2.0 ** -6 * size + 1e-30
        for how, ref in ((dict(), exact), (dict(res=res), exact + res.double())):
            y = P.bsr_linear8_forward(rows, layer, bias, out_dtype=torch.bfloat16, cut_sums=True, **how).double()
            assert bool(((y - ref).abs() <= bound + 2.0 ** -7 * ref.abs()).all())


def test_cut_sums_on_random_rows_and_with_gelu(env):
    """random data, where the cut takes 3e-5 of the size of a sum (the root of its sum of squares, 1 here) on the mean: within 2^-10, thirty times that"""
    torch, P = env
    g = torch.Generator().manual_seed(1)
    M, K, N = 1000, 1536, 512
    x, layer = P.bsr_quantize8_rows(torch.randn(M, K, generator=g).cuda()), P.bsr_quantize8_weight((torch.randn(K, N, generator=g) / K ** 0.5).cuda())
    u, uc = (torch.empty(M, N, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    P.bsr_linear8_forward(x, layer, act=1, u_out=u)
    P.bsr_linear8_forward(x, layer, act=1, u_out=uc, cut_sums=True)
    assert bool(((u.float() - uc.float()).abs() <= 2.0 ** -10 + 2.0 ** -7 * u.float().abs()).all())
    dy = torch.randn(M, N, generator=g).cuda()
    a, b = (P.bsr_linear8_dgrad(dy, layer, u=torch.randn(M, K, generator=torch.Generator().manual_seed(2)).bfloat16().cuda(), out_dtype=torch.bfloat16, cut_sums=c).float()
            for c in (False, True))
    assert bool(((a - b).abs() <= 2.0 ** -10 + 2.0 ** -7 * a.abs()).all())


def test_cut_sums_refused(env):
    torch, P = env
    x, layer = torch.randn(40, 64, device="cuda"), P.bsr_quantize8_weight(torch.randn(64, 32, device="cuda"))
    with pytest.raises(ValueError):
        P.bsr_linear8_forward(x, layer, cut_sums=True)
    with pytest.raises(ValueError):
        P.bsr_linear8_dgrad(torch.randn(40, 32, device="cuda"), layer, cut_sums=True)
