"""Frozen linear layers in 8 bits: the quantised blocks bit for bit, the products against 64 bits.

Tolerance of a product, from the arithmetic alone: operands are exact, a product of two e4m3 values has 8 significand bits and is exact in
fp32, so an element's error is that of adding K numbers in fp32 in any order, at most K 2^-23 sum|a w| (a truncating adder counted), plus the
roundings of bias, residual and result (2^-22 of each), plus half an ulp of bf16 (2^-9) where that is the type.  The GELU's Phi is good to 1e-6."""
import numpy as np
import pytest

from reference8 import blocks8, decode

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device")
    import paper_2405_10951_amd as P
    return torch, P


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def dtypes(torch):
    return {"bf16": torch.bfloat16, "f32": torch.float32}


def check_blocks(x, r, rows_per_scale):
    """8-bit rows `r` = (values, scales) of x [M,K] (host), padding included"""
    M, K = x.shape
    ref, exps = blocks8(x, rows_per_scale, 128)
    v, s = r[0].cpu().numpy(), r[1].cpu().numpy()
    assert v.shape == (M, exps.shape[1] * 128) and s.shape == (exps.shape[0], -(-exps.shape[1] // 4) * 4)
    assert np.array_equal(s[:, :exps.shape[1]].astype(np.int64) - 127, exps)
    got = decode(v, s[:, :exps.shape[1]], rows_per_scale, K)
    assert np.array_equal(got, ref, equal_nan=True)
    assert not v[:, K:].any(), "columns behind the last one are zero"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,extra", [(1, 1, 0), (3, 127, 0), (2, 128, 0), (5, 129, 3), (7, 300, 4), (257, 768, 0), (33, 1000, 24)])
def test_rows_to_8_bits(env, M, K, extra, dtype):
    torch, P = env
    g = torch.Generator().manual_seed(M * 1000 + K)
    x = torch.randn(M, K + extra, generator=g) * torch.exp(3 * torch.randn(M, 1, generator=g))
    x = x.to(dtypes(torch)[dtype]).cuda()[:, :K]
    r = P.bsr_quantize8_rows(x)
    check_blocks(host(x), (r.values, r.scales), 1)


def special_rows(torch):
    """zeros, ties, the ends of the range, subnormals, infinities and NaN"""
    x = torch.zeros(9, 256)
    x[1, 0] = 448.0
    x[1, 1:9] = torch.tensor([17.0, 19.0, 21.0, 1.0625, 2 ** -9, 2 ** -10, 3 * 2 ** -10, -17.0])      # halfway between neighbours
    x[2, 5] = 448.0001                                    # one scale up
    x[3, :] = torch.linspace(-3.3e38, 3.3e38, 256)
    x[4, :] = 1e-44
    x[5, 7] = 1e-38
    x[6, 3], x[6, 4], x[6, 5] = float("inf"), float("nan"), 2.5
    x[7, 128:] = float("-inf")
    x[8, :] = torch.finfo(torch.float32).min
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_with_special_values(env, dtype):
    torch, P = env
    x = special_rows(torch).to(dtypes(torch)[dtype])
    r = P.bsr_quantize8_rows(x.cuda())
    check_blocks(host(x), (r.values, r.scales), 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", [256, 250])
def test_special_values_on_the_way(env, K, dtype):
    """few rows are brought to 8 bits inside the product: row i against a weight that picks columns out one by one gives the values themselves, the very
    ones that the rows in 8 bits give (and NaN where a row has one: 0 times NaN)"""
    torch, P = env
    x = special_rows(torch)[:, :K].to(dtypes(torch)[dtype]).cuda()
    x = torch.cat([x, torch.randn(5, K, device="cuda").to(x.dtype), 1e-3 * torch.randn(2, K, device="cuda").to(x.dtype)])
    layer = P.bsr_quantize8_weight(torch.eye(K, device="cuda"))
    a = P.bsr_linear8_forward(x, layer, out_dtype=torch.float32)
    b = P.bsr_linear8_forward(P.bsr_quantize8_rows(x), layer, out_dtype=torch.float32)
    assert torch.equal(a.nan_to_num(7.0, 8.0, 9.0), b.nan_to_num(7.0, 8.0, 9.0))
    want, _ = blocks8(host(x), 1, 128)
    with np.errstate(over="ignore"):
        finite = np.isfinite(want.astype(np.float32)).all(1)         # (the largest fp32 values round up to 2^128)
    assert 0 < finite.sum() < len(finite)
    assert np.array_equal(np.isnan(host(a)).all(1), ~finite) and np.array_equal(np.isnan(host(a)).any(1), ~finite)
    normal = finite & (np.abs(want).max(1) > 1e-30)
    assert np.array_equal(host(a)[normal], want[normal])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_in,n_out,extra", [(1, 1, 0), (128, 256, 0), (130, 127, 0), (300, 1000, 8), (513, 64, 1)])
def test_weights_to_8_bits(env, n_in, n_out, extra, dtype):
    torch, P = env
    g = torch.Generator().manual_seed(n_in + n_out)
    w = (torch.randn(n_in, n_out + extra, generator=g) * 0.05).to(dtypes(torch)[dtype]).cuda()[:, :n_out]
    q = P.bsr_quantize8_weight(w)
    check_blocks(host(w).T, (q.values, q.scales), 128)
    check_blocks(host(w), (q.values_back, q.scales_back), 128)
    only = P.bsr_quantize8_weight(w, backward=False)
    assert torch.equal(only.values, q.values) and torch.equal(only.scales, q.scales) and only.values_back is None


def phi(u):
    from scipy.special import erfc
    return 0.5 * erfc(-u / np.sqrt(2))


def product(a, w, tol_rows=None):
    """(a w, its error bound)"""
    return a @ w, a.shape[1] * 2.0 ** -23 * (np.abs(a) @ np.abs(w))


def close(got, ref, bound, dtype, what):
    bound = bound + 2.0 ** -22 * np.abs(ref) + 1e-30
    if dtype == "bf16":
        bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref) + 1e-38
    err = np.abs(got - ref)
    assert np.isfinite(got).all() and (err <= bound).all(), f"{what}: {(err / bound).max():.3g} times its bound"


# rows on both sides of every switch between kernels, columns and contractions that end inside tiles, vectors and blocks
SHAPES = [(1, 1, 1), (1, 4096, 520), (3, 128, 16), (16, 200, 130), (17, 513, 15), (33, 1024, 64), (64, 130, 257), (65, 1, 8), (65, 384, 1536), (100, 129, 260),
          (200, 640, 72), (257, 1000, 1111), (1000, 320, 999), (1300, 1536, 512), (2144, 768, 768), (4160, 256, 4104)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_forward(env, M, K, N, dtype):
    torch, P = env
    dt = dtypes(torch)[dtype]
    g = torch.Generator().manual_seed(M + 7 * K + 31 * N)
    x = (torch.randn(M, K, generator=g) * torch.exp(torch.randn(K, generator=g))).to(dt).cuda()
    w = (torch.randn(K, N, generator=g) / K ** 0.5).to(dt).cuda()
    bias = torch.randn(N, generator=g).cuda()
    res = torch.randn(M, N, generator=g).to(dt).cuda()
    layer = P.bsr_quantize8_weight(w)
    y = P.bsr_linear8_forward(x, layer, bias)
    u = torch.full((M, N), float("nan"), dtype=dt, device="cuda")
    act = P.bsr_linear8_forward(x, layer, bias, act=1, u_out=u)
    added = P.bsr_linear8_forward(x, layer, res=res)
    rows8 = P.bsr_quantize8_rows(x)
    from_rows = P.bsr_linear8_forward(rows8, layer, bias, out_dtype=dt)
    other = P.bsr_linear8_forward(rows8, layer, bias, out_dtype=torch.float32 if dtype == "bf16" else torch.bfloat16)
    assert torch.equal(y, from_rows) and torch.equal(u, y), "rows brought to 8 bits before or on the way: the same"
    some = np.unique(np.concatenate([np.random.default_rng(M).choice(M, min(M, 96), replace=False), np.arange(max(0, M - 40), M)]))
    xq = decode(rows8.values.cpu().numpy()[some], rows8.scales.cpu().numpy()[some][:, :-(-K // 128)], 1, K)
    wq = decode(layer.values.cpu().numpy(), layer.scales.cpu().numpy()[:, :-(-K // 128)], 128, K).T
    ref, bound = product(xq, wq)
    b = bias.cpu().numpy().astype(np.float64)
    bound = bound + 2.0 ** -22 * np.abs(b)
    close(host(y)[some], ref + b, bound, dtype, "linear")
    close(host(other)[some], ref + b, bound, "f32" if dtype == "bf16" else "bf16", "linear, the other type")
    v = ref + b
    close(host(act)[some], v * phi(v), 1.2 * bound + 2e-6 * np.abs(v) + 2.0 ** -20 * np.abs(v), dtype, "gelu")
    r = host(res)[some]
    close(host(added)[some], ref + r, bound + 2.0 ** -22 * np.abs(r), dtype, "residual")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,n_in,n_out", [(1, 4096, 520), (5, 130, 1), (64, 257, 300), (70, 1536, 384), (1031, 999, 200), (2144, 768, 768)])
def test_input_gradient(env, M, n_in, n_out, dtype):
    torch, P = env
    dt = dtypes(torch)[dtype]
    g = torch.Generator().manual_seed(M + n_in + n_out)
    w = (torch.randn(n_in, n_out, generator=g) / n_in ** 0.5).to(dt).cuda()
    dy = (1e-4 * torch.randn(M, n_out + 5, generator=g)).to(dt).cuda()[:, :n_out]
    u = torch.randn(M, n_in, generator=g).to(dt).cuda()
    layer = P.bsr_quantize8_weight(w)
    dx, du = P.bsr_linear8_dgrad(dy, layer), P.bsr_linear8_dgrad(dy, layer, u=u)
    rows8 = P.bsr_quantize8_rows(dy)
    assert torch.equal(dx, P.bsr_linear8_dgrad(rows8, layer, out_dtype=dt))
    some = np.unique(np.concatenate([np.random.default_rng(M).choice(M, min(M, 96), replace=False), np.arange(max(0, M - 40), M)]))
    q = decode(rows8.values.cpu().numpy()[some], rows8.scales.cpu().numpy()[some][:, :-(-n_out // 128)], 1, n_out)
    wq = decode(layer.values_back.cpu().numpy(), layer.scales_back.cpu().numpy()[:, :-(-n_out // 128)], 128, n_out)
    ref, bound = product(q, wq.T)
    close(host(dx)[some], ref, bound, dtype, "dgrad")
    v = host(u)[some]
    slope = phi(v) + v * np.exp(-v * v / 2) / np.sqrt(2 * np.pi)
    close(host(du)[some], ref * slope, bound * np.abs(slope) + 4e-6 * np.abs(ref), dtype, "dgrad with GELU'")


def test_gradient_against_differences(env):
    """<dx, d> against (L(x + h d) - L(x - h d)) / 2h of L = sum(c GELU(x W_q)): the layer is linear up to the rounding of x, which a step large against
    it averages out; here x, x + hd and x - hd are 8-bit values themselves, so nothing is rounded and central differences are good to h^2."""
    torch, P = env
    g = torch.Generator().manual_seed(3)
    M, K, N = 70, 256, 136
    layer = P.bsr_quantize8_weight((torch.randn(K, N, generator=g) / 16).cuda())
    d = torch.randint(-1, 2, (M, K), generator=g).float()
    x = torch.randint(-3, 4, (M, K), generator=g).float()
    x[:, 0], x[:, 128], d[:, 0], d[:, 128] = 7.0, 7.0, 0.0, 0.0            # one scale throughout: multiples of 1/16 up to 1, of 1/4 up to 4
    h = 0.25
    c = torch.randn(M, N, generator=g).cuda()

    def loss(v):
        u = torch.empty(M, N, device="cuda")
        y = P.bsr_linear8_forward(v.cuda(), layer, act=1, u_out=u)
        return float((y.double() * c.double()).sum()), u

    (up, _), (down, _), (_, u) = loss(x + h * d), loss(x - h * d), loss(x)
    wq = torch.from_numpy(decode(layer.values.cpu().numpy(), layer.scales.cpu().numpy()[:, :2], 128, K).T.copy())
    ud = host(u)
    slope = phi(ud) + ud * np.exp(-ud * ud / 2) / np.sqrt(2 * np.pi)
    direction = (d.double() @ wq).numpy()
    formula = float((c.cpu().numpy() * slope * direction).sum())
    # the third derivative of GELU is below 1.6 in size
    third = float((np.abs(c.cpu().numpy()) * 1.6 * np.abs(h * direction) ** 3).sum()) / 6 / h
    assert abs((up - down) / (2 * h) - formula) <= third + 1e-4 * float(np.abs(c.cpu().numpy() * direction).sum())
    # the same product by the library: dy = c GELU'(u), brought to 8 bits, is what differs
    dy = (c * torch.from_numpy(slope).float().cuda())
    dx = P.bsr_linear8_dgrad(dy, layer)
    dyq, _ = blocks8(host(dy), 1, 128)
    assert abs(float((host(dx) * d.numpy()).sum()) - float((dyq * direction).sum())) <= 1e-4 * float(np.abs(dyq * direction).sum())


def test_non_finite_rows_show(env):
    torch, P = env
    for M in (4, 100):
        x = torch.randn(M, 300, device="cuda")
        x[1, 7], x[2, 200] = float("inf"), float("nan")
        y = P.bsr_linear8_forward(x, P.bsr_quantize8_weight(torch.randn(300, 40, device="cuda")))
        bad = torch.isnan(y).all(1).cpu()
        assert bad[1] and bad[2] and int(bad.sum()) == 2 and bool(torch.isfinite(y[0]).all())


def test_no_rows(env):
    torch, P = env
    layer = P.bsr_quantize8_weight(torch.randn(64, 48, device="cuda"))
    x = torch.empty(0, 64, device="cuda", dtype=torch.bfloat16)
    assert P.bsr_linear8_forward(x, layer).shape == (0, 48)
    assert P.bsr_linear8_forward(P.bsr_quantize8_rows(x), layer).shape == (0, 48)
    assert P.bsr_linear8_dgrad(torch.empty(0, 48, device="cuda"), layer).shape == (0, 64)


def test_on_another_stream(env):
    torch, P = env
    x, w = torch.randn(500, 700, device="cuda"), torch.randn(700, 300, device="cuda")
    ref = P.bsr_linear8_forward(x, P.bsr_quantize8_weight(w))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y = P.bsr_linear8_forward(x, P.bsr_quantize8_weight(w))
    s.synchronize()
    assert torch.equal(y, ref)


def test_refusals(env):
    torch, P = env
    x, w = torch.randn(8, 64, device="cuda"), torch.randn(64, 32, device="cuda")
    layer = P.bsr_quantize8_weight(w, backward=False)
    for call in (lambda: P.bsr_linear8_forward(x[:, :60], layer), lambda: P.bsr_linear8_forward(x.t(), layer),
                 lambda: P.bsr_linear8_forward(x, layer, bias=torch.zeros(31, device="cuda")),
                 lambda: P.bsr_linear8_forward(x, layer, res=torch.zeros(8, 32, device="cuda", dtype=torch.bfloat16)),
                 lambda: P.bsr_linear8_forward(x, layer, y=torch.empty(8, 64, device="cuda")[:, :32]),
                 lambda: P.bsr_linear8_dgrad(torch.zeros(8, 32, device="cuda"), layer), lambda: P.bsr_quantize8_rows(x.cpu()),
                 lambda: P.bsr_linear8_forward(x.cpu(), layer), lambda: P.bsr_quantize8_rows(x[0])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        P.bsr_quantize8_rows(x.half())
    with pytest.raises(P.BsrError):
        P.bsr_linear8_forward(x, layer, act=2)


# few tiles and long sums, whose k-tiles several groups of wavefronts share: as many for each, one or more left over, the fewest that are shared
SHARED = [(33, 400, 64), (40, 897, 70), (64, 1100, 128), (90, 1300, 200), (50, 1920, 96), (130, 2048, 300), (257, 5000, 1030), (512, 4096, 2048)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N", SHARED)
def test_sums_shared_by_groups(env, M, K, N, dtype):
    test_forward(env, M, K, N, dtype)
    test_input_gradient(env, M, N, K, dtype)
