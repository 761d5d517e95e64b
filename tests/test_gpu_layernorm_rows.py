"""LayerNorm as an operator against 64 bits.

Tolerances, from the arithmetic: statistics are fp32 sums of D terms, two-pass, so mean and 1/std are good to about sqrt(D) 2^-24 of their scale
(1e-6 at D = 8192, held to 4e-6; a row far from zero adds 2^-23 |mean| rstd to every xhat); y and dx follow with a handful of roundings (1e-5 of the row's scale), plus half an ulp of bf16
(2^-9) where that is the type.  Sums over M rows are held to 1e-5 of the sum of the terms' sizes' root mean square times sqrt(M), which a sum in fp32 of
any order keeps by far."""
import numpy as np
import pytest

from reference8 import blocks8, decode

pytestmark = pytest.mark.gpu
EPS = 1e-6

# widths: one, single chunks, each number of chunks a thread, its ends, rows no whole chunks, rows beyond the registers
WIDTHS = [1, 8, 63, 64, 100, 192, 512, 520, 768, 1024, 1032, 1777, 2048, 2056, 4096, 5000, 8192, 8200, 16384, 16392]


@pytest.fixture(scope="module")
def env():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device")
    import paper_2405_10951_amd as P
    return torch, P


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def make(torch, M, D, dtype, extra=0, seed=0):
    g = torch.Generator().manual_seed(seed * 7 + M + 131 * D)
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    x = (torch.randn(M, D + extra, generator=g) * (0.5 + torch.rand(M, 1, generator=g)) + torch.randn(M, 1, generator=g)).to(dt).cuda()[:, :D]
    dy = torch.randn(M, D + extra, generator=g).to(dt).cuda()[:, :D]
    gamma, beta = (1 + 0.2 * torch.randn(D, generator=g)).cuda(), (0.3 * torch.randn(D, generator=g)).cuda()
    return x, dy, gamma, beta


def reference(x, gamma, beta):
    mu = x.mean(1, keepdims=True)
    rstd = 1 / np.sqrt(((x - mu) ** 2).mean(1, keepdims=True) + EPS)
    return mu, rstd, (x - mu) * rstd


def tight(got, ref, scale, dtype, what):
    bound = 1e-5 * scale + (2.0 ** -8 * np.abs(ref) if dtype == "bf16" else 0.0)
    err = np.abs(got - ref)
    assert (err <= bound).all(), f"{what}: {(err / bound).max():.3g} times its bound"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", WIDTHS)
def test_forward(env, D, dtype):
    torch, P = env
    for M, extra in ((1, 0), (7, 8), (66, 3)):
        x, _, gamma, beta = make(torch, M, D, dtype, extra)
        y, mean, rstd = P.bsr_layernorm_forward(x, gamma, beta, EPS)
        r8, mean8, rstd8 = P.bsr_layernorm_forward8(x, gamma, beta, EPS)
        both = torch.empty_like(y)
        r8b, _, _ = P.bsr_layernorm_forward8(x, gamma, beta, EPS, y=both)
        xd, g, b = host(x), host(gamma), host(beta)
        mu, rs, xh = reference(xd, g, b)
        size = np.abs(xd).max(1, keepdims=True)
        assert (np.abs(host(mean) - mu[:, 0]) <= 4e-6 * size[:, 0]).all()
        # a row of one element has no variance: 1/sqrt(eps), whatever the mean's last bit does to it
        assert (np.abs(host(rstd) / rs[:, 0] - 1) <= 4e-6 + 1e-6 * size[:, 0] * rs[:, 0]).all()
        ref = xh * g + b
        tight(host(y), ref, np.abs(g) * (1 + np.abs(xh) + 0.1 * size * rs) + np.abs(b), dtype, f"y {M}x{D}")
        assert torch.equal(mean, mean8) and torch.equal(rstd, rstd8) and torch.equal(both, y)
        assert torch.equal(r8.values, r8b.values) and torch.equal(r8.scales, r8b.scales)
        # the 8-bit rows are the blocks of an fp32 y: a value next to a boundary may fall to its other side
        s = r8.scales.cpu().numpy()[:, :-(-D // 128)]
        got = decode(r8.values.cpu().numpy(), s, 1, D)
        assert not r8.values.cpu().numpy()[:, D:].any()
        want, _ = blocks8(ref, 1, 128)
        far = np.abs(got - ref) - np.abs(want - ref)
        assert (far <= 4e-5 * (np.abs(g) * (1 + np.abs(xh) + 0.1 * size * rs) + np.abs(b))).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", WIDTHS)
def test_backward(env, D, dtype):
    torch, P = env
    for M, extra in ((1, 0), (5, 8), (70, 3), (1031, 0)) if D <= 2056 else ((1, 0), (70, 8)):
        x, dy, gamma, beta = make(torch, M, D, dtype, extra, 1)
        res = make(torch, M, D, dtype, extra, 2)[1]
        xd, d, g = host(x), host(dy), host(gamma)
        mu, rs, xh = reference(xd, g, host(beta))
        mean, rstd = torch.from_numpy(mu[:, 0]).float().cuda(), torch.from_numpy(rs[:, 0]).float().cuda()
        mu, rs = host(mean)[:, None], host(rstd)[:, None]
        xh = (xd - mu) * rs
        gd = d * g
        ref = rs * (gd - gd.mean(1, keepdims=True) - xh * (gd * xh).mean(1, keepdims=True))
        size = np.sqrt((gd ** 2).mean(1, keepdims=True)) * (1 + np.abs(xh)) + np.abs(gd)
        off = rs * size * (1 + 0.1 * np.abs(xd).max(1, keepdims=True) * rs)
        dx, dg, db = P.bsr_layernorm_backward(dy, x, mean, rstd, gamma)
        tight(host(dx), ref, off, dtype, f"dx {M}x{D}")
        dxr, dgr, dbr = P.bsr_layernorm_backward(dy, x, mean, rstd, gamma, res=res)
        tight(host(dxr), ref + host(res), off + np.abs(host(res)), dtype, f"dx + res {M}x{D}")
        for got, term, what in ((dg, d * xh, "dgamma"), (db, d, "dbeta")):
            bound = 1e-5 * np.sqrt(M * (term ** 2).sum(0)) + 1e-6 * (np.abs(d) * (np.abs(mu) * rs)).sum(0) * (what == "dgamma") + 1e-30
            assert (np.abs(host(got) - term.sum(0)) <= bound).all(), f"{what} {M}x{D}"
        assert torch.equal(dg, dgr) and torch.equal(db, dbr)
        only, none, _ = P.bsr_layernorm_backward(dy, x, mean, rstd, gamma, need_params=False)
        assert none is None and torch.equal(only, dx)
        nodx, dg2, db2 = P.bsr_layernorm_backward(dy, x, mean, rstd, gamma, need_dx=False)
        assert nodx is None and torch.equal(dg2, dg) and torch.equal(db2, db)
        # in place of dy
        own = dy.clone()
        inplace, _, _ = P.bsr_layernorm_backward(own, x, mean, rstd, gamma, dx=own)
        assert torch.equal(inplace, dx)


@pytest.mark.parametrize("D", [192, 777])
def test_against_differences(env, D):
    """central differences of L = sum(c y) in 64 bits in the direction of random vectors"""
    torch, P = env
    x, c, gamma, beta = make(torch, 6, D, "f32", 0, 5)
    _, mean, rstd = P.bsr_layernorm_forward(x, gamma, beta, EPS)
    dx, dg, db = P.bsr_layernorm_backward(c, x, mean, rstd, gamma)
    xd, cd, g, b = host(x), host(c), host(gamma), host(beta)

    def loss(x_, g_, b_):
        return float((cd * (reference(x_, g_, b_)[2] * g_ + b_)).sum())

    rng, h = np.random.default_rng(1), 1e-4
    vx, vg, vb = rng.standard_normal(xd.shape), rng.standard_normal(D), rng.standard_normal(D)
    for (ax, ag, ab), grad, v in (((1, 0, 0), dx, vx), ((0, 1, 0), dg, vg), ((0, 0, 1), db, vb)):
        up = loss(xd + ax * h * vx, g + ag * h * vg, b + ab * h * vb)
        down = loss(xd - ax * h * vx, g - ag * h * vg, b - ab * h * vb)
        got = float((host(grad) * v).sum())
        assert abs((up - down) / (2 * h) - got) <= 1e-4 * float(np.linalg.norm(host(grad)) * np.linalg.norm(v))


def test_many_rows_of_one_value(env):
    """constant rows: xhat is 0 (up to the mean's rounding), nothing divides by zero"""
    torch, P = env
    x = torch.full((300, 768), 3.0, device="cuda")
    gamma, beta = torch.ones(768, device="cuda"), torch.full((768,), 0.5, device="cuda")
    y, mean, rstd = P.bsr_layernorm_forward(x, gamma, beta, EPS)
    assert torch.equal(mean, x[:, 0]) and torch.equal(y, torch.full_like(y, 0.5))
    assert (rstd / 1000 - 1).abs().max() < 1e-6
    r8, _, _ = P.bsr_layernorm_forward8(x, gamma, torch.zeros_like(beta), EPS)
    assert not r8.values.any() and bool((r8.scales[:, :6] == 127).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [256, 300, 1024, 8200])
def test_infinities_and_nan_in_8_bit_rows(env, D, dtype):
    """a gain of infinity or NaN in some columns: those are NaN in 8 bits and do not count towards their blocks' maxima"""
    torch, P = env
    x, _, gamma, beta = make(torch, 9, D, dtype)
    plain, _, _ = P.bsr_layernorm_forward8(x, torch.where(torch.arange(D, device="cuda") % 128 == 5, 0.0, gamma), torch.where(torch.arange(D, device="cuda") % 128 == 5, 0.0, beta), EPS)
    gamma[5::128] = float("inf")
    gamma[5] = float("nan")
    r8, _, _ = P.bsr_layernorm_forward8(x, gamma, beta, EPS)
    n = -(-D // 128)
    assert torch.equal(r8.scales[:, :n], plain.scales[:, :n])
    got, want = r8.values[:, :D].clone(), plain.values[:, :D].clone()
    assert bool((got[:, 5::128] & 0x7f == 0x7f).all())
    got[:, 5::128] = 0
    want[:, 5::128] = 0
    assert torch.equal(got, want)


def test_no_rows_zero_the_sums(env):
    torch, P = env
    x = torch.empty(0, 96, device="cuda")
    v = torch.empty(0, device="cuda")
    gamma = torch.ones(96, device="cuda")
    y, _, _ = P.bsr_layernorm_forward(x, gamma, gamma)
    assert y.shape == (0, 96)
    dx, dg, db = P.bsr_layernorm_backward(x, x, v, v, gamma)
    assert dx.shape == (0, 96) and not dg.any() and not db.any()


def test_the_same_bits_twice(env):
    torch, P = env
    x, dy, gamma, beta = make(torch, 5000, 768, "bf16")
    _, mean, rstd = P.bsr_layernorm_forward(x, gamma, beta)
    a, b = (P.bsr_layernorm_backward(dy, x, mean, rstd, gamma) for _ in range(2))
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_refusals(env):
    torch, P = env
    x = torch.randn(8, 64, device="cuda")
    g, v = torch.ones(64, device="cuda"), torch.ones(8, device="cuda")
    for call in (lambda: P.bsr_layernorm_forward(x, g[:63], g), lambda: P.bsr_layernorm_forward(x.t(), g, g), lambda: P.bsr_layernorm_forward(x[0], g, g),
                 lambda: P.bsr_layernorm_forward(x, g.bfloat16(), g), lambda: P.bsr_layernorm_backward(x[:7], x, v, v, g),
                 lambda: P.bsr_layernorm_backward(x, x, v[:7], v, g), lambda: P.bsr_layernorm_forward(x.cpu(), g, g),
                 lambda: P.bsr_layernorm_forward(x[:1].expand(8, 64), g, g)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        P.bsr_layernorm_forward(x.double(), g, g)
    with pytest.raises(P.BsrError):
        P.bsr_layernorm_forward(x, g, g, eps=-1.0)
    with pytest.raises(P.BsrError):
        P.bsr_layernorm_backward(x, x, v, v, g, need_dx=False, need_params=False)
