"""RMSNorm with the residual's addition against 64 bits.

Tolerances, from the arithmetic: a row's sum of squares is an fp32 sum of positive terms, added in chains of at most 257 and then pairwise, so it is good to 270 x 2^-24 =
1.6e-5 and 1/std to half of that; s, y and every term of dx are products and sums of a handful more roundings.  So everything is held to 1.2e-5 of the sizes of the terms it is made of
(FLAT), plus half a step of bf16 (2^-8 of the result) where that is the type.  Sums over rows: chains of at most 64 fp32 additions, 64 x 2^-24 of the sum of the terms' sizes, and
the terms' own 4 roundings."""
import numpy as np
import pytest

from reference8 import blocks8, decode

pytestmark = pytest.mark.gpu
EPS = 1e-6
FLAT = 1.2e-5
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}

# widths: one, single chunks, each number of chunks a thread, its ends, rows no whole chunks, rows beyond the registers
WIDTHS = [1, 3, 8, 63, 100, 192, 512, 520, 768, 1024, 1032, 1777, 2048, 2056, 4096, 5000, 8192, 8200, 16384, 16392]


@pytest.fixture(scope="module")
def env():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device")
    import paper_2405_10951_amd as P
    return torch, P


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def rows(torch, M, D, dtype, seed, extra=0, first=0):
    """rows of D values among rows of D + extra + first"""
    g = torch.Generator().manual_seed(1000 * seed + M + 131 * D)
    t = torch.randn(M, D + extra + first, generator=g) * (0.5 + 3 * torch.rand(M, 1, generator=g))
    return t.to({"bf16": torch.bfloat16, "f32": torch.float32}[dtype]).cuda()[:, first:first + D]


def gains(torch, D):
    return (1 + 0.2 * torch.randn(D, generator=torch.Generator().manual_seed(D))).cuda()


def close(got, ref, size, half, what):
    off = np.abs(got - ref) - half * np.abs(ref)
    assert (off <= FLAT * size + 1e-38).all(), f"{what}: {(off / (size + 1e-38)).max():.3g}"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", WIDTHS)
def test_forward(env, D, dtype):
    torch, P = env
    gamma = gains(torch, D)
    for M, extra, first in ((1, 0, 0), (7, 8, 0), (66, 3, 1)):
        x, r = rows(torch, M, D, dtype, 1, extra, first), rows(torch, M, D, dtype, 2, extra, first)
        for res in (None, r):
            s = host(x) + (0 if res is None else host(res))
            rs = 1 / np.sqrt((s ** 2).mean(1, keepdims=True) + EPS)
            ref = s * rs * host(gamma)
            y, rstd, total = P.bsr_rmsnorm_forward(x, gamma, EPS, res=res)
            what = f"{M}x{D} res {res is not None}"
            close(host(y), ref, np.abs(ref), HALF[dtype], "y " + what)
            close(host(rstd), rs[:, 0], rs[:, 0], 0, "rstd " + what)
            if res is None:
                assert total is x
            else:
                assert (np.abs(host(total) - s) <= HALF[dtype] * np.abs(s) * 1.0001).all()
            both = torch.empty_like(y)
            r8, rstd8, total8 = P.bsr_rmsnorm_forward8(x, gamma, EPS, res=res, y=both)
            alone, _, _ = P.bsr_rmsnorm_forward8(x, gamma, EPS, res=res)
            assert torch.equal(rstd8, rstd) and torch.equal(total8, total) and torch.equal(both, y)
            assert torch.equal(alone.values, r8.values) and torch.equal(alone.scales, r8.scales)
            assert not r8.values[:, D:].any()
            got = decode(r8.values.cpu().numpy(), r8.scales.cpu().numpy()[:, :-(-D // 128)], 1, D)
            want, _ = blocks8(ref, 1, 128)             # (a value next to a boundary may fall to its other side)
            assert (np.abs(got - ref) - np.abs(want - ref) <= 2 * FLAT * np.abs(ref) + 1e-38).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", WIDTHS)
def test_backward(env, D, dtype):
    torch, P = env
    gamma = gains(torch, D)
    for M, extra, first in ((1, 0, 0), (5, 8, 0), (70, 3, 1), (1031, 0, 0)) if D <= 2056 else ((1, 0, 0), (70, 8, 0), (9, 3, 1)):
        x, dy, res = (rows(torch, M, D, dtype, s, extra, first) for s in (3, 4, 5))
        xd, d, g = host(x), host(dy), host(gamma)
        rstd = torch.from_numpy(1 / np.sqrt((xd ** 2).mean(1) + EPS)).float().cuda()
        rs = host(rstd)[:, None]
        xh, gd = xd * rs, d * g
        ref = rs * (gd - xh * (gd * xh).mean(1, keepdims=True))
        size = rs * (np.abs(gd) + np.abs(xh) * np.abs(gd * xh).mean(1, keepdims=True))
        dx, dg = P.bsr_rmsnorm_backward(dy, x, rstd, gamma)
        close(host(dx), ref, size, HALF[dtype], f"dx {M}x{D}")
        dxr, dgr = P.bsr_rmsnorm_backward(dy, x, rstd, gamma, res=res)
        close(host(dxr), ref + host(res), size + np.abs(host(res)), HALF[dtype], f"dx + res {M}x{D}")
        term = d * xh
        assert (np.abs(host(dg) - term.sum(0)) <= 68 * 2.0 ** -24 * np.abs(term).sum(0) + 1e-38).all(), f"dgamma {M}x{D}"
        assert torch.equal(dg, dgr)
        only, none = P.bsr_rmsnorm_backward(dy, x, rstd, gamma, need_params=False)
        assert none is None and torch.equal(only, dx)
        none, dg2 = P.bsr_rmsnorm_backward(dy, x, rstd, gamma, need_dx=False)
        assert none is None and torch.equal(dg2, dg)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,extra", [(64, 0), (777, 3), (5001, 7), (16392, 8), (8200, 0), (5, 1)])
def test_results_in_the_inputs_places(env, D, extra, dtype):
    """and nothing behind a row or the last row is written"""
    torch, P = env
    gamma = gains(torch, D)

    def own(t):
        """the rows in a buffer of their own, a row more behind them"""
        buf = torch.full((t.shape[0] + 1, D + extra), 7.0, dtype=t.dtype, device="cuda")
        buf[:-1, :D] = t
        return buf, buf[:-1, :D]

    def untouched(buf):
        return bool((buf[-1] == 7).all()) and bool((buf[:, D:] == 7).all())

    x, r, dy = (rows(torch, 33, D, dtype, s) for s in (6, 7, 8))
    y, rstd, total = P.bsr_rmsnorm_forward(x, gamma, EPS, res=r)
    for first, second in (("x", "res"), ("res", "x")):
        (bx, ox), (br, orr) = own(x), own(r)
        place = dict(x=ox, res=orr)
        got, rstd2, total2 = P.bsr_rmsnorm_forward(ox, gamma, EPS, res=orr, y=place[first], sum_out=place[second])
        assert torch.equal(got, y) and torch.equal(total2, total) and torch.equal(rstd2, rstd) and untouched(bx) and untouched(br)
    dx, dg = P.bsr_rmsnorm_backward(dy, total, rstd, gamma, res=r)
    for k in range(3):
        held = [own(t) for t in (dy, total, r)]
        a, h, c = (v for _, v in held)
        dx2, dg2 = P.bsr_rmsnorm_backward(a, h, rstd, gamma, res=c, dx=held[k][1])
        assert torch.equal(dx2, dx) and torch.equal(dg2, dg) and all(untouched(b) for b, _ in held)


@pytest.mark.parametrize("D", [192, 777])
def test_against_differences(env, D):
    """central differences of L = sum(c y) + sum(e s) in 64 bits in the direction of random vectors"""
    torch, P = env
    x, r, c, e = (rows(torch, 6, D, "f32", s) for s in (9, 10, 11, 12))
    gamma = gains(torch, D)
    y, rstd, total = P.bsr_rmsnorm_forward(x, gamma, EPS, res=r)
    dx, dg = P.bsr_rmsnorm_backward(c, total, rstd, gamma, res=e)

    def loss(dxs, dgs):
        s = host(x) + host(r) + dxs
        return (host(c) * s / np.sqrt((s ** 2).mean(1, keepdims=True) + EPS) * (host(gamma) + dgs)).sum() + (host(e) * s).sum()

    rng = np.random.default_rng(0)
    for _ in range(3):
        v, w, h = rng.standard_normal((6, D)), rng.standard_normal(D), 1e-5
        slope = (loss(h * v, h * w) - loss(-h * v, -h * w)) / (2 * h)
        got = (host(dx) * v).sum() + (host(dg) * w).sum()
        scale = np.sqrt(((host(dx) * v) ** 2).sum() + ((host(dg) * w) ** 2).sum())
        assert abs(got - slope) <= 1e-5 * scale * np.sqrt(7 * D)


def test_rows_without_anything(env):
    torch, P = env
    gamma = gains(torch, 256)
    empty = torch.empty(0, 256, device="cuda")
    y, rstd, total = P.bsr_rmsnorm_forward(empty, gamma, EPS, res=empty)
    assert y.shape == total.shape == (0, 256) and rstd.shape == (0,)
    dx, dg = P.bsr_rmsnorm_backward(empty, empty, rstd, gamma)
    assert dx.shape == (0, 256) and not dg.any()
    x = torch.zeros(3, 256, device="cuda")
    y, rstd, _ = P.bsr_rmsnorm_forward(x, gamma, EPS)
    assert not y.any() and torch.allclose(rstd, torch.full((3,), EPS ** -0.5, device="cuda"))
    # what is no number stays in its row
    x = rows(torch, 5, 256, "f32", 13).clone()
    good, _, _ = P.bsr_rmsnorm_forward(x, gamma, EPS)
    x[2, 17] = float("nan")
    y, rstd, _ = P.bsr_rmsnorm_forward(x, gamma, EPS)
    assert y[2].isnan().all() and torch.equal(y[[0, 1, 3, 4]], good[[0, 1, 3, 4]])


def test_on_another_stream(env):
    torch, P = env
    x, r = rows(torch, 500, 768, "bf16", 14), rows(torch, 500, 768, "bf16", 15)
    gamma = gains(torch, 768)
    want = P.bsr_rmsnorm_forward(x, gamma, EPS, res=r)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = P.bsr_rmsnorm_forward(x, gamma, EPS, res=r)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_far_rows(env):
    """a row whose offset passes 32 bits"""
    torch, P = env
    M, D, ld = 3, 4096, (1 << 31) + 64
    buf = torch.empty(2 * ld + D, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((M, D), (ld, 1))
    near = rows(torch, M, D, "bf16", 16)
    x.copy_(near)
    gamma = gains(torch, D)
    want = P.bsr_rmsnorm_forward(near, gamma, EPS, res=near)
    got = P.bsr_rmsnorm_forward(x, gamma, EPS, res=x)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    dx, dg = P.bsr_rmsnorm_backward(x, x, want[1], gamma, res=x)
    dx2, dg2 = P.bsr_rmsnorm_backward(near, near, want[1], gamma, res=near)
    assert torch.equal(dx, dx2) and torch.equal(dg, dg2)


@pytest.mark.parametrize("D", [16, 5])
def test_rows_past_one_launch(env, D):
    """2^21 rows are a launch: the rows around its end and the last ones as by themselves"""
    torch, P = env
    M = (1 << 21) + 3
    g = torch.Generator(device="cuda").manual_seed(D)
    x, r, dy = (torch.randn(M, D, generator=g, device="cuda").bfloat16() for _ in range(3))
    gamma = gains(torch, D)
    y, rstd, total = P.bsr_rmsnorm_forward(x, gamma, EPS, res=r)
    r8, _, _ = P.bsr_rmsnorm_forward8(x, gamma, EPS, res=r)
    dx, none = P.bsr_rmsnorm_backward(dy, total, rstd, gamma, res=r, need_params=False)
    dx2, dgamma = P.bsr_rmsnorm_backward(dy, total, rstd, gamma, res=r)
    assert none is None and torch.equal(dx, dx2)
    for part in (slice(0, 70), slice((1 << 21) - 50, M), slice(M - 1, M)):
        a, b, c = (t[part].contiguous() for t in (x, r, dy))
        want = P.bsr_rmsnorm_forward(a, gamma, EPS, res=b)
        q, _, _ = P.bsr_rmsnorm_forward8(a, gamma, EPS, res=b)
        assert torch.equal(y[part], want[0]) and torch.equal(rstd[part], want[1]) and torch.equal(total[part], want[2])
        assert torch.equal(r8.values[part], q.values) and torch.equal(r8.scales[part], q.scales)
        assert torch.equal(dx[part], P.bsr_rmsnorm_backward(c, want[2], want[1], gamma, res=b, need_params=False)[0])
    xhat = total.double() * rstd.double()[:, None]
    want = (dy.double() * xhat).sum(0)
    # (at most 256 chains of 8192 additions, whose running sums of random signs stay below 512: each is off by 8192 x 512 x 2^-24 at the very most)
    assert (dgamma.double() - want).abs().max() < 64
