"""Rows that start at the address of any element: the same bits as from rows on 16-byte boundaries (every row is taken in the same pieces by the same
threads, wherever it lies), and nothing written beside them."""
import pytest

pytestmark = pytest.mark.gpu

# widths: one short of, at and one past whole pieces and each number of pieces a thread; past the registers
WIDTHS = [1, 7, 9, 31, 64, 127, 511, 513, 1023, 1032, 2047, 2049, 4095, 4097, 8191, 8193, 16383, 16385]
LEFT = -77.0


@pytest.fixture(scope="module")
def env():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device")
    import paper_2405_10951_amd as P
    return torch, P


def types(torch):
    return {"bf16": torch.bfloat16, "f32": torch.float32}


def shifted(torch, t, first, gap):
    """t as a view whose first element is element `first` of its memory, rows `gap` elements apart"""
    M, D = t.shape
    whole = torch.full((first + M * (D + gap) + 16,), LEFT, dtype=t.dtype, device="cuda")
    view = whole[first:first + M * (D + gap)].view(M, D + gap)[:, :D]
    view.copy_(t)
    return view, whole


def beside(torch, whole, first, M, D, gap):
    """what lies beside the rows is as it was"""
    rows = whole[first:first + M * (D + gap)].view(M, D + gap)[:, D:]
    return all(bool((part == LEFT).all()) for part in (whole[:first], rows, whole[first + M * (D + gap):]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", WIDTHS)
def test_layernorm(env, D, dtype):
    torch, P = env
    torch.manual_seed(D)
    M = 37
    x, dy, res = (torch.randn(M, D, device="cuda").to(types(torch)[dtype]) for _ in range(3))
    gamma, beta = torch.randn(D, device="cuda"), torch.randn(D, device="cuda")
    y, mean, rstd = P.bsr_layernorm_forward(x, gamma, beta)
    r8, _, _ = P.bsr_layernorm_forward8(x, gamma, beta)
    dx, dg, db = P.bsr_layernorm_backward(dy, x, mean, rstd, gamma, res=res)
    for first, gap in ((1, 0), (3, 5), (0, 1)):
        (xs, _), (dys, _), (ress, _), (out, whole) = (shifted(torch, t, first, gap) for t in (x, dy, res, torch.zeros_like(x)))
        got, m2, r2 = P.bsr_layernorm_forward(xs, gamma, beta, y=out)
        assert torch.equal(got, y) and torch.equal(m2, mean) and torch.equal(r2, rstd) and beside(torch, whole, first, M, D, gap)
        r8s, _, _ = P.bsr_layernorm_forward8(xs, gamma, beta)
        assert torch.equal(r8s.values, r8.values) and torch.equal(r8s.scales, r8.scales)
        out, whole = shifted(torch, torch.zeros_like(x), first, gap)
        got, dg2, db2 = P.bsr_layernorm_backward(dys, xs, mean, rstd, gamma, res=ress, dx=out)
        assert torch.equal(got, dx) and torch.equal(dg2, dg) and torch.equal(db2, db) and beside(torch, whole, first, M, D, gap)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", WIDTHS)
def test_layernorm_gradient_in_place(env, D, dtype):
    """dx in the place of dy, and of the residual's gradient: the same dx and the same sums"""
    torch, P = env
    torch.manual_seed(D + 1)
    x, dy, res = (torch.randn(41, D, device="cuda").to(types(torch)[dtype]) for _ in range(3))
    gamma, beta = torch.randn(D, device="cuda"), torch.randn(D, device="cuda")
    _, mean, rstd = P.bsr_layernorm_forward(x, gamma, beta)
    want = P.bsr_layernorm_backward(dy, x, mean, rstd, gamma, res=res)
    for place in (0, 1):
        mine = [dy.clone(), res.clone()]
        got = P.bsr_layernorm_backward(mine[0], x, mean, rstd, gamma, res=mine[1], dx=mine[place])
        assert got[0].data_ptr() == mine[place].data_ptr()
        assert all(torch.equal(g, w) for g, w in zip(got, want)), "in the place of " + ("dy", "res")[place]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", WIDTHS[:12])
def test_to_8_bits_and_few_rows(env, K, dtype):
    torch, P = env
    torch.manual_seed(K)
    N = 70
    w = torch.randn(K, N, device="cuda").to(types(torch)[dtype])
    w8 = P.bsr_quantize8_weight(w)
    ws, _ = shifted(torch, w, 1, 2)
    w8s = P.bsr_quantize8_weight(ws)
    for name in ("values", "scales", "values_back", "scales_back"):
        assert torch.equal(getattr(w8s, name), getattr(w8, name))
    for M in (1, 19, 33):
        x = torch.randn(M, K, device="cuda").to(types(torch)[dtype])
        r8, y = P.bsr_quantize8_rows(x), P.bsr_linear8_forward(x, w8)
        assert torch.equal(P.bsr_linear8_forward(r8, w8, y=torch.empty_like(y)), y)
        for first, gap in ((1, 0), (3, 5)):
            xs, _ = shifted(torch, x, first, gap)
            r8s = P.bsr_quantize8_rows(xs)
            assert torch.equal(r8s.values, r8.values) and torch.equal(r8s.scales, r8.scales)
            assert torch.equal(P.bsr_linear8_forward(xs, w8), y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 7, 9, 63, 65, 129, 255, 257, 331])
def test_results_of_odd_width(env, N, dtype):
    """rows of results that share lines and 16-byte pieces: each column is what a wider, whole product has there, the residual and the stored input too"""
    torch, P = env
    torch.manual_seed(N)
    M, K, W = 203, 384, 384                               # (sums too short to be shared in ways that depend on the number of tiles)
    dt = types(torch)[dtype]
    w, b = torch.randn(K, W, device="cuda").to(dt), torch.randn(W, device="cuda")
    w[:, N:] = 0                                          # (the same 128 x 128 blocks on both sides)
    x, res = P.bsr_quantize8_rows(torch.randn(M, K, device="cuda").to(dt)), torch.randn(M, W, device="cuda").to(dt)
    narrow, wide = P.bsr_quantize8_weight(w[:, :N].contiguous()), P.bsr_quantize8_weight(w)
    bn, rn = b[:N].contiguous(), res[:, :N].contiguous()

    def fresh(n):
        return torch.empty(M, n, device="cuda", dtype=dt)
    whole = torch.full((M * N + 64,), LEFT, device="cuda", dtype=dt)
    u, uw = fresh(N), fresh(W)
    pairs = [(P.bsr_linear8_forward(x, narrow, bn, y=whole[:M * N].view(M, N)), P.bsr_linear8_forward(x, wide, b, y=fresh(W))),
             (P.bsr_linear8_forward(x, narrow, bn, res=rn, y=fresh(N)), P.bsr_linear8_forward(x, wide, b, res=res, y=fresh(W))),
             (P.bsr_linear8_forward(x, narrow, bn, act=1, u_out=u, y=fresh(N)), P.bsr_linear8_forward(x, wide, b, act=1, u_out=uw, y=fresh(W)))]
    pairs.append((u, uw))
    for got, want in pairs:
        assert torch.equal(got, want[:, :N])
    assert bool((whole[M * N:] == LEFT).all())
