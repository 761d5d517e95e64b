"""The cross-entropy of a linear layer and its gradients against 64 bits.

Tolerances, from the arithmetic.  bf16 operands are exact; fp32 values are two fp16 terms, h off by half a step of 2^-11 and l by 2^-11 of that: 2^-22 of the value, or 2^-39 of the largest
value of its row or feature where the terms are subnormal; the product l l that is left out is another 2^-22.  A logit is a sum of D products in fp32: with the instructions' sums of 16 and
chains of D / 16 it is off by at most (D / 16 + 20) 2^-24 of the sum of the products' sizes (12 of the 20 for what fp32 operands lose), e_z.  exp and log are good to 2^-22 and to their argument's
error: the loss is off by 2 e_z + 2^-20 + 2^-22 of the largest logit's size.  A probability is then off by a factor 1 + 2 e_z + 2^-20 (1 + the distance to the maximum), G's fp16 by 2^-11 of itself and
2^-39 (fp32: 2^-22 and 2^-39), the operand beside it by nothing (fp32: 2^-22, and 2^-22 for l l; 2^-11 in bf16 where a weight multiplies x).  A gradient is a sum of such products: every bound is that times the
sum of the terms' sizes, with (n / 16 + 60) 2^-24 for the sum of n terms, and half a step of the result's type."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
HALF_G = {"bf16": 2.0 ** -11, "f32": 2.0 ** -22}


@pytest.fixture(scope="module")
def env():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device")
    import paper_2405_10951_amd as P
    return torch, P


def host(t):
    return t.detach().double().cpu().numpy()


def kind(torch, dtype):
    return {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]


def make(torch, N, D, V, dtype, seed=0, extra=0, first=0, bias=True, spread=0.0):
    """x and w as views of rows of D + extra + first values; every fifth row has no label"""
    g = torch.Generator().manual_seed(1000 * seed + N + 131 * D + 17 * V)
    by = torch.exp(spread * torch.randn(D + extra + first, generator=g))
    x = (torch.randn(N, D + extra + first, generator=g) * by).to(kind(torch, dtype)).cuda()[:, first:first + D]
    w = (2 * torch.randn(V, D + extra + first, generator=g) / by / D ** 0.5).to(kind(torch, dtype)).cuda()[:, first:first + D]
    labels = torch.randint(V, (N,), generator=g, dtype=torch.int32)
    labels[4::5] = torch.tensor([-1, V, -7, 2 ** 31 - 1, -2 ** 31])[torch.arange(len(labels[4::5])) % 5].int()
    b = (0.5 * torch.randn(V, generator=g)).cuda() if bias else None
    return x, w, labels.cuda(), b


def reference(x, w, labels, bias, weight, f32=True):
    """-> (loss, G with the rows' weights, e_z, the logits)"""
    z = x @ w.T + (0 if bias is None else bias)
    most = z.max(1, keepdims=True)
    ref = np.where(np.isinf(most), 0, most)
    e = np.exp(z - ref)
    s = e.sum(1, keepdims=True)
    some = (labels >= 0) & (labels < w.shape[0])
    at = np.where(some, labels, 0)
    with np.errstate(divide="ignore", invalid="ignore"):
        loss = np.where(some & ~np.isinf(most[:, 0]), np.log(s[:, 0]) + ref[:, 0] - z[np.arange(len(z)), at], 0.0)
        p = np.where(s > 0, e / s, 0)
    G = p - (np.arange(w.shape[0])[None] == at[:, None])
    G *= (some & ~np.isinf(most[:, 0]))[:, None]
    ez = (x.shape[1] / 16 + 20) * 2.0 ** -24 * (np.abs(x) @ np.abs(w).T)
    if f32:
        ez = ez + 2.0 ** -39 * (np.abs(x).max(1)[:, None] * np.abs(w).sum(1) + np.abs(x).sum(1)[:, None] * np.abs(w).max(1))
    return loss, G * weight[:, None], p, ez, z


def check(torch, P, x, w, labels, bias, dtype, row_grad=None, grad_scale=1.0, dw_type=None):
    xd, wd, ld, bd = host(x), host(w), labels.cpu().numpy().astype(np.int64), None if bias is None else host(bias)
    N, D, V = len(xd), xd.shape[1], len(wd)
    weight = np.ones(N) if row_grad is None else host(row_grad)
    ref, G, p, ez, z = reference(xd, wd, ld, bd, weight, dtype == "f32")
    what = f"{N}x{D}x{V} {dtype}"
    loss, stats = P.bsr_linear_ce_forward(x, w, labels, bias=bias)
    most = np.abs(z).max(1)
    assert (np.abs(host(loss) - ref) <= 2 * ez.max(1) + 2.0 ** -20 + 2.0 ** -22 * most).all(), f"loss {what}"
    assert (host(loss)[(ld < 0) | (ld >= V)] == 0).all()
    dw = None if dw_type is None else torch.empty(V, D, dtype=dw_type, device="cuda")
    dx, dw, db = P.bsr_linear_ce_backward(x, w, labels, stats, bias=bias, row_grad=row_grad, grad_scale=grad_scale, dw=dw)
    assert dx.dtype is x.dtype and dw.dtype is (dw_type or w.dtype)
    some = ((ld >= 0) & (ld < V) & (weight != 0))[:, None]
    flat = 2 * ez + 2.0 ** -20 * (1 + z.max(1, keepdims=True) - z)
    off = np.abs(weight)[:, None] * some * (flat * p + HALF_G[dtype] * np.abs(G / np.where(weight == 0, 1, weight)[:, None]) + 2.0 ** -39)      # of G
    beside = 2.0 ** -21 if dtype == "f32" else 0.0
    size = np.abs(G) @ np.abs(wd)
    bound = grad_scale * (off @ np.abs(wd) + (beside + (V / 16 + 60) * 2.0 ** -24) * size + 2.0 ** -39 * np.abs(G).sum(1, keepdims=True) * np.abs(wd).max(0)) + HALF[dtype] * np.abs(grad_scale * (G @ wd))
    err = np.abs(host(dx) - grad_scale * (G @ wd))
    assert (err <= bound + 1e-38).all(), f"dx {what}: {(err / (bound + 1e-38)).max():.3g}"
    if row_grad is not None and dtype == "bf16":
        beside = 2.0 ** -11
    size = np.abs(G).T @ np.abs(xd)
    half = HALF["bf16" if dw.dtype is torch.bfloat16 else "f32"]
    xm = (np.abs(xd) * some).max(0)
    bound = grad_scale * (off.T @ np.abs(xd) + (beside + (N / 16 + 60) * 2.0 ** -24) * size + 2.0 ** -38 * np.abs(weight).max() * xm * (np.abs(G) / np.maximum(np.abs(weight), 1e-30)[:, None]).sum(0)[:, None]) \
        + half * np.abs(grad_scale * (G.T @ xd))
    err = np.abs(host(dw) - grad_scale * (G.T @ xd))
    assert (err <= bound + 1e-38).all(), f"dw {what}: {(err / (bound + 1e-38)).max():.3g}"
    if bias is None:
        assert db is None
    else:
        bound = grad_scale * ((np.abs(weight)[:, None] * some * flat * p).sum(0) + (N + 40) * 2.0 ** -24 * np.abs(G).sum(0))
        assert (np.abs(host(db) - grad_scale * G.sum(0)) <= bound + 1e-38).all(), f"db {what}"
    return loss, stats, dx, dw, db



SIZES = [(1, 1, 1), (1, 64, 2), (2, 3, 5), (5, 64, 256), (31, 100, 257), (32, 128, 300), (33, 192, 77), (65, 65, 1000), (130, 320, 511), (200, 1001, 1300), (257, 256, 513), (1, 4096, 5000),
         (600, 64, 3000), (300, 776, 130), (1100, 128, 2600)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,D,V", SIZES)
def test_against_64_bits(env, N, D, V, dtype):
    torch, P = env
    for seed, extra, first, bias in ((1, 0, 0, True), (2, 8, 0, False), (3, 5, 1, True)):
        x, w, labels, b = make(torch, N, D, V, dtype, seed, extra, first, bias)
        check(torch, P, x, w, labels, b, dtype, grad_scale=1.0 / N)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,D,V", [(16, 1024, 20000), (17, 65, 70000), (32, 512, 20003), (33, 65, 129), (48, 100, 3000), (49, 576, 20001), (64, 1000, 9000), (64, 4096, 1031),
                                   (9, 300, 33000), (20, 300, 40000), (40, 300, 33001), (40, 100, 50000), (12, 100, 40000), (64, 2048, 300),
                                   (1, 64, 3), (7, 100, 256), (32, 768, 100), (40, 193, 200)])
def test_few_rows_of_many_classes(env, N, D, V, dtype):
    torch, P = env
    x, w, labels, b = make(torch, N, D, V, dtype, 50)
    weight = torch.rand(N, generator=torch.Generator().manual_seed(51)).cuda()
    loss, _, *grads = check(torch, P, x, w, labels, b, dtype, row_grad=weight, grad_scale=0.5)
    # in one call the logits may be added in another order, and the results rounded the other way
    half = {"bf16": 2.0 ** -8, "f32": 2.0 ** -13}[dtype]
    both, *got = P.bsr_linear_ce_forward_backward(x, w, labels, bias=b, row_grad=weight, grad_scale=0.5)
    assert (both - loss).abs().max() <= 2.0 ** -13
    for g, want in zip(got, grads):
        assert (g.double() - want.double()).norm() <= half * want.double().norm()
    x2, w2, _, _ = make(torch, N, D, V, dtype, 50, extra=3, first=1)
    check(torch, P, x2, w2, labels, None, dtype, dw_type=torch.float32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weights_of_rows(env, dtype):
    """and rows whose weight is 0, among them one without any number in it"""
    torch, P = env
    x, w, labels, b = make(torch, 70, 96, 400, dtype, 4)
    g = torch.Generator().manual_seed(5)
    weight = torch.randn(70, generator=g).cuda()
    weight[[3, 17]] = 0
    got = check(torch, P, x, w, labels, b, dtype, row_grad=weight, grad_scale=0.125, dw_type=torch.float32)
    x2 = x.clone()
    x2[17], x2[4] = float("nan"), float("inf")                   # weight 0, no label
    loss, stats = P.bsr_linear_ce_forward(x2, w, labels, bias=b)
    dx, dw, db = P.bsr_linear_ce_backward(x2, w, labels, stats, bias=b, row_grad=weight, grad_scale=0.125, dw=torch.empty_like(got[3]))
    rest = [i for i in range(70) if i not in (4, 17)]
    assert torch.equal(loss[rest], got[0][rest]) and loss[17].isnan() and loss[4] == 0
    assert torch.equal(dx[rest], got[2][rest]) and not dx[[4, 17]].any() and torch.equal(dw, got[3]) and torch.equal(db, got[4])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,D,V", [(20, 96, 400), (70, 96, 400), (300, 128, 9000)])
def test_rows_without_a_label_whose_weight_is_no_number(env, N, D, V, dtype):
    """1 / 0 for a sequence that has no labels, for instance"""
    torch, P = env
    x, w, labels, b = make(torch, N, D, V, dtype, 40)
    weight = torch.rand(N, generator=torch.Generator().manual_seed(41)).cuda()
    want = P.bsr_linear_ce_forward_backward(x, w, labels, bias=b, row_grad=weight, grad_scale=0.5)
    none = (labels < 0) | (labels >= V)
    weight[none] = torch.where(torch.arange(int(none.sum()), device="cuda") % 2 == 0, float("inf"), float("nan"))
    got = P.bsr_linear_ce_forward_backward(x, w, labels, bias=b, row_grad=weight, grad_scale=0.5)
    _, stats = P.bsr_linear_ce_forward(x, w, labels, bias=b)
    apart = P.bsr_linear_ce_backward(x, w, labels, stats, bias=b, row_grad=weight, grad_scale=0.5)
    assert not got[1][none].any() and all(torch.equal(g, r) for g, r in zip(got, want)) and not apart[0][none].any() and all(t.isfinite().all() for t in apart)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_features_of_different_sizes(env, dtype):
    """over a factor of 10^5 or so"""
    torch, P = env
    x, w, labels, b = make(torch, 90, 256, 700, dtype, 6, spread=2.0)
    check(torch, P, x, w, labels, b, dtype, grad_scale=1e-4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_classes_that_are_masked(env, dtype):
    """a bias of -inf or of the type's lowest value: probability 0; a label there: loss +inf or as large, finite gradient"""
    torch, P = env
    lowest = torch.finfo(torch.float32).min
    x, w, labels, b = make(torch, 40, 128, 600, dtype, 7)
    for value in (-float("inf"), lowest):
        masked = b.clone()
        masked[100:400] = value
        inside = torch.where((labels >= 100) & (labels < 400), -1, labels)
        left = torch.cat([torch.arange(100), torch.arange(400, 600)]).cuda()
        moved = torch.where(inside >= 400, inside - 300, inside)
        loss, stats = P.bsr_linear_ce_forward(x, w, inside, bias=masked)
        dx, dw, db = P.bsr_linear_ce_backward(x, w, inside, stats, bias=masked)
        few = check(torch, P, x, w[left].contiguous(), moved, b[left].contiguous(), dtype)
        assert torch.allclose(loss, few[0], rtol=1e-5, atol=1e-5) and torch.allclose(dx.float(), few[2].float(), rtol=0.01, atol=1e-4)
        assert not dw[100:400].any() and not db[100:400].any() and torch.allclose(dw[left].float(), few[3].float(), rtol=0.01, atol=1e-4)
        label = torch.full_like(labels, 200)
        loss, stats = P.bsr_linear_ce_forward(x, w, label, bias=masked)
        dx, dw, db = P.bsr_linear_ce_backward(x, w, label, stats, bias=masked)
        assert (loss > 1e30).all() and dx.isfinite().all() and dw.isfinite().all() and torch.allclose(db[200], torch.tensor(-40.0, device="cuda"))
        masked[:] = -float("inf")
        loss, stats = P.bsr_linear_ce_forward(x, w, labels, bias=masked)
        dx, dw, db = P.bsr_linear_ce_backward(x, w, labels, stats, bias=masked)
        assert not loss.any() and not dx.any() and not dw.any() and not db.any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_is_no_number_shows_in_its_row(env, dtype, bad):
    torch, P = env
    x, w, labels, b = make(torch, 40, 128, 300, dtype, 8)
    good, _ = P.bsr_linear_ce_forward(x, w, labels, bias=b)
    for row, logits in ((2, "x"), (3, "bias")):
        x2, b2 = x.clone(), b.clone()
        if logits == "x":
            x2[row, 7] = bad
            loss, stats = P.bsr_linear_ce_forward(x2, w, labels, bias=b2)
            dx, _, _ = P.bsr_linear_ce_backward(x2, w, labels, stats, bias=b2)
            rest = [i for i in range(40) if i != row]
            assert loss[row].isnan() and torch.equal(loss[rest], good[rest]) and dx[row].isnan().all() and dx[rest].isfinite().all()
        else:
            b2[299] = bad
            loss, _ = P.bsr_linear_ce_forward(x2, w, labels, bias=b2)
            assert loss[(labels >= 0) & (labels < 300)].isnan().all()


def test_against_differences(env):
    """central differences of the weighted loss in 64 bits in random directions"""
    torch, P = env
    x, w, labels, b = make(torch, 12, 65, 130, "f32", 9)
    weight = (1 + torch.rand(12, generator=torch.Generator().manual_seed(1))).cuda()
    _, stats = P.bsr_linear_ce_forward(x, w, labels, bias=b)
    dx, dw, db = P.bsr_linear_ce_backward(x, w, labels, stats, bias=b, row_grad=weight, grad_scale=0.5)
    ld = labels.cpu().numpy().astype(np.int64)

    def value(a, c, d):
        return 0.5 * (reference(host(x) + a, host(w) + c, ld, host(b) + d, host(weight))[0] * host(weight)).sum()

    rng, h = np.random.default_rng(0), 1e-5
    for _ in range(3):
        u, v, t = rng.standard_normal((12, 65)), rng.standard_normal((130, 65)), rng.standard_normal(130)
        slope = (value(h * u, h * v, h * t) - value(-h * u, -h * v, -h * t)) / (2 * h)
        terms = np.concatenate([(host(dx) * u).ravel(), (host(dw) * v).ravel(), (host(db) * t).ravel()])
        assert abs(terms.sum() - slope) <= 1e-5 * np.abs(terms).sum()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_is_not_wanted(env, dtype):
    torch, P = env
    x, w, labels, b = make(torch, 50, 192, 333, dtype, 10)
    loss, stats, dx, dw, db = check(torch, P, x, w, labels, b, dtype)
    for want in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 0, 1), (0, 1, 1)):
        got = P.bsr_linear_ce_backward(x, w, labels, stats, bias=b, need_dx=want[0], need_dw=want[1], need_db=want[2])
        for g, r, k in zip(got, (dx, dw, db), want):
            assert torch.equal(g, r) if k else g is None
    both = P.bsr_linear_ce_forward_backward(x, w, labels, bias=b)
    assert all(torch.equal(g, r) for g, r in zip(both, (loss, dx, dw, db)))
    with pytest.raises(P.BsrError):
        P.bsr_linear_ce_backward(x, w, labels, stats, need_dx=False, need_dw=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_results_among_others(env, dtype):
    """gradients to rows of other strides at any address, with nothing written beside them"""
    torch, P = env
    x, w, labels, b = make(torch, 37, 101, 270, dtype, 11)
    _, stats = P.bsr_linear_ce_forward(x, w, labels, bias=b)
    dx, dw, _ = P.bsr_linear_ce_backward(x, w, labels, stats, bias=b)
    bx, bw = (torch.full((t.shape[0] + 1, 110), 7.0, dtype=t.dtype, device="cuda") for t in (x, w))
    P.bsr_linear_ce_backward(x, w, labels, stats, bias=b, dx=bx[:-1, 3:104], dw=bw[:-1, 1:102])
    assert torch.equal(bx[:-1, 3:104], dx) and torch.equal(bw[:-1, 1:102], dw)
    for t, f in ((bx, 3), (bw, 1)):
        assert (t[:, :f] == 7).all() and (t[:, f + 101:] == 7).all() and (t[-1] == 7).all()


def test_nothing_to_do(env):
    torch, P = env
    x, w, labels, b = make(torch, 3, 64, 100, "bf16", 12)
    loss, stats = P.bsr_linear_ce_forward(x[:0], w, labels[:0], bias=b)
    dx, dw, db = P.bsr_linear_ce_backward(x[:0], w, labels[:0], stats, bias=b)
    assert loss.shape == (0,) and dx.shape == (0, 64) and dw.shape == (100, 64) and not dw.any() and not db.any()
    none = torch.full_like(labels, -1)
    loss, stats = P.bsr_linear_ce_forward(x, w, none, bias=b)
    dx, dw, db = P.bsr_linear_ce_backward(x, w, none, stats, bias=b)
    assert not loss.any() and not dx.any() and not dw.any() and not db.any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,D,V", [(300, 192, 1000), (20, 192, 100), (40, 512, 20000), (700, 512, 1500)])
def test_replayed(env, N, D, V, dtype):
    """recorded once, replayed on new inputs with the program's own work between"""
    torch, P = env
    held = make(torch, N, D, V, dtype, 13)
    P.bsr_linear_ce_forward_backward(*held[:3], bias=held[3], grad_scale=0.01)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded = P.bsr_linear_ce_forward_backward(*held[:3], bias=held[3], grad_scale=0.01)
    for k in range(4):
        now = make(torch, N, D, V, dtype, 14 + k)
        want = [t.clone() for t in P.bsr_linear_ce_forward_backward(*now[:3], bias=now[3], grad_scale=0.01)]
        for h, n in zip(held, now):
            h.copy_(n)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(recorded, want))


def test_two_streams_at_once(env):
    torch, P = env
    a, b = make(torch, 500, 256, 3000, "bf16", 20), make(torch, 400, 320, 2000, "bf16", 21)
    want = [P.bsr_linear_ce_forward_backward(*t[:3], bias=t[3]) for t in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = []
        for s, t in zip(streams, (a, b)):
            with torch.cuda.stream(s):
                got.append(P.bsr_linear_ce_forward_backward(*t[:3], bias=t[3]))
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for g, w in zip(got, want) for p, q in zip(g, w))


@pytest.mark.parametrize("N,D,V", [(9000, 64, 20000), (40, 512, 300000), (3, 64, 4300000), (60, 64, 1100000), (130, 72, 200000)])
def test_several_pieces(env, N, D, V):
    """more classes than a piece holds, against torch in 64 bits on the GPU; the bound: that of a few elements' norms"""
    torch, P = env
    x, w, labels, b = make(torch, N, D, V, "bf16", 22)
    loss, dx, dw, db = P.bsr_linear_ce_forward_backward(x, w, labels, bias=b, grad_scale=1.0 / N, dw=torch.empty(V, D, device="cuda"))
    xr, wr, br = (t.double().requires_grad_() for t in (x, w, b))
    ref = torch.nn.functional.cross_entropy(xr @ wr.t() + br, torch.where((labels < 0) | (labels >= V), -1, labels).long(), ignore_index=-1, reduction="none")
    gx, gw, gb = torch.autograd.grad(ref.sum() / N, (xr, wr, br))
    assert (loss - ref).abs().max() < 1e-4
    for got, want, tol in ((dx, gx, 2.0 ** -8), (dw, gw, 2.0 ** -12), (db, gb, 1e-5)):
        assert ((got.double() - want).norm() / want.norm()) < tol
