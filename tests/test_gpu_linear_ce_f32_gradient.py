"""The weight's gradient of the cross-entropy of a linear layer in fp32 beside bf16 operands, against 64 bits: it keeps the bits that an fp32 sum of fp32 terms has, more than
the one fp16 term of G that is enough for a bf16 result.

Tolerances, from the arithmetic, as parts of 2-norms (|A B| <= |A| times the largest singular value of B).  A logit is off by e_z = (D / 16 + 20) 2^-24 of the sum of its terms' sizes, a probability by
a factor 1 + 2 e_z + 2^-20 (1 + the distance to the maximum); G is two fp16 terms, off by 2^-22 of itself, or by 2^-39.  x is exact; times a weight it is two terms as well, off by 2^-22, and the product of the
low terms that is left out is another 2^-22.  The sums have up to three products a row: (3 N / 16 + 60) 2^-24 of the terms' sizes.  Up to 64 rows G is three bf16 terms, off by less.
One fp16 term would be off by up to 2^-11 of itself, half of that over the root of three at least in the root mean square, which is more than all of that together but for the two sizes of many rows and few features."""
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


def check(torch, x, w, labels, bias, weight, scale, dw):
    N, D = x.shape
    V = len(w)
    xd, wd = x.double(), w.double()
    z = xd @ wd.t() + bias.double()
    some = ((labels >= 0) & (labels < V))
    by = torch.where(some, 1.0 if weight is None else weight.double(), 0.0)[:, None]
    p = torch.softmax(z, 1)
    G = p.clone()
    G[torch.arange(N, device="cuda"), torch.where(some, labels, 0).long()] -= 1
    ez = (D / 16 + 20) * 2.0 ** -24 * (xd.abs() @ wd.abs().t())
    off = by.abs() * (p * (2 * ez + 2.0 ** -20 * (1 + z.amax(1, keepdim=True) - z)) + 2.0 ** -22 * G.abs() + 2.0 ** -39)
    G *= by
    want = G.t() @ xd
    terms = (G.abs().t() @ xd.abs()).norm()
    bound = off.norm() * torch.linalg.matrix_norm(xd, 2) + (2.0 ** -21 + (3 * N / 16 + 60) * 2.0 ** -24) * terms + 2.0 ** -24 * want.norm()
    err = (dw.double() / scale - want).norm()
    one_term = 2.0 ** -12 / 3 ** 0.5 * want.norm()
    assert err <= bound, f"off by {err / want.norm():.3g} of the norm, {bound / want.norm():.3g} allowed"
    return err, bound, one_term


# little work, its logits turned into G; tiles of every shape, with x and w as they lie and packed; several workgroups over the rows; several pieces of classes; few rows
@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("N,D,V", [(130, 96, 400), (300, 128, 9000), (700, 512, 1500), (333, 1000, 5003), (65, 64, 1000), (6304, 64, 300), (1100, 200, 2600), (9000, 64, 20000), (2048, 768, 21841),
                                   (64, 512, 3000), (64, 100, 200), (33, 256, 20000), (32, 512, 3000), (17, 130, 250), (16, 768, 9000), (1, 300, 1000)])
def test_dw_in_fp32_beside_bf16(env, N, D, V, weights):
    torch, P = env
    x, w, labels, b = make(torch, N, D, V, "bf16", 60)
    weight = (0.5 + torch.rand(N, generator=torch.Generator().manual_seed(61))).cuda() if weights else None
    scale = 2.0 ** -10
    _, stats = P.bsr_linear_ce_forward(x, w, labels, bias=b)
    dx, dw, db = P.bsr_linear_ce_backward(x, w, labels, stats, bias=b, row_grad=weight, grad_scale=scale, dw=torch.empty(V, D, device="cuda"))
    err, bound, one_term = check(torch, x, w, labels, b, weight, scale, dw)
    print(f"{N}x{D}x{V}: error {err:.3g}, allowed {bound:.3g}, of one term {one_term:.3g}")
    # alone, and in one call with the loss
    _, alone, _ = P.bsr_linear_ce_backward(x, w, labels, stats, bias=b, row_grad=weight, grad_scale=scale, dw=torch.empty(V, D, device="cuda"), need_dx=False, need_db=False)
    check(torch, x, w, labels, b, weight, scale, alone)
    _, dx2, dw2, db2 = P.bsr_linear_ce_forward_backward(x, w, labels, bias=b, row_grad=weight, grad_scale=scale, dw=torch.empty(V, D, device="cuda"))
    check(torch, x, w, labels, b, weight, scale, dw2)
    # the other results as beside a bf16 dw
    ox, ow, ob = P.bsr_linear_ce_backward(x, w, labels, stats, bias=b, row_grad=weight, grad_scale=scale)
    assert torch.equal(dw.bfloat16(), ow) or (dw.double() - ow.double()).norm() < 2.0 ** -8 * dw.double().norm()
    for a, c in ((dx, ox), (dx2, ox), (db, ob), (db2, ob)):
        assert (a.double() - c.double()).norm() <= 2.0 ** -8 * c.double().norm()


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("N,D", [(1 << 22, 16), ((1 << 21) + 100, 200), (1 << 21, 70)])
def test_the_last_of_the_most_rows(env, N, D, weights):
    """of which only some at the ends have labels: offsets of both terms, and 64-bit sums of a few rows to compare with"""
    torch, P = env
    V = 5
    x, w, _, b = make(torch, 64, D, V, "bf16", 62)
    many = torch.zeros(N, D, dtype=torch.bfloat16, device="cuda")
    labels = torch.full((N,), -1, dtype=torch.int32, device="cuda")
    rows = torch.cat([torch.arange(20), torch.arange(N // 2 - 10, N // 2 + 10), torch.arange(N - 24, N)]).cuda()
    many[rows] = x
    few = torch.arange(64, device="cuda").int() % V
    labels[rows] = few
    weight = None
    if weights:
        weight = torch.full((N,), float("nan"), device="cuda")
        weight[rows] = 0.5 + torch.rand(64, generator=torch.Generator().manual_seed(63)).cuda()
    _, dx, dw, db = P.bsr_linear_ce_forward_backward(many, w, labels, bias=b, row_grad=weight, dw=torch.empty(V, D, device="cuda"))
    check(torch, x, w, few, b, None if weight is None else weight[rows], 1.0, dw)
    assert not dx[labels < 0].any() and dx[rows].abs().sum(1).all()


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("N,D,V", [(1, 64, 133), (20, 64, 133), (20, 100, 266), (40, 130, 133), (64, 64, 266), (64, 512, 7424), (65, 64, 133), (100, 200, 266)])
def test_classes_all_alike(env, N, D, V, weights):
    """All logits 0: G is 1 / V - 1 at the label and 1 / V elsewhere, off by 2^-20 of 1 / V and by what its terms leave of it, 2^-22, and a sum over N rows adds (3 N + 4) 2^-24 of its terms.
    Two bf16 terms would leave up to 2^-17 of 1 / V - 1, one fp16 term up to 2^-11."""
    torch, P = env
    x = make(torch, N, D, V, "bf16", 64)[0]
    w, labels = torch.zeros(V, D, dtype=torch.bfloat16, device="cuda"), (torch.arange(N, device="cuda") * 2 % V).int()
    weight = (1 + torch.arange(N, device="cuda") % 3 / 2).float() if weights else torch.ones(N, device="cuda")
    _, _, dw, _ = P.bsr_linear_ce_forward_backward(x, w, labels, row_grad=weight if weights else None, dw=torch.empty(V, D, device="cuda"))
    G = torch.full((N, V), 1 / V, dtype=torch.float64, device="cuda")
    G[torch.arange(N, device="cuda"), labels.long()] -= 1
    G *= weight.double()[:, None]
    xd = x.double()
    bound = 2.0 ** -20 / V * (weight.double()[:, None] * xd.abs()).sum(0) + (2.0 ** -22 + (3 * N + 4) * 2.0 ** -24) * (G.abs().t() @ xd.abs())
    err = (dw.double() - G.t() @ xd).abs()
    assert (err <= bound).all(), f"{float((err / bound).max()):.3g} times the bound"
