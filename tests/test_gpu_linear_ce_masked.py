"""Classes that a bias of -inf or of the type's lowest value masks, whatever finite values their rows of w hold: the other classes' gradients keep their bits.

Such a class has G 0 and so no part in dx: the results are those of a w whose masked rows are zero, to the bit (probability 0 either way, the same sums in the same order)."""
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


@pytest.mark.parametrize("mask", [-float("inf"), -3.4028234663852886e38])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,D,V", [(20, 64, 300), (70, 96, 400), (130, 3, 1000), (300, 128, 9000), (333, 1001, 5003), (65, 64, 70000), (2048, 768, 21841), (9000, 64, 20000)])
def test_what_masked_classes_hold(env, N, D, V, dtype, mask):
    torch, P = env
    x, w, labels, b = make(torch, N, D, V, dtype, 90)
    masked = torch.zeros(V, dtype=torch.bool, device="cuda")
    masked[V // 3:V // 2] = True
    masked[-5:] = True
    masked[0] = True
    free = torch.arange(V, device="cuda")[~masked]
    labels = torch.where((labels >= 0) & (labels < V), free[labels.long().clamp(0, V - 1) % len(free)].int(), labels)
    b[masked] = mask
    zero, junk = w.clone(), w.clone()
    zero[masked] = 0
    junk[masked] = (torch.randn(int(masked.sum()), D, device="cuda") * 1e25).to(w.dtype)
    weight = torch.rand(N, generator=torch.Generator().manual_seed(91)).cuda()
    want = P.bsr_linear_ce_forward_backward(x, zero, labels, bias=b, row_grad=weight, grad_scale=0.5)
    got = P.bsr_linear_ce_forward_backward(x, junk, labels, bias=b, row_grad=weight, grad_scale=0.5)
    assert want[1].abs().sum() > 0 and all(torch.equal(g, r) for g, r in zip(got, want))
    _, stats = P.bsr_linear_ce_forward(x, junk, labels, bias=b)
    apart = P.bsr_linear_ce_backward(x, junk, labels, stats, bias=b, row_grad=weight, grad_scale=0.5)
    again = P.bsr_linear_ce_backward(x, zero, labels, stats, bias=b, row_grad=weight, grad_scale=0.5)
    assert all(torch.equal(g, r) for g, r in zip(apart, again))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,D,V", [(70, 96, 400), (130, 3, 1000), (300, 128, 9000), (333, 201, 5003)])
def test_labels_that_are_masked(env, N, D, V, dtype):
    """loss +inf, and the class's row of w in dx with -1: (the finite parts against 64 bits)"""
    torch, P = env
    x, w, labels, b = make(torch, N, D, V, dtype, 92)
    inside = (labels >= 0) & (labels < V)
    rows = torch.arange(N, device="cuda")[inside][::3]
    b[labels[rows].long()] = -float("inf")
    hit = inside & torch.isin(labels, labels[rows])
    loss, dx, dw, db = P.bsr_linear_ce_forward_backward(x, w, labels, bias=b)
    assert torch.isinf(loss[hit]).all() and loss[~hit].isfinite().all()
    p = torch.softmax(x.double() @ w.double().t() + b.double(), 1)
    p[torch.arange(N, device="cuda"), torch.where(inside, labels, 0).long()] -= 1
    G = p * inside[:, None]
    # (bounds of the norm: G's 2^-11 or 2^-22, a logit's error of some 2^-18, half a step of the result)
    tol = {"bf16": 2.0 ** -7, "f32": 2.0 ** -16}[dtype]
    for got, want in ((dx, G @ w.double()), (dw, G.t() @ x.double()), (db, G.sum(0))):
        assert (got.double() - want).norm() <= tol * want.norm()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,D,V", [(70, 96, 400), (300, 128, 9000), (333, 201, 5003)])
def test_masks_that_leave_nothing(env, N, D, V, dtype):
    """every class of the lowest bias, which takes up x w whole: all are alike, and none counts with 0"""
    torch, P = env
    x, w, labels, _ = make(torch, N, D, V, dtype, 93)
    b = torch.full((V,), torch.finfo(torch.float32).min, device="cuda")
    loss, dx, dw, db = P.bsr_linear_ce_forward_backward(x, w, labels, bias=b)
    some = (labels >= 0) & (labels < V)
    G = torch.full((N, V), 1 / V, dtype=torch.float64, device="cuda")
    G[torch.arange(N, device="cuda"), torch.where(some, labels, 0).long()] -= 1
    G *= some[:, None]
    want = torch.log(torch.tensor(float(V), dtype=torch.float64))
    assert (loss[some] - want.cuda()).abs().max() <= 2.0 ** -20 and not loss[~some].any()
    tol = {"bf16": 2.0 ** -7, "f32": 2.0 ** -17}[dtype]
    for got, ref in ((dx, G @ w.double()), (dw, G.t() @ x.double()), (db, G.sum(0))):
        assert (got.double() - ref).norm() <= tol * ref.norm()
