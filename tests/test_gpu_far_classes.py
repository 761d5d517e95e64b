"""Offsets that pass 32 bits in the cross-entropy of a linear layer: rows 2^30 elements apart, and operands of more than 2^31 elements, against the same rows lying together or alone.

The two sides may add in different orders.  A logit of 8192 features is off by (8192 / 16 + 20) 2^-24 of the sum of its terms' sizes, here 0.64 2 sqrt(8192) = 116: 2^-8.1 on either side, a loss by twice
that, and a probability by as large a part of itself: 2^-6, to which two roundings to bf16 add 2^-8 at most in a tensor's 2-norm (half a step is 2^-9 of it in quadrature).  fp32 of 100 features: 27 2^-24 13, four times: 2^-13.5."""
import pytest

pytestmark = pytest.mark.gpu
STRIDE = (1 << 30) + 3


@pytest.fixture(scope="module")
def env():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device")
    import paper_2405_10951_amd as P
    return torch, P


def apart(torch, t):
    """t with its rows STRIDE elements apart: the last of five starts behind element 2^32"""
    far = torch.empty((t.shape[0] - 1) * STRIDE + t.shape[1], dtype=t.dtype, device="cuda").as_strided(t.shape, (STRIDE, 1))
    far.copy_(t)
    return far


@pytest.mark.parametrize("N,D,V,dtype", [(5, 768, 300, "bf16"), (5, 100, 40, "f32"), (5, 1001, 70000, "bf16"), (64, 128, 5, "bf16"), (40, 65, 5, "f32")])
def test_cross_entropy_of_a_layer(env, N, D, V, dtype):
    """rows of the shorter operand, and of its gradient, far apart"""
    torch, P = env
    torch.manual_seed(D)
    kind = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    x, w = torch.randn(N, D, device="cuda").to(kind), (2 * torch.randn(V, D, device="cuda") / D ** 0.5).to(kind)
    labels = torch.randint(V, (N,), device="cuda", dtype=torch.int32)
    loss, dx, dw, _ = P.bsr_linear_ce_forward_backward(x, w, labels)
    if N == 5:
        far = P.bsr_linear_ce_forward_backward(apart(torch, x), w, labels, dx=apart(torch, torch.zeros_like(x)))
    else:
        far = P.bsr_linear_ce_forward_backward(x, apart(torch, w), labels, dw=apart(torch, torch.zeros_like(w)))
    tol = 2.0 ** -12 if dtype == "f32" else 2.0 ** -6
    assert (loss - far[0]).abs().max() < tol
    for got, want in zip(far[1:3], (dx, dw)):
        assert (got.double() - want.double()).norm() < tol * want.double().norm()


@pytest.mark.parametrize("N", [7, 100])
def test_the_last_classes_of_many(env, N):
    """a weight of more than 2^31 values, of which all but the last rows' classes are masked"""
    torch, P = env
    D, V, L = 4096, 540000, 1000
    torch.manual_seed(N)
    x = torch.randn(N, D, device="cuda").bfloat16()
    w = torch.zeros(V, D, dtype=torch.bfloat16, device="cuda")
    w[-L:] = (2 * torch.randn(L, D, device="cuda") / D ** 0.5).bfloat16()
    b = torch.full((V,), -float("inf"), device="cuda")
    b[-L:] = 0
    labels = torch.randint(V - L, V, (N,), device="cuda", dtype=torch.int32)
    loss, dx, dw, db = P.bsr_linear_ce_forward_backward(x, w, labels, bias=b)
    want = P.bsr_linear_ce_forward_backward(x, w[-L:].contiguous(), labels - (V - L), bias=b[-L:].contiguous())
    assert (loss - want[0]).abs().max() < 2.0 ** -6 and not dw[:-L].any() and not db[:-L].any()
    for got, ref in ((dx, want[1]), (dw[-L:], want[2]), (db[-L:], want[3])):
        assert (got.double() - ref.double()).norm() < 2.0 ** -6 * ref.double().norm()


def test_the_last_rows_of_many(env):
    """x of more than 2^31 values, of which only the last rows have labels"""
    torch, P = env
    N, D, V, L = 270000, 8192, 40, 50
    torch.manual_seed(1)
    x = torch.zeros(N, D, dtype=torch.bfloat16, device="cuda")
    x[-L:] = torch.randn(L, D, device="cuda").bfloat16()
    w = (2 * torch.randn(V, D, device="cuda") / D ** 0.5).bfloat16()
    labels = torch.full((N,), -1, device="cuda", dtype=torch.int32)
    labels[-L:] = torch.randint(V, (L,), device="cuda", dtype=torch.int32)
    loss, dx, dw, _ = P.bsr_linear_ce_forward_backward(x, w, labels)
    want = P.bsr_linear_ce_forward_backward(x[-L:].contiguous(), w, labels[-L:].contiguous())
    assert (loss[-L:] - want[0]).abs().max() < 2.0 ** -6 and not loss[:-L].any() and not dx[:-L].any()
    for got, ref in ((dx[-L:], want[1]), (dw, want[2])):
        assert (got.double() - ref.double()).norm() < 2.0 ** -6 * ref.double().norm()


@pytest.mark.parametrize("N,D,dtype", [(1 << 22, 16, "bf16"), (1 << 21, 5, "f32"), ((1 << 20) + 7, 3, "bf16")])
def test_the_most_rows(env, N, D, dtype):
    """Labels all alike, so that the sums over the rows grow with them: fp32 sums of N rows are off by (N / 16 + 60) 2^-24 of their terms' sizes, 2^-6, of which a class's sum keeps more than half here; the
    tensors of other signs, and half a step of bf16, take it to 2^-4 in the 2-norm.  What is off by a row or a tile misses by far more in dx and loss, which have a row each."""
    torch, P = env
    torch.manual_seed(D)
    kind = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    V = 5
    x, w = (1 + 0.25 * torch.randn(N, D, device="cuda")).to(kind), (torch.randn(V, D, device="cuda") / D ** 0.5).to(kind)
    labels = torch.zeros(N, device="cuda", dtype=torch.int32)
    labels[1::3] = -1
    loss, dx, dw, _ = P.bsr_linear_ce_forward_backward(x, w, labels, dw=torch.empty(V, D, device="cuda"))
    z = x.double() @ w.double().t()
    some = (labels >= 0).double()
    G = torch.softmax(z, 1)
    G[:, 0] -= 1
    G *= some[:, None]
    ref = (torch.logsumexp(z, 1) - z[:, 0]) * some
    assert (loss - ref).abs().max() < 2.0 ** -16
    want = G @ w.double()
    assert (dx.double() - want).abs().max() < {"bf16": 2.0 ** -7, "f32": 2.0 ** -16}[dtype] * want.abs().max()
    want = G.t() @ x.double()
    assert (dw.double() - want).norm() < 2.0 ** -4 * want.norm()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [3, 40, 70])
def test_the_widest_rows(env, N, dtype):
    """2^20 features, of which 64 are not zero in x: sums of 64 terms, off by less than 64 2^-24 of their sizes (8 or so); gradients by 2^-12 (fp32) and half a step of bf16, 2^-8, as parts of their 2-norm"""
    torch, P = env
    torch.manual_seed(N)
    kind = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    D, V = 1 << 20, 20
    at = torch.randperm(D, device="cuda")[:64]
    at[0] = D - 1
    x, w = torch.zeros(N, D, dtype=kind, device="cuda"), torch.randn(V, D, device="cuda").to(kind)
    x[:, at] = (torch.randn(N, 64, device="cuda") / 8).to(kind)
    labels = torch.randint(V, (N,), device="cuda", dtype=torch.int32)
    loss, dx, dw, _ = P.bsr_linear_ce_forward_backward(x, w, labels)
    z = x[:, at].double() @ w[:, at].double().t()
    assert (loss - torch.nn.functional.cross_entropy(z, labels.long(), reduction="none")).abs().max() < 2.0 ** -12
    G = torch.softmax(z, 1)
    G[torch.arange(N), labels.long()] -= 1
    tol = {"bf16": 2.0 ** -8, "f32": 2.0 ** -12}[dtype]
    want = G @ w.double()
    assert (dx.double() - want).norm() < tol * want.norm()
    want = G.t() @ x[:, at].double()
    assert (dw[:, at].double() - want).norm() < tol * want.norm()
    dw[:, at] = 0
    assert not dw.any()
