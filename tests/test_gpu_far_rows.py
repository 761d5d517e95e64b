"""Offsets that pass 32 bits: rows 2^30 elements apart, and results of more than 2^31 elements.  The same bits as from rows that lie together, and as from the
last rows alone."""
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


@pytest.mark.parametrize("D", [768, 1001, 16500])
def test_layernorm(env, D):
    torch, P = env
    torch.manual_seed(D)
    x, dy = (torch.randn(5, D, device="cuda").bfloat16() for _ in range(2))
    gamma, beta = torch.randn(D, device="cuda"), torch.randn(D, device="cuda")
    y, mean, rstd = P.bsr_layernorm_forward(x, gamma, beta)
    r8, _, _ = P.bsr_layernorm_forward8(x, gamma, beta)
    want = P.bsr_layernorm_backward(dy, x, mean, rstd, gamma)
    xf, out = apart(torch, x), apart(torch, torch.zeros_like(x))
    assert torch.equal(P.bsr_layernorm_forward(xf, gamma, beta, y=out)[0], y)
    far8, _, _ = P.bsr_layernorm_forward8(xf, gamma, beta)
    assert torch.equal(far8.values, r8.values) and torch.equal(far8.scales, r8.scales)
    dyf = apart(torch, dy)
    got = P.bsr_layernorm_backward(dyf, xf, mean, rstd, gamma, dx=out)
    assert all(torch.equal(g, w) for g, w in zip(got, want))


@pytest.mark.parametrize("K", [256, 301, 1100])
def test_rows_of_a_product(env, K):
    torch, P = env
    torch.manual_seed(K)
    w = P.bsr_quantize8_weight(torch.randn(K, 90, device="cuda"))
    x = torch.randn(5, K, device="cuda").bfloat16()
    far = apart(torch, x)
    a, b = P.bsr_quantize8_rows(far), P.bsr_quantize8_rows(x)
    assert torch.equal(a.values, b.values) and torch.equal(a.scales, b.scales)
    assert torch.equal(P.bsr_linear8_forward(far, w), P.bsr_linear8_forward(x, w))


@pytest.mark.parametrize("classes", [99, 3003, 140003])           # (rows on the same places within 16 bytes on both sides)
def test_distillation(env, classes):
    torch, P = env
    torch.manual_seed(classes)
    z = torch.randn(5, classes, device="cuda").bfloat16()
    index, logits = torch.randint(classes, (5, 7), device="cuda", dtype=torch.int32), torch.randn(5, 7, device="cuda")
    labels = torch.randint(classes, (5,), device="cuda", dtype=torch.int32)
    far, dz = apart(torch, z), apart(torch, torch.zeros_like(z))
    want, wdz = P.bsr_distill_forward_backward(z, index, logits, labels, 2.0, 0.3)
    got, _ = P.bsr_distill_forward_backward(far, index, logits, labels, 2.0, 0.3, dz=dz)
    assert torch.equal(got, want) and torch.equal(dz, wdz)


def test_more_results_than_31_bits(env):
    torch, P = env
    torch.manual_seed(0)
    M, K, N = (1 << 17) + 5, 96, 16400                    # 2.1 G results
    x, w = torch.randn(M, K, device="cuda").bfloat16(), P.bsr_quantize8_weight(torch.randn(K, N, device="cuda").bfloat16())
    y = P.bsr_linear8_forward(x, w)
    last = P.bsr_linear8_forward(x[-200:], w)
    assert torch.equal(y[-200:], last) and torch.equal(y[:200], P.bsr_linear8_forward(x[:200], w))


def test_more_logits_than_31_bits(env):
    torch, P = env
    torch.manual_seed(0)
    rows, classes = 16500, 131072
    z = torch.empty(rows, classes, dtype=torch.bfloat16, device="cuda").normal_()
    index, logits = torch.randint(classes, (rows, 3), device="cuda", dtype=torch.int32), torch.randn(rows, 3, device="cuda")
    labels = torch.randint(classes, (rows,), device="cuda", dtype=torch.int32)
    want, wdz = P.bsr_distill_forward_backward(z[-600:], index[-600:], logits[-600:], labels[-600:], 1.0, 0.5)
    got, dz = P.bsr_distill_forward_backward(z, index, logits, labels, 1.0, 0.5, dz=z)
    assert torch.equal(got[-600:], want) and torch.equal(dz[-600:], wdz)


# more rows than a launch takes (2^21 of them), and than a launch of 64 threads a row could have threads for (2^26)
@pytest.mark.parametrize("rows,classes,top,kind", [((1 << 21) + 3, 9, 3, "f32"), ((1 << 21) + 3, 1100, 2, "bf16"), ((1 << 26) + 5, 2, 1, "bf16")])
def test_distillation_of_many_rows(env, rows, classes, top, kind):
    torch, P = env
    torch.manual_seed(rows)
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[kind]
    z = torch.empty(rows, classes, dtype=dt, device="cuda").normal_()
    index = torch.randint(classes, (rows, top), device="cuda", dtype=torch.int32)
    logits = torch.empty(rows, top, dtype=torch.bfloat16 if kind == "f32" else torch.float32, device="cuda").normal_()
    labels, weight = torch.randint(classes, (rows,), device="cuda", dtype=torch.int32), torch.rand(rows, device="cuda")
    how = dict(temperature=2.0, hard_weight=0.25)
    loss, stats = P.bsr_distill_forward(z, index, logits, labels, **how)
    both, dz = P.bsr_distill_forward_backward(z, index, logits, labels, row_grad=weight, **how)
    apart = P.bsr_distill_backward(z, index, logits, stats, row_grad=weight, labels=labels, **how)
    assert torch.equal(both, loss)
    for first in {0, (1 << 21) - 64, (rows - 64) // 64 * 64}:
        part = slice(first, first + 128)
        some = [t[part] for t in (z, index, logits, labels, weight)]
        want, wstats = P.bsr_distill_forward(*some[:4], **how)
        wboth, wdz = P.bsr_distill_forward_backward(*some[:4], row_grad=some[4], **how)
        assert torch.equal(loss[part], want) and torch.equal(stats[part], wstats) and torch.equal(dz[part], wdz)
        assert torch.equal(apart[part], P.bsr_distill_backward(*some[:3], wstats, row_grad=some[4], labels=some[3], **how))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("D", [5, 8, 3])
def test_layernorm_of_many_rows(env, D, kind):
    """more than a launch takes: forward, to 8 bits, and dx alone"""
    torch, P = env
    torch.manual_seed(D)
    M = (1 << 21) + 3
    x, dy, res = (torch.randn(M, D, device="cuda").to({"bf16": torch.bfloat16, "f32": torch.float32}[kind]) for _ in range(3))
    gamma, beta = torch.randn(D, device="cuda"), torch.randn(D, device="cuda")
    y, mean, rstd = P.bsr_layernorm_forward(x, gamma, beta)
    r8, mean8, rstd8 = P.bsr_layernorm_forward8(x, gamma, beta)
    dx, _, _ = P.bsr_layernorm_backward(dy, x, mean, rstd, gamma, res=res, need_params=False)
    assert torch.equal(mean, mean8) and torch.equal(rstd, rstd8)
    for part in (slice(0, 100), slice((1 << 21) - 50, M), slice(M - 1, M)):
        wy, wm, wr = P.bsr_layernorm_forward(x[part], gamma, beta)
        w8, _, _ = P.bsr_layernorm_forward8(x[part], gamma, beta)
        wdx, _, _ = P.bsr_layernorm_backward(dy[part], x[part], wm, wr, gamma, res=res[part], need_params=False)
        assert torch.equal(y[part], wy) and torch.equal(mean[part], wm) and torch.equal(rstd[part], wr) and torch.equal(dx[part], wdx)
        assert torch.equal(r8.values[part], w8.values) and torch.equal(r8.scales[part], w8.scales)
