"""The norm of many gradients and their clipping against 64 bits.

Tolerances, from the arithmetic: the sum of squares is fp64, so the norm is off by its rounding to fp32 (2^-24) and hardly more; the factor is rounded once to fp32, the product once to the
gradient's type: 2 x 2^-24 for fp32, 2^-8 and those for bf16."""
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


def host(t):
    return t.detach().double().cpu().numpy()


def gradients(torch, sizes, seed=0, scale=1.0, kinds=("f32", "bf16"), odd=False):
    """odd: tensors at any address, others' values around them"""
    g = torch.Generator().manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        t = (torch.randn(n, generator=g) * scale).to({"bf16": torch.bfloat16, "f32": torch.float32}[kinds[i % len(kinds)]])
        if odd:
            buf = torch.full((n + 9,), 5.0, dtype=t.dtype, device="cuda")
            buf[1 + i % 7:1 + i % 7 + n] = t.cuda()
            t = buf[1 + i % 7:1 + i % 7 + n]
        out.append(t.cuda())
    return out


def check(torch, P, grads, max_norm, **how):
    before = [g.clone() for g in grads]
    norm = P.bsr_clip_grads(grads, max_norm, **how)
    out = how.get("out") or grads
    want = np.sqrt(sum((host(g) ** 2).sum() for g in before))
    assert norm.shape == () and abs(float(norm) - want) <= 1.01 * 2.0 ** -24 * want
    by = min(1.0, max_norm / want) if want else 1.0
    for g, o in zip(before, out):
        assert o.dtype is g.dtype
        if by == 1.0:
            assert torch.equal(o, g)
        else:
            ref = host(g) * by
            half = 2.0 ** -8 if g.dtype is torch.bfloat16 else 0.0
            assert (np.abs(host(o) - ref) <= (half + 2.1 * 2.0 ** -24) * np.abs(ref) + 1e-38).all()
    if how.get("out"):
        assert all(torch.equal(g, b) for g, b in zip(grads, before))
    assert abs(float(P.bsr_grad_norm(before)) - want) <= 1.01 * 2.0 ** -24 * want
    return norm


SIZES = [[1], [7], [16384], [16385, 3], [0, 5, 0], [100003, 1, 16383, 16385, 8, 0, 333333], list(range(1, 145)), [17 * (i % 90) for i in range(1, 300)], [3000000, 40000, 768, 768]]


@pytest.mark.parametrize("max_norm", [0.5, 1e9, 0.0, float("inf")])
@pytest.mark.parametrize("k", range(len(SIZES)))
def test_clip(env, k, max_norm):
    torch, P = env
    check(torch, P, gradients(torch, SIZES[k], k), max_norm)
    grads = gradients(torch, SIZES[k], k)
    check(torch, P, grads, max_norm, out=[torch.full_like(g, 9.0) for g in grads])


@pytest.mark.parametrize("max_norm", [0.5, 1e9])
def test_tensors_at_any_address(env, max_norm):
    """and their neighbours stay as they were"""
    torch, P = env
    sizes = [1, 15, 16, 17, 4099, 16384, 16385, 50001]
    grads, out = gradients(torch, sizes, 1, odd=True), gradients(torch, sizes[:], 2, odd=True)
    check(torch, P, grads, max_norm, out=out)
    check(torch, P, grads, max_norm)
    for t in grads + out:
        whole = torch.empty(0, dtype=t.dtype, device="cuda").set_(t.untyped_storage())
        at = t.storage_offset()
        assert (whole[:at] == 5).all() and (whole[at + t.numel():] == 5).all()


@pytest.mark.parametrize("scale", [1e25, 1e-25])
def test_squares_past_the_range_of_fp32(env, scale):
    torch, P = env
    check(torch, P, gradients(torch, [1000, 333], 3, scale, kinds=("f32",)), 1e-3 * scale)


def test_a_factor_below_the_normal_numbers_of_fp32(env):
    torch, P = env
    check(torch, P, gradients(torch, [1000, 333], 3, 1e36, kinds=("f32",)), 1e-3)


def test_a_norm_past_the_range_of_fp32_scales_nothing(env):
    torch, P = env
    grads = [torch.full((n,), 3e38, device="cuda") for n in (100, 3000)]
    assert torch.isinf(P.bsr_clip_grads(grads, 1.0)) and all((g == 3e38).all() for g in grads)


def test_a_norm_that_is_no_number_scales_nothing(env):
    torch, P = env
    for bad in (float("nan"), float("inf"), -float("inf")):
        grads = gradients(torch, [100, 50], 4)
        grads[1][7] = bad
        before = [g.clone() for g in grads]
        norm = P.bsr_clip_grads(grads, 0.1)
        assert torch.isnan(norm) if bad != bad else torch.isinf(norm)
        assert all(torch.equal(g.nan_to_num(1e3), b.nan_to_num(1e3)) for g, b in zip(grads, before))


def test_shapes_and_the_same_bits(env):
    torch, P = env
    grads = [g.view(-1, 4) for g in gradients(torch, [4096, 40000], 5)]
    again = [g.clone() for g in grads]
    assert torch.equal(P.bsr_clip_grads(grads, 0.25), P.bsr_clip_grads(again, 0.25))
    assert all(torch.equal(a, b) for a, b in zip(grads, again))


def test_replayed(env):
    """recorded once, replayed on new gradients with the program's own work between"""
    torch, P = env
    held = gradients(torch, [70000, 300, 16385], 6)
    out = [torch.empty_like(g) for g in held]
    P.bsr_clip_grads(held, 0.5, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = P.bsr_clip_grads(held, 0.5, out=out)
    for k in range(4):
        now = gradients(torch, [70000, 300, 16385], 7 + k, scale=10.0 ** (2 * k - 5))
        want = [torch.empty_like(g) for g in now]
        length = P.bsr_clip_grads(now, 0.5, out=want)
        for h, n in zip(held, now):
            h.copy_(n)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(norm, length) and all(torch.equal(o, w) for o, w in zip(out, want))


def test_a_step_with_its_gradients_clipped(env):
    """the trainable tensors' gradients of a step, taken together, in front of the optimizer"""
    torch, P = env
    from bsr_synth import get_config, make_inputs, make_params
    cfg = get_config("mini_4blk")
    x, labels = make_inputs(cfg, 2)[:2]
    ctx = P.Context(cfg, make_params(cfg), max_batch=2)
    inp = torch.as_tensor(x).to(ctx.act_dtype).cuda()
    grads = ctx.new_grads()
    ctx.bsr_train_blocks_fwd_bwd(ctx.bsr_forward_frozen(inp), torch.as_tensor(labels, dtype=torch.int32).cuda(), grads)
    want = np.sqrt(sum((host(g) ** 2).sum() for g in grads.values()))
    before = {n: g.clone() for n, g in grads.items()}
    norm = ctx.bsr_clip_grads(grads, 0.5 * want)
    assert abs(float(norm) - want) <= 1.01 * 2.0 ** -24 * want
    for n, g in grads.items():
        assert (np.abs(host(g) - 0.5 * host(before[n])) <= 2.1 * 2.0 ** -24 * np.abs(host(before[n])) + 1e-38).all()
    ctx.bsr_sgd_step(grads, None, 0.1)


def test_far_values(env):
    """a tensor of more than 2^31 values: the last ones count and are scaled"""
    torch, P = env
    n = (1 << 31) + 5
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[-1], g[0] = 3.0, 4.0
    norm = P.bsr_clip_grads([g], 1.0)
    assert float(norm) == 5.0 and abs(float(g[-1]) - 0.6) <= 0.6 * 2.0 ** -8 and abs(float(g[0]) - 0.8) <= 0.8 * 2.0 ** -8
