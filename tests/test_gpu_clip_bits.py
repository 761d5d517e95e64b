"""Clipped gradients to the last bit that their type holds.

Tolerance: squares, sum and factor are fp64, off by some 2^-50; the product is rounded to fp32, 2^-24 of itself, and for bf16 once more, 2^-8 of that."""
import numpy as np
import pytest

from test_gpu_clip import SIZES, gradients, host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device")
    import paper_2405_10951_amd as P
    return torch, P


@pytest.mark.parametrize("scale", [1.0, 1e-12, 1e15])
@pytest.mark.parametrize("k", range(len(SIZES)))
def test_one_rounding(env, k, scale):
    torch, P = env
    for elsewhere in (True, False):
        grads = gradients(torch, SIZES[k], 20 + k, scale)
        before = [host(g) for g in grads]
        norm = np.sqrt(sum((b ** 2).sum() for b in before))
        out = [torch.full_like(g, 9.0) for g in grads] if elsewhere else grads
        limit = float(np.float32(0.3 * norm))
        P.bsr_clip_grads(grads, limit, out=out if elsewhere else None)
        for b, o in zip(before, out):
            want = b * (limit / norm if norm > limit else 1.0)
            half = 2.0 ** -24 + (2.0 ** -8 if o.dtype is torch.bfloat16 else 0)
            assert (np.abs(host(o) - want) <= (half + 2.0 ** -40) * np.abs(want)).all()
