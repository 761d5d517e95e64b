"""The operators recorded into a graph: every replay, on new inputs and with the program's own work between, gives what the calls give."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,classes", [(20, 50), (300, 1000), (7, 140000)])
def test_a_step_in_a_graph(rows, classes):
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device")
    from paper_2405_10951_amd.norm_tuning import random_stack
    stack = random_stack(256, 384, 2, classes)
    gen = torch.Generator(device="cuda").manual_seed(3)

    def inputs():
        return (torch.randn(rows, 256, generator=gen, device="cuda").bfloat16(), torch.randint(classes, (rows, 9), generator=gen, device="cuda", dtype=torch.int32),
                2 * torch.randn(rows, 9, generator=gen, device="cuda"), torch.randint(classes, (rows,), generator=gen, device="cuda", dtype=torch.int32))

    def step(x, index, logits, labels):
        loss, grads = stack.step(x, index, logits, labels, 2.0, 0.25)
        return [loss] + [g for pair in grads for g in pair]

    held = inputs()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*held)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded = step(*held)
    for _ in range(4):
        now = inputs()
        want = [t.clone() for t in step(*now)]
        torch.cuda.synchronize()
        for h, n in zip(held, now):
            h.copy_(n)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.isfinite(t).all() for t in want)
        assert all(torch.equal(r, w) for r, w in zip(recorded, want))
