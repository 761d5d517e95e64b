"""Tuning the head of a frozen model for many classes, and the gains of its norms with it, with the library's operators on their own tensors.

The model is a stack of pre-norm feed-forward blocks, x + fc2(GELU(fc1(RMSNorm(x)))), a final RMSNorm and a linear head.  The blocks' matrices are frozen and kept in 8 bits only; what
learns are the norms' gains and the head.  A step runs, of each block,

    bsr_rmsnorm_forward8 (the branch before is added on the way in) -> bsr_linear8_forward (GELU, its input kept) -> bsr_linear8_forward

the final bsr_rmsnorm_forward, bsr_linear_ce_forward_backward with the head, whose logits nobody keeps, and back

    bsr_rmsnorm_backward -> per block: bsr_linear8_dgrad (GELU' of the kept input) -> bsr_linear8_dgrad -> bsr_rmsnorm_backward (the stream's gradient added)

with the 8-bit rounding of activations counted as the identity; then bsr_clip_grads on all gradients taken together, and a step of gradient descent.

    python -m paper_2405_10951_amd.head_tuning --rows 6304 --width 768 --hidden 1536 --depth 4 --classes 21841 --steps 60
"""
from __future__ import annotations

import argparse
import time

import paper_2405_10951_amd as P

EPS = 1e-6


class TunedHead:
    """`blocks`: [(fc1 [width,hidden], b1 [hidden], fc2 [hidden,width], b2 [width])], matrices bf16 or fp32, biases fp32; `head`: (weight [classes,width], bias [classes]), fp32, learned;
    all on one GPU.  `gains`: a norm's each and the final one's, fp32, learned."""

    def __init__(self, blocks, head):
        import torch
        self.blocks = [(P.bsr_quantize8_weight(fc1), b1, P.bsr_quantize8_weight(fc2), b2) for fc1, b1, fc2, b2 in blocks]
        self.weight, self.bias = head
        self.gains = [torch.ones(self.weight.shape[1], device=self.weight.device) for _ in range(len(blocks) + 1)]

    def gradients(self, x, labels):
        """x [rows,width] bf16, labels [rows] int32 (-1: the row counts for nothing) -> (loss of every row, [gains' gradients ..., the head's, its bias's])"""
        import torch
        kept, stream, branch = [], x, None
        for (fc1, b1, fc2, b2), gamma in zip(self.blocks, self.gains):
            h, rstd, stream = P.bsr_rmsnorm_forward8(stream, gamma, EPS, res=branch)
            u = torch.empty((x.shape[0], fc1.n_out), dtype=x.dtype, device=x.device)
            branch = P.bsr_linear8_forward(P.bsr_linear8_forward(h, fc1, bias=b1, act=1, u_out=u, out_dtype=x.dtype), fc2, bias=b2)
            kept.append((stream, rstd, u))
        h, rstd, stream = P.bsr_rmsnorm_forward(stream, self.gains[-1], EPS, res=branch)
        loss, dh, dw, db = P.bsr_linear_ce_forward_backward(h, self.weight.to(x.dtype), labels, bias=self.bias, grad_scale=1.0 / x.shape[0], dw=torch.empty_like(self.weight))
        d, dgamma = P.bsr_rmsnorm_backward(dh, stream, rstd, self.gains[-1])
        grads = [dgamma]
        for i in reversed(range(len(self.blocks))):
            fc1, _, fc2, _ = self.blocks[i]
            stream, rstd, u = kept[i]
            dh = P.bsr_linear8_dgrad(P.bsr_linear8_dgrad(d, fc2, u=u), fc1)
            d, dgamma = P.bsr_rmsnorm_backward(dh, stream, rstd, self.gains[i], res=d if i else None, need_dx=i > 0)
            grads.append(dgamma)
        return loss, grads[::-1] + [dw, db]

    def step(self, x, labels, lr=0.0, max_norm=None):
        """One step of gradient descent on the mean loss -> (loss of every row, gradients, their norm before the clipping or None)"""
        loss, grads = self.gradients(x, labels)
        norm = None if max_norm is None else P.bsr_clip_grads(grads, max_norm)
        if lr:
            for p, g in zip(self.gains + [self.weight, self.bias], grads):
                p.add_(g, alpha=-lr)
        return loss, grads, norm


def random_model(width, hidden, depth, classes, seed=0, device="cuda"):
    """Random frozen matrices, scaled as trained ones are, and a random head."""
    import torch
    gen = torch.Generator(device=device).manual_seed(seed)

    def normal(*shape, scale=1.0, dtype=torch.float32):
        return (scale * torch.randn(*shape, generator=gen, device=device)).to(dtype)

    blocks = [(normal(width, hidden, scale=width ** -0.5, dtype=torch.bfloat16), normal(hidden, scale=0.1),
               normal(hidden, width, scale=hidden ** -0.5, dtype=torch.bfloat16), normal(width, scale=0.1)) for _ in range(depth)]
    return TunedHead(blocks, (normal(classes, width, scale=width ** -0.5), torch.zeros(classes, device=device)))


def main():
    import torch
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("rows", 6304), ("width", 768), ("hidden", 1536), ("depth", 4), ("classes", 21841), ("steps", 60)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--lr", type=float, default=20.0)
    ap.add_argument("--max-norm", type=float, default=0.1)
    a = ap.parse_args()
    model = random_model(a.width, a.hidden, a.depth, a.classes)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(a.rows, a.width, generator=gen, device="cuda").bfloat16()
    labels = torch.randint(a.classes, (a.rows,), generator=gen, device="cuda", dtype=torch.int32)
    torch.cuda.synchronize()
    start = time.perf_counter()
    for i in range(a.steps):
        loss, _, norm = model.step(x, labels, lr=a.lr, max_norm=a.max_norm)
        if i % 10 == 0 or i == a.steps - 1:
            print(f"step {i}: loss {loss.mean().item():.4f}, gradient norm {norm.item():.4f}", flush=True)
    torch.cuda.synchronize()
    print(f"{(time.perf_counter() - start) / a.steps * 1e3:.3f} ms a step, {a.rows} rows")


if __name__ == "__main__":
    main()
