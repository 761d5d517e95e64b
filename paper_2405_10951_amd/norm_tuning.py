"""Tuning the norms of a frozen model against a teacher's top logits, with the library's operators on their own tensors.

The model is a stack of pre-norm feed-forward blocks, x + fc2(GELU(fc1(LayerNorm(x)))), a final LayerNorm and a head.  Its matrices
are frozen and kept in 8 bits only; what learns are gamma and beta of the LayerNorms.  A step runs, of each block,

    bsr_layernorm_forward8 -> bsr_linear8_forward (GELU, its input kept) -> bsr_linear8_forward (residual added)

the final norm and the head, bsr_distill_forward_backward on the logits, and back

    bsr_linear8_dgrad (GELU' of the kept input) -> bsr_linear8_dgrad -> bsr_layernorm_backward (residual gradient added; dgamma, dbeta)

with the 8-bit rounding of activations counted as the identity.  The products' sums are exact; --cut-sums takes the faster ones of fewer bits.

    python -m paper_2405_10951_amd.norm_tuning --rows 6304 --width 768 --hidden 1536 --depth 4 --classes 1000 --steps 60
"""
from __future__ import annotations

import argparse
import time

import paper_2405_10951_amd as P

EPS = 1e-6


class FrozenStack:
    """`weights`: [(fc1 [width,hidden], b1 [hidden], fc2 [hidden,width], b2 [width]) per block] and (head [width,classes], bias [classes]);
    matrices bf16 or fp32, biases fp32, all on one GPU.  `norms`: [gamma, beta] per block and of the final LayerNorm, fp32, learned.
    cut_sums: the products' sums faster and of fewer bits."""

    def __init__(self, blocks, head, cut_sums=False):
        import torch
        self.sums = dict(cut_sums=cut_sums)
        self.blocks = [(P.bsr_quantize8_weight(fc1), b1, P.bsr_quantize8_weight(fc2), b2) for fc1, b1, fc2, b2 in blocks]
        self.head, self.head_bias = P.bsr_quantize8_weight(head[0]), head[1]
        width = self.head.n_in
        self.norms = [[torch.ones(width, device=head[1].device), torch.zeros(width, device=head[1].device)] for _ in range(len(blocks) + 1)]

    def forward(self, x):
        """x [rows,width] bf16 -> (logits [rows,classes] bf16, what the backward needs)"""
        import torch
        kept = []
        for (fc1, b1, fc2, b2), (gamma, beta) in zip(self.blocks, self.norms):
            h, mean, rstd = P.bsr_layernorm_forward8(x, gamma, beta, EPS)
            u = torch.empty((x.shape[0], fc1.n_out), dtype=x.dtype, device=x.device)
            g = P.bsr_linear8_forward(h, fc1, bias=b1, act=1, u_out=u, out_dtype=x.dtype, **self.sums)
            kept.append((x, mean, rstd, u))
            x = P.bsr_linear8_forward(g, fc2, bias=b2, res=x, **self.sums)
        h, mean, rstd = P.bsr_layernorm_forward8(x, *self.norms[-1], EPS)
        kept.append((x, mean, rstd, None))
        return P.bsr_linear8_forward(h, self.head, bias=self.head_bias, out_dtype=x.dtype, **self.sums), kept

    def backward(self, dlogits, kept):
        """-> [[dgamma, dbeta] per norm]"""
        grads = []
        x, mean, rstd, _ = kept[-1]
        dx, *grad = P.bsr_layernorm_backward(P.bsr_linear8_dgrad(dlogits, self.head, **self.sums), x, mean, rstd, self.norms[-1][0])
        grads.append(grad)
        for i in reversed(range(len(self.blocks))):
            fc1, _, fc2, _ = self.blocks[i]
            x, mean, rstd, u = kept[i]
            dh = P.bsr_linear8_dgrad(P.bsr_linear8_dgrad(dx, fc2, u=u, **self.sums), fc1, **self.sums)
            dx, *grad = P.bsr_layernorm_backward(dh, x, mean, rstd, self.norms[i][0], res=dx if i else None, need_dx=i > 0)
            grads.append(grad)
        return grads[::-1]

    def step(self, x, top_index, top_logits, labels=None, temperature=2.0, hard_weight=0.0, lr=0.0, max_norm=None):
        """One step of gradient descent on the mean loss -> (loss of every row [rows], gradients); max_norm: all of them taken together are brought down to that norm first"""
        logits, kept = self.forward(x)
        loss, dlogits = P.bsr_distill_forward_backward(logits, top_index, top_logits, labels, temperature, hard_weight,
                                                       grad_scale=1.0 / x.shape[0], dz=logits)
        grads = self.backward(dlogits, kept)
        if max_norm is not None:
            P.bsr_clip_grads([g for grad in grads for g in grad], max_norm)
        if lr:
            for norm, grad in zip(self.norms, grads):
                for p, g in zip(norm, grad):
                    p.add_(g, alpha=-lr)
        return loss, grads


def random_stack(width, hidden, depth, classes, seed=0, device="cuda", cut_sums=False):
    """A stack of random frozen matrices, scaled as trained ones are."""
    import torch
    gen = torch.Generator(device=device).manual_seed(seed)

    def normal(*shape, scale=1.0, dtype=torch.float32):
        return (scale * torch.randn(*shape, generator=gen, device=device)).to(dtype)

    blocks = [(normal(width, hidden, scale=width ** -0.5, dtype=torch.bfloat16), normal(hidden, scale=0.1),
               normal(hidden, width, scale=hidden ** -0.5, dtype=torch.bfloat16), normal(width, scale=0.1)) for _ in range(depth)]
    return FrozenStack(blocks, (normal(width, classes, scale=2 * width ** -0.5, dtype=torch.bfloat16), torch.zeros(classes, device=device)), cut_sums)


def main():
    import torch
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("rows", 6304), ("width", 768), ("hidden", 1536), ("depth", 4), ("classes", 1000), ("top", 16), ("steps", 60)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--lr", type=float, default=2.0)
    ap.add_argument("--max-norm", type=float, default=None, help="clip the gradients, all taken together, to this norm")
    ap.add_argument("--cut-sums", action="store_true", help="let the 8-bit matrix instructions add the products")
    a = ap.parse_args()
    student, teacher = (random_stack(a.width, a.hidden, a.depth, a.classes, cut_sums=a.cut_sums) for _ in range(2))
    gen = torch.Generator(device="cuda").manual_seed(1)
    for gamma, beta in teacher.norms:                      # the same frozen matrices under other norms
        gamma.add_(torch.randn(a.width, generator=gen, device="cuda"), alpha=0.3)
        beta.add_(torch.randn(a.width, generator=gen, device="cuda"), alpha=0.3)
    x = torch.randn(a.rows, a.width, generator=gen, device="cuda").bfloat16()
    top_logits, top_index = torch.topk(teacher.forward(x)[0].float(), a.top, dim=1)
    top_index = top_index.int()
    torch.cuda.synchronize()
    start = time.perf_counter()
    for i in range(a.steps):
        loss, _ = student.step(x, top_index, top_logits, lr=a.lr, max_norm=a.max_norm)
        if i % 10 == 0 or i == a.steps - 1:
            print(f"step {i}: loss {loss.mean().item():.4f}", flush=True)
    torch.cuda.synchronize()
    print(f"{(time.perf_counter() - start) / a.steps * 1e3:.3f} ms a step, {a.rows} rows")


if __name__ == "__main__":
    main()
