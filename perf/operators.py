"""The single operators of the library that a program calls on its own tensors, as cases that can be timed and compared.

Three families, which a program that tunes the LayerNorms of a frozen model against a teacher runs one after the other:

  layernorm  LayerNorm of rows, forward (y, mean, 1/std) or backward (dx, dgamma, dbeta)
  linear8    a frozen linear layer whose weights are e4m3 values with a power-of-two scale for each block of 128 x 128:
             forward (the rows are brought to 8 bits, 1 x 128 a block, on the way in; with norm, by the LayerNorm in front of
             the layer), or the input gradient
  distill    the loss of a classifier against a teacher's top logits mixed with the label's cross-entropy, and its gradient

`own` false computes the operators in elementary torch operations in 32 bits; `own` true calls the library.

8-bit blocks.  A block's exponent e is the smallest integer (-127 at least) with max|x| 2^-e <= 448, 448 being the largest e4m3
value; the block holds x 2^-e rounded to e4m3, to nearest and ties to even.  Everything but that rounding is exact.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
BLOCK = 128
EPS = 1e-6
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}

# what no drawn case exceeds: the largest listed ones
MOST_ROWS, MOST_WIDTH = 16384, 8192
MOST_PRODUCT = 16384 * 4096 * 8192
MOST_NORM = 16384 * 8192
MOST_CLASSES, MOST_DISTILL, MOST_TOP = 131072, 4096 * 131072, 64


def _linear8(direction, rows, n_in, n_out, dtype="bf16", norm=False, gelu=False, res=False, **more):
    return dict(what="linear8", dir=direction, rows=rows, n_in=n_in, n_out=n_out, dtype=dtype, norm=norm, gelu=gelu, res=res, **more)


def _layernorm(direction, rows, width, dtype="bf16", res=False, **more):
    return dict(what="layernorm", dir=direction, rows=rows, width=width, dtype=dtype, res=res, **more)


def _distill(direction, rows, classes, top, dtype="bf16", hard=0.0, temperature=1.0, **more):
    return dict(what="distill", dir=direction, rows=rows, classes=classes, top=top, dtype=dtype, hard=hard, temperature=temperature, **more)


def listed():
    return [
        # one token through a square projection, as a model that answers token by token has it: latency and the weights' bytes
        _linear8("fwd", 1, 4096, 4096, name="linear8_token"),
        # LayerNorm and qkv of a frozen ViT-B block, 32 images
        _linear8("fwd", 6304, 768, 2304, norm=True, name="linear8_vit_b_norm_qkv"),
        # back through fc2 and the GELU of a frozen DeiT-S block in the gradient path
        _linear8("dgrad", 6304, 1536, 384, gelu=True, name="linear8_deit_s_fc2_dgrad"),
        # nothing a multiple of anything, fp32 in and out, residual added
        _linear8("fwd", 999, 1000, 1111, dtype="f32", res=True, name="linear8_ragged_f32"),
        # the first layer of a large feed-forward network, GELU behind it
        _linear8("fwd", 16384, 4096, 8192, gelu=True, name="linear8_large_gelu"),
        # the tokens of one image: latency
        _layernorm("fwd", 197, 768, name="layernorm_one_image"),
        # 32 images of ViT-B, backward with the branch's gradient added
        _layernorm("bwd", 6304, 768, res=True, name="layernorm_vit_b_bwd"),
        # odd rows in fp32
        _layernorm("bwd", 1031, 1777, dtype="f32", name="layernorm_odd_f32_bwd"),
        # a long batch of a wide model
        _layernorm("bwd", 16384, 8192, name="layernorm_large_bwd"),
        # the head of the 100-class fine-tuning run, label mixed in
        _distill("both", 32, 100, 10, dtype="f32", hard=0.5, temperature=3.0, name="distill_100_classes"),
        # an odd number of classes, the gradient alone, as an autograd tape asks for it
        _distill("bwd", 2048, 21841, 32, hard=0.1, temperature=2.0, name="distill_21841_classes_bwd"),
        # a vocabulary
        _distill("both", 4096, 131072, 64, name="distill_vocabulary"),
    ]


def _log_uniform(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    what = rng.choice(["linear8", "layernorm", "distill"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if what == "linear8":
        n_in, n_out = _log_uniform(rng, 64, MOST_WIDTH), _log_uniform(rng, 64, MOST_WIDTH)
        if rng.random() < 0.6:                                # most layers are wide in whole vectors
            n_in, n_out = (n_in + 63) // 64 * 64, (n_out + 63) // 64 * 64
        rows = _log_uniform(rng, 1, max(1, min(MOST_ROWS, MOST_PRODUCT // (n_in * n_out))))
        direction = rng.choice(["fwd", "fwd", "dgrad"])
        norm = direction == "fwd" and rng.random() < 0.3
        gelu = rng.random() < 0.4
        return _linear8(direction, rows, n_in, n_out, dtype=dtype, norm=norm, gelu=gelu,
                        res=direction == "fwd" and not gelu and rng.random() < 0.5)
    if what == "layernorm":
        width = _log_uniform(rng, 64, MOST_WIDTH)
        if rng.random() < 0.6:
            width = (width + 63) // 64 * 64
        rows = _log_uniform(rng, 1, min(MOST_ROWS, MOST_NORM // width // SIZE[dtype] * 2))
        direction = rng.choice(["fwd", "bwd"])
        return _layernorm(direction, rows, width, dtype=dtype, res=direction == "bwd" and rng.random() < 0.5)
    classes = _log_uniform(rng, 10, MOST_CLASSES)
    rows = _log_uniform(rng, 1, max(1, min(4096, MOST_DISTILL // classes // SIZE[dtype] * 2)))
    return _distill(rng.choice(["both", "fwd", "bwd"]), rows, classes, _log_uniform(rng, 1, min(MOST_TOP, classes)), dtype=dtype,
                    hard=rng.choice([0.0, 0.1, 0.5]), temperature=rng.choice([1.0, 2.0, 4.0]))


# ------------------------------------------------------------------------------------------------ inputs

def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    dtype = TYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEV)

    state = dict(case=case)
    if case["what"] == "linear8":
        rows, n_in, n_out = case["rows"], case["n_in"], case["n_out"]
        # a few features of a token are far larger than the rest, in every model
        spread = torch.exp(0.7 * normal(n_in if case["dir"] == "fwd" else n_out))
        state["weight"] = (normal(n_in, n_out) / math.sqrt(n_in)).to(dtype)
        if case["dir"] == "fwd":
            state["x"] = (normal(rows, n_in) * spread).to(dtype)
            state["bias"] = 0.1 * normal(n_out)
            if case["norm"]:
                state["gamma"], state["beta"] = 1 + 0.1 * normal(n_in), 0.1 * normal(n_in)
            if case["res"]:
                state["res"] = normal(rows, n_out).to(dtype)
        else:
            state["dy"] = (1e-3 * normal(rows, n_out) * spread).to(dtype)
            if case["gelu"]:
                state["u"] = normal(rows, n_in).to(dtype)
        # the frozen layer as the program keeps it: 8-bit values and scales, not the matrix they came from
        if own:
            import paper_2405_10951_amd as P
            state["frozen"] = P.bsr_quantize8_weight(state["weight"])
        else:
            state["frozen"] = _eight_bits(state["weight"].float(), BLOCK, BLOCK)
        if not case.get("keep_weight"):
            del state["weight"]
    elif case["what"] == "layernorm":
        rows, width = case["rows"], case["width"]
        x = normal(rows, width) * (1 + normal(rows, 1).abs()) + normal(rows, 1)
        state["x"] = x.to(dtype)
        state["gamma"], state["beta"] = 1 + 0.1 * normal(width), 0.1 * normal(width)
        if case["dir"] == "bwd":
            state["dy"] = (0.1 * normal(rows, width)).to(dtype)
            if case["res"]:
                state["res"] = (0.1 * normal(rows, width)).to(dtype)
            xd = state["x"].double()
            state["mean"] = xd.mean(1).float()
            state["rstd"] = torch.rsqrt(xd.var(1, unbiased=False) + EPS).float()
    else:
        rows, classes, top = case["rows"], case["classes"], case["top"]
        z = 2 * normal(rows, classes)
        state["z"] = z.to(dtype)
        # the teacher agrees with the student in the main and is surer of itself
        values, index = [], []
        for part in z.split(512):
            v, i = torch.topk(part + normal(*part.shape), top, dim=1)
            values.append(v)
            index.append(i)
        state["top_index"] = torch.cat(index).to(torch.int32)
        state["top_logits"] = (1.5 * torch.cat(values)).contiguous()
        state["labels"] = torch.randint(classes, (rows,), generator=gen, device=DEV, dtype=torch.int32)
        if rows > 4 and top > 1:                               # a shorter list, no list, no label: as a data set holds them
            state["top_index"][1, top // 2:] = -1
            state["top_index"][3] = -1
            state["labels"][4] = -1
        if case["dir"] == "bwd":
            state["row_grad"] = (1 + 0.1 * normal(rows).abs()) / rows
            # what the forward leaves: the largest logit and the logarithms of both sums of exp(difference to it)
            most = state["z"].float().amax(1, keepdim=True)
            d = state["z"].double() - most
            state["stats"] = torch.cat([most, torch.logsumexp(d / case["temperature"], 1, keepdim=True).float(),
                                        torch.logsumexp(d, 1, keepdim=True).float()], 1)
    return state


# ------------------------------------------------------------------------------------------------ the plain forms

def _blocks(x, br, bc):
    """x padded with zeros to whole blocks, as [blocks down, br, blocks across, bc]"""
    rows, cols = x.shape
    x = torch.nn.functional.pad(x, (0, -cols % bc, 0, -rows % br))
    return x.view(x.shape[0] // br, br, x.shape[1] // bc, bc)


def _two_to(e):
    """2^e in fp32, from the bits of an fp64: torch's ldexp goes through pow, which is not exact on a GPU, and of bf16 values one in
    sixteen lies halfway between two e4m3 values"""
    return ((e.long() + 1023) << 52).view(torch.float64).float()


def _eight_bits(x, br, bc):
    """fp32 x -> (e4m3 values, exponents of its blocks)"""
    b = _blocks(x, br, bc)
    m, e = torch.frexp(b.abs().amax((1, 3), keepdim=True))     # m in [0.5, 1); 448 = 0.875 * 2^9
    e = torch.where(m > 0, e - 9 + (m > 0.875), 0).clamp_min(-127)
    q = (b * _two_to(-e)).to(torch.float8_e4m3fn)
    return q.view(q.shape[0] * br, -1)[:x.shape[0], :x.shape[1]], e.squeeze(3).squeeze(1)


def _values(q, e, br, bc):
    """the fp32 values that 8-bit blocks stand for"""
    rows, cols = q.shape
    s = e.repeat_interleave(br, 0)[:rows].repeat_interleave(bc, 1)[:, :cols]
    return q.float() * _two_to(s)


def _norm(x, gamma, beta):
    x = x.float()
    mean = x.mean(1, keepdim=True)
    c = x - mean
    rstd = torch.rsqrt((c * c).mean(1, keepdim=True) + EPS)
    return c * rstd * gamma + beta, mean.squeeze(1), rstd.squeeze(1)


def _phi(u):
    return 0.5 * (1 + torch.erf(u * math.sqrt(0.5)))


def _run_plain(s, case):
    if case["what"] == "linear8":
        w = _values(*s["frozen"], BLOCK, BLOCK)
        if case["dir"] == "dgrad":
            dtype = s["dy"].dtype
            dx = _values(*_eight_bits(s["dy"].float(), 1, BLOCK), 1, BLOCK) @ w.t()
            if case["gelu"]:
                u = s["u"].float()
                dx = dx * (_phi(u) + u * torch.exp(-0.5 * u * u) / math.sqrt(2 * math.pi))
            return dx.to(dtype)
        x = _norm(s["x"], s["gamma"], s["beta"])[0] if case["norm"] else s["x"].float()
        y = _values(*_eight_bits(x, 1, BLOCK), 1, BLOCK) @ w + s["bias"]
        if case["gelu"]:
            y = y * _phi(y)
        if case["res"]:
            y = y + s["res"].float()
        return y.to(s["x"].dtype)
    if case["what"] == "layernorm":
        if case["dir"] == "fwd":
            y, mean, rstd = _norm(s["x"], s["gamma"], s["beta"])
            return y.to(s["x"].dtype), mean, rstd
        dy = s["dy"].float()
        xhat = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        g = dy * s["gamma"]
        dx = s["rstd"][:, None] * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
        if case["res"]:
            dx = dx + s["res"].float()
        return dx.to(s["x"].dtype), (dy * xhat).sum(0), dy.sum(0)
    z, temperature, hard = s["z"].float(), case["temperature"], case["hard"]
    present = s["top_index"] >= 0
    index = s["top_index"].clamp_min(0).long()
    some = present.any(1)
    t = torch.where(present, s["top_logits"] / temperature, -math.inf)
    t = torch.where(some[:, None], t - t.amax(1, keepdim=True), 0.0)
    p = torch.where(present, torch.exp(t), 0.0)
    p = p / p.sum(1, keepdim=True).clamp_min(1e-30)
    labelled = s["labels"] >= 0
    label = s["labels"].clamp_min(0).long()[:, None]

    def log_sum(v):
        m = v.amax(1, keepdim=True)
        return m + torch.log(torch.exp(v - m).sum(1, keepdim=True))

    if case["dir"] == "bwd":
        z = z - s["stats"][:, :1]
        lse_t, lse_1 = s["stats"][:, 1:2], s["stats"][:, 2:]
        weight = s["row_grad"][:, None]
    else:
        lse_t = log_sum(z / temperature)
        lse_1 = log_sum(z) if hard else lse_t
        weight = 1.0 / z.shape[0]
        log_q = torch.gather(z, 1, index) / temperature - lse_t
        kl = torch.where(p > 0, p * (torch.log(p.clamp_min(1e-30)) - log_q), 0.0).sum(1)
        loss = (1 - hard) * temperature ** 2 * kl
        if hard:
            loss = loss + hard * torch.where(labelled, (lse_1 - torch.gather(z, 1, label)).squeeze(1), 0.0)
        if case["dir"] == "fwd":
            return loss
    soft = (1 - hard) * temperature * weight * some[:, None]
    dz = soft * torch.exp(z / temperature - lse_t)
    dz.scatter_add_(1, index, -soft * p)
    if hard:
        mix = hard * weight * labelled[:, None]
        dz = dz + mix * torch.exp(z - lse_1)
        dz.scatter_add_(1, label, -mix * torch.ones_like(label, dtype=torch.float32))
    dz = dz.to(s["z"].dtype)
    return dz if case["dir"] == "bwd" else (loss, dz)


# ------------------------------------------------------------------------------------------------ the library's calls

def _run_own(s, case):
    import paper_2405_10951_amd as P
    if case["what"] == "linear8":
        if case["dir"] == "dgrad":
            return P.bsr_linear8_dgrad(s["dy"], s["frozen"], u=s.get("u"))
        x = s["x"]
        if case["norm"]:
            x = P.bsr_layernorm_forward8(x, s["gamma"], s["beta"], EPS)[0]
        return P.bsr_linear8_forward(x, s["frozen"], bias=s["bias"], act=int(case["gelu"]), res=s.get("res"), out_dtype=s["x"].dtype)
    if case["what"] == "layernorm":
        if case["dir"] == "fwd":
            return P.bsr_layernorm_forward(s["x"], s["gamma"], s["beta"], EPS)
        return P.bsr_layernorm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["gamma"], res=s.get("res"))
    how = dict(labels=s["labels"], temperature=case["temperature"], hard_weight=case["hard"])
    if case["dir"] == "bwd":
        return P.bsr_distill_backward(s["z"], s["top_index"], s["top_logits"], s["stats"], s["row_grad"], **how)
    if case["dir"] == "fwd":
        return P.bsr_distill_forward(s["z"], s["top_index"], s["top_logits"], **how)[0]
    return P.bsr_distill_forward_backward(s["z"], s["top_index"], s["top_logits"], grad_scale=1.0 / s["z"].shape[0], **how)


def run(state):
    return (_run_own if own else _run_plain)(state, state["case"])


# ------------------------------------------------------------------------------------------------ what a pass cannot do without

def work(case):
    e = SIZE[case["dtype"]]
    if case["what"] == "linear8":
        rows, n_in, n_out = case["rows"], case["n_in"], case["n_out"]
        scales = math.ceil(n_in / BLOCK) * math.ceil(n_out / BLOCK)
        moved = e * rows * (n_in + n_out) + n_in * n_out + scales
        if case["dir"] == "fwd":
            moved += 4 * n_out + (8 * n_in if case["norm"] else 0) + (e * rows * n_out if case["res"] else 0)
        elif case["gelu"]:
            moved += e * rows * n_in
        return {"bytes": moved, "flops": 2 * rows * n_in * n_out}
    if case["what"] == "layernorm":
        rows, width = case["rows"], case["width"]
        tensors = 2 if case["dir"] == "fwd" else 3 + case["res"]
        return {"bytes": tensors * e * rows * width + 8 * rows + (8 if case["dir"] == "fwd" else 12) * width,
                "flops": (8 if case["dir"] == "fwd" else 14) * rows * width}
    rows, classes, top = case["rows"], case["classes"], case["top"]
    passes = 1 if case["dir"] == "fwd" else 2
    return {"bytes": passes * e * rows * classes + 8 * rows * top + 8 * rows, "flops": 4 * passes * rows * classes}


# ------------------------------------------------------------------------------------------------ the same in 64 bits

def _exact_eight_bits(x, br, bc):
    """fp64 x -> the values its 8-bit blocks stand for"""
    rows, cols = x.shape
    powers = torch.tensor([2.0 ** k for k in range(-300, 301)], dtype=torch.float64, device=x.device)

    def two_to(e):
        return powers[e.long() + 300]

    b = _blocks(x, br, bc)
    most = b.abs().amax((1, 3), keepdim=True)
    e = torch.where(most > 0, torch.ceil(torch.log2(most / 448)), torch.zeros_like(most))
    e = torch.where(most > 448 * two_to(e), e + 1, e)           # (the logarithm's own rounding)
    e = torch.where((most > 0) & (most <= 448 * two_to(e - 1)), e - 1, e).clamp_min(-127)
    v = b * two_to(-e)
    step = two_to(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)      # e4m3: 3 bits behind the first, down to 2^-9
    v = torch.round(v / step) * step * two_to(e)
    return v.view(v.shape[0] * br, -1)[:rows, :cols]


def exact(case, seed):
    s = prepare(dict(case, keep_weight=True), seed)
    f = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    if case["what"] == "linear8":
        w = _exact_eight_bits(f["weight"], BLOCK, BLOCK)
        if case["dir"] == "dgrad":
            dx = _exact_eight_bits(f["dy"], 1, BLOCK) @ w.t().contiguous()
            if case["gelu"]:
                u = f["u"].cpu() if f["u"].numel() < 1 << 22 else f["u"]
                dx = dx * (0.5 * torch.erfc(-u / math.sqrt(2)) + u * torch.exp(-u * u / 2) / math.sqrt(2 * math.pi)).to(DEV)
            return dx
        x = f["x"]
        if case["norm"]:
            x = torch.nn.functional.layer_norm(x, (x.shape[1],), f["gamma"], f["beta"], EPS)
        y = torch.addmm(f["bias"], _exact_eight_bits(x, 1, BLOCK), w)
        if case["gelu"]:
            y = y * 0.5 * torch.erfc(-y / math.sqrt(2))
        return y + f["res"] if case["res"] else y
    if case["what"] == "layernorm":
        x = f["x"].clone().requires_grad_()
        gamma, beta = f["gamma"].requires_grad_(), f["beta"].requires_grad_()
        y = torch.nn.functional.layer_norm(x, (x.shape[1],), gamma, beta, EPS)
        if case["dir"] == "fwd":
            var, mean = torch.var_mean(f["x"], 1, unbiased=False)
            return y.detach(), mean, 1 / torch.sqrt(var + EPS)
        dx, dgamma, dbeta = torch.autograd.grad(y, (x, gamma, beta), f["dy"])
        return (dx + f["res"] if case["res"] else dx), dgamma, dbeta
    temperature, hard, rows = case["temperature"], case["hard"], case["rows"]
    z = f["z"].requires_grad_()
    present = s["top_index"] >= 0
    t = (f["top_logits"] / temperature).masked_fill(~present, -math.inf)
    p = torch.softmax(t, 1).nan_to_num(0.0)                      # (a row without entries has no distribution)
    log_q = torch.log_softmax(z / temperature, 1).gather(1, s["top_index"].clamp_min(0).long())
    kl = (torch.special.xlogy(p, p) - p * log_q).masked_fill(~present, 0.0).sum(1)
    loss = (1 - hard) * temperature ** 2 * kl
    if hard:
        loss = loss + hard * torch.nn.functional.cross_entropy(z, s["labels"].long(), ignore_index=-1, reduction="none")
    if case["dir"] == "fwd":
        return loss.detach()
    weight = f["row_grad"] if case["dir"] == "bwd" else torch.full((rows,), 1.0 / rows, dtype=torch.float64, device=DEV)
    dz, = torch.autograd.grad(loss, z, weight)
    return dz if case["dir"] == "bwd" else (loss.detach(), dz)
