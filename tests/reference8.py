"""8-bit blocks in numpy and 64 bits, from their definition: e is the smallest integer >= -127 with max|x| 2^-e <= 448 (0 for zeros), the
values are x 2^-e on the grid of e4m3 (steps of 2^(floor(log2|v|) - 3), 2^-9 at least), to nearest and ties to even."""
import numpy as np


def exponent(most):
    """most >= 0, finite -> e"""
    if most == 0:
        return 0
    m, e = np.frexp(most)                # most = m 2^e, m in [0.5, 1); 448 = 0.875 2^9
    return max(int(e) - 9 + (1 if m > 0.875 else 0), -127)


def to_e4m3(v):
    v = np.asarray(v, np.float64)
    a = np.abs(v)
    _, e = np.frexp(np.where(a > 0, a, 1.0))
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.sign(v) * np.round(a / step) * step          # (np.round: halves to even)


def blocks8(x, br, bc):
    """x [M,K] -> (values that the 8-bit form stands for, exponents [blocks down, blocks across]); non-finite x: NaN, not in the maximum"""
    x = np.asarray(x, np.float64)
    out = np.empty_like(x)
    nr, nc = -(-x.shape[0] // br), -(-x.shape[1] // bc)
    exps = np.zeros((nr, nc), np.int64)
    for i in range(nr):
        for j in range(nc):
            s = (slice(i * br, (i + 1) * br), slice(j * bc, (j + 1) * bc))
            b = x[s]
            ok = np.isfinite(b)
            e = exponent(np.abs(b[ok]).max() if ok.any() else 0.0)
            exps[i, j] = e
            q = np.full_like(b, np.nan)
            q[ok] = np.ldexp(to_e4m3(np.ldexp(b[ok], -e)), e)
            out[s] = q
    return out, exps


def decode(values, scales, rows_per_scale, cols):
    """uint8 values [M, ldv], scales [.., lds] (numpy) -> fp64 [M, cols]"""
    import torch
    v = torch.from_numpy(np.ascontiguousarray(values)).view(torch.float8_e4m3fn).double().numpy()
    e = scales.astype(np.int64) - 127
    e = np.repeat(np.repeat(e, rows_per_scale, 0)[:v.shape[0]], 128, 1)[:, :v.shape[1]]
    return np.ldexp(v, e)[:, :cols]
