"""Plain attention in 64 bits, with what its bf16 form may be off by."""
import torch

F64 = torch.float64


def attend(q, k, v, ok, weight=2.0 ** -8):
    """(out, tolerance) for q [n, d], k and v [m, d] (bf16) and ok [n, m], in 64 bits; zeros where a row has no key.

    The tensor cores' scores, fp32 sums of d exact products, are off by at most s = (d / 16 + 32) 2^-23 |q| . |k|, which moves a weight
    by 2 s of itself (its own score and the sum); its power of two and the running maximum's products by 2^-20; its rounding to bf16 by
    `weight`, 2^-8, or as the sum of two bf16 by 2^-8 of the first one's rest, 2^-16.  The sum of weighted values is then rounded once more, 2^-8 of the result, after fp32 sums over the keys (2^-23 of
    the magnitudes for each sixteen keys)."""
    q, k, v = q.to(F64), k.to(F64), v.to(F64)
    s = (q @ k.T).masked_fill(~ok, -torch.inf)
    m = s.amax(1, keepdim=True).clamp_min(-1e300) if k.shape[0] else s.sum(1, keepdim=True)
    p = torch.exp(s - m)
    p = p / p.sum(1, keepdim=True).clamp_min(1e-300)
    out, mag = p @ v, p @ v.abs()
    off = ((q.shape[1] / 16 + 32) * 2.0 ** -23 * (q.abs() @ k.abs().T)).masked_fill(~ok, 0)
    off = off.amax(1, keepdim=True) if k.shape[0] else 0.0
    return out, 2.0 ** -8 * out.abs() + mag * (weight + 2 * off + 2.0 ** -20 + (k.shape[0] / 16 + 32) * 2.0 ** -23) + 1e-30
