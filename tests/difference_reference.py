"""Differential attention from its definition in 64 bits, with bounds for what its roundings may do."""
import torch

from token_reference import STEP, cross_bounds, cross, half_step


def difference(q, k, v, vectors, lambda_init, scale, norm=True, weight=None, eps=1e-5, out_scale=1.0, kv_lengths=None, mask=None, once=0.0, dtype=torch.float32):
    """-> (out, bound).  Each map is cross attention of one half of the heads, with its bounds."""
    half, Tk = q.shape[-1] // 2, k.shape[1]
    H = q.shape[2]
    a = vectors.double().expand(H, 4, half) if vectors.dim() == 2 else vectors.double()
    lam = (torch.exp((a[:, 0] * a[:, 1]).sum(-1)) - torch.exp((a[:, 2] * a[:, 3]).sum(-1)) + lambda_init)[None, None, :, None]
    # both exponents are sums of `half` products, and the difference is off by what they are
    lam_off = (half + 4) * STEP * (torch.exp((a[:, 0] * a[:, 1]).abs().sum(-1)) + torch.exp((a[:, 2] * a[:, 3]).abs().sum(-1)) + abs(lambda_init))[None, None, :, None]
    y, off = 0.0, 0.0
    for at, gain, more in ((slice(0, half), torch.ones_like(lam), 0.0), (slice(half, None), -lam, lam_off)):
        # values are wider than a half: two calls, of either half of them
        parts = [cross(q[..., at], k[..., at], v[..., i], scale, kv_lengths, mask) for i in (slice(0, half), slice(half, None))]
        o, size = (torch.cat([p[i] for p in parts], -1) for i in (0, 1))
        share = cross_bounds(torch.zeros_like(o), size, parts[0][2], half, Tk, torch.float64, once)
        y, off = y + gain * o, off + gain.abs() * share + more * o.abs()
    off = off + 4 * STEP * y.abs()
    if norm:
        rms = torch.sqrt((y * y).mean(-1, keepdim=True) + eps)
        g = torch.where(rms == 0, 0.0, 1 / torch.where(rms == 0, 1.0, rms)) * abs(out_scale) * (1.0 if weight is None else weight.double().abs())
        moved = torch.sqrt((off * off).mean(-1, keepdim=True)) / torch.where(rms == 0, 1.0, rms)
        out = y / torch.where(rms == 0, 1.0, rms) * out_scale * (1.0 if weight is None else weight.double())
        # the row's length moves with its elements, to either side; where that is not small against it the row may be anything of its length
        bound = g * off / (1 - moved).clamp(min=1e-3) + out.abs() * (moved / (1 - moved).clamp(min=1e-3) + (q.shape[-1] + 8) * STEP)
    else:
        out, bound = y * out_scale, off * abs(out_scale) + y.abs() * abs(out_scale) * STEP
    return out, bound * (1 + half_step(dtype)) + half_step(dtype) * out.abs()
