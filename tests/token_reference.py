"""The operators over tokens from their definitions in 64 bits, with the sizes their rounding errors are measured against.

Each reference returns the value and, for sums, the same sum over absolute values: an fp32 sum of n terms is off by at
most n * 2^-23 of that (each addition by half a step of 2^-24 when rounded, by a whole one where an adder cuts off)."""
import math

import torch

STEP = 2.0 ** -23


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def norm_rope(x, w, positions, inv_freq, eps, norm, interleaved, gain):
    """-> (value, size): size is the largest absolute value of the normed row."""
    y = x.double()
    if norm:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps)
        if w is not None:
            y = y * w.double()
    size = y.abs().amax(-1, keepdim=True) * max(1.0, abs(gain)) * 2
    half = 0 if inv_freq is None else inv_freq.shape[0]
    if half:
        t = positions.double()[..., None] * inv_freq
        t = t.expand(x.shape[0], x.shape[1], half)[:, :, None]
        i = torch.arange(half, device=x.device)
        first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        a, b = y[..., first].clone(), y[..., second].clone()
        y[..., first] = gain * (a * t.cos() - b * t.sin())
        y[..., second] = gain * (b * t.cos() + a * t.sin())
    return y, size


def linear(q, k, v, log_decay, state, scale, lengths=None):
    """state [B][H][D][D] -> (out, its size, last state, its size), token by token."""
    B, T, H, D = q.shape
    g = H // k.shape[2]
    q, k, v = q.double() * scale, k.double().repeat_interleave(g, 2), v.double().repeat_interleave(g, 2)
    d = torch.exp(log_decay.double())[None, :, None, None]
    S, A = state.double().clone(), state.double().abs()
    out, size = torch.zeros(B, T, H, D, dtype=torch.float64, device=q.device), torch.zeros(B, T, H, D, dtype=torch.float64, device=q.device)
    n = [T] * B if lengths is None else [max(0, min(T, int(x))) for x in lengths]
    for b in range(B) if lengths is not None else [slice(None)]:
        for t in range(n[b] if lengths is not None else T):
            kv = k[b, t][..., :, None] * v[b, t][..., None, :]
            S[b] = torch.where(d[0] == 0, 0.0, S[b] * d[0]) + kv
            A[b] = torch.where(d[0] == 0, 0.0, A[b] * d[0]) + kv.abs()
            out[b, t] = (q[b, t][..., None, :] @ S[b])[..., 0, :]
            size[b, t] = (q[b, t][..., None, :].abs() @ A[b])[..., 0, :]
    return out, size, S, A


def cross(q, k, v, scale, kv_lengths=None, mask=None):
    """-> (out, size of the weighted sum, largest size of a score's sum per row).  Keys out of sight are left out before anything is computed."""
    B, Tq, H, D = q.shape
    Tk, g = k.shape[1], H // k.shape[2]
    out = torch.zeros(B, Tq, H, D, dtype=torch.float64, device=q.device)
    size, score = torch.zeros_like(out), torch.zeros(B, Tq, H, 1, dtype=torch.float64, device=q.device)
    for b in range(B):
        n = Tk if kv_lengths is None else max(0, min(Tk, int(kv_lengths[b])))
        rows = [(slice(None), torch.arange(n, device=q.device))]
        if mask is not None and mask.dim() == 2:
            rows = [(slice(None), torch.nonzero(mask[b, :n])[:, 0])]
        elif mask is not None:
            rows = [(slice(i, i + 1), torch.nonzero(mask[b, i, :n])[:, 0]) for i in range(Tq)]
        for at, seen in rows:
            if not len(seen):
                continue
            for h in range(H):
                x, y, z = q[b, at, h].double(), k[b, seen, h // g].double(), v[b, seen, h // g].double()
                w = torch.softmax(x @ y.T * scale, -1)
                out[b, at, h] = w @ z
                size[b, at, h] = w @ z.abs()
                score[b, at, h] = (x.abs() @ y.abs().T * scale).amax(-1, keepdim=True)
    return out, size, score


def linear_bounds(out, size, state_size, D, T, dtype, exact_products):
    """A chain is at most D products, 128 tokens of a chunk and two roundings per chunk, and of those the smallest has 32 tokens; where
    the products run on 16-bit operands the weights of a chunk and the state before it are rounded to them once each."""
    n = 2 * D + 128 + 2 * (T // 32 + 1) + 16
    once = 0.0 if exact_products else 2.0 ** -8
    return half_step(dtype) * out.abs() + (n * STEP + once) * size, n * STEP * state_size


def cross_bounds(out, size, score, D, Tk, dtype, once):
    """A score is off by D steps of its size, and its exponential by that share and that of forming the argument and evaluating it (2^-20);
    both sums carry it.  `once`: weights' own rounding."""
    share = 2 * ((D + 2) * STEP * score + 2.0 ** -20) + once + (Tk + 64) * STEP
    return half_step(dtype) * out.abs() + share * size


def check(got, want, bound, name):
    err = (got.double() - want).abs()
    bad = ~(err <= bound)
    if bad.any():
        i = tuple(int(x) for x in torch.nonzero(bad)[0])
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.numel()} outside; first at {i}: {float(got[i])} for {float(want[i])}, "
                             f"off by {float(err[i]):.3e}, bound {float(bound.expand_as(err)[i]):.3e}")
