"""The gated delta rule from its definition in 64 bits, with the sizes its rounding errors are measured against.

Each token turns the state's error E into exp(log_decay) (1 - beta k k^T) E plus what the token's own roundings add.  With
0 <= beta |k|^2 <= 2 the matrix lengthens no column of E, so an error at a token stays at most what it was, and a column of the state is
off by the sum of what its tokens added.  That is measured against the column's length as it stood, faded to the end (state_size), and, for what q
reads of it, times the length of q (size)."""
import torch

from token_reference import half_step

STEP = 2.0 ** -23


def delta(q, k, v, log_decay, beta, state, scale=1.0, lengths=None):
    """state [B][H][D][D] -> (out, its size, last state, its size), token by token."""
    B, T, H, D = v.shape
    g = H // k.shape[2]
    q, k, v = q.double().repeat_interleave(g, 2), k.double().repeat_interleave(g, 2), v.double()
    a = torch.ones(B, T, H, dtype=torch.float64, device=v.device) if log_decay is None else torch.exp(log_decay.double())
    beta = beta.double()
    S = state.double().clone()
    A = S.norm(dim=-2, keepdim=True)
    out, size = torch.zeros(B, T, H, D, dtype=torch.float64, device=v.device), torch.zeros(B, T, H, D, dtype=torch.float64, device=v.device)
    n = [T] * B if lengths is None else [max(0, min(T, int(x))) for x in lengths]
    order = sorted(set(n), reverse=True)
    for t in range(order[0] if order else 0):
        at = [b for b in range(B) if n[b] > t]
        at = slice(None) if len(at) == B else torch.tensor(at, device=v.device)
        f = a[at, t][..., None, None]
        old = torch.where(f == 0, torch.where(torch.isfinite(S[at]), 0.0, S[at] * f), S[at] * f)
        kt, u = k[at, t][..., None], None
        u = beta[at, t][..., None, None] * (v[at, t][..., None, :] - kt.transpose(-1, -2) @ old)
        S[at] = old + kt * u
        A[at] = torch.maximum(A[at] * f, S[at].norm(dim=-2, keepdim=True))
        qt = q[at, t][..., None, :]
        out[at, t] = (qt @ S[at])[..., 0, :] * scale
        size[at, t] = (qt.norm(dim=-1, keepdim=True) * A[at])[..., 0, :] * abs(scale)
    return out, size, S, A


def bounds(out, size, state_size, D, T, dtype, several):
    """A token's own roundings: its sums of D products (half a step each when rounded, a whole one where an adder cuts off) with windows of up to 64 tokens, of which two
    in a row are taken where a window's inverse is; the number of tokens whose errors add up is what their decay leaves of T, and independent
    errors add up as the root of that.  Of several bf16 tokens out reads the state, the corrections of a window and their weights with 16 bits each, which is off by up to
    2^-15, and a window's corrections are up to 32 of the column's length: 3 * 32 * 2^-15 of it are less than 2^-8."""
    n = (2 * D + 2 * 64 + 16) * max(1.0, T) ** 0.5 / 4
    # what fades below fp32's normal range (2^-126, whole steps of 2^-149) keeps fewer bits, the factor exp(log_decay) itself among it
    low = 2.0 ** -126
    once = 2.0 ** -8 if several and dtype == torch.bfloat16 else 0.0
    return half_step(dtype) * out.abs() + (n * STEP + once) * size + low, (n * STEP * state_size + low).expand(*state_size.shape[:-2], D, D)
