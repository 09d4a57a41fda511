"""The gated delta rule: gates at their ends token by token, and what several bf16 tokens' rows lose beyond their own rounding."""
import math

import pytest
import torch

import delta_reference as ref
from paper_2402_04466_b200 import binding
from test_gpu_delta_overflow import _element_by_element
from test_gpu_delta_rule import BF16, FP32, TYPES, _case, _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("T", [1, 5, 8])
@pytest.mark.parametrize("B", [2, 40])
def test_gates_at_their_ends(cuda_device, dtype, D, T, B):
    """No decay at all, decays of 0, -infinity and far below what 32 bits can hold at the first, a middle and the last token; beta of 0, 1 and nearly 2, with few and with many states."""
    H = 6
    q, k, v, decay, beta, state = _case(cuda_device, D + T, B, T, H, H, D, dtype)
    call = lambda f: binding.delta_rule(q, k, v, f, beta, state, state_out=torch.full_like(state, math.nan))      # noqa: E731
    _element_by_element(call(None), q, k, v, None, beta, state)
    decay[:, :, 0], decay[:, 0, 1], decay[:, T // 2, 2], decay[:, T - 1, 3], decay[:, 0, 4], decay[:, :, 5] = 0.0, -math.inf, -1e4, -90.0, -300.0, -1e-3
    beta[:, 0, 0], beta[:, :, 1], beta[:, :, 2], beta[:, T - 1, 3], beta[:, :, 5] = 0.0, 1.0, 2.0 - 2.0 ** -6, 0.0, 0.0
    _element_by_element(call(decay), q, k, v, decay, beta, state)


@pytest.mark.parametrize("B,T,H,K,D", [(2, 60, 2, 2, 64), (3, 33, 4, 2, 32), (4, 300, 4, 4, 64), (30, 100, 8, 4, 128), (2, 500, 2, 1, 128), (2, 700, 2, 2, 32), (40, 70, 8, 8, 64)])
@pytest.mark.parametrize("alike", [0.0, 0.7, 3.0])
def test_rows_of_several_bf16_tokens(cuda_device, B, T, H, K, D, alike):
    """Against the rounded value of the definition.  Two terms of bf16 keep 16 bits of S, U and P: what is cut off is less than 2^-14 of each, with either sign in a row's sum, so that
    a row before its rounding is off by less than 3 * 2^-14 of what it is in the mean, d.  It then rounds to the other neighbour, 2^-7 of the value away at most, for a share d / 2^-7 of the
    elements: sqrt(3 * 2^-14 * 2^-7) = 1.2e-3 of the whole in the mean.  (S, U or P rounded to bf16 once would be 2^-8 / sqrt(3) = 2.3e-3 of it by themselves.)"""
    q, k, v, decay, beta, state = _case(cuda_device, T + D, B, T, H, K, D, BF16, alike=alike)
    out, _ = binding.delta_rule(q, k, v, decay, beta, state.clone())
    want = ref.delta(q, k, v, decay, beta, state)[0]
    rounded = want.to(BF16).double()
    off = float((out.double() - rounded).norm() / want.norm())
    assert off < 3 ** 0.5 * 2.0 ** -10.5, f"off by {off:.2e}"


@pytest.mark.parametrize("B,T", [(74, 25), (74, 33), (74, 48), (74, 49), (73, 25), (80, 47)])
def test_many_fp32_states_of_heads_of_128(cuda_device, B, T):
    """On either side of the border between token by token and windows, with lengths and slots."""
    q, k, v, decay, beta, state = _case(cuda_device, B + T, B, T, 4, 2, 128, FP32, slots=B + 1)
    n = [T - b % 5 if b % 7 else b % 3 for b in range(B)]
    lengths, slots = torch.tensor(n, dtype=torch.int32, device=cuda_device), torch.arange(B, 0, -1, dtype=torch.int32, device=cuda_device)
    before = state.clone()
    out, _ = binding.delta_rule(q, k, v, decay, beta, state, lengths=lengths, slots=slots)
    at = slots.long()
    _check(out, state[at], q, k, v, decay, beta, before[at], 1.0, n, "many")
    assert torch.equal(state[0], before[0]) and all((out[b, n[b]:] == 0).all() for b in range(B))
