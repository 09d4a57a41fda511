"""The gated delta rule where products pass what 32 bits hold although the rule itself stays finite: sums over a window that the formula never forms, and states that a decay takes back."""
import math

import pytest
import torch

import delta_reference as ref
from paper_2402_04466_b200 import binding
from test_gpu_delta_rule import TYPES, _case, _check
from token_reference import check

pytestmark = pytest.mark.gpu

HEADS = [(2, 32), (2, 64), (2, 128), (40, 32), (20, 64), (10, 128)]


def _call(q, k, v, decay, beta, state, **kw):
    return binding.delta_rule(q, k, v, decay, beta, state, state_out=torch.full_like(state, math.nan), **kw)


def _element_by_element(got, q, k, v, decay, beta, state):
    """Against the columns as they stood.  (In the mean _check counts errors as independent and against the state that is left.  Where one large state fades, exp(log_decay) is off by
    up to two steps for all of it alike, 2^-22 by itself against 2.6 * 2^-23 in the mean that heads of 32 are allowed, and a correction that takes 1 - beta |k|^2 of it, a fiftieth,
    leaves fifty times the share.)"""
    want, size, S, A = ref.delta(q, k, v, decay, beta, state)
    assert torch.isfinite(want).all() and torch.isfinite(S).all()
    bound, state_bound = ref.bounds(want, size, A, v.shape[3], v.shape[1], v.dtype, v.shape[1] > 1)
    check(got[0], want, bound, "out")
    check(got[1], S, state_bound, "state")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,D", HEADS)
@pytest.mark.parametrize("T", [60, 65, 150])
def test_products_of_two_keys(cuda_device, dtype, H, D, T):
    """Two keys of 1e20 whose corrections are 0: k_i . k_j is no number of 32 bits, and the rule never asks for it."""
    B = 4
    q, k, v, decay, beta, state = _case(cuda_device, D + T, B, T, H, H, D, dtype)
    for b, (i, j) in enumerate(((5, 9), (12, 20), (33, 59))):      # in a half of a window, over both halves, in the second window
        k[b, i, 0], k[b, j, 0] = 1e20, 1e20
        beta[b, i, 0] = beta[b, j, 0] = 0.0
    _check(*_call(q, k, v, decay, beta, state), q, k, v, decay, beta, state, 1.0, None, "keys")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,D", HEADS)
@pytest.mark.parametrize("T", [60, 65, 150])
def test_products_of_a_query_and_an_earlier_key(cuda_device, dtype, H, D, T):
    """A query of 1e20 behind a key of 1e20 that corrected nothing, and one behind a decay that forgot what the key left."""
    B = 4
    q, k, v, decay, beta, state = _case(cuda_device, D + T, B, T, H, H, D, dtype)
    for b, (i, j) in enumerate(((5, 9), (12, 20), (33, 59))):
        k[b, i, 0], q[b, j, 0], beta[b, i, 0] = 1e20, 1e20, 0.0
    k[3, 8, 1], q[3, 14, 1], decay[3, 11, 1] = 1e15, 1e25, -math.inf
    beta[3, 8, 1] = 2.0 ** -110      # beta |k|^2 is 0.1 at most
    _check(*_call(q, k, v, decay, beta, state), q, k, v, decay, beta, state, 1.0, None, "queries")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,D", HEADS)
@pytest.mark.parametrize("T", [60, 65, 150])
@pytest.mark.parametrize("length", [3.0, 10.0])
def test_tokens_before_a_state_overflows(cuda_device, dtype, H, D, T, length):
    """One key again and again, so long that every token makes the state eight times, or a hundred times, larger: what is not finite at last is not
    finite for the tokens before."""
    B, first = 2, 35
    q, k, v, _, beta, state = _case(cuda_device, D, B, T, H, H, D, dtype)
    k[0, first:, 0] = length * D ** -0.5
    beta[0, first:, 0] = 1.0
    out, new = _call(q, k, v, None, beta, state)
    want, size, S, A = ref.delta(q, k, v, None, beta, state)
    # An error grows as the state does, by |k|^2 - 1 a token, in every column alike: it is measured against the longest column, and a token adds a sum's roundings of that.
    widest = size.amax(-1, keepdim=True)
    some = ((2 * D + 16) * T * ref.STEP + (2.0 ** -8 if dtype == torch.bfloat16 else 0.0)) * widest + ref.half_step(dtype) * want.abs()
    held = (widest < 1e34).expand_as(want)
    assert held[0, :first + 13, 0].all() and held[1].all() and held[0, :, 1].all()
    check(out[held], want[held], some[held], "before")
    assert torch.isfinite(new[1]).all() and torch.isfinite(new[0, 1:]).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,D", HEADS)
@pytest.mark.parametrize("T", [1, 2, 8, 60, 150])
def test_product_of_a_token_s_query_and_key(cuda_device, dtype, H, D, T):
    """Both of 1e20, with a correction of 0, at the first and last token."""
    q, k, v, decay, beta, state = _case(cuda_device, D + T, 3, T, H, H, D, dtype)
    for b, t in ((0, 0), (1, T - 1)):
        q[b, t, 0], k[b, t, 0], beta[b, t, 0] = 1e20, 1e20, 0.0
    _check(*_call(q, k, v, decay, beta, state), q, k, v, decay, beta, state, 1.0, None, "one token")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,D", HEADS + [(8, 128)])
@pytest.mark.parametrize("T", [1, 2, 8])
def test_a_state_that_is_forgotten(cuda_device, dtype, H, D, T):
    """Elements of 1e38, which a key of length 1 adds up to more than 32 bits hold: all of it fades before it is read, at once or to some thousand."""
    B = 20 if D == 128 and H == 8 else 3
    q, k, v, decay, beta, state = _case(cuda_device, D + T, B, T, H, H, D, dtype)
    q[:2, 0, 0], k[:2, 0, 0] = 0.9 * D ** -0.5, 0.9 * D ** -0.5
    state[:2, 0] = 1e38
    decay[0, 0, 0], decay[1, 0, 0] = -math.inf, -80.0
    _element_by_element(_call(q, k, v, decay, beta, state), q, k, v, decay, beta, state)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,D", HEADS)
@pytest.mark.parametrize("T", [60, 65, 150])
def test_a_state_that_is_forgotten_within_a_window(cuda_device, dtype, H, D, T):
    """The same by windows, with keys of which such a state says nothing, so that only the queries' sums pass 32 bits: at the first token, and where the second window begins."""
    q, k, v, decay, beta, state = _case(cuda_device, D + T, 4, T, H, H, D, dtype)
    sign = torch.ones(D, device=cuda_device)
    sign[1::2] = -1
    state[:3, 0] = 1e38
    q[:2, 0, 0], k[:2, 0, 0] = 0.9 * D ** -0.5, (0.9 * D ** -0.5 * sign).to(dtype)
    decay[0, 0, 0], decay[1, 0, 0] = -math.inf, -80.0
    q[2, :32, 0], k[2, :32, 0], beta[2, :32, 0], decay[2, :32, 0] = 0.0, 0.0, 0.0, 0.0
    q[2, 32, 0], k[2, 32, 0], decay[2, 32, 0] = 0.9 * D ** -0.5, (0.9 * D ** -0.5 * sign).to(dtype), -math.inf
    _element_by_element(_call(q, k, v, decay, beta, state), q, k, v, decay, beta, state)
