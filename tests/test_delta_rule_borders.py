"""Which calls of the gated delta rule go token by token (no GPU needed): those ask for no scratch."""
import ctypes as C

import pytest

from paper_2402_04466_b200 import binding

S = binding.tt_delta_rule_args


def _room(states, tokens, D, precision):
    heads = 2
    view = binding.tt_tokens(0x7F0000000000, tokens * heads * D, heads * D, D)
    a = S(C.sizeof(S), precision, states // heads, tokens, heads, heads, D, states, 1.0, 0, view, view, view, view, None, 0x7F0000000000, 0x7F0000000000, 0x7F0000000000, None, None, None, 0)
    return binding.load_library().tt_delta_rule_scratch_bytes(C.byref(a))


@pytest.mark.parametrize("states,tokens", [(10, 12), (146, 12), (148, 24), (294, 24), (296, 48), (2048, 48)])
def test_fp32_heads_of_128_go_token_by_token_as_far_as_that_is_faster(states, tokens):
    assert _room(states, tokens, 128, 0) == 0 < _room(states, tokens + 1, 128, 0)


@pytest.mark.parametrize("D", [32, 64])
@pytest.mark.parametrize("states", [400, 2048])
def test_other_heads_have_one_border(states, D):
    assert _room(states, 12, D, 0) == 0 < _room(states, 13, D, 0)
    assert _room(states, 8, D, 1) == 0 < _room(states, 9, D, 1)
