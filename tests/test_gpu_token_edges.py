"""The operators over tokens where their kernels change course."""
import math

import pytest
import torch

from paper_2402_04466_b200 import binding
import token_reference as ref
from token_reference import check

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32
TYPES = [BF16, FP32]


def _normal(g, dev, shape, dtype, gain=1.0, shift=0.0):
    return (torch.randn(shape, generator=g, device=dev) * gain + shift).to(dtype)


def _same_kind(got, want, name, signs=True):
    """Finite where the definition is, and else the same infinity, or NaN."""
    assert torch.equal(torch.isfinite(got), torch.isfinite(want)), name
    if signs:
        assert torch.equal(torch.isnan(got), torch.isnan(want)), name
        assert torch.equal(got == math.inf, want == math.inf) and torch.equal(got == -math.inf, want == -math.inf), name


def _finite_check(got, want, bound, name):
    fine = torch.isfinite(want) & torch.isfinite(bound)
    check(got.double()[fine], want[fine], bound[fine], name)


# ------------------------------------------------------------------------------- infinities
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,Tq,Tk,H,K,D", [(2, 7, 480, 2, 2, 64), (2, 1, 63, 2, 2, 32), (2, 40, 200, 2, 1, 128), (2, 7, 20001, 2, 1, 64),
                                           (2, 300, 2500, 4, 4, 64), (2, 260, 3000, 2, 2, 128), (2, 700, 1100, 4, 2, 32),
                                           (2, 700, 3001, 4, 4, 64), (2, 700, 3000, 2, 2, 128), (2, 1300, 1100, 8, 4, 32)])
@pytest.mark.parametrize("masked", [False, True])
def test_an_infinity_that_a_query_sees_is_an_infinity_of_its_row(cuda_device, dtype, B, Tq, Tk, H, K, D, masked):
    """Whichever kernel a size goes to: weights above 0 of one infinity are that infinity, of two that differ a NaN, and other columns and rows are finite."""
    g = torch.Generator(device=cuda_device).manual_seed(Tq + Tk)
    q = _normal(g, cuda_device, (B, Tq, H, D), dtype, 0.5)
    k, v = (_normal(g, cuda_device, (B, Tk, K, D), dtype, 0.5) for _ in range(2))
    at = Tk // 3
    v[0, at, 0, 3], v[0, Tk - 1, 0, D - 1] = math.inf, -math.inf
    v[1, 0, K - 1, 0], v[1, at, K - 1, 0], v[1, at, K - 1, 9] = math.inf, -math.inf, math.inf
    mask = None
    if masked:
        mask = (torch.rand(B, Tq, Tk, generator=g, device=cuda_device) < 0.5).to(torch.uint8)
        mask[:, :, at] = (torch.arange(Tq, device=cuda_device) % 2 == 0)
        mask[:, :, 1] = 1
    got = binding.cross_attention(q, k, v, mask=mask)
    want, size, score = ref.cross(q, k, v, D ** -0.5, None, mask)
    assert not torch.isfinite(want).all() and torch.isinf(want).any()
    _same_kind(got, want, "out")
    _finite_check(got, want, ref.cross_bounds(want, size, score, D, Tk, dtype, 0.0 if dtype == FP32 else 2.0 ** -8), "out")
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,T,H,K,D", [(3, 1, 2, 1, 64), (3, 60, 2, 2, 64), (3, 333, 2, 1, 32), (3, 333, 2, 2, 128), (3, 1300, 4, 4, 64),
                                       (3, 2900, 2, 2, 128), (40, 300, 4, 4, 64), (40, 500, 4, 2, 128), (8, 2500, 4, 4, 32)])
def test_an_infinity_of_a_key_or_value_is_an_infinity_of_the_state(cuda_device, dtype, B, T, H, K, D):
    """k v^T of an infinity is one wherever the other factor is not 0, and it stays one while no decay has faded to 0."""
    g = torch.Generator(device=cuda_device).manual_seed(T + D)
    q, k, v = (_normal(g, cuda_device, (B, T, n, D), dtype) for n in (H, K, K))
    for x in (q, k, v):
        x[x == 0] = 1
    decay = torch.tensor([-0.01, -0.002, 0.0, -0.02], device=cuda_device)[:H]
    state = torch.randn(B, H, D, D, generator=g, device=cuda_device)
    late, early = T - 1 - T // 5, T // 7
    k[0, late, 0, 5], k[0, early, 0, D - 1] = math.inf, -math.inf
    v[1, late, 0, 7], v[1, early, 0, 0] = -math.inf, math.inf
    state[2, 0, 3, 4], state[2, H - 1, 9, 0] = math.inf, -math.inf
    v[2, T - 1, 0, D - 1] = math.inf
    out, new = binding.linear_attention(q, k, v, decay, state, scale=0.1, state_out=torch.empty_like(state))
    want, size, S, A = ref.linear(q, k, v, decay, state, 0.1, None)
    assert torch.isinf(S).any(-1).any(-1)[:3].any(-1).all()
    _same_kind(new, S, "state")
    _same_kind(out, want, "out", signs=False)      # an infinity of the state meets q's signs, a chunk's own q k first: either sum is not finite
    bound, state_bound = ref.linear_bounds(want, size, A, D, T, dtype, dtype == FP32 or T == 1)
    _finite_check(new, S, state_bound, "state")
    _finite_check(out, want, bound, "out")


# ------------------------------------------------------------------------------- views
def _odd(x):
    """The same tensor, its axes of extent 1 with a stride that fits nothing."""
    return x.as_strided(x.shape, [7 if n == 1 else s for n, s in zip(x.shape[:3], x.stride())] + [1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,T,Tk,H", [(1, 1, 1, 1), (1, 7, 300, 1), (3, 1, 200, 2), (1, 1, 9000, 2), (1, 2000, 4000, 4), (2, 1, 1, 1), (1, 300, 1, 2)])
def test_strides_of_axes_of_extent_one_change_nothing(cuda_device, dtype, B, T, Tk, H):
    g = torch.Generator(device=cuda_device).manual_seed(B + T)
    q = _normal(g, cuda_device, (B, T, H, 64), dtype)
    k, v = (_normal(g, cuda_device, (B, T, 1, 64), dtype) for _ in range(2))
    ck, cv = (_normal(g, cuda_device, (B, Tk, 1, 64), dtype) for _ in range(2))
    new = lambda x: _odd(torch.zeros_like(x))      # noqa: E731
    a, b = binding.qk_norm_rope(q, k), binding.qk_norm_rope(_odd(q), _odd(k), out=(new(q), new(k)))
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    decay, state = torch.full((H,), -0.1, device=cuda_device), torch.randn(B, H, 64, 64, generator=g, device=cuda_device)
    a, b = (binding.linear_attention(*x, decay, state, scale=0.1, state_out=torch.empty_like(state), out=o)
            for x, o in (((q, k, v), None), ((_odd(q), _odd(k), _odd(v)), new(q))))
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    assert torch.equal(binding.cross_attention(q, ck, cv), binding.cross_attention(_odd(q), _odd(ck), _odd(cv), out=new(q)))
