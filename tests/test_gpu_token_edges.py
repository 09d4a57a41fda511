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
