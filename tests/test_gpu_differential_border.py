"""Which weights differential attention rounds to bf16: those of large calls only, on either side of the border between its kernels."""
import pytest
import torch

import difference_reference as ref
from paper_2402_04466_b200 import binding
from test_gpu_differential_attention import BF16, _case
from token_reference import check

pytestmark = pytest.mark.gpu


def _rounded(B, Tq, Tk, K, group):
    """More than 32 queries and a fifth of a million keys x tiles of 16 rows."""
    return Tq > 32 and -(-Tq * group // 16) * B * K >= 200000 // Tk + 1


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("B,Tq,Tk,H,K,rounded", [(2, 320, 1000, 5, 5, False), (2, 321, 1000, 5, 5, True), (2, 160, 1000, 10, 5, False), (2, 161, 1000, 10, 5, True), (1, 256, 4800, 2, 2, False),
                                                 (1, 400, 4800, 2, 2, True), (5, 33, 4800, 2, 2, False), (5, 65, 4800, 2, 2, True), (8, 32, 14400, 2, 1, False), (8, 33, 14400, 2, 1, True)])
def test_weights_count_with_16_bits_below_the_border(cuda_device, D, B, Tq, Tk, H, K, rounded):
    assert _rounded(B, Tq, Tk, K, H // K) == rounded
    # sharp maps: a few weights of a row are most of it, so that their own rounding shows
    q, k, v, vectors, _ = _case(cuda_device, Tq + D, B, Tq, Tk, H, K, D, BF16, sharp=3.0)
    got = binding.differential_attention(q, k, v, vectors, 0.3, norm=False)
    want, bound = ref.difference(q, k, v, vectors, 0.3, (D // 2) ** -0.5, norm=False, once=2.0 ** -8 if rounded else 2.0 ** -16, dtype=BF16)
    check(got, want, bound, "rounded once" if rounded else "16 bits")
