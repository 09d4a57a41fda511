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


# ------------------------------------------------------------------------------- long runs of chunks
@pytest.mark.parametrize("B,T,H,D", [(8, 14400, 4, 64), (38, 4000, 4, 64), (8, 14400, 4, 32), (8, 14400, 2, 128), (75, 3000, 2, 128)])
def test_sums_of_a_long_sequence_are_rounded_not_cut_off(cuda_device, B, T, H, D):
    """Keys and values above 0, no decay: whatever an addition cuts off is missing from the state, always on the same side.  Products start from nothing every two
    chunks at most, 16 instructions for the largest term, which lose half a step of a sum that is half grown: 17 / 2 of at most 0.75 / 2 * 2^-23, 3.8e-7 of
    it; what is rounded is off to either side and not in the mean.  (One sum over all chunks lost 1.3e-6.)"""
    g = torch.Generator(device=cuda_device).manual_seed(T + D)
    q, k, v = (torch.rand(B, T, H, D, generator=g, device=cuda_device).to(BF16) for _ in range(3))
    _, new = binding.linear_attention(q, k, v, torch.zeros(H, device=cuda_device), torch.zeros(B, H, D, D, device=cuda_device), scale=0.01)
    want = torch.stack([torch.einsum("thd,the->hde", x.double(), y.double()) for x, y in zip(k, v)])
    lost = ((want - new) / want).flatten(2).mean(-1)
    assert lost.abs().max() < 5e-7, f"{float(lost.abs().max()):.2e}"


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("B,T,H,K", [(10, 1100, 15, 15), (8, 2000, 4, 2), (8, 2500, 4, 4), (8, 4500, 4, 4), (2, 5300, 30, 10)])
def test_linear_attention_of_many_chunks_to_a_block(cuda_device, B, T, H, K, D):
    """Four to nine chunks to a segment, odd and even, and nine to a sequence that is not cut: every place of operands, scores and sums is used more than once."""
    g = torch.Generator(device=cuda_device).manual_seed(T + D)
    q, k, v = (_normal(g, cuda_device, (B, T, n, D), BF16) for n in (H, K, K))
    decay = torch.tensor([-0.002, -0.03, 0.0, -0.7, -6.0, -math.inf], device=cuda_device).repeat(5)[:H]
    state = torch.randn(B, H, D, D, generator=g, device=cuda_device)
    lengths = [T - 97 * b for b in range(B)]
    for n in (None, torch.tensor(lengths, dtype=torch.int32, device=cuda_device)):
        out, new = binding.linear_attention(q, k, v, decay, state, scale=D ** -0.5, state_out=torch.empty_like(state), lengths=n)
        if n is None:
            want, size, S, A = ref.linear(q, k, v, decay, state, D ** -0.5, None)
            bound, state_bound = ref.linear_bounds(want, size, A, D, T, BF16, False)
            check(out, want, bound, "out")
            check(new, S, state_bound, "state")
        else:
            for b, m in enumerate(lengths):
                assert (out[b, m:] == 0).all()
            # a sequence that ends sooner: the same rows, and the state of a call with no more tokens
            check(out[0], want[0], bound[0], "out of the longest")
            b, m = B - 1, lengths[-1]
            short = ref.linear(q[b:, :m], k[b:, :m], v[b:, :m], decay, state[b:], D ** -0.5, None)
            limits = ref.linear_bounds(short[0], short[1], short[3], D, m, BF16, False)
            check(out[b:, :m], short[0], limits[0], "out of the shortest")
            check(new[b:], short[2], limits[1], "state of the shortest")


# ------------------------------------------------------------------------------- few queries, keys over several clusters
def _scratch(B, Tq, Tk, H, K, D, masked):
    import ctypes as C
    a = binding.tt_cross_attention_args(C.sizeof(binding.tt_cross_attention_args), 1, B, Tq, Tk, H, K, D, 0.125)
    a.mask = 16 if masked else None
    return binding.load_library().tt_cross_attention_scratch_bytes(C.byref(a))


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("B,Tq,Tk,H,K", [(1, 7, 14400, 4, 4), (1, 3, 20001, 2, 1), (2, 7, 14400, 2, 2), (1, 9, 33333, 4, 2)])
@pytest.mark.parametrize("masked", [False, True])
def test_cross_attention_of_few_queries_on_keys_split_over_clusters(cuda_device, B, Tq, Tk, H, K, D, masked):
    assert _scratch(B, Tq, Tk, H, K, D, masked) >= 2 * B * K * Tq * (H // K) * (D + 2) * 4      # two clusters to a tile of rows at least
    g = torch.Generator(device=cuda_device).manual_seed(Tk + D)
    q = _normal(g, cuda_device, (B, Tq, H, D), BF16, 3.0)
    k, v = (_normal(g, cuda_device, (B, Tk, K, D), BF16, 1.0, s) for s in (0.0, 0.3))
    mask = None
    if masked:
        mask = (torch.rand(B, Tq, Tk, generator=g, device=cuda_device) < 0.2).to(torch.uint8)
        mask[:, 0] = 0                                   # sees nothing
        mask[:, 1, :Tk - 5] = 0                          # the last piece only
        mask[:, 2, 100:] = 0                             # the first only
    for n in (None, 0, 1, 300, 9000, Tk - 1):
        lengths = None if n is None else torch.tensor([n, Tk][:B], dtype=torch.int32, device=cuda_device)
        got = binding.cross_attention(q, k, v, mask=mask, kv_lengths=lengths)
        want, size, score = ref.cross(q, k, v, D ** -0.5, lengths, mask)
        # weights are two bf16 terms: off by half a step of half a step, 2^-18, and they are summed before they are cut
        check(got, want, ref.cross_bounds(want, size, score, D, Tk, BF16, 2.0 ** -17), f"{n} keys")


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("Tq,Tk,H,K", [(1, 2, 2, 2), (7, 480, 2, 2), (3, 5, 4, 1), (16, 70, 2, 2), (40, 1000, 4, 2)])
def test_weights_of_few_queries_count_with_more_bits_than_a_value_has(cuda_device, Tq, Tk, H, K, D):
    """Values that cancel: out is small beside what is summed, so a weight rounded to bf16 once (2^-8 of the sum) would show."""
    g = torch.Generator(device=cuda_device).manual_seed(Tk + D)
    q, k = _normal(g, cuda_device, (3, Tq, H, D), BF16, 0.5), _normal(g, cuda_device, (3, Tk, K, D), BF16)
    v = _normal(g, cuda_device, (3, Tk, K, D), BF16, 0.1) + torch.where(torch.arange(Tk, device=cuda_device) % 2 == 0, 1.0, -1.0)[None, :, None, None].to(BF16)
    for mask in (None, torch.ones(3, Tq, Tk, dtype=torch.uint8, device=cuda_device)):
        want, size, score = ref.cross(q, k, v, D ** -0.5, None, mask)
        check(binding.cross_attention(q, k, v, mask=mask), want, ref.cross_bounds(want, size, score, D, Tk, BF16, 2.0 ** -17), "out")


def test_results_carry_no_gradient(cuda_device):
    q = torch.randn(1, 5, 2, 64, device=cuda_device, requires_grad=True)
    w = torch.ones(64, device=cuda_device, requires_grad=True)
    decay, state = torch.zeros(2, device=cuda_device), torch.zeros(1, 2, 64, 64, device=cuda_device)
    for x in (*binding.qk_norm_rope(q, q, q_weight=w, k_weight=w), *binding.linear_attention(q, q, q, decay, state), binding.cross_attention(q, q, q)):
        assert not x.requires_grad and torch.isfinite(x).all()


@pytest.mark.parametrize("name", ["rope", "linear", "cross"])
def test_tensors_let_go_before_another_stream_has_read_them(cuda_device, name):
    """A call for another stream returns before its kernels have run.  Its tensors' memory is nobody else's until they have."""
    g = torch.Generator(device=cuda_device).manual_seed(3)
    x = _normal(g, cuda_device, (2, 600, 2, 64), FP32)
    decay, state = torch.full((2,), -0.1, device=cuda_device), torch.zeros(2, 2, 64, 64, device=cuda_device)
    pos, inv = torch.arange(600, device=cuda_device), torch.from_numpy(binding.rope_frequencies(64)[0]).to(cuda_device)
    calls = {"rope": lambda y, s: binding.qk_norm_rope(y, None, pos, inv, stream=s)[0],
             "linear": lambda y, s: binding.linear_attention(y, y, y, decay, state, state_out=torch.zeros_like(state), stream=s)[0],
             "cross": lambda y, s: binding.cross_attention(y, y, y, stream=s)}
    want = calls[name](x, None)
    side = torch.cuda.Stream()
    calls[name](x, side)                                  # what is set up once is there
    torch.cuda.synchronize()
    y = x.clone()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(40_000_000)                     # some 20 ms
    got = calls[name](y, side)
    del y
    others = [torch.full_like(x, math.nan) for _ in range(8)]
    torch.cuda.synchronize()
    assert torch.equal(got, want) and len(others) == 8
