"""The operators over tokens against their definitions in 64 bits (token_reference.py), at the sizes and masks where they can go wrong."""
import math

import pytest
import torch

import tt_synth
from paper_2402_04466_b200 import binding
import token_reference as ref
from token_reference import check, half_step

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32
TYPES = [BF16, FP32]


def _gen(dev, seed):
    return torch.Generator(device=dev).manual_seed(seed)


def _tokens(g, dev, shape, dtype, layout="plain", pad=float("nan"), shift=0.0, gain=1.0):
    """[B][T][H][D] normal values; 'fused': the first heads of a wider row, 'heads first': [B][H][T][D] in memory, 'padded': room behind the rows."""
    B, T, H, D = shape
    x = (torch.randn(shape, generator=g, device=dev) * gain + shift).to(dtype)
    if layout == "plain":
        return x
    if layout == "fused":
        y = torch.full((B, T, H + 3, D), pad, dtype=dtype, device=dev)[:, :, 1:H + 1]
    elif layout == "heads first":
        y = torch.full((B, H, T, D), pad, dtype=dtype, device=dev).transpose(1, 2)
    else:
        y = torch.full((B, T + 5, H, D + 8), pad, dtype=dtype, device=dev)[:, 2:T + 2, :, :D]
    y.copy_(x)
    return y


# ------------------------------------------------------------------------------- norm and rotation
def _rope_case(dev, seed, B, T, H, K, D, rot, dtype, layout="fused", far=False):
    g = _gen(dev, seed)
    q, k = _tokens(g, dev, (B, T, H, D), dtype, layout, gain=1.7, shift=0.1), _tokens(g, dev, (B, T, K, D), dtype, layout, gain=0.4)
    w = [1 + 0.3 * torch.randn(D, generator=g, device=dev) for _ in range(2)]
    pos = torch.randint(0, 2 ** 40 if far else 5_000_000, (B, T), generator=g, device=dev)
    inv = torch.from_numpy(binding.rope_frequencies(rot)[0]).to(dev)
    return q, k, w, pos, inv


def _rope_check(got, x, w, pos, inv, eps, norm, interleaved, gain, name):
    want, size = ref.norm_rope(x, w, pos, inv, eps, norm, interleaved, gain)
    # a row's sum of squares, its root, weight and turn: a dozen roundings of 2^-24, the angle's 2^-23 and the functions' 2^-22
    check(got, want, half_step(got.dtype) * want.abs() + 2.0 ** -19 * size, name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,T,H,K,D,rot,interleaved", [
    (1, 1, 1, 1, 32, 32, False), (8, 1, 4, 4, 64, 64, False), (2, 7, 3, 1, 64, 32, True), (1, 33, 2, 2, 128, 128, True),
    (3, 65, 5, 1, 32, 8, False), (2, 130, 8, 2, 128, 40, False), (2, 19, 1, 7, 64, 24, True), (1, 501, 2, 2, 64, 0, False),
    (1, 3, 70, 70, 32, 16, True), (5, 300, 2, 2, 128, 96, False)])
def test_norm_rope(cuda_device, dtype, B, T, H, K, D, rot, interleaved):
    for layout in ("plain", "fused", "heads first", "padded"):
        q, k, w, pos, inv = _rope_case(cuda_device, B * 1000 + T, B, T, H, K, D, rot, dtype, layout)
        a, b = binding.qk_norm_rope(q, k, pos, inv, w[0], w[1], eps=1e-5, interleaved=interleaved, rot_scale=1.25)
        _rope_check(a, q, w[0], pos, inv, 1e-5, True, interleaved, 1.25, f"q {layout}")
        _rope_check(b, k, w[1], pos, inv, 1e-5, True, interleaved, 1.25, f"k {layout}")


@pytest.mark.parametrize("dtype", TYPES)
def test_norm_rope_parts_that_can_be_left_out(cuda_device, dtype):
    q, k, w, pos, inv = _rope_case(cuda_device, 3, 2, 21, 2, 1, 64, 48, dtype)
    a, b = binding.qk_norm_rope(q, k, pos, inv, w[0], w[1], norm=False)
    _rope_check(a, q, None, pos, inv, 0, False, False, 1.0, "rotation alone")
    _rope_check(b, k, None, pos, inv, 0, False, False, 1.0, "rotation alone, keys")
    a, b = binding.qk_norm_rope(q, k, None, None, None, w[1])
    _rope_check(a, q, None, pos, None, 1e-6, True, False, 1.0, "norm alone, no weight")
    _rope_check(b, k, w[1], pos, None, 1e-6, True, False, 1.0, "norm alone")
    a, b = binding.qk_norm_rope(None, k, pos[0], inv, k_weight=w[1])
    assert a is None
    _rope_check(b, k, w[1], pos[:1], inv, 1e-6, True, False, 1.0, "keys alone, positions shared")
    a, b = binding.qk_norm_rope(q, None, pos, inv, w[0])
    assert b is None
    _rope_check(a, q, w[0], pos, inv, 1e-6, True, False, 1.0, "queries alone")
    assert binding.qk_norm_rope(q[:, :0], k[:, :0], pos[:, :0], inv)[0].shape == (2, 0, 2, 64)


def test_norm_rope_far_positions_and_rows_of_zeros(cuda_device):
    q, k, w, pos, inv = _rope_case(cuda_device, 4, 2, 40, 2, 2, 64, 64, FP32, far=True)
    q[0, 3] = 0
    # 2^40 positions: the product in 64 bits has 2^-13 radians left to be wrong by, the reference's own too
    for x, y, wt in zip(binding.qk_norm_rope(q, k, pos % 2 ** 30, inv, w[0], w[1]), (q, k), w):
        want, size = ref.norm_rope(y, wt, pos % 2 ** 30, inv, 1e-6, True, False, 1.0)
        check(x, want, 2.0 ** -24 * want.abs() + (2.0 ** -19 + 2.0 ** 30 * 2.0 ** -51) * size, "far")
    assert torch.isfinite(binding.qk_norm_rope(q, k, pos, inv, w[0], w[1])[0]).all()
    assert (binding.qk_norm_rope(q, k, -pos % 7, inv)[0][0, 3] == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_norm_rope_leaves_rows_behind_the_length_and_works_in_place(cuda_device, dtype):
    q, k, w, pos, inv = _rope_case(cuda_device, 5, 4, 37, 2, 3, 64, 64, dtype, "plain")
    n = torch.tensor([37, 0, 20, 99], dtype=torch.int32, device=cuda_device)
    whole = binding.qk_norm_rope(q, k, pos, inv, w[0], w[1])
    q0, k0 = q.clone(), k.clone()
    a, b = binding.qk_norm_rope(q, k, pos, inv, w[0], w[1], lengths=n, out=(q, k))
    assert a is q and b is k
    for got, before, full in ((q, q0, whole[0]), (k, k0, whole[1])):
        for e, m in enumerate((37, 0, 20, 37)):
            assert torch.equal(got[e, :m], full[e, :m]) and torch.equal(got[e, m:], before[e, m:])
    fresh = binding.qk_norm_rope(q0, k0, pos, inv, w[0], w[1], lengths=n)
    assert (fresh[0][1] == 0).all() and (fresh[1][2, 20:] == 0).all()


# ------------------------------------------------------------------------------- linear attention
DECAYS = [0.0, -0.002, -0.03, -0.7, -6.0, -math.inf]


def _linear_case(dev, seed, B, T, H, K, D, dtype, layout="fused", slots=None):
    g = _gen(dev, seed)
    q, k = _tokens(g, dev, (B, T, H, D), dtype, layout), _tokens(g, dev, (B, T, K, D), dtype, layout)
    v = _tokens(g, dev, (B, T, K, D), dtype, layout, shift=0.2)
    decay = torch.tensor([DECAYS[(seed + h) % len(DECAYS)] for h in range(H)], device=dev)
    state = torch.randn(slots or B, H, D, D, generator=g, device=dev)
    return q, k, v, decay, state


def _linear_check(got, got_state, q, k, v, decay, state, scale, lengths, name, rows=None):
    out, size, S, A = ref.linear(q, k, v, decay, state, scale, lengths)
    # a reference that starts a state of decay 0 from nothing: the sizes count what is there
    bound, state_bound = ref.linear_bounds(out, size, A, q.shape[3], q.shape[1], q.dtype, q.dtype == FP32 or q.shape[1] == 1)
    check(got, out, bound, name + " out")
    check(got_state, S, state_bound, name + " state")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,T,H,K,D", [
    (1, 1, 1, 1, 32), (5, 1, 2, 2, 64), (3, 1, 6, 2, 128), (40, 1, 8, 8, 64), (75, 1, 8, 4, 32), (38, 1, 8, 8, 128),
    (1, 2, 1, 1, 64), (2, 31, 3, 1, 32), (1, 32, 2, 2, 128), (2, 33, 2, 2, 128), (3, 63, 2, 1, 64), (1, 64, 6, 6, 64), (2, 65, 2, 2, 64),
    (1, 127, 2, 2, 32), (1, 128, 6, 3, 128), (2, 129, 1, 1, 64), (1, 257, 6, 6, 64), (2, 300, 2, 1, 128), (1, 700, 4, 2, 32), (1, 1025, 1, 1, 64),
    (8, 1300, 4, 4, 32), (8, 1300, 4, 2, 64), (8, 1300, 4, 4, 128), (40, 300, 8, 8, 64)])      # segments of several chunks; sequences enough without
def test_linear_attention(cuda_device, dtype, B, T, H, K, D):
    for i, layout in enumerate(("plain", "fused", "heads first", "padded")):
        q, k, v, decay, state = _linear_case(cuda_device, 17 * T + i, B, T, H, K, D, dtype, layout)
        before = state.clone()
        out, new = binding.linear_attention(q, k, v, decay, state, scale=D ** -0.5, state_out=torch.empty_like(state))
        assert torch.equal(state, before)
        _linear_check(out, new, q, k, v, decay, state, D ** -0.5, None, layout)
        again, same = binding.linear_attention(q, k, v, decay, state, scale=D ** -0.5)
        assert same is state and torch.equal(again, out) and torch.equal(state, new)      # in place: the same bits


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [1, 60, 400])
def test_linear_attention_slots_and_lengths(cuda_device, dtype, T):
    B, H, K, D, slots = 6, 2, 1, 64, 9
    q, k, v, decay, state = _linear_case(cuda_device, T, B, T, H, K, D, dtype, "plain", slots)
    at = torch.tensor([7, 2, 7, 9, -1, 0], dtype=torch.int32, device=cuda_device)      # the third repeats the first, two lie outside
    n = torch.tensor([T, T // 2, T, T, T, -3], dtype=torch.int32, device=cuda_device)
    for b, m in ((1, T // 2), (5, 0)):
        for x in (q, k, v):
            x[b, m:] = math.nan
    out = torch.full_like(q, 77.0)
    new = torch.full_like(state, 55.0)
    binding.linear_attention(q, k, v, decay, state, scale=0.2, slots=at, lengths=n, out=out, state_out=new)
    keep = [0, 1, 5]
    rows = n[keep].clamp(min=0)
    want = ref.linear(q[keep], k[keep], v[keep], decay, state[at[keep].long()], 0.2, rows.tolist())
    bound, state_bound = ref.linear_bounds(want[0], want[1], want[3], D, T, dtype, dtype == FP32 or T == 1)
    for i, (b, m) in enumerate(zip(keep, rows.tolist())):
        check(out[b, :m], want[0][i, :m], bound[i, :m], f"entry {b}")
        assert (out[b, m:] == 77).all()
        check(new[at[b]], want[2][i], state_bound[i], f"state of entry {b}")
    assert torch.equal(new[0], state[0])                                               # no token: the state as it was
    for b in (2, 3, 4):
        assert (out[b] == 77).all()
    for s in (1, 3, 4, 5, 6, 8):
        assert (new[s] == 55).all()
    old = state.clone()
    binding.linear_attention(q, k, v, decay, state, scale=0.2, slots=at, lengths=n, out=out)
    named = [7, 2, 0]
    assert torch.equal(state[named], new[named])
    rest = [s for s in range(slots) if s not in named]
    assert torch.equal(state[rest], old[rest])


@pytest.mark.parametrize("B,T,H", [(38, 4000, 4), (8, 6000, 4), (1, 9000, 2)])      # a block to a sequence, segments of many chunks and of few
def test_linear_attention_state_of_a_long_sequence_is_not_cut_short(cuda_device, B, T, H):
    """Keys and values above 0 and no decay: sums that only grow, of which every addition that cuts off where it should round takes a part."""
    g = _gen(cuda_device, T)
    q, k, v = (torch.rand(B, T, H, 64, generator=g, device=cuda_device).to(BF16) for _ in range(3))
    state = torch.zeros(B, H, 64, 64, device=cuda_device)
    out, new = binding.linear_attention(q, k, v, torch.zeros(H, device=cuda_device), state.clone(), scale=0.01)
    want = torch.einsum("bthd,bthe->bhde", k.double(), v.double())
    # a product of two chunks is 48 instructions, whose sums may each be short of two steps of fp32; products, segments and the state are added with a
    # rounding each.  (A sum of all chunks in one accumulator is short of a step for every instruction: 24 in a chunk, 1.1e-4 of 6000 tokens.)
    check(new, want, (48 * 2.0 ** -22 + (T // 128 + 8) * 2.0 ** -24) * want, "state")


def test_two_linear_calls_at_once(cuda_device):
    """Side by side on two streams, eager and captured: each has scratch of its own."""
    cases = [_linear_case(cuda_device, 40 + i, 3, 2000, 4, 2, 64, BF16) for i in range(2)]
    want = [[x.clone() for x in binding.linear_attention(q, k, v, d, s.clone(), scale=0.1)] for q, k, v, d, s in cases]
    streams, graphs, got = [torch.cuda.Stream() for _ in range(2)], [], []
    torch.cuda.synchronize()
    for (q, k, v, d, s), st in zip(cases, streams):
        graph, out = torch.cuda.CUDAGraph(), (torch.empty_like(want[0][0]), torch.empty_like(s))
        with torch.cuda.graph(graph, stream=st):
            binding.linear_attention(q, k, v, d, s, scale=0.1, out=out[0], state_out=out[1])
        graphs.append(graph)
        got.append(out)
    for _ in range(5):
        for graph, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    for _ in range(5):
        for i, ((q, k, v, d, s), st) in enumerate(zip(cases, streams)):
            binding.linear_attention(q, k, v, d, s, scale=0.1, out=got[i][0], state_out=got[i][1], stream=st)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [32, 64, 128])
def test_linear_attention_does_not_look_ahead(cuda_device, dtype, D):
    """What is not finite in a token's key or value reaches that token's row and later ones, and no earlier one."""
    B, T, H, K = 2, 333, 2, 1
    for name, at in (("v", 200), ("k", 200), ("v", 332), ("v", 128), ("v", 1)):
        q, k, v, decay, state = _linear_case(cuda_device, at + D, B, T, H, K, D, dtype, "plain")
        decay = torch.tensor([-0.01, -0.5], device=cuda_device)
        x = {"k": k, "v": v}[name]
        clean = x.clone()
        clean[:, at:] = 0
        args = (q, clean, v) if name == "k" else (q, k, clean)
        want, _ = binding.linear_attention(*args, decay, state.clone(), scale=0.1)
        x[0, at, 0, D // 2], x[1, at, 0, 1] = math.inf, math.nan
        x[1, at, 0, D - 1] = -math.inf
        got, new = binding.linear_attention(q, k, v, decay, state.clone(), scale=0.1)
        out, size, _, A = ref.linear(args[0], args[1], args[2], decay, state, 0.1, None)
        bound, _ = ref.linear_bounds(out, size, A, D, T, dtype, dtype == FP32)
        check(got[:, :at], out[:, :at], bound[:, :at], f"{name} before {at}")
        assert not torch.isfinite(got[0, at:]).all(-1).any() and torch.isnan(got[1, at:]).any(-1).all()
        assert not torch.isfinite(new).flatten(2).all(-1).any()
        if name == "v":                # columns of the state are apart from each other
            others = [c for c in range(D) if c not in (1, D // 2, D - 1)]
            assert torch.isfinite(got[..., others]).all() and torch.isfinite(new[..., others]).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_linear_attention_in_pieces_is_linear_attention(cuda_device, dtype):
    """A clip and then single tokens, as a stream that is brought up to date and goes on: the states meet."""
    q, k, v, decay, state = _linear_case(cuda_device, 1, 3, 210, 2, 2, 64, dtype)
    whole, last = binding.linear_attention(q, k, v, decay, state, state_out=torch.empty_like(state))
    outs = [binding.linear_attention(q[:, :203], k[:, :203], v[:, :203], decay, state)[0]]
    for t in range(203, 210):
        outs.append(binding.linear_attention(q[:, t:t + 1], k[:, t:t + 1], v[:, t:t + 1], decay, state)[0])
    _linear_check(torch.cat(outs, 1), state, q, k, v, decay, last * 0 + _linear_case(cuda_device, 1, 3, 210, 2, 2, 64, dtype)[4], 1.0, None, "pieces")
    assert binding.linear_attention(q[:, :0], k[:, :0], v[:, :0], decay, state, state_out=last)[0].shape == (3, 0, 2, 64)
    assert torch.equal(last, state)


# ------------------------------------------------------------------------------- cross attention
def _cross_case(dev, seed, B, Tq, Tk, H, K, D, dtype, layout="fused", sharp=1.0):
    g = _gen(dev, seed)
    return (_tokens(g, dev, (B, Tq, H, D), dtype, layout, gain=sharp), _tokens(g, dev, (B, Tk, K, D), dtype, layout),
            _tokens(g, dev, (B, Tk, K, D), dtype, layout, shift=0.3))


def _cross_check(got, q, k, v, scale, n, mask, name):
    want, size, score = ref.cross(q, k, v, scale, n, mask)
    check(got, want, ref.cross_bounds(want, size, score, q.shape[3], k.shape[1], q.dtype, 0.0 if q.dtype == FP32 else 2.0 ** -8), name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,Tq,Tk,H,K,D", [
    (1, 1, 1, 1, 1, 32), (2, 1, 63, 2, 2, 64), (5, 7, 480, 2, 2, 64), (1, 7, 1201, 4, 1, 128), (8, 3, 130, 4, 4, 64), (2, 16, 64, 1, 1, 128),
    (2, 17, 65, 2, 1, 64), (1, 33, 127, 8, 2, 32), (1, 64, 128, 2, 2, 128), (2, 127, 129, 2, 2, 64), (1, 128, 257, 1, 1, 32), (1, 129, 200, 2, 1, 128),
    (1, 255, 1000, 2, 2, 64), (2, 300, 385, 3, 3, 64), (1, 520, 3, 1, 1, 64), (1, 1, 5000, 1, 1, 128), (3, 257, 640, 4, 2, 128), (1, 700, 128, 2, 2, 32)])
def test_cross_attention(cuda_device, dtype, B, Tq, Tk, H, K, D):
    for i, layout in enumerate(("plain", "fused", "heads first", "padded")):
        q, k, v = _cross_case(cuda_device, Tq * 31 + Tk + i, B, Tq, Tk, H, K, D, dtype, layout, sharp=(0.3, 1.0, 3.0, 12.0)[i])
        _cross_check(binding.cross_attention(q, k, v), q, k, v, D ** -0.5, None, None, layout)


@pytest.mark.parametrize("B,Tq,Tk,H,K,D", [
    (3, 513, 4001, 4, 4, 64), (2, 700, 3001, 6, 3, 64), (4, 129, 4100, 8, 8, 32), (1, 1000, 2500, 4, 2, 128), (2, 257, 9000, 2, 2, 128),
    (1, 8000, 130, 8, 8, 64), (1, 4000, 64, 32, 32, 64), (1, 66000, 1, 128, 128, 32), (300, 70, 60, 8, 8, 32), (2, 1300, 777, 8, 8, 128)])
def test_cross_attention_of_many_queries(cuda_device, B, Tq, Tk, H, K, D):
    """Work enough for the tensor-core kernel: tiles of queries and of keys that are not whole, more entries than one launch takes, tiles
    that several blocks share."""
    for i, layout in enumerate(("fused", "heads first")):
        q, k, v = _cross_case(cuda_device, Tq * 31 + Tk + i, B, Tq, Tk, H, K, D, BF16, layout, sharp=(1.0, 8.0)[i])
        _cross_check(binding.cross_attention(q, k, v), q, k, v, D ** -0.5, None, None, layout)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Tq,Tk,D", [(7, 700, 64), (150, 300, 64), (300, 130, 128), (260, 1000, 32), (400, 3000, 64), (300, 2001, 128), (700, 1100, 32)])
def test_cross_attention_lengths(cuda_device, dtype, Tq, Tk, D):
    """Rows behind the lengths hold NaN; rows of the output behind q_lengths are left alone."""
    B = 6
    q, k, v = _cross_case(cuda_device, Tk, B, Tq, Tk, 4, 2, D, dtype, "plain")
    n = torch.tensor([Tk, 0, 1, Tk // 2 + 1, -5, Tk + 100], dtype=torch.int32, device=cuda_device)
    m = torch.tensor([Tq, Tq // 2, Tq, 0, Tq, 1], dtype=torch.int32, device=cuda_device)
    for b in range(B):
        lo = max(0, min(Tk, int(n[b])))
        k[b, lo:], v[b, lo:] = math.nan, (math.nan if b % 2 else math.inf)
    out = torch.full_like(q, 7.0)
    binding.cross_attention(q, k, v, kv_lengths=n, q_lengths=m, out=out)
    want, size, score = ref.cross(q, k, v, D ** -0.5, n)
    bound = ref.cross_bounds(want, size, score, D, Tk, dtype, 0.0 if dtype == FP32 else 2.0 ** -8)
    for b in range(B):
        r = max(0, min(Tq, int(m[b])))
        check(out[b, :r], want[b, :r], bound[b, :r], f"entry {b}")
        assert (out[b, r:] == 7).all()
    assert (out[4] == 0).all()                                              # nothing to read
    fresh = binding.cross_attention(q, k, v, kv_lengths=n, q_lengths=m)
    assert (fresh[3] == 0).all() and torch.equal(fresh[0], out[0])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Tq,Tk,H,K,D", [(7, 480, 2, 2, 64), (7, 1301, 4, 1, 64), (40, 200, 2, 1, 128), (130, 257, 2, 2, 64), (300, 64, 1, 1, 32)])
def test_cross_attention_masks(cuda_device, dtype, Tq, Tk, H, K, D):
    """A byte mask per query with empty rows, the same as a bool, and one mask for all queries; infinities and NaN in K and V where a query does not look."""
    g = _gen(cuda_device, Tk)
    q, k, v = _cross_case(cuda_device, Tq + Tk, 3, Tq, Tk, H, K, D, dtype, "heads first")
    mask = (torch.rand(3, Tq, Tk, generator=g, device=cuda_device) < 0.3).to(torch.uint8) * 200
    mask[1, Tq // 2] = 0
    mask[2, :, :Tk - 1] = 0
    got = binding.cross_attention(q, k, v, mask=mask)
    _cross_check(got, q, k, v, D ** -0.5, None, mask, "bytes")
    assert (got[1, Tq // 2] == 0).all()
    assert torch.equal(binding.cross_attention(q, k, v, mask=mask != 0), got)
    n = torch.tensor([Tk, Tk // 2, Tk], dtype=torch.int32, device=cuda_device)
    _cross_check(binding.cross_attention(q, k, v, mask=mask, kv_lengths=n), q, k, v, D ** -0.5, n, mask, "bytes and lengths")
    shared = (torch.rand(3, Tk, generator=g, device=cuda_device) < 0.6)
    shared[0, 0] = True
    bad_k, bad_v = k.clone(), v.clone()
    bad_k[~shared], bad_v[~shared] = math.nan, math.inf
    _cross_check(binding.cross_attention(q, bad_k, bad_v, mask=shared), q, bad_k, bad_v, D ** -0.5, None, shared, "one mask for all")
    # a key that one query alone does not see
    bad_v = v.clone()
    bad_v[0, 5] = math.nan
    lone = torch.ones(3, Tq, Tk, dtype=torch.uint8, device=cuda_device)
    lone[0, 1, 5] = 0
    got = binding.cross_attention(q, k, bad_v, mask=lone)
    assert torch.isnan(got[0, 0]).all() and torch.isnan(got[0, 2:]).all()
    want, size, score = ref.cross(q, k, bad_v, D ** -0.5, None, lone)
    check(got[0, 1], want[0, 1], ref.cross_bounds(want, size, score, D, Tk, dtype, 0.0 if dtype == FP32 else 2.0 ** -8)[0, 1], "the query that does not see it")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Tq", [5, 200, 3001])
def test_cross_attention_of_sharp_and_large_scores(cuda_device, dtype, Tq):
    """Scores in the thousands, rising along the keys so that the running maximum changes in every tile; and one key far above all others."""
    q, k, v = _cross_case(cuda_device, 9, 2, Tq, 700, 2, 2, 64, dtype, "plain")
    k = (k.float() * 0.05 + torch.linspace(-20, 20, 700, device=cuda_device)[None, :, None, None] * q[:, :1, :1].float().sign()).to(dtype)
    _cross_check(binding.cross_attention(q, k, v, scale=1.0), q, k, v, 1.0, None, None, "rising")
    k[:, 333] = (q[:, 0].float() * 40).to(dtype)
    _cross_check(binding.cross_attention(q, k, v, scale=0.5), q, k, v, 0.5, None, None, "one key")
    same = binding.cross_attention(q * 0, k, v)
    mean = v.double().mean(1, keepdim=True).expand(-1, Tq, -1, -1)
    check(same, mean, half_step(dtype) * mean.abs() + (2.0 ** -8 if dtype == BF16 else 2.0 ** -14) * v.double().abs().mean(1, keepdim=True), "even weights")


def test_cross_attention_of_no_keys(cuda_device):
    for dtype in TYPES:
        for Tq in (3, 200):
            q, k, v = _cross_case(cuda_device, 2, 2, Tq, 0, 2, 1, 64, dtype, "plain")
            assert (binding.cross_attention(q, k, v, out=torch.ones_like(q)) == 0).all()
            assert binding.cross_attention(q[:, :0], k, v).shape == (2, 0, 2, 64)


# ------------------------------------------------------------------------------- common to all
def _calls(dev, dtype, size):
    """(name, call) of each operator on fixed inputs; a call takes keyword arguments and returns a tuple of tensors."""
    T, Tk = [(1, 300), (260, 700), (1100, 2000)][size]
    q, k, w, pos, inv = _rope_case(dev, 21, 2, T, 2, 2, 64, 64, dtype)
    lq, lk, lv, decay, state = _linear_case(dev, 22, 2, T, 2, 2, 64, dtype)
    cq, ck, cv = _cross_case(dev, 23, 2, T, Tk, 2, 2, 64, dtype)
    new = torch.empty_like(state)
    return [("rope", lambda **kw: binding.qk_norm_rope(q, k, pos, inv, w[0], w[1], **kw)),
            ("linear", lambda **kw: tuple(x.clone() for x in binding.linear_attention(lq, lk, lv, decay, state, state_out=new, **kw))),
            ("cross", lambda **kw: (binding.cross_attention(cq, ck, cv, **kw),))]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [0, 1, 2])
def test_streams_and_graphs_give_the_same_bits(cuda_device, dtype, size):
    for name, call in _calls(cuda_device, dtype, size):
        want = [x.clone() for x in call()]
        for _ in range(3):
            assert all(torch.equal(a, b) for a, b in zip(call(), want)), name
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = call()
        other = call(stream=side) if name != "linear" else got
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and all(torch.equal(a, b) for a, b in zip(other, want)), name
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = call()
        for _ in range(2):
            for x in got:
                x.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want)), name


@pytest.mark.parametrize("Tq,Tk", [(7, 90000), (1100, 2000)])
def test_two_graphs_at_once(cuda_device, Tq, Tk):
    """Captured apart, replayed side by side on two streams: each has scratch of its own."""
    q, k, v = _cross_case(cuda_device, 5, 1, Tq, Tk, 4, 4, 64, BF16)
    q2, k2, v2 = _cross_case(cuda_device, 6, 1, Tq, Tk, 4, 4, 64, BF16)
    want, want2 = binding.cross_attention(q, k, v), binding.cross_attention(q2, k2, v2)
    graphs, outs = [], []
    for a in ((q, k, v), (q2, k2, v2)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(binding.cross_attention(*a))
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(20):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want) and torch.equal(outs[1], want2)


def test_rows_more_than_32_bits_apart(cuda_device):
    """Entries, tokens and heads whose offsets pass 2^32 elements."""
    far = 2 ** 32 + 64
    room = torch.empty(far + 64 * 4000, dtype=BF16, device=cuda_device)
    g = _gen(cuda_device, 8)
    for strides in ((far, 64, 64), (64, far, 64)):
        # two entries, or two tokens of one
        B, T = (2, 4000) if strides[0] == far else (1, 2)
        x = room.as_strided((B, T, 1, 64), strides[:2] + (64, 1))
        x.copy_(torch.randn(B, T, 1, 64, generator=g, device=cuda_device).to(BF16))
        near = x.contiguous()
        q = torch.randn(B, 2000, 1, 64, generator=g, device=cuda_device).to(BF16)
        assert torch.equal(binding.cross_attention(q, x, x), binding.cross_attention(q, near, near))
        assert torch.equal(binding.cross_attention(q[:, :3], x, x), binding.cross_attention(q[:, :3], near, near))
        assert torch.equal(binding.qk_norm_rope(x, None)[0], binding.qk_norm_rope(near, None)[0])
        decay, state = torch.tensor([-0.1], device=cuda_device), torch.randn(B, 1, 64, 64, generator=g, device=cuda_device)
        a, b = (binding.linear_attention(y, y, y, decay, state, state_out=torch.empty_like(state)) for y in (x, near))
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        y = x.clone(memory_format=torch.contiguous_format)
        binding.qk_norm_rope(x, None, out=(x, None))
        assert torch.equal(x, binding.qk_norm_rope(y, None)[0])


def test_shared_inputs(cuda_device):
    """Keys and values that all entries, or all heads, share through a stride of 0."""
    for Tq, Tk in ((3, 200), (300, 200), (1000, 1500)):
        q, k, v = _cross_case(cuda_device, 3, 3, Tq, Tk, 2, 2, 64, BF16, "plain")
        for a, b in ((k[:1].expand(3, -1, -1, -1), v[:1].expand(3, -1, -1, -1)), (k[:, :, :1].expand(-1, -1, 2, -1), v[:, :, :1].expand(-1, -1, 2, -1))):
            assert torch.equal(binding.cross_attention(q, a, b), binding.cross_attention(q, a.contiguous(), b.contiguous()))
            d, s = torch.tensor([-0.1, 0.0], device=cuda_device), torch.zeros(3, 2, 64, 64, device=cuda_device)
            x = binding.linear_attention(a, a, b, d, s, state_out=torch.empty_like(s))
            y = binding.linear_attention(a.contiguous(), a.contiguous(), b.contiguous(), d, s, state_out=torch.empty_like(s))
            assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])


def test_refusals_of_tensors(cuda_device):
    q = torch.zeros(2, 4, 2, 64, dtype=BF16, device=cuda_device)
    d, s = torch.zeros(2, device=cuda_device), torch.zeros(2, 2, 64, 64, device=cuda_device)
    n = torch.zeros(2, dtype=torch.int32, device=cuda_device)
    inv, pos = torch.ones(32, dtype=torch.float64, device=cuda_device), torch.zeros(2, 4, dtype=torch.int64, device=cuda_device)
    mask = torch.ones(2, 4, 4, dtype=torch.uint8, device=cuda_device)
    for bad in (lambda: binding.cross_attention(q.half(), q.half(), q.half()), lambda: binding.cross_attention(q, q.float(), q.float()),
                lambda: binding.cross_attention(q, q, q[:, :3]), lambda: binding.cross_attention(q, q[:1], q[:1]),
                lambda: binding.cross_attention(q, q, q, kv_lengths=n.long()), lambda: binding.cross_attention(q, q, q, kv_lengths=n[:1]),
                lambda: binding.cross_attention(q, q, q, mask=mask[:, :3]), lambda: binding.cross_attention(q, q, q, mask=mask.int()),
                lambda: binding.cross_attention(q, q, q, mask=mask.transpose(1, 2)[:, :, ::2]), lambda: binding.cross_attention(q, q, q, scale=0.0),
                lambda: binding.cross_attention(q[..., ::2], q[..., ::2], q[..., ::2]), lambda: binding.cross_attention(q[..., 4:36], q[..., 4:36], q[..., 4:36]),
                lambda: binding.cross_attention(q, q, q, out=q[:1].expand(2, -1, -1, -1)), lambda: binding.cross_attention(q, q.cpu(), q.cpu()),
                lambda: binding.linear_attention(q, q, q, d, s[:1]), lambda: binding.linear_attention(q, q, q, d[:1], s),
                lambda: binding.linear_attention(q, q, q, d, s.double()), lambda: binding.linear_attention(q, q, q, d, s.transpose(2, 3)),
                lambda: binding.linear_attention(q, q, q, d, s, slots=n.long()), lambda: binding.linear_attention(q, q, q, d, s, state_out=s[:1]),
                lambda: binding.qk_norm_rope(q, q[:, :3]), lambda: binding.qk_norm_rope(q, q, pos.int(), inv), lambda: binding.qk_norm_rope(q, q, None, inv),
                lambda: binding.qk_norm_rope(q, q, pos, inv.float()), lambda: binding.qk_norm_rope(q, q, pos, inv[:30]), lambda: binding.qk_norm_rope(q, q, pos[:1], inv),
                lambda: binding.qk_norm_rope(q, q, q_weight=d), lambda: binding.qk_norm_rope(q, q, out=(q, q[:, :, :1]))):
        with pytest.raises(binding.TTError):
            bad()
    torch.cuda.synchronize()


def test_a_tick_of_a_token_model(cuda_device):
    """The operators as a model of K streams uses them behind the framework's own path: each stream's frame goes through the tick; per
    tool a query is normed and turned by the frame's number, runs through the recurrent cell in the stream's slot, and reads the
    stream's map where the tool's mask is set.  Two frames, held against the definitions in 64 bits."""
    wl = tt_synth.workload("cfg1-gain").with_(name="tokens", src_w=214, src_h=120, net_w=160, net_h=120, hidden=128)
    K, T, H, D = 3, wl.n_tools, 2, 64
    ctx = binding.Context(binding.make_config(wl, max_streams=K), tt_synth.make_weights(wl))
    states = [ctx.state_create() for _ in range(K)]
    g = _gen(cuda_device, 12)
    first = (torch.randn(K, T, H, D, generator=g, device=cuda_device)).to(BF16)      # the tools' queries
    w = 1 + 0.2 * torch.randn(D, generator=g, device=cuda_device)
    to_kv = torch.randn(wl.hidden, 2 * H * D, generator=g, device=cuda_device).to(BF16) * 0.09
    decay = torch.tensor([-0.05, -0.5], device=cuda_device)
    cell = torch.zeros(K, H, D, D, device=cuda_device)
    inv = torch.from_numpy(binding.rope_frequencies(32)[0]).to(cuda_device)
    slots = torch.tensor([2, 0, 1], dtype=torch.int32, device=cuda_device)
    hm, wm = ctx.hm, ctx.wm
    for frame in range(2):
        fr = [tt_synth.make_frame(wl.frame_kind, wl.stream_seed(s), frame, wl.src_w, wl.src_h) for s in range(K)]
        ctx.submit_frames([torch.from_numpy(f).to(cuda_device) for f in fr], states, frame_index=frame)
        res = ctx.sync()
        maps = torch.stack([torch.from_numpy(ctx.state_export(s)[0]).reshape(wl.hidden, hm * wm).T for s in states]).to(cuda_device).to(BF16)
        masks = torch.stack([torch.from_numpy(ctx.fetch_masks(r)).reshape(T, hm * wm) for r in res]).to(cuda_device)
        pos = torch.full((K, T), 1_000_000 + frame, dtype=torch.int64, device=cuda_device)
        q, k = binding.qk_norm_rope(first, first, pos, inv, w, w)
        for got in (q, k):
            _rope_check(got, first, w, pos, inv, 1e-6, True, False, 1.0, "norm and rotation")
        before = cell.clone()
        r, cell = binding.linear_attention(q, k, first, decay, cell, scale=D ** -0.5, slots=slots)
        _linear_check(r, cell[slots.long()], q, k, first, decay, before[slots.long()], D ** -0.5, None, "cell")
        kv = (maps @ to_kv).view(K, hm * wm, 2 * H, D)
        out = binding.cross_attention(r, kv[:, :, :H], kv[:, :, H:], mask=masks)
        _cross_check(out, r, kv[:, :, :H], kv[:, :, H:], D ** -0.5, None, masks, "reading the map")
        assert (out[masks.sum(-1) == 0] == 0).all() and out.abs().sum() > 0
    ctx.destroy()
