"""The gated delta rule against its definition in 64 bits (delta_reference.py), at the sizes and values where it can go wrong."""
import math

import pytest
import torch

from paper_2402_04466_b200 import binding
import delta_reference as ref
from token_reference import check

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32
TYPES = [BF16, FP32]


def _place(x, layout, pad=float("nan")):
    """The same tensor in memory as a projection or a view leaves it, with NaN around it."""
    B, T, H, D = x.shape
    if layout == "plain":
        return x
    if layout == "fused":
        y = torch.full((B, T, H + 3, D), pad, dtype=x.dtype, device=x.device)[:, :, 1:H + 1]
    elif layout == "heads first":
        y = torch.full((B, H, T, D), pad, dtype=x.dtype, device=x.device).transpose(1, 2)
    else:
        y = torch.full((B, T + 5, H, D + 8), pad, dtype=x.dtype, device=x.device)[:, 2:T + 2, :, :D]
    y.copy_(x)
    return y


def _case(dev, seed, B, T, H, K, D, dtype, layout="plain", slots=None, alike=0.7):
    """Queries and keys of length 1 that resemble each other, gates from a model's: rates from a few tokens to hundreds."""
    g = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev)

    qk = [normal(B, T, K, D) + alike * normal(B, 1, K, D) for _ in range(2)]
    q, k = ((x / x.norm(dim=-1, keepdim=True)).to(dtype) for x in qk)
    if dtype == BF16:
        k = (k.float() * (1 - 2.0 ** -8)).to(dtype)      # beta |k|^2 stays at 2 or below whichever way k was rounded
    v = (normal(B, T, H, D) + 0.2).to(dtype)
    rate = torch.exp(torch.linspace(-6, 0, H, device=dev))
    decay = -rate * torch.nn.functional.softplus(normal(B, T, H))
    beta = torch.sigmoid(normal(B, T, H)) * 1.9
    state = normal(slots or B, H, D, D)
    return *(_place(x, layout) for x in (q, k, v)), decay, beta, state


def _check(out, state, q, k, v, decay, beta, before, scale, lengths, name):
    want, size, S, A = ref.delta(q, k, v, decay, beta, before, scale, lengths)
    B, T, H, D = v.shape
    bound, state_bound = ref.bounds(want, size, A, D, T, v.dtype, T > 1)
    n = [T] * B if lengths is None else [max(0, min(T, int(x))) for x in lengths]
    for b in range(B):
        check(out[b, :n[b]], want[b, :n[b]], bound[b, :n[b]], f"{name}, out of {b}")
    check(state, S, state_bound, f"{name}, state")
    # And as a whole, where errors are independent.  A token's sum of D products is rounded D times by half a step, 2^-24 / sqrt(3) in the mean, of a partial sum that
    # is on average half grown: sqrt(D) 2^-24 / sqrt(12) of the column.  beta up to 1.9 adds as much of it to the state, and of an error's square a token takes
    # (2 beta - beta^2) / D away, 0.8 / D in the mean, so that those of 2 D tokens are left at most: 1.9 sqrt(D min(T, 2 D)) 2^-24 / sqrt(12).  Two more
    # half steps for the element itself.
    off, most = float((state.double() - S).norm() / S.norm()), (0.55 * (D * min(T, 2 * D)) ** 0.5 + 2) * 2.0 ** -24
    assert off < most, f"{name}: state off by {off:.2e} of {most:.2e}"


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,T,H,K,D", [
    (1, 1, 1, 1, 32), (5, 1, 2, 2, 64), (3, 1, 4, 2, 128), (200, 1, 4, 4, 64), (2, 2, 2, 1, 64), (2, 3, 1, 1, 128), (2, 8, 2, 2, 64), (1, 9, 4, 2, 64), (200, 6, 4, 4, 64), (90, 5, 2, 1, 32), (80, 4, 2, 2, 128), (2, 12, 2, 2, 32), (3, 13, 2, 1, 64),
    (40, 24, 4, 4, 128), (40, 25, 4, 4, 128), (1, 15, 2, 2, 64), (1, 16, 3, 3, 32), (2, 17, 4, 1, 128),
    (2, 31, 2, 2, 64), (2, 32, 2, 2, 128), (2, 33, 2, 1, 32), (3, 60, 2, 2, 64), (1, 63, 2, 2, 128), (2, 64, 2, 2, 64), (2, 65, 2, 2, 32), (2, 127, 2, 1, 128), (2, 128, 2, 2, 64),
    (1, 129, 4, 2, 64), (2, 200, 2, 2, 32), (2, 333, 2, 1, 128), (1, 1000, 2, 2, 64), (40, 97, 4, 4, 64), (20, 190, 8, 4, 128), (90, 70, 4, 2, 32)])
def test_delta_rule(cuda_device, dtype, B, T, H, K, D):
    for layout, scale in (("fused", 1.0), ("heads first", 0.3), ("padded", -2.0)):
        q, k, v, decay, beta, state = _case(cuda_device, B + T, B, T, H, K, D, dtype, layout)
        before = state.clone()
        out, new = binding.delta_rule(q, k, v, decay, beta, state, scale=scale, state_out=torch.full_like(state, float("nan")))
        assert torch.equal(state, before)
        _check(out, new, q, k, v, decay, beta, before, scale, None, layout)
        again, same = binding.delta_rule(q, k, v, decay, beta, state, scale=scale)
        assert same is state and torch.equal(state, new) and torch.equal(again, out)      # in place, the same bits


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [1, 2, 60, 65, 400])
@pytest.mark.parametrize("H,D", [(2, 64), (2, 128), (40, 32), (14, 64), (8, 128)])
def test_slots_and_lengths(cuda_device, dtype, T, H, D):
    """Slots in any order; entries without tokens, of one, of all and of more; rows behind the last token hold NaN and stay as they are, as do slots that no entry has."""
    B, n = 9, 13
    q, k, v, decay, beta, state = _case(cuda_device, T, B, T, H, 1, D, dtype, "fused", slots=n)
    want_lengths = [T, 0, 1, T // 2, T + 7, -3, T, T, T]
    slots = torch.tensor([4, 12, 0, 7, 9, 3, 4, -1, 13], dtype=torch.int32, device=cuda_device)      # the sixth takes the first's, two are out of range
    for b, m in enumerate(want_lengths[:6]):
        for x in (q, k, v, decay, beta):
            x[b, max(m, 0):] = float("nan")
    for b in (6, 7, 8):
        for x in (q, k, v, decay, beta):
            x[b] = float("nan")
    for i in set(range(n)) - set(slots[:6].tolist()):
        state[i] = float("nan")
    lengths = torch.tensor(want_lengths, dtype=torch.int32, device=cuda_device)
    out = torch.full((B, T, H, D), 7.0, dtype=dtype, device=cuda_device)
    new = torch.full_like(state, 5.0)
    binding.delta_rule(q, k, v, decay, beta, state, lengths=lengths, slots=slots, out=out, state_out=new)
    at = slots[:6].long()
    clean = [x[:6].nan_to_num(0.0) for x in (q, k, v, decay, beta)]
    _check(out[:6], new[at], *clean, state[at], 1.0, want_lengths[:6], "slots")
    for b, m in enumerate(want_lengths[:6]):
        assert (out[b, min(T, max(m, 0)):] == 7).all()
    assert (out[6:] == 7).all()
    assert all((new[i] == 5).all() for i in range(n) if i not in at.tolist())
    # in place, and the same bits
    there = state.clone()
    out2, _ = binding.delta_rule(q, k, v, decay, beta, there, lengths=lengths, slots=slots)
    assert torch.equal(there[at], new[at])
    others = [i for i in range(n) if i not in at.tolist()]
    assert there[others].isnan().all()
    for b, m in enumerate(want_lengths[:6]):
        m = min(T, max(m, 0))
        assert torch.equal(out2[b, :m], out[b, :m]) and (out2[b, m:] == 0).all()
    assert (out2[6:] == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("T", [60, 150])
def test_gates_at_their_ends(cuda_device, dtype, D, T):
    """No decay at all, decays of 0 and -infinity and far below what 32 bits can hold, beta of 0, 1 and 2: beside tokens that hardly fade."""
    B, H = 2, 6
    q, k, v, decay, beta, state = _case(cuda_device, D, B, T, H, H, D, dtype)
    _check(*binding.delta_rule(q, k, v, None, beta, state, state_out=torch.empty_like(state)), q, k, v, None, beta, state, 1.0, None, "no decay")
    decay[:, :, 0], decay[:, ::7, 1], decay[:, 40::9, 2], decay[:, 10, 3], decay[:, :, 4] = 0.0, -math.inf, -1e4, -90.0, -0.001
    decay[:, 20:25, 4] = -300.0
    beta[:, ::3, 0], beta[:, :, 1], beta[:, :, 2], beta[:, 5:100, 3] = 0.0, 1.0, 2.0 - 2.0 ** -6, 0.0
    _check(*binding.delta_rule(q, k, v, decay, beta, state, state_out=torch.empty_like(state)), q, k, v, decay, beta, state, 1.0, None, "ends")


@pytest.mark.parametrize("dtype", TYPES)
def test_keys_that_repeat(cuda_device, dtype):
    """One key for every token: with beta 1 the state says the last value of it, whatever came before."""
    B, T, H, D = 2, 200, 2, 64
    q, k, v, decay, beta, state = _case(cuda_device, 1, B, T, H, H, D, dtype)
    k = torch.zeros_like(k)
    k[..., 5] = 1
    out, new = binding.delta_rule(k, k, v, None, torch.ones_like(beta), state, state_out=torch.empty_like(state))
    # u is at most 10 and counts with 16 bits, 10 * 2^-17; up to 64 of them add up to a value of at most 10, half a step of 2^-24 each
    assert ((out.double() - v.double()).abs() <= ref.half_step(dtype) * v.double().abs() + 2.0 ** -13 + 64 * 10 * 2.0 ** -24).all()
    assert torch.allclose(new[:, :, 5], v[:, -1].float(), rtol=0, atol=64 * 10 * 2.0 ** -24) and torch.equal(new[:, :, 6:], state[:, :, 6:])
    k = torch.full_like(k, D ** -0.5)
    _check(*binding.delta_rule(k, k, v, decay, beta, state, state_out=torch.empty_like(state)), k, k, v, decay, beta, state, 1.0, None, "dense")


@pytest.mark.parametrize("dtype", TYPES)
def test_in_pieces_is_the_same_rule(cuda_device, dtype):
    B, T, H, D = 3, 259, 4, 64
    q, k, v, decay, beta, state = _case(cuda_device, 3, B, T, H, 2, D, dtype)
    cell, at = state.clone(), 0
    parts = []
    for n in (1, 64, 2, 130, 1, 61):
        s = slice(at, at + n)
        parts.append(binding.delta_rule(q[:, s], k[:, s], v[:, s], decay[:, s].contiguous(), beta[:, s].contiguous(), cell)[0])
        at += n
    assert at == T
    _check(torch.cat(parts, 1), cell, q, k, v, decay, beta, state, 1.0, None, "pieces")


@pytest.mark.parametrize("B,T,H,D", [(8, 6000, 4, 64), (2, 9000, 1, 32), (3, 5001, 2, 128)])
@pytest.mark.parametrize("dtype", TYPES)
def test_long_sequences(cuda_device, dtype, B, T, H, D):
    q, k, v, decay, beta, state = _case(cuda_device, T, B, T, H, 1, D, dtype)
    decay[..., 0] *= 0.02      # memories of thousands of tokens
    _check(*binding.delta_rule(q, k, v, decay, beta, state, state_out=torch.empty_like(state)), q, k, v, decay, beta, state, 1.0, None, "long")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,D", [(2, 32), (2, 64), (2, 128), (40, 32), (20, 64), (10, 128)])
@pytest.mark.parametrize("T", [1, 60, 130])
def test_what_is_not_finite_goes_where_the_formula_takes_it(cuda_device, dtype, H, D, T):
    """An infinity or NaN in q makes its own row of out not finite, one in v its column, one in k or a gate its head, each from its token on; nothing before it."""
    B = 6
    for seed, at in ((0, 0), (1, T // 2), (2, T - 1)):
        q, k, v, decay, beta, state = _case(cuda_device, seed + D, B, T, H, H, D, dtype)
        k[k == 0] = 0.01
        other = T - 1 - at
        q[0, at, 0, 3] = math.nan
        k[1, at, 1, 7] = math.inf
        v[2, at, 0, D - 1], v[2, other, 1, 0] = -math.inf, math.nan
        decay[3, at, 1] = math.nan
        beta[4, at, 0] = math.inf
        state[5, 1, 2, 9] = math.inf
        out, new = binding.delta_rule(q, k, v, decay, beta, state, state_out=torch.empty_like(state))
        want, size, S, A = ref.delta(q, k, v, decay, beta, state)
        assert not torch.isfinite(want).all() and torch.isfinite(want).any()
        assert torch.equal(torch.isfinite(out), torch.isfinite(want)) and torch.equal(torch.isfinite(new), torch.isfinite(S))
        bound, state_bound = ref.bounds(want, size, A, D, T, dtype, T > 1)
        for got, exact, off in ((out, want, bound), (new, S, state_bound)):
            fine = torch.isfinite(exact) & torch.isfinite(off)
            check(got[fine], exact[fine], off[fine], "finite part")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,T,H,D", [(64, 1000, 8, 32), (70, 70, 190, 32), (24, 1700, 10, 64)])
def test_more_windows_than_are_prepared_at_once(cuda_device, dtype, B, T, H, D):
    """Entries that end in each of the ranges of windows, at their borders, and before the first; slots, of which two entries share one."""
    q, k, v, decay, beta, state = _case(cuda_device, T, B, T, H, 1, D, dtype, slots=B + 2)
    n = [(0, 1, 32, 33, 511, 512, 513, T // 2, T - 1, T)[b % 10] for b in range(B)]
    n = [min(x, T) for x in n]
    slots = torch.arange(B + 1, 1, -1, dtype=torch.int32, device=cuda_device)
    slots[7] = slots[3]
    lengths, before, new = torch.tensor(n, dtype=torch.int32, device=cuda_device), state.clone(), torch.full_like(state, 5.0)
    out, _ = binding.delta_rule(q, k, v, decay, beta, state, scale=0.7, slots=slots, lengths=lengths, state_out=new)
    assert torch.equal(state, before)
    own = [b for b in range(B) if b != 7]
    at, mine = slots[own].long(), torch.tensor(own, device=cuda_device)
    _check(out[mine], new[at], *(x[mine] for x in (q, k, v, decay, beta)), before[at], 0.7, [n[b] for b in own], "ranges")
    left = [i for i in range(B + 2) if i not in at.tolist()]
    assert (new[left] == 5).all() and (out[7] == 0).all() and all((out[b, n[b]:] == 0).all() for b in own)
    again, _ = binding.delta_rule(q, k, v, decay, beta, state, scale=0.7, slots=slots, lengths=lengths)
    assert torch.equal(again, out) and torch.equal(state[at], new[at]) and torch.equal(state[left], before[left])
    # captured, and replayed twice in place
    want = [binding.delta_rule(q, k, v, decay, beta, state, scale=0.7, slots=slots, lengths=lengths)[0] for _ in range(2)][1]
    cell, graph = before.clone(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got, _ = binding.delta_rule(q, k, v, decay, beta, cell, scale=0.7, slots=slots, lengths=lengths)
    cell.copy_(before)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(cell, state)


def test_no_tokens(cuda_device):
    for dtype in TYPES:
        q, k, v, decay, beta, state = _case(cuda_device, 1, 2, 3, 2, 1, 64, dtype)
        new = torch.zeros_like(state)
        out, _ = binding.delta_rule(q[:, :0], k[:, :0], v[:, :0], decay[:, :0].contiguous(), beta[:, :0].contiguous(), state, state_out=new)
        assert out.shape == (2, 0, 2, 64) and torch.equal(new, state)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [1, 5, 50, 300])
def test_streams_and_graphs_give_the_same_bits(cuda_device, dtype, T):
    q, k, v, decay, beta, state = _case(cuda_device, T, 3, T, 4, 2, 64, dtype)
    new = torch.empty_like(state)

    def call(**kw):
        return tuple(x.clone() for x in binding.delta_rule(q, k, v, decay, beta, state, state_out=new, **kw))

    want = call()
    assert all(torch.equal(a, b) for a, b in zip(call(), want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out, _ = binding.delta_rule(q, k, v, decay, beta, state, state_out=new, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(out, want[0]) and torch.equal(new, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for _ in range(2):
        for x in got:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_two_graphs_at_once(cuda_device):
    """Captured apart, replayed side by side on two streams, each advancing states of its own in place."""
    cases = [_case(cuda_device, s, 2, 500, 4, 4, 64, BF16) for s in (1, 2)]
    graphs, outs, cells = [], [], []
    for c in cases:
        cells.append(c[5].clone())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(binding.delta_rule(*c[:5], cells[-1])[0])
        graphs.append(g)
    torch.cuda.synchronize()
    for x, c in zip(cells, cases):
        x.copy_(c[5])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(4):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for c, cell, out in zip(cases, cells, outs):
        own = c[5].clone()
        for _ in range(4):
            last = binding.delta_rule(*c[:5], own)[0]
        assert torch.equal(own, cell) and torch.equal(last, out)


def test_shared_and_far_inputs(cuda_device):
    """Keys and values that all entries or heads share through a stride of 0, and tokens and entries whose offsets pass 2^32 elements."""
    q, k, v, decay, beta, state = _case(cuda_device, 4, 3, 70, 2, 2, 64, BF16)
    for x, y in ((k[:1].expand(3, -1, -1, -1), v[:1].expand(3, -1, -1, -1)), (k[:, :, :1].expand(-1, -1, 2, -1), v[:, :, :1].expand(-1, -1, 2, -1))):
        a = binding.delta_rule(x, x, y, decay, beta, state, state_out=torch.empty_like(state))
        b = binding.delta_rule(x.contiguous(), x.contiguous(), y.contiguous(), decay, beta, state, state_out=torch.empty_like(state))
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    far = 2 ** 32 + 64
    room = torch.empty(far + 64 * 100, dtype=BF16, device=cuda_device)
    for B, T, strides in ((2, 100, (far, 64, 64)), (1, 2, (64, far, 64)), (2, 1, (far, 64, 64))):
        x = room.as_strided((B, T, 1, 64), strides + (1,))
        _, near, _, decay, beta, state = _case(cuda_device, 5, B, T, 1, 1, 64, BF16)
        x.copy_(near)
        a, b = (binding.delta_rule(y, y, y, decay, beta, state, state_out=torch.empty_like(state)) for y in (x, near))
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        binding.delta_rule(near, near, near, decay, beta, state.clone(), out=x)
        assert torch.equal(x, b[0])


def test_refusals_of_tensors(cuda_device):
    q = torch.zeros(2, 4, 2, 64, dtype=BF16, device=cuda_device)
    g, s = torch.zeros(2, 4, 2, device=cuda_device), torch.zeros(2, 2, 64, 64, device=cuda_device)
    n = torch.zeros(2, dtype=torch.int32, device=cuda_device)
    for bad in (lambda: binding.delta_rule(q.half(), q.half(), q.half(), g, g, s), lambda: binding.delta_rule(q, q.float(), q, g, g, s),
                lambda: binding.delta_rule(q, q, q[:, :3], g, g, s), lambda: binding.delta_rule(q, q[:, :, :1], q, g, g, s),
                lambda: binding.delta_rule(q, q, q, g[:, :3], g, s), lambda: binding.delta_rule(q, q, q, g, g.double(), s),
                lambda: binding.delta_rule(q, q, q, g, g.transpose(0, 1), s), lambda: binding.delta_rule(q, q, q, g, g, s[:1]),
                lambda: binding.delta_rule(q, q, q, g, g, s.double()), lambda: binding.delta_rule(q, q, q, g, g, s, slots=n.long()),
                lambda: binding.delta_rule(q, q, q, g, g, s, lengths=n[:1]), lambda: binding.delta_rule(q, q, q, g, g, s, state_out=s[:1]),
                lambda: binding.delta_rule(q, q, q, g, None, s), lambda: binding.delta_rule(q, q, q, g, g.cpu(), s),
                lambda: binding.delta_rule(q, q, q, g, g, s, scale=math.nan), lambda: binding.delta_rule(q, q, q, g, g, s, out=q[:1].expand(2, -1, -1, -1))):
        with pytest.raises(binding.TTError):
            bad()
    torch.cuda.synchronize()


def test_results_carry_no_gradient(cuda_device):
    for T in (1, 40):
        x = torch.randn(1, T, 2, 64, device=cuda_device, requires_grad=True)
        g = torch.full((1, T, 2), 0.01, device=cuda_device, requires_grad=True)
        for y in binding.delta_rule(x, x, x, None, g, torch.zeros(1, 2, 64, 64, device=cuda_device)):
            assert not y.requires_grad and torch.isfinite(y).all()


@pytest.mark.parametrize("T", [1, 50, 600])
def test_tensors_let_go_before_another_stream_has_read_them(cuda_device, T):
    x, _, _, decay, beta, state = _case(cuda_device, 6, 2, T, 2, 2, 64, FP32)
    call = lambda y, f, s: binding.delta_rule(y, y, y, f, beta, state, state_out=torch.zeros_like(state), stream=s)[0]      # noqa: E731
    want = call(x, decay, None)
    side = torch.cuda.Stream()
    call(x, decay, side)                                  # what is set up once is there
    torch.cuda.synchronize()
    y, f = x.clone(), decay.clone()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(40_000_000)                     # some 20 ms
    got = call(y, f, side)
    del y, f
    others = [torch.full_like(z, math.nan) for _ in range(8) for z in (x, decay)]
    torch.cuda.synchronize()
    assert torch.equal(got, want) and len(others) == 16


def test_two_calls_at_once(cuda_device):
    """On two streams, each with records and states of its own."""
    cases = [_case(cuda_device, s, 3, 700, 6, 3, 64, BF16) for s in (7, 8)]
    want = [[x.clone() for x in binding.delta_rule(*c, state_out=torch.empty_like(c[5]))] for c in cases]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(10):
        got = [binding.delta_rule(*c, state_out=torch.empty_like(c[5]), stream=s) for c, s in zip(cases, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for x, y in zip(got, want) for a, b in zip(x, y))
