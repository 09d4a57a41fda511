"""Differential attention against its definition in 64 bits (difference_reference.py), at the sizes and masks where it can go wrong."""
import math

import pytest
import torch

from paper_2402_04466_b200 import binding
import difference_reference as ref
from token_reference import check

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32
TYPES = [BF16, FP32]


def _place(x, layout, pad=float("nan")):
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


def _case(dev, seed, B, Tq, Tk, H, K, D, dtype, layout="plain", sharp=1.0, each=False):
    g = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev)

    q, k, v = (normal(B, Tq, H, D) * sharp).to(dtype), normal(B, Tk, K, D).to(dtype), (normal(B, Tk, K, D) + 0.2).to(dtype)
    return *(_place(x, layout) for x in (q, k, v)), 0.3 * normal(*([H] if each else []), 4, D // 2), 1 + 0.3 * normal(D)


def _once(Tq, dtype, mask):
    """How weights may be rounded: to 16 bits, in large calls without a mask to bf16."""
    return 0.0 if dtype == FP32 else 2.0 ** -16 if Tq <= 32 or mask is not None else 2.0 ** -8


def _check(got, q, k, v, vectors, init, name, scale=None, n=None, mask=None, rows=None, **kw):
    scale = (q.shape[-1] // 2) ** -0.5 if scale is None else scale
    want, bound = ref.difference(q, k, v, vectors, init, scale, kv_lengths=n, mask=mask, once=_once(q.shape[1], q.dtype, mask), dtype=q.dtype, **kw)
    for b in range(q.shape[0]):
        m = q.shape[1] if rows is None else rows[b]
        check(got[b, :m], want[b, :m], bound[b, :m], f"{name}, entry {b}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,Tq,Tk,H,K,D", [
    (1, 1, 1, 1, 1, 32), (2, 1, 2, 2, 1, 64), (1, 1, 17, 2, 2, 128), (3, 7, 60, 2, 2, 64), (2, 5, 63, 4, 1, 128), (2, 16, 64, 2, 2, 32), (1, 17, 65, 3, 3, 64),
    (2, 7, 1000, 4, 2, 64), (1, 7, 5001, 2, 2, 128), (1, 3, 20000, 1, 1, 32), (2, 33, 130, 6, 2, 64), (2, 64, 300, 2, 2, 128), (1, 65, 129, 2, 1, 64),
    (2, 127, 257, 2, 2, 64), (1, 129, 511, 2, 2, 128), (2, 200, 333, 2, 2, 32), (3, 300, 1, 1, 1, 64)])
def test_differential_attention(cuda_device, dtype, B, Tq, Tk, H, K, D):
    for i, layout in enumerate(("fused", "heads first", "padded")):
        q, k, v, vectors, w = _case(cuda_device, Tq + Tk, B, Tq, Tk, H, K, D, dtype, layout, each=i == 1)
        kw = [dict(norm=True, weight=w, eps=1e-5, out_scale=0.8), dict(norm=True, weight=None, eps=1e-3, out_scale=-0.5), dict(norm=False, out_scale=1.5)][i]
        init = [0.2, 0.65, -0.4][i]
        got = binding.differential_attention(q, k, v, vectors, init, norm=kw["norm"], norm_weight=kw.get("weight"), eps=kw.get("eps", 0.0), out_scale=kw["out_scale"])
        _check(got, q, k, v, vectors, init, layout, **kw)


@pytest.mark.parametrize("B,Tq,Tk,H,K,D", [(2, 1100, 1300, 4, 4, 64), (2, 700, 2049, 2, 1, 128), (3, 999, 1500, 4, 2, 32), (1, 4000, 700, 2, 2, 64), (5, 150, 4800, 2, 2, 128), (3, 33, 14400, 4, 2, 128), (8, 40, 9001, 4, 4, 64),
                                           (300, 70, 130, 2, 2, 64)])
def test_many_queries(cuda_device, B, Tq, Tk, H, K, D):
    q, k, v, vectors, w = _case(cuda_device, Tq, B, Tq, Tk, H, K, D, BF16, "fused", each=True)
    for kw in (dict(norm=True, weight=w, eps=1e-5, out_scale=0.8), dict(norm=False, out_scale=1.0)):
        got = binding.differential_attention(q, k, v, vectors, 0.3, norm=kw["norm"], norm_weight=kw.get("weight"), out_scale=kw["out_scale"])
        _check(got, q, k, v, vectors, 0.3, "many", **kw)


def test_defaults_are_the_usual_ones(cuda_device):
    q, k, v, vectors, _ = _case(cuda_device, 1, 2, 7, 100, 2, 2, 64, FP32)
    a = binding.differential_attention(q, k, v, vectors, 0.25)
    assert torch.equal(a, binding.differential_attention(q, k, v, vectors, 0.25, scale=32 ** -0.5, norm=True, eps=1e-5, out_scale=0.75))
    assert torch.equal(binding.differential_attention(q, k, v, vectors, 0.25, norm=False), binding.differential_attention(q, k, v, vectors, 0.25, norm=False, out_scale=1.0))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Tq,Tk,D", [(7, 700, 64), (150, 300, 64), (300, 130, 128), (260, 1000, 32), (400, 3000, 64), (300, 2001, 128), (700, 1100, 32)])
def test_lengths(cuda_device, dtype, Tq, Tk, D):
    """Entries of no keys and queries, of one, of some and of more than there are; what lies behind a length is NaN, and rows there stay as they are."""
    B, H = 6, 2
    q, k, v, vectors, w = _case(cuda_device, Tk, B, Tq, Tk, H, 1, D, dtype, "fused")
    nk, nq = [0, 1, Tk // 2, Tk, Tk + 9, -4], [Tq, 1, Tq // 2 + 1, 0, Tq + 5, Tq]
    for b in range(B):
        for x in (k, v):
            x[b, max(0, nk[b]):] = float("nan")
        q[b, max(0, nq[b]):] = float("nan")
    out = torch.full((B, Tq, H, D), 3.0, dtype=dtype, device=cuda_device)
    at = [torch.tensor(x, dtype=torch.int32, device=cuda_device) for x in (nk, nq)]
    kw = dict(norm=True, weight=w, eps=1e-5, out_scale=0.8)
    binding.differential_attention(q, k, v, vectors, 0.3, norm_weight=w, out_scale=0.8, kv_lengths=at[0], q_lengths=at[1], out=out)
    rows = [min(Tq, max(0, n)) for n in nq]
    _check(out, q.nan_to_num(0.0), k.nan_to_num(0.0), v.nan_to_num(0.0), vectors, 0.3, "lengths", n=nk, rows=rows, **kw)
    for b in range(B):
        assert (out[b, rows[b]:] == 3).all()
    assert (out[0] == 0).all() and (out[5] == 0).all()
    fresh = binding.differential_attention(q, k, v, vectors, 0.3, norm_weight=w, out_scale=0.8, kv_lengths=at[0], q_lengths=at[1])
    for b in range(B):
        assert torch.equal(fresh[b, :rows[b]], out[b, :rows[b]]) and (fresh[b, rows[b]:] == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Tq,Tk,H,K,D", [(7, 480, 2, 2, 64), (7, 1301, 4, 1, 64), (40, 200, 2, 1, 128), (130, 257, 2, 2, 64), (300, 64, 1, 1, 32)])
def test_masks(cuda_device, dtype, Tq, Tk, H, K, D):
    """Rows that see nothing, one key, the last one, or NaN and infinities only where they do not look; bytes other than 1; a mask for all queries; with a length too."""
    B = 3
    q, k, v, vectors, w = _case(cuda_device, Tk, B, Tq, Tk, H, K, D, dtype, "heads first")
    g = torch.Generator(device=cuda_device).manual_seed(1)
    mask = (torch.rand(B, Tq, Tk, generator=g, device=cuda_device) < 0.4).to(torch.uint8) * 255
    mask[:, 0] = 0
    mask[:, 1 % Tq] = 0
    mask[:, 1 % Tq, Tk // 2] = 1
    mask[:, 2 % Tq] = 0
    mask[:, 2 % Tq, -1] = 2
    dark = Tk // 3
    mask[:, :, dark] = 0
    k[:, dark], v[0, dark], v[1, dark], v[2, dark] = float("nan"), math.inf, float("nan"), -math.inf
    if Tq > 3:
        mask[:, 3] = 0      # nothing, between rows that see something
    clean = [x.nan_to_num(0.0, 0.0, 0.0) for x in (q, k, v)]
    for norm in (True, False):
        kw = dict(norm=norm, weight=w if norm else None, eps=1e-5, out_scale=0.8)
        out = binding.differential_attention(q, k, v, vectors, 0.3, norm=norm, norm_weight=w, out_scale=0.8, mask=mask)
        _check(out, *clean, vectors, 0.3, "mask", mask=mask, **kw)
        assert (out[:, 0] == 0).all()
        n = torch.tensor([Tk // 2, 1, 0], dtype=torch.int32, device=cuda_device)
        _check(binding.differential_attention(q, k, v, vectors, 0.3, norm=norm, norm_weight=w, out_scale=0.8, mask=mask.bool(), kv_lengths=n), *clean, vectors, 0.3, "mask and length",
               n=n, mask=mask, **kw)
        one = mask[:, -1].contiguous()
        _check(binding.differential_attention(q, k, v, vectors, 0.3, norm=norm, norm_weight=w, out_scale=0.8, mask=one), *clean, vectors, 0.3, "one mask", mask=one, **kw)
    wide = torch.zeros(B, Tq, Tk + 3, dtype=torch.uint8, device=cuda_device)[:, :, 1:Tk + 1]
    wide.copy_(mask)
    assert torch.equal(binding.differential_attention(q, k, v, vectors, 0.3, mask=wide), binding.differential_attention(q, k, v, vectors, 0.3, mask=mask))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Tq,Tk", [(5, 700), (200, 900), (1500, 1500)])
def test_what_is_not_finite_stays_in_its_column(cuda_device, dtype, Tq, Tk):
    q, k, v, vectors, w = _case(cuda_device, Tq, 2, Tq, Tk, 2, 2, 64, dtype, sharp=0.5)
    clean = v.clone()
    v[0, Tk // 3, 0, 5], v[1, 0, 1, 63] = math.inf, float("nan")
    out = binding.differential_attention(q, k, v, vectors, 0.3, norm=False)
    assert not torch.isfinite(out[0, :, 0, 5]).any() and not torch.isfinite(out[1, :, 1, 63]).any()
    fine = torch.ones(2, Tq, 2, 64, dtype=torch.bool, device=cuda_device)
    fine[0, :, 0, 5] = fine[1, :, 1, 63] = False
    want, bound = ref.difference(q, k, clean, vectors, 0.3, 32 ** -0.5, norm=False, once=_once(Tq, dtype, None), dtype=dtype)
    check(out[fine], want[fine], bound[fine], "the others")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Tq", [5, 200, 3001])
def test_sharp_and_large_scores(cuda_device, dtype, Tq):
    """Maxima that keep moving, in one map only, and scores far from 0."""
    q, k, v, vectors, w = _case(cuda_device, 2, 1, Tq, 600, 2, 2, 64, dtype, sharp=6.0)
    k = (k.float() * torch.linspace(0.05, 2, 600, device=cuda_device)[None, :, None, None]).to(dtype)
    q[..., 32:] = (q[..., 32:].float() * 0.01).to(dtype)
    _check(binding.differential_attention(q, k, v, vectors, 0.3, norm=False), q, k, v, vectors, 0.3, "sharp", norm=False)


def test_no_keys_and_rows_of_zeros(cuda_device):
    for dtype in TYPES:
        q, k, v, vectors, w = _case(cuda_device, 3, 2, 70, 40, 2, 2, 64, dtype)
        for eps in (0.0, 1e-5):
            assert (binding.differential_attention(q, k[:, :0], v[:, :0], vectors, 0.3, eps=eps) == 0).all()
            assert (binding.differential_attention(q, k, torch.zeros_like(v), vectors, 0.3, eps=eps) == 0).all()
        assert binding.differential_attention(q[:, :0], k, v, vectors, 0.3).shape == (2, 0, 2, 64)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Tq,Tk", [(1, 300), (7, 9000), (260, 700), (1100, 2000)])
def test_streams_and_graphs_give_the_same_bits(cuda_device, dtype, Tq, Tk):
    q, k, v, vectors, w = _case(cuda_device, Tq, 2, Tq, Tk, 2, 2, 64, dtype)

    def call(**kw):
        return binding.differential_attention(q, k, v, vectors, 0.3, norm_weight=w, **kw)

    want = call().clone()
    assert all(torch.equal(call(), want) for _ in range(3))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = call(stream=side)
    with torch.cuda.stream(side):
        got = call()
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(other, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for _ in range(2):
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)


@pytest.mark.parametrize("Tq,Tk", [(7, 90000), (1100, 2000)])
def test_two_graphs_at_once(cuda_device, Tq, Tk):
    """Captured apart, replayed side by side on two streams: each has scratch of its own."""
    cases = [_case(cuda_device, s, 1, Tq, Tk, 4, 4, 64, BF16) for s in (5, 6)]
    want = [binding.differential_attention(*c[:4], 0.3) for c in cases]
    graphs, outs = [], []
    for c in cases:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(binding.differential_attention(*c[:4], 0.3))
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(20):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])


def test_shared_and_far_inputs(cuda_device):
    for Tq, Tk in ((3, 200), (300, 200), (1000, 1500)):
        q, k, v, vectors, _ = _case(cuda_device, 3, 3, Tq, Tk, 2, 2, 64, BF16)
        for a, b in ((k[:1].expand(3, -1, -1, -1), v[:1].expand(3, -1, -1, -1)), (k[:, :, :1].expand(-1, -1, 2, -1), v[:, :, :1].expand(-1, -1, 2, -1))):
            assert torch.equal(binding.differential_attention(q, a, b, vectors, 0.3), binding.differential_attention(q, a.contiguous(), b.contiguous(), vectors, 0.3))
    far = 2 ** 32 + 64
    room = torch.empty(far + 64 * 4000, dtype=BF16, device=cuda_device)
    for B, T, strides in ((2, 4000, (far, 64, 64)), (1, 2, (64, far, 64))):
        x = room.as_strided((B, T, 1, 64), strides + (1,))
        q, near, _, vectors, _ = _case(cuda_device, 5, B, 2000, T, 1, 1, 64, BF16)
        x.copy_(near)
        for n in (3, 2000):
            assert torch.equal(binding.differential_attention(q[:, :n], x, x, vectors, 0.3), binding.differential_attention(q[:, :n], near, near, vectors, 0.3))


def test_refusals_of_tensors(cuda_device):
    q = torch.zeros(2, 4, 2, 64, dtype=BF16, device=cuda_device)
    a, n = torch.zeros(4, 32, device=cuda_device), torch.zeros(2, dtype=torch.int32, device=cuda_device)
    mask = torch.ones(2, 4, 4, dtype=torch.uint8, device=cuda_device)
    f = binding.differential_attention
    for bad in (lambda: f(q.half(), q.half(), q.half(), a, 0.3), lambda: f(q, q.float(), q.float(), a, 0.3), lambda: f(q, q, q[:, :3], a, 0.3), lambda: f(q, q[:1], q[:1], a, 0.3),
                lambda: f(q, q, q, None, 0.3), lambda: f(q, q, q, a[:, :16], 0.3), lambda: f(q, q, q, a.double(), 0.3), lambda: f(q, q, q, a[None], 0.3), lambda: f(q, q, q, a.cpu(), 0.3),
                lambda: f(q, q, q, a.T.contiguous().T, 0.3), lambda: f(q, q, q, a, math.nan), lambda: f(q, q, q, a, 0.3, norm_weight=a[0]), lambda: f(q, q, q, a, 0.3, eps=-1.0),
                lambda: f(q, q, q, a, 0.3, scale=0.0), lambda: f(q, q, q, a, 0.3, kv_lengths=n.long()), lambda: f(q, q, q, a, 0.3, mask=mask[:, :3]),
                lambda: f(q, q, q, a, 0.3, mask=mask.int()), lambda: f(q, q, q, a, 0.3, out=q[:1].expand(2, -1, -1, -1)), lambda: f(q[..., ::2], q[..., ::2], q[..., ::2], a, 0.3)):
        with pytest.raises(binding.TTError):
            bad()
    torch.cuda.synchronize()


def test_results_carry_no_gradient(cuda_device):
    x = torch.randn(1, 40, 2, 64, device=cuda_device, requires_grad=True)
    a = torch.zeros(4, 32, device=cuda_device, requires_grad=True)
    for y in (binding.differential_attention(x, x, x, a, 0.3), binding.differential_attention(x[:, :1], x, x, a, 0.3)):
        assert not y.requires_grad and torch.isfinite(y).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_tensors_let_go_before_another_stream_has_read_them(cuda_device, dtype):
    q, k, v, vectors, w = _case(cuda_device, 6, 2, 600, 600, 2, 2, 64, dtype)
    call = lambda y, a, s: binding.differential_attention(q, k, y, a, 0.3, norm_weight=w, stream=s)      # noqa: E731
    want = call(v, vectors, None)
    side = torch.cuda.Stream()
    call(v, vectors, side)                                # what is set up once is there
    torch.cuda.synchronize()
    y, a = v.clone(), vectors.clone()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(40_000_000)                     # some 20 ms
    got = call(y, a, side)
    del y, a
    others = [torch.full_like(z, math.nan) for _ in range(8) for z in (v, vectors)]
    torch.cuda.synchronize()
    assert torch.equal(got, want) and len(others) == 16
