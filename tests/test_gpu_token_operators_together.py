"""The gated delta rule and differential attention as a model uses them, behind the framework's own path."""
import pytest
import torch

import delta_reference
import difference_reference
import tt_synth
from paper_2402_04466_b200 import binding
from test_gpu_delta_rule import _check as _delta_check
from test_gpu_differential_attention import _check as _difference_check

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def test_frames_of_a_token_model(cuda_device):
    """Each stream's frame goes through the tick.  Per tool a query is normed and turned by the frame's number, corrects the stream's cell in its slot, reads it, and reads
    the stream's map with two maps' difference where the tool's mask is set; then the places of the map go through a cell of their own, one behind the other.  Two
    frames, each step held against its definition in 64 bits."""
    wl = tt_synth.workload("cfg1-gain").with_(name="tokens", src_w=214, src_h=120, net_w=160, net_h=120, hidden=128)
    K, T, H, D = 3, wl.n_tools, 2, 64
    ctx = binding.Context(binding.make_config(wl, max_streams=K), tt_synth.make_weights(wl))
    states = [ctx.state_create() for _ in range(K)]
    g = torch.Generator(device=cuda_device).manual_seed(21)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=cuda_device)

    first = normal(K, T, H, D).to(BF16)
    unit = torch.full((D,), D ** -0.5 * (1 - 2.0 ** -7), device=cuda_device)      # keys of length 1, and not above it however they are rounded
    to_kv = (0.09 * normal(wl.hidden, 2 * H * D)).to(BF16)
    vectors, w = 0.3 * normal(4, D // 2), 1 + 0.2 * normal(D)
    decay, beta = -0.1 * torch.rand(K, T, H, generator=g, device=cuda_device), torch.rand(K, T, H, generator=g, device=cuda_device)
    cell, places = torch.zeros(K, H, D, D, device=cuda_device), torch.zeros(K, H, D, D, device=cuda_device)
    inv = torch.from_numpy(binding.rope_frequencies(32)[0]).to(cuda_device)
    slots = torch.tensor([2, 0, 1], dtype=torch.int32, device=cuda_device)
    hm, wm = ctx.hm, ctx.wm
    for frame in range(2):
        fr = [tt_synth.make_frame(wl.frame_kind, wl.stream_seed(s), frame, wl.src_w, wl.src_h) for s in range(K)]
        ctx.submit_frames([torch.from_numpy(f).to(cuda_device) for f in fr], states, frame_index=frame)
        res = ctx.sync()
        maps = torch.stack([torch.from_numpy(ctx.state_export(s)[0]).reshape(wl.hidden, hm * wm).T for s in states]).to(cuda_device).to(BF16)
        masks = torch.stack([torch.from_numpy(ctx.fetch_masks(r)).reshape(T, hm * wm) for r in res]).to(cuda_device)
        pos = torch.full((K, T), 1000 + frame, dtype=torch.int64, device=cuda_device)
        q, k = binding.qk_norm_rope(first, first, pos, inv, unit, unit)
        before = cell.clone()
        r, cell = binding.delta_rule(q, k, first, decay, beta, cell, slots=slots)
        _delta_check(r, cell[slots.long()], q, k, first, decay, beta, before[slots.long()], 1.0, None, "cell")
        kv = (maps @ to_kv).view(K, hm * wm, 2 * H, D)
        out = binding.differential_attention(r, kv[:, :, :H], kv[:, :, H:], vectors, 0.3, norm_weight=w, mask=masks)
        _difference_check(out, r, kv[:, :, :H], kv[:, :, H:], vectors, 0.3, "reading the map", mask=masks, weight=w, out_scale=0.7)
        assert (out[masks.sum(-1) == 0] == 0).all() and out.abs().sum() > 0
        q, k = binding.qk_norm_rope(kv[:, :, :H], kv[:, :, :H], None, None, unit, unit)
        gates = torch.sigmoid(kv[..., 0].float())
        fade, gain = (-0.05 * gates[:, :, :H]).contiguous(), gates[:, :, H:].contiguous()
        before = places.clone()
        r, _ = binding.delta_rule(q, k, kv[:, :, H:], fade, gain, places)
        _delta_check(r, places, q, k, kv[:, :, H:], fade, gain, before, 1.0, None, "places")
    ctx.destroy()
