"""The operators over tokens on the host: structures, refusals, frequencies, scratch (no GPU needed).

Addresses are made up; every call here is refused or needs nothing launched."""
import ctypes as C
import math
import os
import subprocess
import tempfile

import numpy as np
import pytest
import torch

from paper_2402_04466_b200 import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 0x7F0000000000
STRUCTS = (binding.tt_tokens, binding.tt_qk_norm_rope_args, binding.tt_linear_attention_args, binding.tt_cross_attention_args)


def test_structures_match_the_header():
    fields = [(s.__name__, n) for s in STRUCTS for n, _ in s._fields_]
    src = '#include "tt.h"\n#include <stddef.h>\n#include <stdio.h>\nint main(){%s%sreturn 0;}\n' % (
        "".join(f'printf("%zu\\n", sizeof({s.__name__}));' for s in STRUCTS),
        "".join(f'printf("%zu\\n", offsetof({s}, {n}));' for s, n in fields))
    with tempfile.TemporaryDirectory() as d:
        open(os.path.join(d, "s.c"), "w").write(src)
        subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), os.path.join(d, "s.c"), "-o", os.path.join(d, "s")], check=True)
        got = [int(x) for x in subprocess.run([os.path.join(d, "s")], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [C.sizeof(s) for s in STRUCTS] + [getattr(next(s for s in STRUCTS if s.__name__ == n), f).offset for n, f in fields]
    for packed, s in ((binding._ROPE_ARGS, STRUCTS[1]), (binding._LINEAR_ARGS, STRUCTS[2]), (binding._CROSS_ARGS, STRUCTS[3])):
        assert packed.size == C.sizeof(s)


def _view(at, B, T, H, D):
    return binding.tt_tokens(at, T * H * D, H * D, D)


def _rope(**over):
    B, T, H, K, D = 2, 3, 4, 2, 64
    a = binding.tt_qk_norm_rope_args(C.sizeof(binding.tt_qk_norm_rope_args), 1, B, T, H, K, D, D, 0, 1, 1e-6, 1.0, _view(A, B, T, H, D),
                                     _view(A + 0x10000, B, T, K, D), _view(A + 0x20000, B, T, H, D), _view(A + 0x30000, B, T, K, D),
                                     A, A, A, T, A, None)
    return _set(a, over)


def _linear(**over):
    B, T, H, K, D = 2, 3, 4, 2, 64
    a = binding.tt_linear_attention_args(C.sizeof(binding.tt_linear_attention_args), 1, B, T, H, K, D, 5, 0.125, 0, _view(A, B, T, H, D),
                                         _view(A + 0x10000, B, T, K, D), _view(A + 0x20000, B, T, K, D), _view(A + 0x30000, B, T, H, D),
                                         A, A, A, None, None, None, None, 0)
    return _set(a, over)


def _cross(**over):
    B, Q, T, H, K, D = 2, 3, 5, 4, 2, 64
    a = binding.tt_cross_attention_args(C.sizeof(binding.tt_cross_attention_args), 1, B, Q, T, H, K, D, 0.125, 0, _view(A, B, Q, H, D),
                                        _view(A + 0x10000, B, T, K, D), _view(A + 0x20000, B, T, K, D), _view(A + 0x30000, B, Q, H, D),
                                        None, None, None, 0, 0, None, None, 0)
    return _set(a, over)


def _set(a, over):
    for name, value in over.items():
        at, part = (getattr(a, name.split("__")[0]), name.split("__")[1]) if "__" in name else (a, name)
        setattr(at, part, value)
    return a


CALLS = {"tt_qk_norm_rope": _rope, "tt_linear_attention": _linear, "tt_cross_attention": _cross}
ANY = [dict(struct_size=8), dict(precision=2), dict(batch=0), dict(batch=65536), dict(q__data=None), dict(q__data=A + 8), dict(k__data=A + 2),
       dict(q__token_stride=4), dict(k__head_stride=1), dict(q__batch_stride=-64), dict(k__token_stride=1 << 50)]


@pytest.mark.parametrize("call", sorted(CALLS))
@pytest.mark.parametrize("over", ANY)
def test_refusals_common_to_all(call, over):
    lib = binding.load_library()
    assert getattr(lib, call)(C.byref(CALLS[call](**over)), None) == 1
    assert call.encode() in lib.tt_last_error(None)
    assert getattr(lib, call)(None, None) == 1


@pytest.mark.parametrize("call", sorted(CALLS))
@pytest.mark.parametrize("d", [0, 16, 48, 96, 256])
def test_other_head_dims_are_unsupported(call, d):
    lib = binding.load_library()
    assert getattr(lib, call)(C.byref(CALLS[call](head_dim=d)), None) == 2


@pytest.mark.parametrize("call,over", [
    ("tt_qk_norm_rope", o) for o in (dict(rot_dim=4), dict(rot_dim=72), dict(rot_dim=-8), dict(positions=None), dict(inv_freq=None),
                                     dict(positions=A + 4), dict(inv_freq=A + 4), dict(q_weight=A + 2), dict(eps=-1.0), dict(eps=math.nan),
                                     dict(rot_scale=math.inf), dict(q_heads=0, k_heads=0), dict(q_heads=-1), dict(tokens=-1),
                                     dict(q_out__data=None), dict(q_out__head_stride=0), dict(k_out__token_stride=64), dict(position_stride=-1))] + [
    ("tt_linear_attention", o) for o in (dict(heads=3), dict(kv_heads=0), dict(num_slots=0), dict(num_slots=1), dict(log_decay=None),
                                         dict(state=None), dict(state_out=None), dict(state=A + 4), dict(state_out=A + 8), dict(slots=A + 2),
                                         dict(lengths=A + 1), dict(scale=math.nan), dict(tokens=-1), dict(out__data=None),
                                         dict(out__batch_stride=0), dict(tokens=5000), dict(tokens=5000, scratch=A, scratch_bytes=64),
                                         dict(tokens=5000, scratch=A + 8, scratch_bytes=1 << 40), dict(status_dev=A + 2))] + [
    ("tt_cross_attention", o) for o in (dict(heads=3), dict(kv_heads=8), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf),
                                        dict(scale=math.nan), dict(q_tokens=-1), dict(kv_tokens=-1), dict(v__data=None), dict(out__data=A + 4),
                                        dict(mask=A, mask_batch_stride=-1), dict(mask=A, mask_query_stride=1 << 50), dict(q_lengths=A + 1),
                                        dict(kv_lengths=A + 2), dict(out__token_stride=0), dict(kv_tokens=40000),
                                        dict(kv_tokens=40000, scratch=A + 4, scratch_bytes=1 << 40), dict(kv_tokens=40000, scratch=A, scratch_bytes=8))])
def test_refusals(call, over):
    lib = binding.load_library()
    assert getattr(lib, call)(C.byref(CALLS[call](**over)), None) == 1
    assert call.encode() in lib.tt_last_error(None)


def test_a_call_without_rows_launches_nothing():
    lib = binding.load_library()
    assert lib.tt_qk_norm_rope(C.byref(_rope(tokens=0, q__data=None, positions=None)), None) == 0
    assert lib.tt_cross_attention(C.byref(_cross(q_tokens=0, q__data=None, out__data=None)), None) == 0


def test_scratch_is_asked_for_only_where_work_is_split():
    lib = binding.load_library()
    assert lib.tt_linear_attention_scratch_bytes(C.byref(_linear())) == 0
    assert lib.tt_linear_attention_scratch_bytes(C.byref(_linear(tokens=1))) == 0
    assert lib.tt_linear_attention_scratch_bytes(C.byref(_linear(tokens=14400))) > 0
    assert lib.tt_linear_attention_scratch_bytes(C.byref(_linear(tokens=14400, batch=65535, num_slots=65535))) == 0    # sequences enough
    assert lib.tt_linear_attention_scratch_bytes(C.byref(_linear(head_dim=7))) == 0
    assert lib.tt_linear_attention_scratch_bytes(None) == 0
    assert lib.tt_cross_attention_scratch_bytes(C.byref(_cross())) == 0
    assert lib.tt_cross_attention_scratch_bytes(C.byref(_cross(kv_tokens=14400))) > 0
    assert lib.tt_cross_attention_scratch_bytes(C.byref(_cross(kv_tokens=0))) == 0
    assert lib.tt_cross_attention_scratch_bytes(None) == 0


@pytest.mark.parametrize("rot", [0, 8, 64, 128])
def test_frequencies(rot):
    i = np.arange(0, rot, 2)
    plain = 10000.0 ** (-i / max(rot, 1))
    inv, gain = binding.rope_frequencies(rot)
    assert np.allclose(inv, plain, rtol=1e-14) and gain == 1
    inv, gain = binding.rope_frequencies(rot, scaling="linear", factor=4.0)
    assert np.allclose(inv, plain / 4, rtol=1e-14) and gain == 1
    inv, gain = binding.rope_frequencies(rot, base=500.0, scaling="base", factor=4.0)
    if rot:      # the fastest pair stays, the slowest is divided by the factor
        assert inv[0] == 1 and np.isclose(inv[-1], 500.0 ** (-(rot - 2) / rot) / 4, rtol=1e-13)
        assert np.allclose(np.diff(np.log(inv)), np.log(inv[1]), rtol=1e-12)
    inv, gain = binding.rope_frequencies(rot, scaling="by_parts", factor=4.0, trained=4096, slow_turns=1, fast_turns=32)
    turns = 4096 * plain / (2 * math.pi)
    assert np.allclose(inv[turns >= 32], plain[turns >= 32], rtol=1e-14) and np.allclose(inv[turns <= 1], plain[turns <= 1] / 4, rtol=1e-14)
    between = (turns > 1) & (turns < 32)
    keep = (turns[between] - 1) / 31
    assert np.allclose(inv[between], plain[between] * (keep + (1 - keep) / 4), rtol=1e-13)
    assert np.isclose(gain, 0.1 * math.log(4) + 1, rtol=1e-7)


@pytest.mark.parametrize("kw", [dict(rot_dim=7), dict(rot_dim=-2), dict(rot_dim=130), dict(rot_dim=8, base=1.0), dict(rot_dim=8, base=math.nan),
                                dict(rot_dim=8, scaling="linear", factor=0.5), dict(rot_dim=2, scaling="base", factor=2.0),
                                dict(rot_dim=8, scaling="by_parts", factor=2.0), dict(rot_dim=8, scaling="other"),
                                dict(rot_dim=8, scaling="by_parts", factor=2.0, trained=10, slow_turns=4, fast_turns=4)])
def test_frequencies_refused(kw):
    with pytest.raises(binding.TTError):
        binding.rope_frequencies(**{"rot_dim": 8, **kw})


def test_host_tensors_are_refused():
    x = torch.zeros(1, 2, 2, 64)
    with pytest.raises(binding.TTError, match="CUDA"):
        binding.qk_norm_rope(x, x)
    with pytest.raises(binding.TTError, match="CUDA"):
        binding.linear_attention(x, x, x, torch.zeros(2), torch.zeros(1, 2, 64, 64))
    with pytest.raises(binding.TTError, match="CUDA"):
        binding.cross_attention(x, x, x)
    with pytest.raises(binding.TTError):
        binding.qk_norm_rope(None, None)


@pytest.mark.parametrize("call,later,text", [("tt_qk_norm_rope", dict(positions=None), b"positions"), ("tt_linear_attention", dict(log_decay=None), b"log_decay"),
                                             ("tt_cross_attention", dict(mask=A, mask_batch_stride=-1), b"mask stride")])
@pytest.mark.parametrize("view", ["q", "k", "out"])
@pytest.mark.parametrize("axis,extents", [("batch", ("batch",)), ("token", ("tokens", "q_tokens", "kv_tokens")), ("head", ("heads", "kv_heads", "q_heads", "k_heads"))])
@pytest.mark.parametrize("stride", [3, 0, -64, 1 << 60])
def test_strides_of_axes_of_extent_one_are_not_looked_at(call, later, text, view, axis, extents, stride):
    """What is refused is the argument that is checked behind the views (nothing is launched), as with strides that would do for any extent."""
    lib = binding.load_library()
    over = {n: 1 for n in extents if n in dict(CALLS[call]()._fields_)}
    names = [n for n, _ in CALLS[call]()._fields_ if n in ((view,) if view != "out" else ("out", "q_out", "k_out"))]
    assert getattr(lib, call)(C.byref(CALLS[call](**over, **later, **{f"{n}__{axis}_stride": stride for n in names})), None) == 1
    assert text in lib.tt_last_error(None)
