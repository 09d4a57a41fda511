"""The gated delta rule on the host: structure and refusals (no GPU needed).  Addresses are made up; every call here is refused."""
import ctypes as C
import math
import os
import subprocess
import tempfile

import pytest
import torch

from paper_2402_04466_b200 import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 0x7F0000000000
S = binding.tt_delta_rule_args


def test_structure_matches_the_header():
    names = [n for n, _ in S._fields_]
    src = '#include "tt.h"\n#include <stddef.h>\n#include <stdio.h>\nint main(){printf("%%zu\\n", sizeof(tt_delta_rule_args));%sreturn 0;}\n' % "".join(
        f'printf("%zu\\n", offsetof(tt_delta_rule_args, {n}));' for n in names)
    with tempfile.TemporaryDirectory() as d:
        open(os.path.join(d, "s.c"), "w").write(src)
        subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), os.path.join(d, "s.c"), "-o", os.path.join(d, "s")], check=True)
        got = [int(x) for x in subprocess.run([os.path.join(d, "s")], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [C.sizeof(S)] + [getattr(S, n).offset for n in names]
    assert binding._DELTA_ARGS.size == C.sizeof(S)


def _view(at, B, T, H, D):
    return binding.tt_tokens(at, T * H * D, H * D, D)


def _delta(**over):
    B, T, H, K, D = 2, 70, 4, 2, 64
    a = S(C.sizeof(S), 1, B, T, H, K, D, 5, 0.125, 0, _view(A, B, T, K, D), _view(A + 0x10000, B, T, K, D), _view(A + 0x20000, B, T, H, D),
          _view(A + 0x30000, B, T, H, D), A, A, A, A, None, None, A, 1 << 40)
    for name, value in over.items():
        at, part = (getattr(a, name.split("__")[0]), name.split("__")[1]) if "__" in name else (a, name)
        setattr(at, part, value)
    return a


@pytest.mark.parametrize("over", [
    dict(struct_size=8), dict(precision=2), dict(batch=0), dict(batch=65536), dict(tokens=-1), dict(heads=3), dict(heads=0), dict(qk_heads=0), dict(qk_heads=8),
    dict(heads=8192, qk_heads=8192), dict(num_slots=0), dict(num_slots=1), dict(scale=math.nan), dict(scale=math.inf), dict(q__data=None), dict(q__data=A + 8),
    dict(k__data=A + 2), dict(v__data=None), dict(out__data=A + 4), dict(q__token_stride=4), dict(k__head_stride=1), dict(v__batch_stride=-64),
    dict(v__token_stride=1 << 50), dict(k__token_stride=0), dict(out__batch_stride=0), dict(out__head_stride=32), dict(beta=None), dict(beta=A + 2),
    dict(log_decay=A + 1), dict(state=None), dict(state_out=None), dict(state=A + 4), dict(state_out=A + 8), dict(slots=A + 2), dict(lengths=A + 1), dict(scratch=None),
    dict(scratch=A + 8), dict(scratch_bytes=64)])
def test_refusals(over):
    lib = binding.load_library()
    assert lib.tt_delta_rule(C.byref(_delta(**over)), None) == 1
    assert b"tt_delta_rule" in lib.tt_last_error(None)
    assert lib.tt_delta_rule(None, None) == 1


@pytest.mark.parametrize("d", [0, 16, 48, 96, 256])
def test_other_head_dims_are_unsupported(d):
    assert binding.load_library().tt_delta_rule(C.byref(_delta(head_dim=d)), None) == 2


def test_scratch_is_asked_for_only_where_windows_are_prepared_apart():
    lib = binding.load_library()
    room = lambda **over: lib.tt_delta_rule_scratch_bytes(C.byref(_delta(**over)))      # noqa: E731
    assert room() > 0 and room(tokens=64, precision=0) > 0 and room(tokens=64, batch=40, num_slots=40) > 0 and room(tokens=64, head_dim=128) > 0
    assert room(tokens=0) == room(tokens=1) == room(tokens=8) == room(tokens=64) == room(tokens=12, precision=0) == 0
    assert room(tokens=24, precision=0, batch=40, num_slots=40, head_dim=128) == 0 < room(tokens=25, precision=0, batch=40, num_slots=40, head_dim=128)
    assert room(heads=3) == 0 and lib.tt_delta_rule_scratch_bytes(None) == 0
    # a long call asks for the records of two ranges of windows, not of all
    assert room(tokens=1 << 20) <= 2 * (48 << 20) < room(tokens=1 << 20) * 1.1


def test_host_tensors_are_refused():
    x = torch.zeros(1, 2, 2, 64)
    with pytest.raises(binding.TTError, match="CUDA"):
        binding.delta_rule(x, x, x, None, torch.ones(1, 2, 2), torch.zeros(1, 2, 64, 64))
