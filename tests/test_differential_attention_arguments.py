"""Differential attention on the host: structure, refusals, scratch (no GPU needed).  Addresses are made up; every call here is refused or needs nothing launched."""
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
S = binding.tt_differential_attention_args


def test_structure_matches_the_header():
    names = [n for n, _ in S._fields_]
    src = '#include "tt.h"\n#include <stddef.h>\n#include <stdio.h>\nint main(){printf("%%zu\\n", sizeof(tt_differential_attention_args));%sreturn 0;}\n' % "".join(
        f'printf("%zu\\n", offsetof(tt_differential_attention_args, {n}));' for n in names)
    with tempfile.TemporaryDirectory() as d:
        open(os.path.join(d, "s.c"), "w").write(src)
        subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), os.path.join(d, "s.c"), "-o", os.path.join(d, "s")], check=True)
        got = [int(x) for x in subprocess.run([os.path.join(d, "s")], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [C.sizeof(S)] + [getattr(S, n).offset for n in names]
    assert binding._DIFF_ARGS.size == C.sizeof(S)


def _view(at, B, T, H, D):
    return binding.tt_tokens(at, T * H * D, H * D, D)


def _diff(**over):
    B, Q, T, H, K, D = 2, 3, 5, 4, 2, 64
    a = S(C.sizeof(S), 1, B, Q, T, H, K, D, 0.125, 0.3, 1e-5, 0.7, 1, 0, _view(A, B, Q, H, D), _view(A + 0x10000, B, T, K, D),
          _view(A + 0x20000, B, T, K, D), _view(A + 0x30000, B, Q, H, D), A, 0, A, None, None, None, 0, 0, None, None, 0)
    for name, value in over.items():
        at, part = (getattr(a, name.split("__")[0]), name.split("__")[1]) if "__" in name else (a, name)
        setattr(at, part, value)
    return a


@pytest.mark.parametrize("over", [
    dict(struct_size=8), dict(precision=2), dict(batch=0), dict(batch=65536), dict(heads=3), dict(kv_heads=8), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf),
    dict(scale=math.nan), dict(q_tokens=-1), dict(kv_tokens=-1), dict(lambda_init=math.nan), dict(out_scale=math.inf), dict(eps=-1.0), dict(eps=math.nan),
    dict(lambda_vectors=None), dict(lambda_vectors=A + 2), dict(lambda_head_stride=-4), dict(norm_weight=A + 1), dict(q__data=None), dict(q__data=A + 8), dict(k__data=A + 2),
    dict(v__data=None), dict(out__data=A + 4), dict(q__token_stride=4), dict(k__head_stride=1), dict(q__batch_stride=-64), dict(k__token_stride=1 << 50),
    dict(out__token_stride=0), dict(mask=A, mask_batch_stride=-1), dict(mask=A, mask_query_stride=1 << 50), dict(q_lengths=A + 1), dict(kv_lengths=A + 2),
    dict(status_dev=A + 2), dict(kv_tokens=40000), dict(kv_tokens=40000, scratch=A + 4, scratch_bytes=1 << 40), dict(kv_tokens=40000, scratch=A, scratch_bytes=8)])
def test_refusals(over):
    lib = binding.load_library()
    assert lib.tt_differential_attention(C.byref(_diff(**over)), None) == 1
    assert b"tt_differential_attention" in lib.tt_last_error(None)
    assert lib.tt_differential_attention(None, None) == 1


@pytest.mark.parametrize("d", [0, 16, 48, 96, 256])
def test_other_head_dims_are_unsupported(d):
    assert binding.load_library().tt_differential_attention(C.byref(_diff(head_dim=d)), None) == 2


def test_scratch_is_asked_for_only_where_keys_are_split():
    lib = binding.load_library()
    assert lib.tt_differential_attention_scratch_bytes(C.byref(_diff())) == 0
    assert lib.tt_differential_attention_scratch_bytes(C.byref(_diff(kv_tokens=14400))) > 0
    assert lib.tt_differential_attention_scratch_bytes(C.byref(_diff(kv_tokens=14400, precision=0))) > 0
    assert lib.tt_differential_attention_scratch_bytes(C.byref(_diff(kv_tokens=0))) == 0
    assert lib.tt_differential_attention_scratch_bytes(C.byref(_diff(kv_heads=3))) == 0
    assert lib.tt_differential_attention_scratch_bytes(None) == 0


def test_a_call_without_queries_launches_nothing():
    assert binding.load_library().tt_differential_attention(C.byref(_diff(q_tokens=0, q__data=None, out__data=None)), None) == 0


def test_host_tensors_are_refused():
    x = torch.zeros(1, 2, 2, 64)
    with pytest.raises(binding.TTError, match="CUDA"):
        binding.differential_attention(x, x, x, torch.zeros(4, 32), 0.2)
