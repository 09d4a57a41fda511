"""What the plan of cross and differential attention takes for granted of their kernels (no GPU needed)."""
import ctypes as C
import os
import re

import pytest

from paper_2402_04466_b200 import binding

TOKENS = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2402_04466_b200", "csrc", "tokens")
SIZES = {"uint64_t": 8, "float2": 8, "float": 4}


def _shared_bytes(D, warps, maps):
    """-> (static, dynamic) bytes of a block, from the declarations."""
    code = re.sub(r"/\*.*?\*/|//[^\n]*", "", open(os.path.join(TOKENS, "cross_few.cu")).read(), flags=re.S)
    few = dict(D=D, W=warps, M=maps)
    for name, value in re.findall(r"static constexpr int (\w+) = ([^;]+);", code[code.index("struct Few"):code.index("run_at")]):
        value = re.sub(r"(.+?) \? (.+?) : (.+)", r"(\2) if (\1) else (\3)", value).replace("/", "//")
        few[name] = eval(value, {}, few)
    static = 0
    for kind, dims in re.findall(r"(?<!extern )__shared__ (?:__align__\(\d+\) )?(\w+) \w+((?:\[[^\]]+\])+);", code):
        n = SIZES[kind]
        for d in re.findall(r"\[([^\]]+)\]", dims):
            n *= eval(d.replace("F::", ""), {}, few | dict(MAPS=maps))
        static += n
    return static, few["SMEM"]


@pytest.mark.parametrize("maps", [1, 2])
@pytest.mark.parametrize("D", [32, 64, 128])
def test_as_many_blocks_fit_a_multiprocessor_as_the_plan_counts_on(D, maps):
    """cross_plan makes up to two blocks of four warps to a multiprocessor, or one of eight.  A multiprocessor has 228 KB, of which each block takes 1 KB more than it asks for."""
    for warps, blocks in ((4, 2), (8, 1)):
        static, dynamic = _shared_bytes(D, warps, maps)
        assert static >= warps * 3 * 8 + maps * 17 * 8 * warps // 2 and dynamic >= warps * 24576      # the declarations were read
        assert blocks * (static + dynamic + 1024) <= 228 * 1024, (static, dynamic)


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("B,Tq,Tk,H", [(1, 1023, 4096, 2), (1, 300, 4096, 2), (5, 7, 4800, 2), (2, 100, 2000, 4), (1, 1, 100000, 1)])
def test_fp32_keys_of_two_maps_are_split_over_the_blocks_that_fit(B, Tq, Tk, H, D):
    """One block to a multiprocessor, or two of 64 rows with heads of 32; the number of splits is what the scratch has room for."""
    view = lambda T: binding.tt_tokens(0x7F0000000000, T * H * D, H * D, D)      # noqa: E731
    args = binding.tt_differential_attention_args(C.sizeof(binding.tt_differential_attention_args), 0, B, Tq, Tk, H, H, D, 0.125, 0.3, 1e-5, 0.7, 1, 0, view(Tq), view(Tk), view(Tk),
                                                  view(Tq), 0x7F0000000000, 0, None, None, None, None, 0, 0, None, None, 0)
    room = binding.load_library().tt_differential_attention_scratch_bytes(C.byref(args))
    splits, rest = divmod(room, Tq * 2 * B * H * (D + 2) * 4)
    rows = 16 if Tq <= 16 else 64
    assert rest == 0 and splits > 1 and -(-Tq // rows) * B * H * splits <= 148 * (2 if D == 32 and rows == 64 else 1)
