"""Rules of the device code of the operators over tokens that no run on a healthy device can show broken (no GPU needed)."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2402_04466_b200", "csrc")


def _code(path):
    """Source without comments."""
    return re.sub(r"/\*.*?\*/|//[^\n]*", "", open(path).read(), flags=re.S)


SOURCES = {os.path.basename(f): _code(f) for f in sorted(glob.glob(os.path.join(CSRC, "tokens", "*.cu*")))}
WAITING = {"cross_tc.cu": "WAIT_CROSS_TC", "linear_tc.cu": "WAIT_LINEAR_TC", "cross_few.cu": "WAIT_CROSS_FEW"}


def test_every_kernel_that_waits_is_looked_at():
    assert {n for n, c in SOURCES.items() if "mbar_wait" in c} == set(WAITING)
    assert {n for n, c in SOURCES.items() if "tcgen05.alloc" in c} == {"cross_tc.cu", "linear_tc.cu"}
    assert [n for n, c in SOURCES.items() if "__activemask" in c or "__trap" in c or re.search(r"\bassert\(", c)] == []
    assert [n for n, c in SOURCES.items() if "multicast" in c or "atomicAdd" in c] == []      # sums are taken in a fixed order


@pytest.mark.parametrize("name", WAITING)
def test_waits_are_bounded_and_report_a_code_of_their_own(name):
    code = SOURCES[name]
    assert "try_wait" not in code and not re.search(r"while \(!mbar_test", code)      # single looks go on to a wait with a limit
    calls = re.findall(r"mbar_wait\w*\((?:[^()]|\([^()]*\))*\)", code)
    assert calls and all(c.endswith("WAIT_LIMIT)") for c in calls)
    # the code goes along with the wait, or is left behind it by a kernel whose warps wait each for themselves
    assert all(WAITING[name] in c for c in calls) or f"atomicCAS(p.status, 0, {WAITING[name]} + " in code
    assert "atomicCAS(p.status" in code


def test_status_codes_name_the_kernel():
    bases = {}
    for path in (os.path.join(CSRC, "tc_ptx.cuh"), os.path.join(CSRC, "tokens", "token_ptx.cuh")):
        bases.update(re.findall(r"(WAIT_[A-Z0-9_]+) = (0x[0-9A-F]+)", _code(path)))
    values = [int(v, 16) for v in bases.values()]
    assert set(WAITING.values()) <= set(bases)
    assert len({v >> 8 for v in values}) == len(values) and all(v & 0xFF == 0 for v in values)


def _without_lambdas(code):
    """Their bodies return to the kernel, not from it."""
    while True:
        m = re.search(r"\[[&=]?\]\((?:[^()]|\([^()]*\))*\)\s*\{", code)
        if not m:
            return code
        depth, end = 1, m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(code[end], 0)
            end += 1
        code = code[:m.start()] + code[end:]


@pytest.mark.parametrize("name", ["cross_tc.cu", "linear_tc.cu"])
def test_tensor_memory_is_given_back_on_every_way_out(name):
    """A block takes its columns once, all of its warps meet behind that and before they are given back, and no way out lies between."""
    code = SOURCES[name]
    assert code.count("tcgen05.alloc") == code.count("tcgen05.dealloc") == code.count("tcgen05.relinquish_alloc_permit") == 1
    between = code[code.index("tcgen05.alloc"):code.index("tcgen05.dealloc")]
    assert "__syncthreads()" in between[:between.index("tmem_slot", between.index("__syncthreads()"))]
    assert between.rindex("__syncthreads()") > between.index("abort_flag)")
    kernel = _without_lambdas(between)
    assert not re.search(r"\breturn\b", kernel)
    assert "__nanosleep" in between      # copies and products in flight land before their memory goes


def test_no_spin_without_a_limit():
    for name, code in SOURCES.items():
        assert "cuda::barrier" not in code and not re.search(r"while \(true\)|for \(;;\)|ld\.acquire|volatile.*while", code), name


def _block(code, at):
    """From the brace that opens at or behind `at` to the one that closes it."""
    start = code.index("{", at)
    depth, end = 1, start + 1
    while depth:
        depth += {"{": 1, "}": -1}.get(code[end], 0)
        end += 1
    return code[start:end]


PARTS = r"if \(lane == 0\)|if \(here\)|if \(has_row\)|if \(!has_row\)|\? __uint_as_float|\bcontinue;|\bown_\w+<|\barrive\(\w"
MEETS = r"__syncwarp\(\)|__syncthreads\(\)|__(?:all|any)_sync\(|\bwait\w*\(\w+ [+,]"


@pytest.mark.parametrize("name,loops", [("cross_tc.cu", 3), ("linear_tc.cu", 3)])
def test_lanes_meet_before_a_warp_touches_tensor_memory(name, loops):
    """Loads and stores of tensor memory are of a whole warp in step.  Going round each loop that has one, no lane-dependent step comes last
    before it: the lanes have met in between."""
    code = SOURCES[name]
    bodies = [b for b in (_block(code, m.end() - 1) for m in re.finditer(r"\bfor \([^;{}]*;[^;{}]*;[^{};]*\)\s*\{", code))
              if re.search(r"\btmem_(?:ld|st)\d", b) and re.search(PARTS, b)]
    assert len(bodies) >= loops
    for body in bodies:
        apart = None
        for e in re.finditer(f"(?P<part>{PARTS})|(?P<meet>{MEETS})|(?P<take>\\btmem_(?:ld|st)\\d\\w*\\()", body + body):
            if e.lastgroup == "part":
                apart = e.group()
            elif e.lastgroup == "meet":
                apart = None
            else:
                assert apart is None, (name, apart, (body + body)[max(0, e.start() - 400):e.end()])


@pytest.mark.parametrize("name", ["cross_tc.cu", "linear_tc.cu"])
def test_a_wait_that_ran_out_is_reported_whichever_warp_it_was(name):
    """One thread reports for its block, and its own warp may long have been through when another one's wait runs out: it looks behind the
    barrier at which all of them meet, and nothing leaves the block before."""
    code = SOURCES[name]
    assert code.count("atomicCAS(p.status") == 1 and not re.search(r"p\.status, WAIT_", code)
    tail = code[code.rindex("__syncthreads()", 0, code.index("tcgen05.dealloc")):code.index("tcgen05.dealloc")]
    assert re.search(r"if \(threadIdx\.x == 0 && \*abort_flag && p\.status\) atomicCAS\(p\.status, 0, ", tail)


@pytest.mark.parametrize("name,kernels", [("linear_step.cu", 1), ("linear_tc.cu", 1), ("linear_chunk.cu", 3)])
def test_nothing_of_an_entry_is_read_before_its_slot_is_known_to_be_its_own(name, kernels):
    """An entry that is passed over shares its slot with an earlier one, which may be writing it: the block leaves before it reads states or tokens."""
    bodies = [_block(SOURCES[name], m.end()) for m in re.finditer(r"__global__", SOURCES[name])]
    assert len(bodies) == kernels
    for body in bodies:
        slot = body.index("slot_of(")
        gone = re.search(r"slot_of\([^)]*\) < 0\) return;|if \(slot < 0\) return;", body[slot:]).start() + slot
        reads = [m.start() for m in re.finditer(r"p\.(?:state|seg_state)\b|\*reinterpret_cast<const|to_float\(|tma_load|run_chunks<|\.load\(", body)]
        assert reads and min(reads) > gone
