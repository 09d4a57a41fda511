"""Rules of the gated delta rule's device code that no run on a healthy device can show broken (no GPU needed)."""
import os
import re

import pytest

TOKENS = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2402_04466_b200", "csrc", "tokens")
NAMES = ["delta_step.cu", "delta_prepare.cu", "delta_chunk.cu"]


def _body(name):
    code = re.sub(r"/\*.*?\*/|//[^\n]*", "", open(os.path.join(TOKENS, name)).read(), flags=re.S)
    assert code.count("__global__") == 1
    at = code.index("{", code.index("__global__"))
    depth, end = 0, at
    for end in range(at, len(code)):
        depth += {"{": 1, "}": -1}.get(code[end], 0)
        if depth == 0:
            break
    return code[at:end]


@pytest.mark.parametrize("name", NAMES)
def test_nothing_of_an_entry_is_read_before_its_slot_is_known_to_be_its_own(name):
    """An entry that is passed over shares its slot with an earlier one, which may be writing it."""
    body = _body(name)
    slot = body.index("slot_of(")
    gone = slot + re.search(r"\breturn;", body[slot:]).start()
    reads = [m.start() for m in re.finditer(r"p\.(?:state|log_decay|beta)\b|\*reinterpret_cast<const float4|\.fetch\(|\bfetch\(", body)]
    # where the state goes may be asked before
    reads = [r for r in reads if not re.match(r"p\.state\)\)", body[r:])]
    assert reads and min(reads) > gone


def test_records_are_read_behind_the_preparation():
    """The chain's grid is launched ahead of the preparation's end: every way through it waits, and the warps that read records do so behind it."""
    body = _body("delta_chunk.cu")
    before = body[:body.index("return;")]
    assert "pdl_wait();" in before
    loads, rest = body[body.index("left ="):].split("pdl_wait();", 1)
    assert "copy16(" not in loads and "copy16(" in rest and body.count("p.records") == 1
    # the next range's preparation, which writes the other records, begins when this one's is through, and ends behind this chain
    assert body.count("pdl_launch_dependents();") == 1 and body.index("pdl_launch_dependents();") > body.index("left =") + len(loads)
    assert re.search(r"if \(p\.first_window > 0\) pdl_wait\(\);", body[:body.index("= p.state[")])      # and the states of the range before
    prepare = _body("delta_prepare.cu")
    assert prepare.count("if (holds) pdl_wait();") == 2 and prepare.rstrip().endswith("if (holds) pdl_wait();")
    assert re.search(r"holds = p\.first_window > 0 && \(blockIdx\.x \| blockIdx\.y \| blockIdx\.z\) == 0", prepare)
