"""Rules that the sources of the 8-bit products have to keep and that no output shows."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_32882_b200", "csrc")

# waits on barriers; barriers of a group of threads (VSA2_GROUP_SYNC) stand for themselves.  Operations on tensor memory, those in functions of the products' own among them
TOKEN = re.compile(r"(?P<wait>\bVSA2_WAIT\w*\s*\(|\bmbar_wait\w*\s*\(|\bwait_pair\s*<)|(?P<fence>\btc_fence_after\s*\()"
                   r"|(?P<op>\btc::tmem_(?:ld|st)_?\d\w*\s*\(|\b(?:mma_int8|mma_scaled|copy_scales)\s*<|\b(?:load_columns|take_tile)\s*\()")


def lines_of(name):
    with open(os.path.join(CSRC, name)) as f:
        return [re.sub(r"//.*", "", line) for line in f]


def unfenced(lines):
    """(Lines of operations that follow a wait without a fence, in the order of the source; number of operations)."""
    pending, bad, operations = False, [], 0
    for number, line in enumerate(lines, 1):
        for m in TOKEN.finditer(line):
            if m.group("wait"):
                pending = True
            elif m.group("fence"):
                pending = False
            else:
                operations += 1
                if pending:
                    bad.append(number)
    return bad, operations


@pytest.mark.parametrize("name,least", [("fp8_matmul.cu", 9), ("int8_matmul.cu", 5)])
def test_tensor_memory_is_touched_behind_a_fence_after_every_wait(name, least):
    """Behind a wait for tcgen05 work of other threads the next tcgen05 operation needs tcgen05.fence::after_thread_sync between the two: without it the operation may run ahead."""
    bad, operations = unfenced(lines_of(name))
    assert bad == [] and operations >= least


@pytest.mark.parametrize("name", ["fp8_matmul.cu", "int8_matmul.cu"])
def test_the_rule_sees_a_fence_that_is_missing(name):
    """Each fence behind a wait of the kernels taken out of the text by itself."""
    lines = lines_of(name)
    fences = [i for i, line in enumerate(lines) if "tc_fence_after" in line and "VSA2_WAIT" in lines[i - 1]]
    assert len(fences) >= 3
    for i in fences:
        assert unfenced(lines[:i] + [""] + lines[i + 1:])[0], i + 1


@pytest.mark.parametrize("name", ["fp8_matmul.cu", "int8_matmul.cu"])
def test_accumulators_are_released_behind_a_fence(name):
    """What was read of tensor memory is told to the products' warp behind tcgen05.fence::before_thread_sync."""
    text = "".join(lines_of(name))
    released = [m.start() for m in re.finditer(r"mbar_arrive\(&misc->d_empty", text)]
    assert released
    for at in released:
        assert "tc_fence_before" in text[max(0, at - 200):at]
