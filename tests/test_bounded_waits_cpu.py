"""Waits with a limit, by reading the sources (a wait that runs out in earnest has no place in a test): where a whole warp goes on together --
shuffles, votes and products of the warp follow -- its lanes must agree on whether the wait ran out, or those that go on wait for those
that left."""
import os
import re

import pytest

from test_dependent_launch_cpu import CSRC

WAIT = re.compile(r"\b(?:mbar_wait_bounded|mbar_try_wait|a_bar_wait)\(")


def without_comments(text):
    return re.sub(r"/\*.*?\*/", "", re.sub(r"//[^\n]*", "", text), flags=re.S)


def unvoted(text):
    """Waits whose answer is used without the warp's vote.  (A wait that is a statement of its own waits for copies in flight.)"""
    found = []
    for m in WAIT.finditer(text):
        before = text[:m.start()].rstrip()
        if not before.endswith("__all_sync(0xffffffffu,") and before[-1] not in ";{})":
            found.append(text[m.start() - 30:m.end() + 30])
    return found


def test_the_reader_tells_the_cases_apart():
    text = without_comments("""{ ok = __all_sync(0xffffffffu, a_bar_wait(b, p)); /* ok = a_bar_wait(b, p); */ if (c) ok = mbar_wait_bounded(b, p); // a_bar_wait(
                               if (!a_bar_wait(b, 0)) return; for (k = 0; k < n; ++k) mbar_wait_bounded(b + k, k & 1u); }""")
    assert len(unvoted(text)) == 2


@pytest.mark.parametrize("name", ["paged4_attention.cu", "paged4_attention_tc.cu", "paged_tc.cuh"])
def test_waits_of_the_4_bit_kernels_are_voted_on(name):
    text = without_comments(open(os.path.join(CSRC, name)).read())
    assert WAIT.search(text)
    assert unvoted(text) == []


def test_copies_of_the_4_bit_decode_kernel_land_before_their_warp_leaves():
    """The warps that bring tiles wait for the last copies of every ring, whether or not there was more to bring: a warp that gave up leaves the
    copies it asked for in flight, and shared memory goes to the next block."""
    text = without_comments(open(os.path.join(CSRC, "paged4_attention.cu")).read())
    block = text[text.index("if (warp >= S::WARPS) {"):text.index("const unsigned char* ring")]
    depth, waits = 0, []
    for i, ch in enumerate(block):
        depth += {"{": 1, "}": -1}.get(ch, 0)
        if block.startswith("mbar_wait_bounded(", i):
            waits.append((depth, block[block.rfind(";", 0, block.rfind("for (", 0, i)) + 1:i]))
    assert len(waits) == 1 and waits[0][0] == 1               # of the block itself, under no condition
    assert "if" not in waits[0][1] and "for (unsigned k" in waits[0][1]


def test_no_paged_kernel_promises_that_its_memory_stays():
    """All files of the paged caches, whatever their launch bounds look like: a kernel that is placed before the one ahead of it has finished must
    not promise the compiler that memory does not change."""
    files = [f for f in sorted(os.listdir(CSRC)) if f.startswith("paged") and f.endswith((".cu", ".cuh"))]
    assert {"paged4_attention.cu", "paged4_attention_tc.cu", "paged4_append.cu", "paged_share.cu", "paged_move.cu"} <= set(files)
    assert [f for f in files if "__restrict__" in without_comments(open(os.path.join(CSRC, f)).read())] == []
