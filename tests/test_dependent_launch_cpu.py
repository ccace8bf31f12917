"""Kernels that may be resident while the kernel before them still writes (programmatic dependent launches) must not promise
the compiler that their memory stays as it is: `__restrict__` on a parameter covers the whole kernel, the part before
grid_dependency_wait() too, so loads could be moved before the wait or take the path that is not kept coherent."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_09649_b200", "csrc")


def _kernels(path):
    """(name, parameter list, body) of each __global__ function of a file."""
    text = re.sub(r"//[^\n]*", "", open(path).read())
    for m in re.finditer(r"__global__\s+void\s+(?:__launch_bounds__\((?:[^()]|\([^()]*\))*\)\s*)?(\w+)\s*\(", text):
        depth, i = 1, m.end()
        while depth:
            depth += {"(": 1, ")": -1}.get(text[i], 0)
            i += 1
        params, start = text[m.end():i - 1], text.index("{", i)
        depth, j = 1, start + 1
        while depth:
            depth += {"{": 1, "}": -1}.get(text[j], 0)
            j += 1
        yield m.group(1), params, text[start:j]


def _waiting(prefix):
    files = [f for f in sorted(os.listdir(CSRC)) if f.startswith(prefix) and f.endswith((".cu", ".cuh"))]
    return [(name, params) for f in files for name, params, body in _kernels(os.path.join(CSRC, f)) if "grid_dependency_wait()" in body]


def test_paged_kernels_promise_nothing_about_memory():
    found = _waiting("paged")
    assert {"paged_plan_kernel", "paged_append_kernel", "paged_attn_f32_kernel", "paged_join_kernel", "paged_attn_warp_kernel", "paged_attn_tc_kernel",
            "paged_select_kernel", "paged_select_mma_kernel"} <= {name for name, _ in found}
    assert [name for name, params in found if "__restrict__" in params] == []


def test_selection_kernels_promise_it_of_the_scores_alone():
    """(no kernel of the selection writes the scores, and the first is an ordinary launch behind whatever wrote them)"""
    found = _waiting("select")
    assert {"flat_bracket_kernel", "flat_refine_kernel", "flat_main_kernel", "flat_cand_kernel"} <= {name for name, _ in found}
    for name, params in found:
        assert [p.strip() for p in params.split(",") if "__restrict__" in p] in ([], ["const float* __restrict__ s"]), name
