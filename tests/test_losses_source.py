"""What the kernels of the losses on rows must hold and no run can show: read
from their sources, without a GPU."""

import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_20739_gb300", "csrc")


def functions(name):
    """{function: body} of a source file, comments left out."""
    with open(os.path.join(CSRC, name)) as f:
        text = re.sub(r"//[^\n]*|__launch_bounds__\([^()]*\)", "", f.read())
    out = {}
    for m in re.finditer(r"\b(\w+)\([^;{}]*\)\s*\{\n", text):
        depth, at = 1, m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(text[at], 0)
            at += 1
        out[m.group(1)] = text[m.end():at]
    return out


def test_clusters_have_started_before_they_are_written():
    """A store to another CTA's shared memory needs that CTA to run: behind
    the barrier that every CTA of the cluster reaches at its start."""
    body = functions("row_losses.cu")
    exchanges = [f for f in body if "st.shared::cluster" in body[f]]
    assert sorted(exchanges) == ["gather", "merge"]
    callers = [f for f in body if re.search(r"\b(gather|merge)<", body[f])]
    assert sorted(callers) == ["policy_held_kernel", "policy_long_kernel", "row_stats"]
    for f in callers:
        say, wait = body[f].index("cluster_say_started("), body[f].index("cluster_wait_started(")
        assert say < wait < re.search(r"\b(gather|merge)<", body[f]).start(), f


def test_indexes_of_elements_do_not_overflow():
    """A row may have 2^31 - 1 classes, so an index that steps through its single
    elements by the threads of a group passes 2^31 before the loop's test."""
    loops = []
    for name in ("row_losses.cu", "row_slice.cuh"):
        for f, body in functions(name).items():
            loops += [(f, t) for t, bound in re.findall(r"for \((\w+) \w+ = [^;]*tid; \w+ < ([^;]*); \w+ \+= (?:G|threads)\)", body)
                      if "last" in bound]
    assert {f for f, _ in loops} == {"row_stats", "policy_long_kernel", "slice_grad_extreme"}
    step = 1024
    for f, kind in loops:
        last = (1 << 31) - 1
        beyond = last - 1 + step                    # the last element's thread, one step on
        wrapped = {"int": (beyond + (1 << 31)) % (1 << 32) - (1 << 31), "unsigned": beyond % (1 << 32), "int64_t": beyond}[kind]
        assert wrapped >= last, f
