"""Launch order of the decoder operators' kernels (CPU, read from the sources).

A kernel that is launched while the one ahead of it may still run
(programmatic dependent launch) must not end before it: what the stream does
next waits for the last kernel alone, and may overwrite the inputs that the one
ahead still reads.  So each of these kernels waits on every path, whatever the
lengths on the device are."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2606_07317_gb300", "csrc")
# always launched dependently (the scans themselves, which are only sometimes, wait in the
# warps that read the states before them, and where a CTA has nothing to do)
DEPENDENT = [("gbla_rotate.cu", "rotate_kernel"), ("gbla_rotate.cu", "rotate_bwd_kernel"),
             ("gbla_rotate.cu", "rotate_dw_kernel"), ("gbla_decay.cu", "prefix_kernel"),
             ("gbla_decay.cu", "shared_sum_kernel"), ("gbla_decay.cu", "step_kernel"),
             ("gbla_decay_tc.cu", "before_kernel")]


def _body(path, kernel):
    """The kernel's body without comments, nested blocks cut out."""
    with open(os.path.join(CSRC, path)) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    at = re.search(r"__global__[^;{]*?\b" + kernel + r"\(", text).end()
    depth = 1
    while depth:  # the parameter list
        depth += {"(": 1, ")": -1}.get(text[at], 0)
        at += 1
    at, depth, out = text.index("{", at) + 1, 1, []
    while depth:
        c = text[at]
        depth += {"{": 1, "}": -1}.get(c, 0)
        if depth == 1 and c not in "{}":
            out.append(c)
        at += 1
    return "".join(out)


@pytest.mark.parametrize("path,kernel", DEPENDENT)
def test_every_path_waits(path, kernel):
    before, wait, _ = _body(path, kernel).partition("grid_dep_wait();")
    assert wait, "no wait outside nested blocks"
    assert "return" not in before, "a path that ends before the wait"
    assert before.strip()[-1:] in ("", ";"), "the wait is conditional"
