"""The rule for kernels that are launched before the one in front of them has ended (tc_ptx.cuh): a kernel that waits for the one
in front lets the next one in behind that wait, not before it, so that the next may rely on everything that came before."""
import glob
import os
import re

import pytest

from paper_2410_01623_b200 import build as fbuild

SOURCES = sorted(glob.glob(os.path.join(fbuild.CSRC, "*.cu*")))


def kernels(text):
    for part in re.split(r"^(?=__global__)", text, flags=re.M)[1:]:
        body = part[:part.index("\n}\n")] if "\n}\n" in part else part
        yield re.search(r"\b(k_\w+)\s*\(", part).group(1), body


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_the_next_kernel_is_let_in_behind_the_wait(path):
    with open(path) as f:
        text = f.read()
    for name, body in kernels(text):
        waits, lets_in = body.find("ptx::grid_wait();"), body.find("ptx::grid_launch_next();")
        assert waits < 0 or lets_in < 0 or waits < lets_in, name


def test_the_kernels_are_found():
    found = {name: body for path in SOURCES for name, body in kernels(open(path).read())}
    assert {"k_token_gather", "k_part_step", "k_grad_scale", "k_finalize"} <= set(found)
    assert "grid_wait" in found["k_token_gather"] and "grid_launch_next" in found["k_token_gather"]
