"""Clipping into the tensors of the list itself, in another order: each would be read after it is written, or not."""
import ctypes as C

import pytest

from paper_2410_01623_b200 import binding as fb
from paper_2410_01623_b200 import build as fbuild

INVALID, SMALL = 1, 2
A, B, X, Y = (k << 20 for k in range(1, 5))            # made-up addresses: every case is refused before one is used


@pytest.mark.parametrize("G,out,status", [
    ([A, B], [B, A], INVALID), ([A, B], [X, A], INVALID), ([A, B], [B, X], INVALID), ([A, B, X], [B, X, A], INVALID),
    ([A, B], [A, B], SMALL), ([A, B], [X, Y], SMALL), ([A, X], [B, Y], SMALL), ([A, B], [A, X], SMALL), ([X, A], [Y, B], SMALL)])
def test_outputs_over_other_inputs(G, out, status):
    fbuild.build()
    lib = fb.lib()
    n = len(G)
    descs = (fb.GradDesc * n)(*[fb.GradDesc(1, 8, 0, 0, 0, 0)] * n)
    arrays = [(C.c_void_p * n)(*p) for p in (G, out)]
    assert lib.fira_clip_grads(n, descs, *arrays, 1.0, 4096, 4096, 4096, 8, None) == status
    if status == INVALID:
        assert b"output of another" in lib.fira_last_error()
    empty = (fb.GradDesc * n)(*[fb.GradDesc(0, 8, 0, 0, 0, 0)] * n)
    assert lib.fira_clip_grads(n, empty, *arrays, 1.0, 4096, 4096, 4096, 8, None) == SMALL
