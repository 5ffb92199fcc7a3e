"""Lists around the number of tensors that a launch holds (480), and launches that hold empty tensors alone."""
import ctypes as C
import math

import pytest
import torch

from paper_2410_01623_b200 import binding as fb
from paper_2410_01623_b200 import build as fbuild

SMALL = 2


@pytest.mark.parametrize("count,launches", [(1, 1), (479, 1), (480, 1), (481, 2), (960, 2), (961, 3)])
def test_the_workspace_of_a_list(count, launches):
    fbuild.build()
    lib = fb.lib()
    need, one = lib.fira_grad_work_bytes(count), lib.fira_grad_work_bytes(1)
    assert need == launches * one
    descs = (fb.GradDesc * count)(*[fb.GradDesc(1, 8, 0, 0, 0, 0)] * count)
    at = (C.c_void_p * count)(*[(i + 1) << 20 for i in range(count)])       # (made up: the call is refused before one is used)
    assert lib.fira_clip_grads(count, descs, at, None, 1.0, 4096, 4096, 4096, need - 1, None) == SMALL


def sizes(count, empty):
    """empty: which tensors have no element."""
    return [0 if i in empty else 1 + (977 * i) % 9001 for i in range(count)]


@pytest.mark.gpu
@pytest.mark.parametrize("count,empty", [(479, ()), (480, ()), (481, ()), (960, ()), (961, ()), (481, range(480, 481)), (700, range(480, 700)),
                                         (700, range(480)), (1000, range(480, 960)), (961, range(961)), (49, range(48))])
@pytest.mark.parametrize("place", ["in place", "out"])
def test_lists(count, empty, place):
    gen = torch.Generator(device="cuda").manual_seed(count)
    types = [torch.float32, torch.bfloat16]
    Gs = [torch.randint(-9, 10, (n,), generator=gen, device="cuda").to(types[i % 2]) for i, n in enumerate(sizes(count, empty))]
    was = [g.clone() for g in Gs]
    # whole numbers: the sum of squares is exact
    squares = sum(float(g.double().square().sum()) for g in Gs)
    norm32 = float(torch.tensor(math.sqrt(squares), dtype=torch.float64).float())
    outs = [torch.full_like(g, 99.0) for g in Gs] if place == "out" else Gs
    norm, scale = fb.clip_grads(Gs, norm32 / 4 if norm32 else 1.0, out=None if place == "in place" else outs)
    assert float(norm) == norm32
    # norm32 is the norm rounded once, the factor the quotient rounded once: 2 roundings of 2^-24; the product and bf16's storage
    want = 0.25 if norm32 else 1.0
    assert abs(float(scale) - want) <= 2 * 2.0 ** -24 * want
    for w, o in zip(was, outs):
        ref = w.double() * want
        assert bool(((o.double() - ref).abs() <= (3 * 2.0 ** -24 + (2.0 ** -8 if o.dtype == torch.bfloat16 else 0.0)) * ref.abs()).all())
    if place == "out":
        assert all(torch.equal(g, w) for g, w in zip(Gs, was))
