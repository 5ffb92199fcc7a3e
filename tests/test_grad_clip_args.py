"""Refusals of fira_grad_norm and fira_clip_grads: arguments are checked before anything reaches the device."""
import ctypes as C

import pytest
import torch

from paper_2410_01623_b200 import binding as fb
from paper_2410_01623_b200 import build as fbuild

INVALID, SMALL = 1, 2


@pytest.fixture(scope="module")
def lib():
    fbuild.build()
    return fb.lib()


def call(lib, descs, G=None, out=None, max_norm=1.0, norm=4096, scale=4096, work=4096, work_bytes=1 << 20, norm_only=False):
    """The call with made-up addresses: every case here is refused before one is used."""
    n = len(descs)
    table = (fb.GradDesc * max(n, 1))(*descs)
    ptrs = (C.c_void_p * max(n, 1))(*(G if G is not None else [(i + 1) << 20 for i in range(n)]))
    outs = None if out is None else (C.c_void_p * max(n, 1))(*out)
    if norm_only:
        return lib.fira_grad_norm(n, table, ptrs, norm, work, work_bytes, None)
    return lib.fira_clip_grads(n, table, ptrs, outs, max_norm, norm, scale, work, work_bytes, None)


D = fb.GradDesc


@pytest.mark.parametrize("max_norm", [0.0, -1.0, float("nan")])
def test_max_norm_must_be_positive(lib, max_norm):
    assert call(lib, [D(1, 8, 0, 0, 0, 0)], max_norm=max_norm) == INVALID
    assert b"max_norm" in lib.fira_last_error()


@pytest.mark.parametrize("desc", [
    D(-1, 8, 0, 0, 0, 0), D(1, -8, 0, 0, 0, 0), D(2, 8, 7, 0, 0, 0), D(1, 8, 0, 0, 2, 0),
    D(1 << 41, 1, 0, 0, 0, 0), D(1, 1 << 41, 0, 0, 0, 0), D(1 << 22, 1 << 22, 0, 0, 0, 0), D(2, 1 << 31, 0, 0, 0, 0),
    D(1 << 30, 4, 1 << 20, 0, 0, 0), D(1 << 40, 1, 1 << 40, 0, 0, 0)])
@pytest.mark.parametrize("norm_only", [False, True])
def test_bad_tensors_are_refused(lib, desc, norm_only):
    assert call(lib, [D(1, 8, 0, 0, 0, 0), desc], norm_only=norm_only) == INVALID
    assert b"tensor 1" in lib.fira_last_error()


@pytest.mark.parametrize("desc", [D(2, 8, 8, 7, 0, 0), D(1, 8, 0, 0, 0, 9)])
def test_bad_outputs_are_refused(lib, desc):
    assert call(lib, [desc], out=[1 << 24]) == INVALID


def test_empty_list_and_null_pointers_are_refused(lib):
    one = [D(1, 8, 0, 0, 0, 0)]
    assert call(lib, []) == INVALID
    assert call(lib, [], norm_only=True) == INVALID
    assert call(lib, one, G=[None]) == INVALID
    assert call(lib, one, out=[None]) == INVALID
    assert call(lib, one, norm=None) == INVALID
    assert call(lib, one, scale=None) == INVALID
    assert call(lib, one, work=None) == INVALID
    assert lib.fira_grad_norm(1, None, None, 4096, 4096, 1 << 20, None) == INVALID
    assert lib.fira_clip_grads(1, None, None, None, 1.0, 4096, 4096, 4096, 1 << 20, None) == INVALID


def test_misaligned_pointers_are_refused(lib):
    assert call(lib, [D(1, 8, 0, 0, 0, 0)], G=[(1 << 20) + 2]) == INVALID
    assert call(lib, [D(1, 8, 0, 0, 1, 1)], G=[(1 << 20) + 1]) == INVALID
    assert call(lib, [D(1, 8, 0, 0, 1, 0)], out=[(1 << 24) + 2]) == INVALID
    assert call(lib, [D(1, 8, 0, 0, 0, 0)], work=4100) == INVALID
    assert call(lib, [D(1, 8, 0, 0, 0, 0)], norm=4097) == INVALID


def test_small_workspace_is_refused(lib):
    for count in (1, 48, 49, 512, 513, 1500):
        need = lib.fira_grad_work_bytes(count)
        assert call(lib, [D(1, 8, 0, 0, 0, 0)] * count, work_bytes=need - 1) == SMALL
        assert b"workspace" in lib.fira_last_error()


def test_a_tensor_written_twice_is_refused(lib):
    two = [D(1, 8, 0, 0, 0, 0)] * 2
    assert call(lib, two, G=[1 << 20, 1 << 20]) == INVALID
    assert b"twice" in lib.fira_last_error()
    assert call(lib, two, out=[1 << 24, 1 << 24]) == INVALID


def test_in_place_needs_one_type_and_one_pitch(lib):
    assert call(lib, [D(1, 8, 0, 0, 0, 1)], G=[1 << 20], out=[1 << 20]) == INVALID
    assert call(lib, [D(2, 8, 8, 16, 0, 0)], G=[1 << 20], out=[1 << 20]) == INVALID
    assert b"in place" in lib.fira_last_error()


def test_binding_refuses_what_it_cannot_pass_on():
    with pytest.raises(ValueError, match="empty list"):
        fb.grad_norm([])
    with pytest.raises(ValueError, match="CUDA"):
        fb.grad_norm([torch.zeros(4)])
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        fb.grad_norm([torch.zeros(4, dtype=torch.float16)])
    with pytest.raises(ValueError, match="strides"):
        fb.grad_norm([torch.zeros(4, 8)[:, ::2]])
    with pytest.raises(ValueError, match="strides"):
        fb.grad_norm([torch.zeros(1, 8).expand(4, 8)])
    with pytest.raises(ValueError, match="strides"):
        fb.grad_norm([torch.zeros(4, 8, 6)[:, :, :3]])
    with pytest.raises(ValueError, match="outputs"):
        fb.clip_grads([torch.zeros(4)], 1.0, out=[])
    with pytest.raises(ValueError, match="output"):
        fb.clip_grads([torch.zeros(4)], 1.0, out=[torch.zeros(5)])
    with pytest.raises(ValueError, match="transposed"):
        fb.clip_grads([torch.zeros(4, 8)], 1.0, out=[torch.zeros(8, 4).t()])
