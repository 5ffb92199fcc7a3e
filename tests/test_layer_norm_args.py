"""Refusals of fira_layer_norm and fira_layer_norm_grad: arguments are checked before anything reaches the device."""
import pytest
import torch

from paper_2410_01623_b200 import binding as fb
from paper_2410_01623_b200 import build as fbuild

INVALID, SMALL, UNSUPPORTED = 1, 2, 3
P = [(i + 1) << 20 for i in range(10)]                 # made-up addresses: every case is refused before one is used


@pytest.fixture(scope="module")
def lib():
    fbuild.build()
    return fb.lib()


def forward(lib, **change):
    a = dict(x=P[0], ld_x=0, dtype=0, rows=4, hidden=8, gain=P[1], bias=P[2], param_dtype=0, eps=1e-5, y=P[3], ld_y=0,
             mean=P[4], rstd=P[5])
    assert not set(change) - set(a)
    return lib.fira_layer_norm(*{**a, **change}.values(), None)


def backward(lib, **change):
    a = dict(dY=P[6], ld_dy=0, x=P[0], ld_x=0, dtype=0, rows=4, hidden=8, gain=P[1], param_dtype=0, mean=P[4], rstd=P[5],
             dX=P[3], ld_dx=0, dgain=P[7], dbias=P[8], grad_dtype=0, accumulate=0, work=P[9], work_bytes=1 << 30)
    assert not set(change) - set(a)
    return lib.fira_layer_norm_grad(*{**a, **change}.values(), None)


@pytest.mark.parametrize("change", [
    dict(rows=-1), dict(rows=1 << 41), dict(hidden=0), dict(hidden=-3), dict(dtype=2), dict(param_dtype=-1), dict(ld_x=7),
    dict(x=None), dict(x=P[0] + 2), dict(gain=None), dict(gain=P[1] + 2), dict(rstd=None), dict(rstd=P[5] + 2), dict(mean=P[4] + 1),
    dict(mean=None)])                                  # (without a mean there is no bias)
def test_bad_arguments_are_refused(lib, change):
    assert forward(lib, **change) == INVALID
    assert len(lib.fira_last_error()) > 0
    assert backward(lib, **change) == INVALID


@pytest.mark.parametrize("change", [dict(y=None), dict(y=P[3] + 2), dict(ld_y=5), dict(bias=P[2] + 2), dict(eps=-1.0), dict(eps=float("nan")),
                                    dict(eps=float("inf"))])
def test_bad_forward_arguments_are_refused(lib, change):
    assert forward(lib, **change) == INVALID


@pytest.mark.parametrize("change", [
    dict(dY=None), dict(dY=P[6] + 2), dict(ld_dy=5), dict(dX=None), dict(dX=P[3] + 2), dict(ld_dx=5), dict(dgain=None), dict(dgain=P[7] + 2),
    dict(dbias=P[8] + 2), dict(grad_dtype=9), dict(work=None), dict(work=P[9] + 16)])
def test_bad_backward_arguments_are_refused(lib, change):
    assert backward(lib, **change) == INVALID


def test_rows_that_are_too_long(lib):
    assert forward(lib, hidden=16385) == UNSUPPORTED and backward(lib, hidden=16385) == UNSUPPORTED
    assert lib.fira_layer_norm_grad_work_bytes(4, 16385, 0) == 0


@pytest.mark.parametrize("rows,hidden", [(0, 1), (1, 1), (4, 8), (4096, 1707), (1 << 20, 16384)])
@pytest.mark.parametrize("dtype", [0, 1])
def test_small_workspaces_are_refused(lib, rows, hidden, dtype):
    need = lib.fira_layer_norm_grad_work_bytes(rows, hidden, dtype)
    assert need >= 8 * hidden
    assert backward(lib, rows=rows, hidden=hidden, dtype=dtype, work_bytes=need - 1) == SMALL


def test_a_norm_of_nothing_is_done(lib):
    assert forward(lib, rows=0, x=None, y=None) == 0


def test_binding_refuses_what_it_cannot_pass_on():
    x, g = torch.zeros(4, 8), torch.ones(8)
    rstd = torch.ones(4)
    with pytest.raises(ValueError, match="vectors of 8"):
        fb.layer_norm(x, torch.ones(7))
    with pytest.raises(ValueError, match="vectors of 8"):
        fb.layer_norm(x, g, torch.zeros(8, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        fb.layer_norm(x.half(), g)
    with pytest.raises(ValueError, match="strides"):
        fb.layer_norm(torch.zeros(8, 4).t(), g)
    with pytest.raises(ValueError, match="CUDA"):
        fb.layer_norm(x, g)
    with pytest.raises(ValueError, match="for x"):
        fb.layer_norm_grad(x[:3], x, g, rstd, rstd)
    with pytest.raises(ValueError, match="mean"):
        fb.layer_norm_grad(x, x, g, None, rstd)
    with pytest.raises(ValueError, match="mean"):
        fb.layer_norm_grad(x, x, g, rstd, rstd, rms=True)
    with pytest.raises(ValueError, match="no bias"):
        fb.layer_norm_grad(x, x, g, None, rstd, rms=True, dbias=g)
    with pytest.raises(ValueError, match="needed"):
        fb.layer_norm_grad(x, x, g, rstd, rstd[:3])
    with pytest.raises(ValueError, match="dgain and dbias are needed"):
        fb.layer_norm_grad(x, x, g, rstd, rstd, dgain=g, accumulate=True)
