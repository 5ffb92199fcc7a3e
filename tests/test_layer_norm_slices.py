"""Layer norm over slices of a batch: what its backward pass takes as the gradient, the forward pass takes as its input."""
import itertools

import pytest
import torch

from paper_2410_01623_b200 import binding as fb
from tests.test_gpu_layer_norm import check_backward, check_forward

BATCH = torch.arange(6 * 10 * 24, dtype=torch.float32).reshape(6, 10, 24)
SLICES = {                                     # (the slice, and its rows' pitch: None where there is no one)
    "columns": (lambda b: b[:, :, 5:12], 24), "positions": (lambda b: b[:, 2:7], None), "every other": (lambda b: b[:, ::2], 48),
    "both": (lambda b: b[:, :-1, :8], None), "swapped": (lambda b: b.transpose(0, 1), None), "one sequence": (lambda b: b[2:3, 1:4], 0),
    "one position": (lambda b: b[:, 3:4], 240), "expanded": (lambda b: b[:, :1].expand(6, 10, 24), None), "one column": (lambda b: b[:, :, 4:5], 24)}


@pytest.mark.parametrize("name", SLICES)
def test_pitches(name):
    make, pitch = SLICES[name]
    x = make(BATCH)
    assert fb._pitch_of(x) == pitch
    if pitch is not None:                      # the rows lie where the pitch says
        base, ld = x.storage_offset(), pitch or x.shape[-1]
        for k, index in enumerate(itertools.product(*map(range, x.shape[:-1]))):
            assert float(x[index][0]) == base + k * ld


@pytest.mark.parametrize("name", SLICES)
def test_slices_get_as_far_as_the_device(name):
    x = SLICES[name][0](BATCH)
    gain, stats = torch.ones(x.shape[-1]), torch.ones(x.shape[:-1])
    with pytest.raises(ValueError, match="CUDA"):
        fb.layer_norm(x, gain)
    with pytest.raises(ValueError, match="CUDA"):
        fb.layer_norm_grad(x.contiguous(), x, gain, stats, stats)
    with pytest.raises(ValueError, match="strides"):
        fb.layer_norm(BATCH.transpose(1, 2), torch.ones(10))


@pytest.mark.gpu
@pytest.mark.parametrize("name", SLICES)
@pytest.mark.parametrize("rms", [False, True])
def test_slices(name, rms):
    """Against the formulas in 64 bits, with the tolerances of the contiguous forms."""
    gen = torch.Generator().manual_seed(1)
    x = SLICES[name][0](torch.randn(6, 10, 24, generator=gen).cuda())
    dY = SLICES[name][0](torch.randn(6, 10, 24, generator=gen).cuda())
    gain = torch.randn(x.shape[-1], generator=gen).cuda()
    kept = x.clone()
    y, mean, rstd = fb.layer_norm(x, gain, rms=rms)
    assert torch.equal(x, kept) and y.shape == x.shape and rstd.shape == x.shape[:-1]
    check_forward(x, gain, None, 1e-5, rms, y, mean, rstd)
    dX, dgain, dbias = fb.layer_norm_grad(dY, x, gain, mean, rstd, rms=rms)
    assert dX.shape == x.shape
    check_backward(dY, x, gain, mean, rstd, rms, dX, dgain, dbias)


@pytest.mark.gpu
def test_a_slice_in_place():
    """Columns of a wider batch, over themselves; the others stay."""
    gen = torch.Generator().manual_seed(2)
    wide = torch.randn(6, 10, 24, generator=gen).cuda()
    was, gain = wide.clone(), torch.ones(8, device="cuda")
    x = wide[..., 4:12]
    y, mean, rstd = fb.layer_norm(x, gain, out=x)
    assert y is x
    check_forward(was[..., 4:12], gain, None, 1e-5, False, y, mean, rstd)
    assert torch.equal(wide[..., :4], was[..., :4]) and torch.equal(wide[..., 12:], was[..., 12:])
    with pytest.raises(ValueError, match="out"):
        fb.layer_norm(was[:, :5], torch.ones(24, device="cuda"), out=was[:, :5])
