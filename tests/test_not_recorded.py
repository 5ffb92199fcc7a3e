"""The forward calls return tensors without a graph: where autograd would have recorded them, that is said."""
import warnings

import pytest
import torch

from paper_2410_01623_b200 import binding as fb

X, GAIN, TOKENS = torch.zeros(4, 8), torch.ones(8), torch.zeros(4, dtype=torch.int64)


def leaf(t):
    return t.clone().requires_grad_()


CALLS = {
    "embedding": (lambda: fb.embedding(leaf(X), TOKENS), lambda: fb.embedding(X, TOKENS)),
    "layer_norm of x": (lambda: fb.layer_norm(leaf(X), GAIN), lambda: fb.layer_norm(X, GAIN)),
    "layer_norm's gain": (lambda: fb.layer_norm(X, leaf(GAIN)), lambda: fb.layer_norm(X, GAIN, GAIN)),
    "layer_norm's bias": (lambda: fb.layer_norm(X, GAIN, leaf(GAIN)), lambda: fb.layer_norm(X, GAIN, rms=True))}


@pytest.mark.parametrize("name", CALLS)
def test_lost_gradients_are_said(name):
    lost, kept = CALLS[name]
    with pytest.warns(UserWarning, match="not recorded"), pytest.raises(ValueError, match="CUDA"):
        lost()
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        with pytest.raises(ValueError, match="CUDA"):
            kept()
        with torch.no_grad(), pytest.raises(ValueError, match="CUDA"):
            lost()
