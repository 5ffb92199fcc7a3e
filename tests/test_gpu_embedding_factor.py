"""Positions without a token are rows of zeros whatever the factor: also where the factor times zero is not zero."""
import pytest
import torch

from paper_2410_01623_b200 import binding as fb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("hidden", [16, 37, 1024])
@pytest.mark.parametrize("scale", [float("inf"), float("nan"), -2.0])
def test_positions_without_a_token(dtype, hidden, scale):
    table = torch.ones(10, hidden, dtype=dtype, device="cuda")
    tokens = torch.tensor([3, -1, 10, 9, -1], device="cuda")
    Y = fb.embedding(table, tokens, scale=scale)
    none = torch.zeros(3, hidden, dtype=dtype, device="cuda")
    assert torch.equal(Y[[1, 2, 4]], none) and not bool(Y[[1, 2, 4]].signbit().any())
    assert torch.equal(Y[[0, 3]].nan_to_num(nan=5.0), torch.full((2, hidden), scale, dtype=dtype, device="cuda").nan_to_num(nan=5.0))
    G = fb.embedding_grad(tokens, torch.ones(5, hidden, dtype=dtype, device="cuda"), 10, scale=scale)
    assert not G[[0, 1, 2, 4, 5, 6, 7, 8]].any()
