"""Workspaces that are given to the binding: their size is what they hold."""
import pytest
import torch

from paper_2410_01623_b200 import binding as fb

X, ROW, TOKENS = torch.zeros(4, 8), torch.ones(8), torch.zeros(4, dtype=torch.int64)


@pytest.mark.parametrize("call", [
    lambda work: fb.grad_norm([X], work=work),
    lambda work: fb.clip_grads([X], 1.0, work=work),
    lambda work: fb.embedding_grad(TOKENS, X, 10, work=work),
    lambda work: fb.layer_norm_grad(X, X, ROW, torch.zeros(4), torch.ones(4), work=work)])
def test_expanded_workspaces_are_refused(call):
    """One byte that says it is a million: the library would write behind it."""
    with pytest.raises(ValueError, match="work"):
        call(torch.zeros(1, dtype=torch.uint8).expand(1 << 20))
    with pytest.raises(ValueError, match="CUDA"):
        call(torch.zeros(1 << 20, dtype=torch.uint8))
