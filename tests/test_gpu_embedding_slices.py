"""Lookup into, and gradient from, columns of a wider batch, in place."""
import pytest
import torch

from paper_2410_01623_b200 import binding as fb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("wide,first,hidden", [(48, 16, 16), (40, 3, 21), (24, 0, 24), (9, 8, 1)])
def test_columns_of_a_batch(dtype, wide, first, hidden):
    gen = torch.Generator(device="cuda").manual_seed(wide)
    tokens = torch.randint(-1, 50, (5, 70), generator=gen, device="cuda")
    batch = torch.randint(-8, 8, (5, 70, wide), generator=gen, device="cuda").to(dtype)        # whole numbers: exact sums
    dY = batch[..., first:first + hidden]
    want = torch.zeros(51, hidden, dtype=torch.float64, device="cuda").index_add_(0, tokens.reshape(-1) % 51, dY.reshape(-1, hidden).double())
    G = fb.embedding_grad(tokens, dY, 50)
    assert torch.equal(G, want[:50].float().to(dtype))         # (-1 % 51: the row behind)
    was = batch.clone()
    out = batch[..., first:first + hidden]
    assert fb.embedding(G, tokens, out=out) is out
    rows = torch.cat([G, torch.zeros(1, hidden, dtype=dtype, device="cuda")])[tokens]          # (-1: the last one)
    assert torch.equal(out, rows)
    was[..., first:first + hidden] = rows
    assert torch.equal(batch, was)
    with pytest.raises(ValueError, match="out"):
        fb.embedding(G, tokens.t(), out=torch.empty(5, 70, hidden, dtype=dtype, device="cuda").transpose(0, 1))
