"""The table's gradient where the vocabulary asks for more remainders than the tokens are dealt to at once.

dY holds small whole numbers, so that every sum is a whole number below 2^24, which fp32 adds without rounding in any order:
the results are equal, not near.  The workspace of such sizes holds the dealt entries (8 bytes per position) beside the order:
the batch is dealt once, and not read anew by each of the blocks, of which there are a thousandth of the vocabulary."""
import pytest
import torch

from paper_2410_01623_b200 import binding as fb
from paper_2410_01623_b200 import build as fbuild


@pytest.mark.parametrize("n", [16385, 1 << 20, 1 << 30])
@pytest.mark.parametrize("vocab", [(1 << 19) + 1, 1 << 20, 1 << 30])
def test_the_batch_is_dealt_once(n, vocab):
    fbuild.build()
    L = fb.lib()
    small = 1 << 19
    spans = 8 * (vocab - small)                # what the larger vocabulary needs more
    assert L.fira_embedding_grad_work_bytes(n, vocab, 8, 0) - spans >= L.fira_embedding_grad_work_bytes(n, small, 8, 0) - 256


def tokens_of(kind, n, vocab, gen):
    if kind == "one":
        return torch.full((n,), vocab - 2, device="cuda")
    if kind == "zipf":
        u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
        return (2.7 * ((vocab + 2.7) / 2.7) ** u - 2.7).long().clamp_(0, vocab - 1)
    if kind == "one remainder":                # tokens 512 apart: dealt alike, of different blocks
        return torch.randint(0, vocab // 512, (n,), generator=gen, device="cuda") * 512 + 7
    t = torch.randint(-vocab // 8, vocab + vocab // 8, (n,), generator=gen, device="cuda")
    t[n // 2:n // 2 + 3000] = vocab - 1
    return t


@pytest.mark.gpu
@pytest.mark.parametrize("n,vocab,hidden", [(16385, 524289, 8), (40000, 600000, 16), (1 << 20, 1 << 20, 3), (20000, 3_000_001, 4), (16384, 3_000_001, 4)])
@pytest.mark.parametrize("kind", ["one", "zipf", "one remainder", "mixed"])
@pytest.mark.parametrize("index", [torch.int32, torch.int64])
def test_gradient(n, vocab, hidden, kind, index):
    gen = torch.Generator(device="cuda").manual_seed(n + vocab)
    tokens = tokens_of(kind, n, vocab, gen).to(index)
    dY = torch.randint(-8, 8, (n, hidden), generator=gen, device="cuda").float()
    ok = (tokens >= 0) & (tokens < vocab)
    want = torch.zeros(vocab, hidden, dtype=torch.float64, device="cuda").index_add_(0, tokens[ok].long(), dY[ok].double())
    assert torch.equal(fb.embedding_grad(tokens, dY, vocab).double(), want)
    G = torch.ones(vocab, hidden, device="cuda")
    fb.embedding_grad(tokens, dY, vocab, out=G, accumulate=True)
    assert torch.equal(G.double(), want + 1)
