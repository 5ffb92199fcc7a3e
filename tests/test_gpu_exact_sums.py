"""Long sums with exact answers: whole numbers whose sums, in any order, stay below 2^24, so that fp32 rounds nowhere and every
element has to be equal.  (A tolerance that allows for each rounding of a sum of 10^5 terms of either sign is larger than the sum,
and than what a lost part of it would change.)"""
import pytest
import torch

from paper_2410_01623_b200 import binding as fb

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def whole(gen, lo, hi, *shape):
    return torch.randint(lo, hi, shape, generator=gen, device="cuda").float()


def tokens_of(kind, n, vocab, gen):
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    if kind == "one":
        return torch.full((n,), vocab // 2, device="cuda")
    if kind == "zipf":
        return (2.7 * ((vocab + 2.7) / 2.7) ** u - 2.7).long().clamp_(0, vocab - 1)
    if kind == "few":                          # rows of many parts, one behind another
        return (u * min(vocab, 9)).long()
    t = (u * vocab).long()                     # "mixed": stretches of one token beside single ones, and positions without
    t[n // 3:n // 2] = vocab - 1
    t[:n // 5] = 0
    return torch.where(torch.rand(n, generator=gen, device="cuda") < 0.1, -1, t)


@pytest.mark.parametrize("dtype,grad_dtype", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("n,vocab,hidden", [(4096, 1000, 512), (16384, 300, 256), (16385, 300, 257), (131072, 5000, 512), (150001, 700, 24), (131072, 5000, 130),
                                            (70000, 900, 1024), (1 << 20, 40, 8), (1 << 20, 200003, 5), (30000, 50, 2048), (9000, 20, 4100)])
@pytest.mark.parametrize("kind", ["one", "few", "zipf", "mixed"])
@pytest.mark.parametrize("accumulate", [False, True])
def test_table_gradient(dtype, grad_dtype, n, vocab, hidden, kind, accumulate):
    gen = torch.Generator(device="cuda").manual_seed(n + hidden)
    tokens = tokens_of(kind, n, vocab, gen)
    dY = whole(gen, -8, 8, n, hidden)          # sums of at most 2^20 of them: 2^23
    want = torch.zeros(vocab, hidden, dtype=torch.float64, device="cuda")
    keep = tokens >= 0
    want.index_add_(0, tokens[keep], dY[keep].double())
    want *= 0.5
    old = whole(gen, -4, 4, vocab, hidden).to(grad_dtype)
    G = old.clone()
    fb.embedding_grad(tokens, dY.to(dtype), vocab, scale=0.5, out=G, accumulate=accumulate)
    if accumulate:
        want += old.double()
    assert torch.equal(G, want.float().to(grad_dtype))


SHAPES = [(40000, 64), (65536, 32), (65536, 1), (33333, 7), (4097, 33), (1529, 43), (50000, 100), (20001, 512), (12345, 520), (9000, 1024), (7001, 1707),
          (5000, 4096), (5001, 4099), (2500, 8192), (2501, 8195), (1100, 12000), (1000, 12001), (700, 16384), (700, 16383)]


@pytest.mark.parametrize("rows,hidden", SHAPES)
@pytest.mark.parametrize("dtype,param_dtype", [(F32, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("shift", [0, 1])      # dY begins elsewhere than x: element by element
def test_gains_and_biases(rows, hidden, dtype, param_dtype, rms, shift):
    gen = torch.Generator(device="cuda").manual_seed(rows + hidden)
    x = whole(gen, -4, 5, rows, hidden)
    dY = whole(gen, -4, 5, rows, hidden)
    mean, rstd = whole(gen, -1, 2, rows), 2.0 ** whole(gen, 0, 2, rows)
    h = (x if rms else x - mean[:, None]) * rstd[:, None]               # at most 10; dY h at most 40, and 65536 of them 2.7e6
    gain = torch.ones(hidden, dtype=param_dtype, device="cuda")
    at = torch.empty(rows * hidden + 8, dtype=dtype, device="cuda")[shift:shift + rows * hidden].view(rows, hidden).copy_(dY)
    for accumulate in (False, True):
        old = [whole(gen, -4, 5, hidden).to(param_dtype) for _ in range(2)]
        dgain, dbias = old[0].clone(), None if rms else old[1].clone()
        fb.layer_norm_grad(at, x.to(dtype), gain, None if rms else mean, rstd, rms=rms, dgain=dgain, dbias=dbias, accumulate=accumulate)
        for got, terms, was in ((dgain, dY.double() * h.double(), old[0]), (dbias, dY.double(), old[1])):
            if got is not None:
                want = terms.sum(0) + (was.double() if accumulate else 0.0)
                assert torch.equal(got, want.float().to(param_dtype))


@pytest.mark.parametrize("count", [1, 479, 480, 481, 960, 961])
def test_norms(count):
    """Squares of whole numbers: their sum is exact in double and in each thread's fp32 sum, whatever the launches."""
    gen = torch.Generator(device="cuda").manual_seed(count)
    Gs = [whole(gen, -9, 10, 1 + (977 * i) % 30011).to([F32, BF16][i % 2]) for i in range(count)]
    want = sum(float(g.double().square().sum()) for g in Gs) ** 0.5
    assert float(fb.grad_norm(Gs)) == float(torch.tensor(want, dtype=torch.float64).float())
