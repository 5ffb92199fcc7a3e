"""GPU parity of fira_embedding and fira_embedding_grad with the definitions in 64 bits.

Tolerances.  The lookup is one fp32 product and one rounding: exact at scale 1.  A row of the gradient that k positions
name is a sum of k fp32 terms in some fixed order (fewer than k additions besides those of the parts: below 2 k), one product
and one rounding: within (2 k + 1) 2^-24 |scale| sum |dY| of the true sum, and 2^-24 (fp32) or 2^-8 (bf16) of the
result; added to an old gradient, the product and sum are one rounding more of their result."""
import pytest
import torch

from paper_2410_01623_b200 import binding as fb

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
STORE = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
F32, BF16 = torch.float32, torch.bfloat16


def make_tokens(gen, kind, n, vocab, dtype=torch.int64):
    if kind == "uniform":
        t = torch.randint(0, vocab, (n,), generator=gen)
    elif kind == "zipf":
        t = (2.7 * ((vocab + 2.7) / 2.7) ** torch.rand(n, generator=gen, dtype=torch.float64) - 2.7).long().clamp(0, vocab - 1)
    elif kind == "one":
        t = torch.full((n,), vocab // 2)
    elif kind == "none":
        t = torch.full((n,), -1)
    else:                                      # "mixed": sorted stretches, repeats, positions that hold no token
        t = torch.randint(0, vocab, (n,), generator=gen)
        t[: n // 3] = t[: n // 3].sort().values
        t[n // 3: n // 2] = vocab - 1
        bad = torch.rand(n, generator=gen)
        t[bad < 0.1] = -1
        t[bad > 0.95] = vocab
        t[bad > 0.97] = torch.iinfo(dtype).max
        t[bad > 0.98] = torch.iinfo(dtype).min
        if dtype == torch.int64:
            t[bad > 0.99] = 1 << 32            # its low half is a token
    return t.to(dtype)


def exact_grad(tokens, dY, vocab, scale, old=None):
    """The gradient in 64 bits, and per element the allowance of its sum."""
    t, rows = tokens.long().reshape(-1).cpu(), dY.double().reshape(tokens.numel(), -1).cpu()
    ok = (t >= 0) & (t < vocab)
    t, rows = t[ok], rows[ok]
    G = torch.zeros(vocab, rows.shape[1], dtype=torch.float64).index_add_(0, t, rows)
    size = torch.zeros_like(G).index_add_(0, t, rows.abs())
    k = torch.bincount(t, minlength=vocab).double()[:, None]
    return G * scale, (2 * k + 1) * U * abs(scale) * size


def check_grad(tokens, dY, vocab, scale, G, old=None):
    want, allow = exact_grad(tokens, dY, vocab, scale)
    if old is not None:
        want = want + old.double().cpu()
        allow = allow + U * want.abs()
    got = G.double().cpu()
    assert bool(((got - want).abs() <= allow * (1 + 2 * STORE[G.dtype]) + STORE[G.dtype] * want.abs() + 1e-44).all())


def f32(x):
    return float(torch.tensor(x, dtype=F32))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("index", [torch.int32, torch.int64])
@pytest.mark.parametrize("n,vocab,hidden", [(1, 1, 1), (3, 5, 8), (4, 7, 3), (257, 1000, 64), (1000, 333, 257), (65, 50, 1707),
                                            (33, 20, 4096), (2, 3, 9000)])
@pytest.mark.parametrize("scale", [1.0, 22.627])
def test_lookup(dtype, index, n, vocab, hidden, scale):
    gen = torch.Generator().manual_seed(n)
    table = torch.randn(vocab, hidden, generator=gen).to(dtype).cuda()
    tokens = make_tokens(gen, "mixed", n, vocab, index).cuda()
    Y = fb.embedding(table, tokens, scale=scale)
    assert Y.shape == (n, hidden) and Y.dtype == dtype
    ok = (tokens.long() >= 0) & (tokens.long() < vocab)
    rows = table[tokens.long().clamp(0, vocab - 1)].float() * torch.tensor(scale, device="cuda")
    assert torch.equal(Y, torch.where(ok[:, None], rows, 0.0).to(dtype))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,vocab,hidden", [(1, 1, 1), (1, 70000, 8), (7, 5, 3), (32, 32, 64), (100, 11, 129), (1000, 777, 65), (513, 40, 1707),
                                            (5000, 3000, 512), (20000, 200, 24), (300, 200003, 16)])
@pytest.mark.parametrize("kind", ["uniform", "zipf", "one", "none", "mixed"])
def test_gradient(dtype, n, vocab, hidden, kind):
    gen = torch.Generator().manual_seed(n + vocab)
    tokens = make_tokens(gen, kind, n, vocab).cuda()
    dY = torch.randn(n, hidden, generator=gen).to(dtype).cuda()
    G = fb.embedding_grad(tokens, dY, vocab, scale=3.5)
    assert G.dtype == dtype and G.shape == (vocab, hidden)
    check_grad(tokens, dY, vocab, 3.5, G)


@pytest.mark.parametrize("dtype,grad_dtype", [(F32, BF16), (BF16, F32), (F32, F32), (BF16, BF16)])
@pytest.mark.parametrize("hidden", [8, 20, 21, 256, 260])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("index", [torch.int32, torch.int64])
def test_gradient_types_and_accumulation(dtype, grad_dtype, hidden, accumulate, index):
    gen = torch.Generator().manual_seed(hidden)
    n, vocab = 3000, 500
    tokens = make_tokens(gen, "mixed", n, vocab, index).view(30, 100).cuda()
    dY = torch.randn(30, 100, hidden, generator=gen).to(dtype).cuda()
    G = torch.randn(vocab, hidden, generator=gen).to(grad_dtype).cuda()
    old = G.clone()
    scale = f32(0.3)
    assert fb.embedding_grad(tokens, dY, vocab, scale=scale, out=G, accumulate=accumulate) is G
    check_grad(tokens, dY, vocab, scale, G, old if accumulate else None)
    if accumulate:
        named = torch.zeros(vocab + 1, dtype=torch.bool, device="cuda")
        t = tokens.long().reshape(-1)
        named[torch.where((t >= 0) & (t < vocab), t, vocab)] = True
        assert torch.equal(G[~named[:vocab]], old[~named[:vocab]])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("hidden,pitch", [(64, 72), (64, 67), (37, 40), (37, 37), (1, 5)])
def test_pitched_rows(dtype, hidden, pitch):
    """What lies behind the rows is neither read nor written."""
    gen = torch.Generator().manual_seed(pitch)
    n, vocab = 400, 90
    tokens = make_tokens(gen, "zipf", n, vocab).cuda()
    dY = torch.full((n, pitch), float("nan"), dtype=dtype, device="cuda")
    dY[:, :hidden] = torch.randn(n, hidden, generator=gen).to(dtype).cuda()
    G = torch.full((vocab, pitch), 7.0, dtype=dtype, device="cuda")
    fb.embedding_grad(tokens, dY[:, :hidden], vocab, out=G[:, :hidden])
    check_grad(tokens, dY[:, :hidden], vocab, 1.0, G[:, :hidden])
    assert bool((G[:, hidden:] == 7.0).all())
    Y = torch.full((n, pitch), 9.0, dtype=dtype, device="cuda")
    fb.embedding(G[:, :hidden], tokens, out=Y[:, :hidden])
    assert torch.equal(Y[:, :hidden], G[tokens, :hidden]) and bool((Y[:, hidden:] == 9.0).all())


@pytest.mark.parametrize("shift", [1, 2, 3])
@pytest.mark.parametrize("index", [torch.int32, torch.int64])
def test_tensors_off_the_16_byte_boundaries(shift, index):
    gen = torch.Generator().manual_seed(shift)
    n, vocab, hidden = 1003, 64, 32
    tokens = make_tokens(gen, "mixed", n + 8, vocab, index).cuda()[shift:shift + n]
    buf = torch.randn(n * hidden + 8, generator=gen).cuda()
    dY = buf[shift:shift + n * hidden].view(n, hidden)
    G = torch.zeros(vocab * hidden + 8, device="cuda")[shift:shift + vocab * hidden].view(vocab, hidden)
    fb.embedding_grad(tokens, dY, vocab, out=G)
    check_grad(tokens, dY, vocab, 1.0, G)
    Y = fb.embedding(G, tokens)
    ok = (tokens.long() >= 0) & (tokens.long() < vocab)
    assert torch.equal(Y, torch.where(ok[:, None], G[tokens.long().clamp(0, vocab - 1)], 0.0))


@pytest.mark.parametrize("n,hidden,dtype", [(131072, 512, BF16), (150001, 256, F32), (70000, 1024, BF16)])
@pytest.mark.parametrize("kind", ["one", "zipf", "mixed"])
def test_large_batches(n, hidden, dtype, kind):
    """Long stretches per warp, and rows cut into many parts."""
    gen = torch.Generator().manual_seed(2)
    vocab = 5000
    tokens = make_tokens(gen, kind, n, vocab).cuda()
    dY = torch.randn(n, hidden, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(dtype)
    check_grad(tokens, dY, vocab, 1.0, fb.embedding_grad(tokens, dY, vocab))


@pytest.mark.parametrize("n,vocab,hidden", [(20000, 200003, 16), (20000, 600000, 8), (16384, 3000, 33), (16385, 3000, 33), (1 << 20, 40, 8), (70000, 32000, 3),
                                            (40, 30, 20000), (40, 30, 20001)])
@pytest.mark.parametrize("dtype,kind", [(F32, "zipf"), (BF16, "mixed")])
def test_large_vocabularies_batches_and_widths(n, vocab, hidden, dtype, kind):
    """More remainders than the smallest number, more than the two launches take, batches on both sides of the border between one
    and two launches, a batch of a million positions, rows of many slices."""
    gen = torch.Generator().manual_seed(n + hidden)
    tokens = make_tokens(gen, kind, n, vocab).cuda()
    dY = torch.randn(n, hidden, generator=gen).to(dtype).cuda()
    G = fb.embedding_grad(tokens, dY, vocab)
    check_grad(tokens, dY, vocab, 1.0, G)
    Y = fb.embedding(G, tokens)
    ok = (tokens.long() >= 0) & (tokens.long() < vocab)
    assert torch.equal(Y, torch.where(ok[:, None], G[tokens.long().clamp(0, vocab - 1)], 0.0).to(dtype))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shift,gshift", [(0, 1), (1, 0), (1, 1), (1, 2), (3, 1)])
@pytest.mark.parametrize("hidden", [24, 33, 300, 1023])
def test_rows_that_begin_anywhere(dtype, shift, gshift, hidden):
    """dY, G, table and output each begin elsewhere between two 16-byte boundaries; guards around G and the output stay."""
    gen = torch.Generator().manual_seed(hidden)
    n, vocab = 500, 41
    tokens = make_tokens(gen, "mixed", n, vocab).cuda()
    dY = torch.randn(n * hidden + 8, generator=gen).to(dtype).cuda()[shift:shift + n * hidden].view(n, hidden)
    buf = torch.full((vocab * hidden + 16,), 5.0, dtype=dtype, device="cuda")
    G = buf[gshift:gshift + vocab * hidden].view(vocab, hidden)
    fb.embedding_grad(tokens, dY, vocab, out=G)
    check_grad(tokens, dY, vocab, 1.0, G)
    assert bool((buf[:gshift] == 5.0).all()) and bool((buf[gshift + vocab * hidden:] == 5.0).all())
    outs = torch.full((n * hidden + 16,), 5.0, dtype=dtype, device="cuda")
    Y = outs[shift:shift + n * hidden].view(n, hidden)
    fb.embedding(G, tokens, out=Y)
    ok = (tokens.long() >= 0) & (tokens.long() < vocab)
    assert torch.equal(Y, torch.where(ok[:, None], G[tokens.long().clamp(0, vocab - 1)], 0.0).to(dtype))
    assert bool((outs[:shift] == 5.0).all()) and bool((outs[shift + n * hidden:] == 5.0).all())


def test_two_calls_at_once_on_two_streams():
    gen = torch.Generator().manual_seed(16)
    calls = []
    for k in range(2):
        tokens = make_tokens(gen, "zipf", 30000, 4000).cuda()
        dY = torch.randn(30000, 96, generator=gen).cuda()
        calls.append((tokens, dY, torch.empty(4000, 96, device="cuda"), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(5):
        for tokens, dY, G, stream in calls:
            with torch.cuda.stream(stream):
                fb.embedding_grad(tokens, dY, 4000, out=G)
    torch.cuda.synchronize()
    for tokens, dY, G, _ in calls:
        check_grad(tokens, dY, 4000, 1.0, G)


def test_no_positions():
    empty = torch.zeros(0, dtype=torch.int64, device="cuda")
    G = torch.full((1000, 40), 3.0, device="cuda")
    fb.embedding_grad(empty, torch.zeros(0, 40, device="cuda"), 1000, out=G, accumulate=True)
    assert bool((G == 3.0).all())
    fb.embedding_grad(empty, torch.zeros(0, 40, device="cuda"), 1000, out=G)
    assert not G.any()
    assert fb.embedding(G, empty).shape == (0, 40)


def test_not_contiguous_inputs():
    gen = torch.Generator().manual_seed(12)
    batch = torch.randint(0, 100, (8, 33), generator=gen).cuda()
    dY = torch.randn(8, 40, 16, generator=gen).cuda()[:, :32]
    G = fb.embedding_grad(batch[:, :-1], dY, 100)
    check_grad(batch[:, :-1].contiguous(), dY, 100, 1.0, G)
    assert torch.equal(fb.embedding(G, batch[:, 1:]), G[batch[:, 1:]])


def test_infinities_and_nans_stay_in_their_rows():
    gen = torch.Generator().manual_seed(13)
    tokens = torch.arange(64).repeat(40).cuda()
    dY = torch.randn(2560, 48, generator=gen).cuda()
    dY[3, 5], dY[64 * 7 + 9, 0] = float("inf"), float("nan")
    tokens[17] = -1
    dY[17] = float("nan")                      # at a position that has no part
    G = fb.embedding_grad(tokens, dY, 64)
    assert float(G[3, 5]) == float("inf") and bool(G[9, 0].isnan())
    G[3, 5] = G[9, 0] = 0
    assert bool(G.isfinite().all())


@pytest.mark.parametrize("kind", ["zipf", "one"])
def test_the_same_call_gives_the_same_bits(kind):
    gen = torch.Generator().manual_seed(14)
    tokens = make_tokens(gen, kind, 60000, 3000).cuda()
    dY = torch.randn(60000, 128, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    first = fb.embedding_grad(tokens, dY, 3000)
    for _ in range(10):
        assert torch.equal(fb.embedding_grad(tokens, dY, 3000), first)


def test_captured_and_replayed_on_another_stream():
    gen = torch.Generator().manual_seed(15)
    tokens = make_tokens(gen, "zipf", 4000, 70000).cuda()     # (so many rows that the counts take a larger shared memory)
    dY = torch.randn(4000, 64, generator=gen).cuda()
    G = torch.empty(70000, 64, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        fb.embedding_grad(tokens, dY, 70000, out=G)
        Y = fb.embedding(G, tokens)
    for k in range(3):
        tokens.copy_(make_tokens(gen, "zipf" if k else "mixed", 4000, 70000).clamp(0))
        tokens.clamp_(max=69999)
        dY.copy_(torch.randn(4000, 64, generator=gen))
        G.fill_(5.0)
        graph.replay()
        check_grad(tokens, dY, 70000, 1.0, G)
        assert torch.equal(Y, G[tokens])


def test_offsets_beyond_32_bits():
    """A table of more than 2^32 bytes, and of more than 2^31 elements."""
    vocab, hidden = 300000, 8192
    table = torch.zeros(vocab, hidden, dtype=BF16, device="cuda")
    table[-1], table[vocab // 2] = 2.0, 3.0
    tokens = torch.tensor([vocab - 1, 0, vocab // 2, vocab - 1], device="cuda")
    Y = fb.embedding(table, tokens)
    assert [float(y.float().mean()) for y in Y] == [2.0, 0.0, 3.0, 2.0]
    table.fill_(1.0)
    fb.embedding_grad(tokens, Y, vocab, out=table)
    assert float(table[-1].float().mean()) == 4.0 and float(table[vocab // 2].float().mean()) == 3.0
    assert float(table.float().sum(dtype=torch.float64)) == 7.0 * hidden
