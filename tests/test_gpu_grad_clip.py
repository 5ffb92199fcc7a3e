"""GPU parity of fira_grad_norm and fira_clip_grads with the definition in 64 bits.

Tolerances.  A thread adds 32 squares in fp32 (one rounding each, all terms positive), the rest is in double: the sum
is within 32 * 2^-24 of itself, the norm within 16 * 2^-24, and 2^-24 for its own rounding.  The factor carries the
norm's error before that rounding, max_norm's conversion and its own: 18 * 2^-24.  An output element carries the
factor's, the product's rounding and, in bf16, 2^-8 for the storage."""
import math

import numpy as np
import pytest
import torch

from paper_2410_01623_b200 import binding as fb

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
NORM, SCALE = 17 * U, 18 * U
STORE = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133}    # half a step among the smallest numbers, and some


def exact(Gs, max_norm):
    total = math.sqrt(math.fsum(float(g.double().square().sum()) for g in Gs))
    scale = min(1.0, max_norm / total) if total > 0 else 1.0
    return total, scale


def check(Gs, outs, norm, scale, max_norm):
    """Gs: the gradients as they were."""
    want, s = exact(Gs, max_norm)
    assert abs(float(norm) - want) <= NORM * want
    assert abs(float(scale) - s) <= SCALE * s
    for i, (g, o) in enumerate(zip(Gs, outs)):
        ref = g.double() * s
        off = (o.double() - ref).abs()
        assert bool((off <= (SCALE + U + STORE[o.dtype]) * ref.abs() + TINY[o.dtype]).all()), i


def lists(gen, dtype, sizes, pattern=1.0):
    return [(torch.randn(n, generator=gen) * pattern).to(dtype).cuda() for n in sizes]


SIZES = [1, 2, 7, 8, 9, 2047, 2048, 8191, 8192, 8193, 70001, 0, 1]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("max_norm", [1e-3, 1.0, 1e6, float("inf")])
@pytest.mark.parametrize("place", ["in", "f32", "bf16"])
def test_flat_lists(dtype, max_norm, place):
    gen = torch.Generator().manual_seed(11)
    Gs = lists(gen, dtype, SIZES)
    was = [g.clone() for g in Gs]
    if place == "in":
        out = Gs
        norm, scale = fb.clip_grads(Gs, max_norm)
    else:
        out = [torch.full_like(g, 7.0, dtype={"f32": torch.float32, "bf16": torch.bfloat16}[place]) for g in Gs]
        norm, scale = fb.clip_grads(Gs, max_norm, out=out)
        assert all(torch.equal(g, w) for g, w in zip(Gs, was))
    check(was, out, norm, scale, max_norm)
    alone = fb.grad_norm(was)
    assert alone.shape == norm.shape == scale.shape == () and float(alone) == float(norm)
    if max_norm >= 1e6:
        assert float(scale) == 1.0
        assert all(torch.equal(o, w.to(o.dtype)) for o, w in zip(out, was))


@pytest.mark.parametrize("count", [1, 47, 48, 49, 511, 512, 513, 1100])
def test_lists_of_any_length(count):
    gen = torch.Generator().manual_seed(count)
    Gs = [torch.randn(1 + (37 * i) % 3000, generator=gen).to([torch.float32, torch.bfloat16][i % 2]).cuda() for i in range(count)]
    was = [g.clone() for g in Gs]
    norm, scale = fb.clip_grads(Gs, 2.5)
    check(was, Gs, norm, scale, 2.5)


@pytest.mark.parametrize("dtype,out_dtype", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16),
                                             (torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("rows,cols,pitch,out_pitch", [
    (3, 5, 5, 5), (17, 64, 72, 64), (64, 1707, 1712, 1707), (100, 33, 40, 48), (5, 9000, 9008, 9016), (300, 1, 8, 3), (2, 4099, 4101, 4103)])
def test_pitched_rows(dtype, out_dtype, rows, cols, pitch, out_pitch):
    """Rows with elements behind them that are neither read (NaN there) nor written."""
    gen = torch.Generator().manual_seed(5)
    wide = torch.full((rows, pitch), float("nan"), dtype=dtype, device="cuda")
    wide[:, :cols] = torch.randn(rows, cols, generator=gen).to(dtype).cuda()
    other = torch.randn(100, generator=gen).cuda()
    into = torch.full((rows, out_pitch), 3.0, dtype=out_dtype, device="cuda")
    into_other = torch.empty_like(other)
    norm, scale = fb.clip_grads([wide[:, :cols], other], 0.5, out=[into[:, :cols], into_other])
    check([wide[:, :cols], other], [into[:, :cols], into_other], norm, scale, 0.5)
    assert bool((into[:, cols:] == 3.0).all())
    was = wide.clone()
    norm, scale = fb.clip_grads([wide[:, :cols], other.clone()], 0.5)
    check([was[:, :cols], other], [wide[:, :cols], into_other], norm, scale, 0.5)
    assert bool(wide[:, cols:].isnan().all())


def test_lists_read_natively_and_in_python_are_the_same(monkeypatch):
    """The two ways to the library's arrays; what the native one leaves to the other, it does not touch."""
    pytest.importorskip("paper_2410_01623_b200._native_lists")
    gen = torch.Generator().manual_seed(7)
    f32 = [torch.randn(s, generator=gen).cuda() for s in ((3, 4), (7,), (0,), (), (2, 3, 5))]
    mixed = [g.to([torch.float32, torch.bfloat16][i % 2]) for i, g in enumerate(f32)]
    cases = [(f32, None), (mixed, None), (tuple(mixed), f32), (f32, [g.bfloat16() for g in f32])]
    native = [fb._native_grad_list(*c) for c in cases]
    assert all(x is not None and len(x) == 4 for x in native)
    flat = torch.zeros(4, 6, device="cuda")
    for other in ([flat[:, :3]], [flat.t()], [flat.half()], [flat.cpu()], [flat, flat.cpu()], [], iter([flat]), [1], [None]):
        assert fb._native_grad_list(other, None) is None
    assert fb._native_grad_list([flat], [flat.t()]) is None and fb._native_grad_list([flat], []) is None
    monkeypatch.setattr(fb, "_native_grad_list", lambda Gs, out: None)
    assert [fb._grad_list(*c) for c in cases] == native
    norm = fb.grad_norm(mixed)
    monkeypatch.undo()
    assert float(fb.grad_norm(mixed)) == float(norm)


def test_transposed_and_column_sliced_gradients():
    gen = torch.Generator().manual_seed(6)
    whole = torch.randn(96, 80, generator=gen).cuda()
    parts = [whole[:, :33], whole[:, 33:], torch.randn(40, 24, generator=gen).cuda().t(), torch.randn(24, 40, generator=gen).cuda()]
    was = [p.clone() for p in parts]
    out = [torch.empty_like(p) for p in parts]
    assert out[2].stride() == parts[2].stride()
    check(was, out, *fb.clip_grads(parts, 3.0, out=out), 3.0)
    check(was, parts, *fb.clip_grads(parts, 3.0), 3.0)


@pytest.mark.parametrize("dtype,shift", [(torch.float32, 1), (torch.float32, 3), (torch.bfloat16, 1), (torch.bfloat16, 7)])
def test_tensors_off_the_16_byte_boundaries(dtype, shift):
    gen = torch.Generator().manual_seed(8)
    buf = torch.randn(40000, generator=gen).to(dtype).cuda()
    Gs = [buf[shift:10001], buf[10001:10001 + 8192], buf[20000 + shift:]]
    was = [g.clone() for g in Gs]
    keep = buf.clone()
    check(was, Gs, *fb.clip_grads(Gs, 1.0), 1.0)
    outside = torch.ones(40000, dtype=torch.bool)
    outside[shift:10001 + 8192] = False
    outside[20000 + shift:] = False
    assert torch.equal(buf.cpu()[outside], keep.cpu()[outside])


@pytest.mark.parametrize("dtype,out_dtype", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16),
                                             (torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("shift,out_shift", [(1, 1), (3, 3), (0, 1), (2, 0), (5, 5), (3, 7), (1, 5)])
@pytest.mark.parametrize("rows,cols,pitch", [(1, 40000, 40000), (1, 5, 5), (50, 500, 504), (2, 9000, 9008), (30, 3, 8)])
def test_tensors_that_begin_anywhere(dtype, out_dtype, shift, out_shift, rows, cols, pitch):
    """G and out begin elsewhere between two 16-byte boundaries, alike or not; what lies around them stays."""
    gen = torch.Generator().manual_seed(rows)
    buf = torch.full((shift + rows * pitch + 16,), float("nan"), dtype=dtype, device="cuda")
    into = torch.full((out_shift + rows * pitch + 16,), 4.0, dtype=out_dtype, device="cuda")
    G = buf[shift:shift + rows * pitch].view(rows, pitch)[:, :cols]
    out = into[out_shift:out_shift + rows * pitch].view(rows, pitch)[:, :cols]
    G.copy_(torch.randn(rows, cols, generator=gen))
    was = G.clone()
    check([was], [out], *fb.clip_grads([G], 1.0, out=[out]), 1.0)
    outside = torch.ones_like(into, dtype=torch.bool)
    outside[out_shift:out_shift + rows * pitch].view(rows, pitch)[:, :cols] = False
    assert bool((into[outside] == 4.0).all()) and torch.equal(G, was)
    check([was], [G], *fb.clip_grads([G], 1.0), 1.0)
    outside = torch.ones_like(buf, dtype=torch.bool)
    outside[shift:shift + rows * pitch].view(rows, pitch)[:, :cols] = False
    assert bool(buf[outside].isnan().all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", [1e-38, 1e-30, 1e-22, 1e-19, 1e15, 1e19, 1e25, 1e36])
def test_the_range_of_the_types(dtype, size):
    """Squares that underflow or overflow in fp32 do not reach the norm."""
    gen = torch.Generator().manual_seed(9)
    Gs = [(torch.rand(n, generator=gen) + 0.5).mul(size).to(dtype).cuda() for n in (1, 31, 4096)]
    mixed = torch.zeros(9000, dtype=dtype, device="cuda")
    mixed[17] = size
    Gs.append(mixed)
    want = exact(Gs, 1.0)[0]
    assert abs(float(fb.grad_norm(Gs)) - want) <= NORM * want + 2.0 ** -150      # (the last: half a step of the smallest floats)
    max_norm = float(np.float32(0.25 * want))
    if max_norm > 1e-37:
        was = [g.clone() for g in Gs]
        check(was, Gs, *fb.clip_grads(Gs, max_norm), max_norm)


def test_large_and_small_in_one_tile():
    g = torch.full((64,), 1e-30, device="cuda")
    g[3] = 1e30
    assert abs(float(fb.grad_norm([g])) / 1e30 - 1) <= NORM + U
    z = torch.zeros(100000, device="cuda")
    assert float(fb.grad_norm([z])) == 0.0
    norm, scale = fb.clip_grads([z], 1.0)
    assert float(norm) == 0.0 and float(scale) == 1.0 and not z.any()


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norms_that_are_not_finite_leave_the_gradients(bad, dtype):
    Gs = [torch.full((5000,), 2.0, dtype=dtype, device="cuda"), torch.full((33,), 1.0, dtype=dtype, device="cuda")]
    Gs[0][4321] = bad
    was = [g.clone() for g in Gs]
    norm, scale = fb.clip_grads(Gs, 1.0)
    assert float(scale) == 1.0
    assert math.isnan(float(norm)) if math.isnan(bad) else float(norm) == math.inf
    assert all(torch.equal(g.nan_to_num(nan=5.0), w.nan_to_num(nan=5.0)) for g, w in zip(Gs, was))
    out = [torch.zeros_like(g) for g in Gs]
    fb.clip_grads(Gs, 1.0, out=out)
    assert all(torch.equal(g.nan_to_num(nan=5.0), w.nan_to_num(nan=5.0)) for g, w in zip(out, was))


def test_an_empty_tensor_alone():
    norm, scale = fb.clip_grads([torch.zeros(0, device="cuda"), torch.zeros(0, 5, device="cuda")], 1.0)
    assert float(norm) == 0.0 and float(scale) == 1.0


def test_the_same_call_gives_the_same_bits():
    gen = torch.Generator(device="cuda").manual_seed(3)
    Gs = [torch.randn(n, generator=gen, device="cuda") for n in (3_000_001, 12345, 1 << 20)]
    norms = {float(fb.grad_norm(Gs)) for _ in range(20)}
    assert len(norms) == 1


def test_captured_and_replayed_on_another_stream():
    gen = torch.Generator(device="cuda").manual_seed(4)
    Gs = [torch.randn(n, generator=gen, device="cuda") for n in (100_000, 77)]
    out = [torch.empty_like(g) for g in Gs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    fb.grad_norm(Gs)
    with torch.cuda.graph(graph, stream=side):
        norm, scale = fb.clip_grads(Gs, 1.0, out=out)
    for k in range(3):
        for g in Gs:
            g.mul_(1.5 + k)
        graph.replay()
        check(Gs, out, norm, scale, 1.0)
    with torch.cuda.stream(side):
        norm, scale = fb.clip_grads(Gs, 0.5)
    side.synchronize()
    assert abs(float(fb.grad_norm(Gs)) - 0.5) <= 0.5 * (NORM + SCALE + U)


@pytest.mark.parametrize("count", [60, 500])
def test_a_long_list_captured_and_replayed(count):
    gen = torch.Generator(device="cuda").manual_seed(5)
    Gs = [torch.randn(1 + 53 * i, generator=gen, device="cuda").to([torch.float32, torch.bfloat16][i % 2]) for i in range(count)]
    out = [torch.empty_like(g) for g in Gs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm, scale = fb.clip_grads(Gs, 1.0, out=out)
    for _ in range(2):
        for g in Gs:
            g.mul_(0.5)
        graph.replay()
        check(Gs, out, norm, scale, 1.0)


def test_two_calls_at_once_on_two_streams():
    gen = torch.Generator(device="cuda").manual_seed(6)
    lists = [[torch.randn(n, generator=gen, device="cuda") for n in (2_000_000, 333)] for _ in range(2)]
    outs = [[torch.empty_like(g) for g in Gs] for Gs in lists]
    streams = [torch.cuda.Stream() for _ in lists]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        got = []
        for Gs, out, stream in zip(lists, outs, streams):
            with torch.cuda.stream(stream):
                got.append(fb.clip_grads(Gs, 2.0, out=out))
    torch.cuda.synchronize()
    for Gs, out, (norm, scale) in zip(lists, outs, got):
        check(Gs, out, norm, scale, 2.0)


def test_many_elements_in_one_tensor():
    """Offsets beyond 2^32 bytes, and beyond 2^31 elements."""
    n = (1 << 31) + 12345
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[-5] = 3.0
    g[7] = 4.0
    norm, scale = fb.clip_grads([g], 1.0)
    assert float(norm) == 5.0
    assert abs(float(g[-5]) - 0.6) <= 0.6 * 2.0 ** -8 + 1e-6 and abs(float(g[7]) - 0.8) <= 0.8 * 2.0 ** -8 + 1e-6
