"""GPU parity of fira_layer_norm and fira_layer_norm_grad with the formulas in 64 bits, and of the gradients with differences.

Tolerances.  U = 2^-24.  A thread adds at most 16 elements of a row one after another, then come at most ten levels of
a tree (two more for safety): a sum over a row is within D U of itself in absolute values, D = 28.  So mu is within
(D + 1) U mean|x|; a difference to it, squared and summed, is within (D + 3) U relative to the variance (and the square of
mu's own error, which is added), s within half of that and 3 U, and the output's own three operations follow.  The backward pass is
held to the formula with the statistics that it is given: products and sums as above.  A sum over R rows is R fp32
additions in some fixed order: R U of its absolute values.  Storage: 2^-24 (fp32), 2^-8 (bf16) of the result."""
import pytest
import torch

from paper_2410_01623_b200 import binding as fb

pytestmark = pytest.mark.gpu

U, D = 2.0 ** -24, 28
STORE = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
F32, BF16, F64 = torch.float32, torch.bfloat16, torch.float64


def inputs(rows, hidden, dtype, param_dtype, seed=0, shift=0.5):
    gen = torch.Generator().manual_seed(seed)
    scale = torch.exp(0.7 * torch.randn(hidden, generator=gen))
    x = (torch.randn(rows, hidden, generator=gen) * scale + shift * torch.randn(rows, 1, generator=gen)).to(dtype).cuda()
    dY = (torch.randn(rows, hidden, generator=gen) * 1e-2).to(dtype).cuda()
    gain = (1 + 0.3 * torch.randn(hidden, generator=gen)).to(param_dtype).cuda()
    bias = torch.randn(hidden, generator=gen).to(param_dtype).cuda()
    return x, dY, gain, bias


def within(got, want, allow):
    return bool(((got.to(F64) - want).abs() <= allow * 1.01 + STORE[got.dtype] * want.abs() + 1e-40).all())


def check_forward(x, gain, bias, eps, rms, y, mean, rstd):
    u, g = x.to(F64).reshape(-1, x.shape[-1]), gain.to(F64)
    h = u.shape[1]
    mu = torch.zeros_like(u[:, :1]) if rms else u.mean(1, keepdim=True)
    dmu = 0.0 * mu if rms else (D + 1) * U * u.abs().mean(1, keepdim=True)
    d = u - mu
    var = d.square().mean(1, keepdim=True)
    s = 1 / torch.sqrt(var + eps)
    ds = s * (((D + 3) * U * var + dmu ** 2) / (2 * (var + eps)) + 3 * U)
    if not rms:
        assert within(mean.reshape(-1, 1), mu, dmu)
    assert within(rstd.reshape(-1, 1), s, ds)
    b = 0.0 if bias is None else bias.to(F64)
    want = d * s * g + b
    allow = g.abs() * (s * (dmu + U * d.abs()) + d.abs() * ds) + 3 * U * ((d * s * g).abs() + (0.0 if bias is None else b.abs()))
    assert within(y.reshape(-1, h), want, allow)


def check_backward(dY, x, gain, mean, rstd, rms, dX, dgain, dbias, old=None):
    u, dy, g = (t.to(F64).reshape(-1, x.shape[-1]) for t in (x, dY, gain))
    s = rstd.to(F64).reshape(-1, 1)
    h = (u if rms else u - mean.to(F64).reshape(-1, 1)) * s
    q = dy * g
    level = 0.0 if rms else q.mean(1, keepdim=True)
    along = (q * h).mean(1, keepdim=True)
    dx = s * (q - level - h * along)
    dlevel = 0.0 if rms else (D + 2) * U * q.abs().mean(1, keepdim=True)
    dalong = (D + 5) * U * (q * h).abs().mean(1, keepdim=True)
    size = q.abs() + (0.0 if rms else level.abs()) + (h * along).abs()
    allow = s * (dlevel + h.abs() * dalong + 5 * U * size)
    assert within(dX.reshape(dx.shape), dx, allow)
    R = u.shape[0]
    for name, got, terms in (("dgain", dgain, dy * h), ("dbias", dbias, dy)):
        if got is None:
            continue
        want, allow = terms.sum(0), (R + 4) * U * terms.abs().sum(0)
        if old is not None:
            want = want + old[name].to(F64)
            allow = allow + U * want.abs()
        assert within(got, want, allow), name


SHAPES = [(1529, 43), (1000, 21), (700, 100), (333, 200), (4097, 33), (1, 1), (3, 2), (5, 7), (4, 8), (33, 64), (100, 255), (64, 256), (9, 257), (130, 512), (50, 1000), (300, 1024), (77, 1707),
          (40, 2048), (21, 4096), (10, 4100), (6, 5461), (5, 8192), (4, 8200), (3, 11008), (2, 16384), (2, 16383)]


@pytest.mark.parametrize("rows,hidden", SHAPES)
@pytest.mark.parametrize("dtype,param_dtype", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("rms", [False, True])
def test_forward_and_backward(rows, hidden, dtype, param_dtype, rms):
    x, dY, gain, bias = inputs(rows, hidden, dtype, param_dtype, seed=rows)
    if rms:
        bias = None
    y, mean, rstd = fb.layer_norm(x, gain, bias, eps=1e-5, rms=rms)
    assert y.dtype == dtype and rstd.shape == (rows,) and (mean is None) == rms
    check_forward(x, gain, bias, 1e-5, rms, y, mean, rstd)
    dX, dgain, dbias = fb.layer_norm_grad(dY, x, gain, mean, rstd, rms=rms)
    assert dX.dtype == dtype and dgain.dtype == param_dtype and (dbias is None) == rms
    check_backward(dY, x, gain, mean, rstd, rms, dX, dgain, dbias)


@pytest.mark.parametrize("rows,hidden", [(40000, 64), (20001, 512), (9000, 1024), (7001, 1707), (5000, 4096), (2500, 8192)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rms", [False, True])
def test_many_rows(rows, hidden, dtype, rms):
    x, dY, gain, bias = inputs(rows, hidden, dtype, dtype, seed=3)
    y, mean, rstd = fb.layer_norm(x, gain, None, rms=rms)
    check_forward(x, gain, None, 1e-5, rms, y, mean, rstd)
    out = fb.layer_norm_grad(dY, x, gain, mean, rstd, rms=rms)
    check_backward(dY, x, gain, mean, rstd, rms, *out)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("hidden,pitch", [(64, 72), (64, 67), (37, 40), (1, 5), (1707, 1712)])
def test_pitched_rows(dtype, hidden, pitch):
    """What lies behind the rows is neither read nor written."""
    rows = 45
    x, dY, gain, bias = inputs(rows, hidden, dtype, F32)
    wide = [torch.full((rows, pitch), float("nan"), dtype=dtype, device="cuda") for _ in range(2)]
    wide[0][:, :hidden], wide[1][:, :hidden] = x, dY
    out = [torch.full((rows, pitch), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    y, mean, rstd = fb.layer_norm(wide[0][:, :hidden], gain, bias, out=out[0][:, :hidden])
    check_forward(x, gain, bias, 1e-5, False, y, mean, rstd)
    got = fb.layer_norm_grad(wide[1][:, :hidden], wide[0][:, :hidden], gain, mean, rstd, out=out[1][:, :hidden])
    check_backward(dY, x, gain, mean, rstd, False, *got)
    assert bool((out[0][:, hidden:] == 7.0).all()) and bool((out[1][:, hidden:] == 7.0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("hidden", [64, 1707])
def test_in_place(dtype, hidden):
    x, dY, gain, bias = inputs(70, hidden, dtype, dtype)
    y, mean, rstd = fb.layer_norm(x, gain, bias)
    z = x.clone()
    assert fb.layer_norm(z, gain, bias, out=z)[0] is z and torch.equal(z, y)
    want = fb.layer_norm_grad(dY, x, gain, mean, rstd)
    for over in ("dY", "x"):
        a = dict(dY=dY.clone(), x=x.clone())
        got = fb.layer_norm_grad(a["dY"], a["x"], gain, mean, rstd, out=a[over])
        assert got[0] is a[over] and all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("grad_dtype", [F32, BF16])
@pytest.mark.parametrize("rms", [False, True])
def test_accumulation(grad_dtype, rms):
    x, dY, gain, bias = inputs(500, 96, BF16, BF16)
    y, mean, rstd = fb.layer_norm(x, gain, None, rms=rms)
    old = dict(dgain=torch.randn(96, device="cuda").to(grad_dtype), dbias=torch.randn(96, device="cuda").to(grad_dtype))
    dgain, dbias = old["dgain"].clone(), None if rms else old["dbias"].clone()
    got = fb.layer_norm_grad(dY, x, gain, mean, rstd, rms=rms, dgain=dgain, dbias=dbias, accumulate=True)
    assert got[1] is dgain
    check_backward(dY, x, gain, mean, rstd, rms, *got, old=old)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shifts", [(1, 1, 1, 1), (0, 1, 0, 1), (3, 3, 2, 3), (1, 2, 3, 0)])
@pytest.mark.parametrize("hidden", [16, 37, 520, 4097])
def test_rows_that_begin_anywhere(dtype, shifts, hidden):
    """x, y, dY and dX each begin elsewhere between two 16-byte boundaries, alike or not; what lies around them stays."""
    rows = 37
    x, dY, gain, bias = inputs(rows, hidden, dtype, F32, seed=hidden)
    flat = [torch.full((rows * hidden + 16,), 6.0, dtype=dtype, device="cuda") for _ in range(4)]
    xs, ys, dys, dxs = [f[k:k + rows * hidden].view(rows, hidden) for f, k in zip(flat, shifts)]
    xs.copy_(x)
    dys.copy_(dY)
    y, mean, rstd = fb.layer_norm(xs, gain, bias, out=ys)
    check_forward(x, gain, bias, 1e-5, False, y, mean, rstd)
    check_backward(dY, x, gain, mean, rstd, False, *fb.layer_norm_grad(dys, xs, gain, mean, rstd, out=dxs))
    assert torch.equal(xs, x) and torch.equal(dys, dY)
    for f, k in zip(flat, shifts):
        assert bool((f[:k] == 6.0).all()) and bool((f[k + rows * hidden:] == 6.0).all())


def test_backward_pass_without_the_bias_gradient():
    x, dY, gain, bias = inputs(200, 72, F32, F32)
    y, mean, rstd = fb.layer_norm(x, gain, bias)
    want = fb.layer_norm_grad(dY, x, gain, mean, rstd)
    dX, dgain = torch.empty_like(x), torch.empty_like(gain)
    L = fb.lib()
    work = torch.empty(L.fira_layer_norm_grad_work_bytes(200, 72, 0), dtype=torch.uint8, device="cuda")
    fb.check(L.fira_layer_norm_grad(dY.data_ptr(), 0, x.data_ptr(), 0, 0, 200, 72, gain.data_ptr(), 0, mean.data_ptr(), rstd.data_ptr(),
                                    dX.data_ptr(), 0, dgain.data_ptr(), None, 0, 0, work.data_ptr(), work.nbytes,
                                    torch.cuda.current_stream().cuda_stream))
    assert torch.equal(dX, want[0]) and torch.equal(dgain, want[1])


def test_more_dimensions_and_no_rows():
    x, dY, gain, bias = inputs(60, 40, F32, F32)
    y, mean, rstd = fb.layer_norm(x.view(3, 20, 40), gain, bias)
    assert y.shape == (3, 20, 40) and mean.shape == rstd.shape == (3, 20)
    check_forward(x, gain, bias, 1e-5, False, y, mean, rstd)
    got = fb.layer_norm_grad(dY.view(3, 20, 40).transpose(0, 1).contiguous().transpose(0, 1), x.view(3, 20, 40), gain, mean, rstd)
    check_backward(dY, x, gain, mean, rstd, False, *got)
    one = fb.layer_norm(x[0], gain, bias)
    assert one[0].shape == (40,) and torch.equal(one[0], y[0, 0]) and one[2].shape == ()
    empty = x[:0]
    y, mean, rstd = fb.layer_norm(empty, gain, bias)
    assert y.shape == (0, 40) and mean.shape == rstd.shape == (0,)
    dX, dgain, dbias = fb.layer_norm_grad(empty, empty, gain, mean, rstd)
    assert dX.shape == (0, 40) and not dgain.any() and not dbias.any()
    kept = torch.ones(40, device="cuda")
    fb.layer_norm_grad(empty, empty, gain, None, rstd, rms=True, dgain=kept, accumulate=True)
    assert bool((kept == 1).all())


@pytest.mark.parametrize("rms", [False, True])
def test_rows_of_one_value_and_rows_that_are_not_finite(rms):
    x, dY, gain, bias = inputs(6, 200, F32, F32)
    x[1] = 3.0
    x[2] = 0.0
    x[3, 7] = float("nan")
    x[4, 9] = float("inf")
    y, mean, rstd = fb.layer_norm(x, gain, None, rms=rms)
    check_forward(x[[0, 1, 2, 5]], gain, None, 1e-5, rms, y[[0, 1, 2, 5]], None if rms else mean[[0, 1, 2, 5]], rstd[[0, 1, 2, 5]])
    assert bool(y[3].isnan().all()) and bool(y[4].isnan().any())
    dX = fb.layer_norm_grad(dY, x, gain, mean, rstd, rms=rms)[0]
    assert bool(dX[[0, 1, 2, 5]].isfinite().all()) and bool(dX[3].isnan().any())


def test_a_large_mean_beside_a_small_variance():
    gen = torch.Generator().manual_seed(1)
    x = (1000.0 + torch.randn(50, 1024, generator=gen)).cuda()
    gain = torch.ones(1024, device="cuda")
    y, mean, rstd = fb.layer_norm(x, gain)
    check_forward(x, gain, None, 1e-5, False, y, mean, rstd)


@pytest.mark.parametrize("rms", [False, True])
def test_gradients_against_differences(rms):
    """Central differences of the formula in 64 bits, in every direction of a small case."""
    x, dY, gain, bias = inputs(3, 11, F32, F32)
    dY = dY * 100
    y, mean, rstd = fb.layer_norm(x, gain, None if rms else bias, eps=1e-5, rms=rms)
    got = fb.layer_norm_grad(dY, x, gain, mean, rstd, rms=rms)

    def loss(x, gain, bias):
        d = x if rms else x - x.mean(1, keepdim=True)
        y = d / torch.sqrt(d.square().mean(1, keepdim=True) + 1e-5) * gain + (0.0 if rms else bias)
        return float((y * dY.to(F64)).sum())

    args = [t.to(F64) for t in (x, gain, bias)]
    for k, grad in enumerate(got):
        if grad is None:
            continue
        want = torch.zeros_like(args[k])
        for i in range(want.numel()):
            ends = []
            for step in (1e-5, -1e-5):
                moved = [a.clone() for a in args]
                moved[k].view(-1)[i] += step
                ends.append(loss(*moved))
            want.view(-1)[i] = (ends[0] - ends[1]) / 2e-5
        # the differences are good to about 1e-5^2 of the third derivative, and to 1e-16 / 1e-5 of the loss
        assert float((grad.to(F64) - want).abs().max()) <= 1e-5 * float(want.abs().max())


def test_the_same_call_gives_the_same_bits():
    x, dY, gain, bias = inputs(3000, 640, BF16, F32)
    y, mean, rstd = fb.layer_norm(x, gain, bias)
    first = fb.layer_norm_grad(dY, x, gain, mean, rstd)
    for _ in range(10):
        assert all(torch.equal(a, b) for a, b in zip(fb.layer_norm_grad(dY, x, gain, mean, rstd), first))


def test_captured_and_replayed_on_another_stream():
    x, dY, gain, bias = inputs(300, 320, BF16, BF16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        y, mean, rstd = fb.layer_norm(x, gain, bias)
        got = fb.layer_norm_grad(dY, x, gain, mean, rstd)
    for k in range(3):
        nx, ndy, _, _ = inputs(300, 320, BF16, BF16, seed=10 + k)
        x.copy_(nx)
        dY.copy_(ndy)
        graph.replay()
        check_forward(x, gain, bias, 1e-5, False, y, mean, rstd)
        check_backward(dY, x, gain, mean, rstd, False, *got)


def test_offsets_beyond_32_bits():
    rows, hidden = 530000, 4096
    x = torch.ones(rows, hidden, dtype=BF16, device="cuda")
    x[-1, ::2] = -3.0
    gain = torch.ones(hidden, dtype=BF16, device="cuda")
    y, mean, rstd = fb.layer_norm(x, gain, out=x)
    assert float(mean[-1]) == -1.0 and abs(float(rstd[-1]) - 0.5) <= 1e-5
    assert [float(v) for v in x[-1, :4]] == [-1.0, 1.0, -1.0, 1.0] and not x[:-1].any()
