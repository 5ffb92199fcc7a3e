"""The operators in the order in which a training program calls them: lookup and norm forward, the rest of the model by
torch, norm and table backward over two micro-batches, one norm over projected and unprojected gradients, clipping, and
the two optimizer steps.  Gradients are held to 64-bit automatic differentiation of the same model at the same
parameters, the clipped list to the definition, the steps to the oracle.

Tolerances.  Gradients, as Frobenius norms per parameter: fp32 products and sums over at most 96 terms here, about
sqrt(96) 2^-24 each and a handful of them one behind another, 1e-5 allowed.  The factor and the clipped gradients: 20 roundings of
2^-24 (the norm's 16, as a sum of 32 squares per thread, its own, max_norm's, the factor's, the product's).  Steps: 1e-5 of the weights, as the
other fp32 tests have."""
import math

import numpy as np
import pytest
import torch

from oracle import fira_oracle as fo
from paper_2410_01623_b200 import binding as fb
from tests.parity_util import oracle_hyper, rel_err, to_np64

pytestmark = pytest.mark.gpu

VOCAB, HIDDEN, INNER, RANK, BATCH, LENGTH = 131, 64, 96, 8, 6, 17
U = 2.0 ** -24
EMBED_SCALE, EPS, MAX_NORM = 8.0, 1e-6, 0.5


def loss64(params, tokens, targets):
    """The model in 64 bits: scaled lookup, RMS norm, two projected matrices with a tanh, layer norm, head."""
    E, g1, W1, W2, g2, b2, head = params
    keep = tokens >= 0
    x = torch.where(keep[..., None], E[tokens.clamp_min(0)] * EMBED_SCALE, 0.0).reshape(-1, HIDDEN)
    h = x / torch.sqrt(x.square().mean(1, keepdim=True) + EPS) * g1
    z = x + torch.tanh(h @ W1) @ W2
    n = torch.nn.functional.layer_norm(z, (HIDDEN,), g2, b2, EPS)
    logits = (n @ head.T)[keep.reshape(-1)]
    return torch.nn.functional.cross_entropy(logits, targets[keep], reduction="sum")


def backward(p, tokens, targets, into, first):
    """The same model's gradients by the library's operators and torch, added to `into` unless it is the first micro-batch."""
    E, g1, W1, W2, g2, b2, head = p
    keep = tokens >= 0
    x = fb.embedding(E, tokens, scale=EMBED_SCALE).view(-1, HIDDEN)
    h, _, r1 = fb.layer_norm(x, g1, eps=EPS, rms=True)
    a = torch.tanh(h @ W1)
    z = x + a @ W2
    n, m2, r2 = fb.layer_norm(z, g2, b2, eps=EPS)
    logits = n @ head.T
    dlogits = torch.softmax(logits, 1)
    rows = keep.reshape(-1).nonzero()[:, 0]
    dlogits[rows, targets.reshape(-1)[rows]] -= 1.0
    dlogits[~keep.reshape(-1)] = 0.0
    add = not first
    dE, dg1, dW1, dW2, dg2, db2, dhead = into
    dn = dlogits @ head
    dz, _, _ = fb.layer_norm_grad(dn, z, g2, m2, r2, dgain=dg2, dbias=db2, accumulate=add)
    da = (dz @ W2.T) * (1 - a.square())
    dh = da @ W1.T
    for g, new in ((dhead, dlogits.T @ n), (dW2, a.T @ dz), (dW1, h.T @ da)):
        g.add_(new) if add else g.copy_(new)
    dx, _, _ = fb.layer_norm_grad(dh, x, g1, None, r1, rms=True, dgain=dg1, accumulate=add)
    fb.embedding_grad(tokens, (dx + dz).view(*tokens.shape, HIDDEN), VOCAB, scale=EMBED_SCALE, out=dE, accumulate=add)


def test_training_steps():
    gen = torch.Generator().manual_seed(21)
    shapes = [(VOCAB, HIDDEN), (HIDDEN,), (HIDDEN, INNER), (INNER, HIDDEN), (HIDDEN,), (HIDDEN,), (VOCAB, HIDDEN)]
    p = [torch.randn(s, generator=gen).mul_(0.1).cuda() for s in shapes]
    for k in (1, 4):
        p[k].add_(1.0)
    projected, dense = [2, 3], [0, 1, 4, 5, 6]
    hp = fb.make_hparams(lr=1e-3, alpha=0.5)
    f = fb.Fira([shapes[k] for k in projected], RANK, torch.float32, hp)
    ohp = oracle_hyper(hp)
    moments = [[torch.zeros_like(p[k]) for k in dense] for _ in range(2)]
    states = {k: fo.new_state(*shapes[k], RANK) for k in projected}
    states.update({k: fo.State(M=np.zeros(shapes[k]), V=np.zeros(shapes[k])) for k in dense})
    grads = [torch.full_like(q, float("nan")) for q in p]
    clipped = 0
    for t in range(4):
        batches = []
        for k in range(2):
            tokens = torch.randint(0, VOCAB, (BATCH, LENGTH), generator=gen)
            tokens[torch.arange(LENGTH) >= torch.randint(5, LENGTH + 1, (BATCH, 1), generator=gen)] = -1
            batches.append((tokens.cuda(), torch.randint(0, VOCAB, (BATCH, LENGTH), generator=gen).cuda()))
        for k, (tokens, targets) in enumerate(batches):
            backward(p, tokens, targets, grads, k == 0)
        leaves = [q.double().requires_grad_() for q in p]
        sum(loss64(leaves, *b) for b in batches).backward()
        for k, (g, leaf) in enumerate(zip(grads, leaves)):
            assert float((g.double() - leaf.grad).norm()) <= 1e-5 * float(leaf.grad.norm()), (t, k)
        total = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
        max_norm = MAX_NORM * total if t != 2 else 2.0 * total          # (the third step is not clipped)
        out = [torch.empty_like(g) for g in grads]
        norm, scale = fb.clip_grads(grads, max_norm, out=out)
        want = min(1.0, max_norm / total)
        clipped += want < 1
        assert abs(float(norm) - total) <= 20 * U * total and abs(float(scale) - want) <= 20 * U * want
        for g, o in zip(grads, out):
            assert bool(((o.double() - g.double() * want).abs() <= 20 * U * g.double().abs() * want).all())
        if t == 0:
            f.refresh_projection([out[k] for k in projected])
        before = [to_np64(q) for q in p]
        f.step([p[k] for k in projected], [out[k] for k in projected])
        fb.adam_dense(hp, [p[k] for k in dense], [out[k] for k in dense], *moments, t)
        for i, k in enumerate(projected):
            W, _ = fo.fira_step(before[k], to_np64(out[k]), to_np64(f.get_projection(i)), states[k], ohp, store="f32")
            assert rel_err(to_np64(p[k]), W) <= 1e-5, (t, k)
        for k in dense:
            W = fo.adam_dense_step(before[k], to_np64(out[k]), states[k], ohp, store="f32")
            assert rel_err(to_np64(p[k]), W) <= 1e-5, (t, k)
    assert clipped == 3
    assert f.poll() == 0
    f.close()


def test_bf16_gradients_summed_in_fp32_are_clipped_into_bf16():
    """Two micro-batches of bf16 activations whose gradients are summed in fp32, clipped into bf16 and stepped."""
    gen = torch.Generator().manual_seed(22)
    E = torch.randn(VOCAB, HIDDEN, generator=gen).to(torch.bfloat16).cuda()
    gain = (1 + 0.1 * torch.randn(HIDDEN, generator=gen)).to(torch.bfloat16).cuda()
    dE, dgain = torch.zeros(VOCAB, HIDDEN, device="cuda"), torch.zeros(HIDDEN, device="cuda")
    wantE, want_gain = torch.zeros(VOCAB, HIDDEN, dtype=torch.float64), torch.zeros(HIDDEN, dtype=torch.float64)
    for _ in range(2):
        tokens = torch.randint(-1, VOCAB, (BATCH, LENGTH), generator=gen).cuda()
        x = fb.embedding(E, tokens)
        y, _, rstd = fb.layer_norm(x, gain, eps=EPS, rms=True)
        dY = torch.randn(x.shape, generator=gen).to(torch.bfloat16).cuda()
        dx, _, _ = fb.layer_norm_grad(dY, x, gain, None, rstd, rms=True, dgain=dgain, accumulate=True)
        fb.embedding_grad(tokens, dx, VOCAB, out=dE, accumulate=True)
        keep = (tokens >= 0).reshape(-1).cpu()
        wantE.index_add_(0, tokens.reshape(-1).cpu()[keep], dx.double().reshape(-1, HIDDEN).cpu()[keep])
        want_gain += (dY.double() * x.double() * rstd.double()[..., None]).reshape(-1, HIDDEN).sum(0).cpu()
    # sums of up to 204 terms in fp32: 204 roundings of 2^-24 of their absolute values, which are below 20 each
    assert float((dE.double().cpu() - wantE).abs().max()) <= 204 * U * 204 * 20
    assert float((dgain.double().cpu() - want_gain).abs().max()) <= 208 * U * 204 * 20
    out = [torch.empty_like(E), torch.empty_like(gain)]
    norm, scale = fb.clip_grads([dE, dgain], 1.0, out=out)
    total = math.sqrt(float(dE.double().square().sum()) + float(dgain.double().square().sum()))
    assert total > 1 and abs(float(scale) - 1 / total) <= 20 * U / total
    for g, o in zip((dE, dgain), out):
        assert bool(((o.double() - g.double() / total).abs() <= (2.0 ** -8 + 20 * U) * g.double().abs() / total + 1e-40).all())
    M, V = [torch.zeros_like(o, dtype=torch.float32) for o in out], [torch.zeros_like(o, dtype=torch.float32) for o in out]
    before = [E.clone(), gain.clone()]
    fb.adam_dense(fb.make_hparams(lr=1e-2), [E, gain], out, M, V, 0)
    assert all(bool((a != b).any()) and bool(a.isfinite().all()) for a, b in zip((E, gain), before))
