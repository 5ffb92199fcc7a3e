"""Timed cases of the operators around the two optimizer steps: what makes the gradients of the parameters that are
not projected (embedding table, norm gains), and what looks at all gradients of a step together.

Each is a `kind` here:

  clip           the global norm over a list of gradients, and the list scaled so that the norm is at most max_norm
                 (clip_grads): every iteration, before Fira.step and adam_dense;
  grad_norm      the norm alone (grad_norm);
  lookup         rows of the embedding table for a batch of tokens, times a factor (embedding);
  lookup_grad    the table's gradient from the gradient of those rows (embedding_grad);
  norm           layer norm, or the form without mean and bias that LLaMA models have (layer_norm);
  norm_grad      its backward pass, with the gradients of gain and bias (layer_norm_grad).

A list of gradients is that of a model: per layer four hidden x hidden, two hidden x mlp and one mlp x hidden matrices
and two gains, one gain more, and (vocab > 0) embedding and head.  Token ids follow a Zipf law, as words do, so a few
rows of the table take a large part of the batch; positions behind the end of a sequence hold -1.
"""
from __future__ import annotations

import math

import torch

own = False

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "i32": torch.int32, "i64": torch.int64}
SIZE = {"f32": 4, "bf16": 2, "i32": 4, "i64": 8}
ZIPF = 2.7                                     # token v has a probability in proportion to 1 / (v + ZIPF)


def _clip(layers, hidden, mlp, vocab, dtype, out, limit, kind="clip"):
    """limit: max_norm as a multiple of the norm that is expected (below 1: the gradients are scaled)."""
    return dict(kind=kind, layers=layers, hidden=hidden, mlp=mlp, vocab=vocab, dtype=dtype, out=out, limit=limit)


def _tokens(kind, batch, length, hidden, vocab, dtype, out, index, padding, scale):
    """padding: share of the positions that lie behind the end of their sequence."""
    return dict(kind=kind, batch=batch, length=length, hidden=hidden, vocab=vocab, dtype=dtype, out=out, index=index,
                padding=padding, scale=scale)


def _norm(kind, rows, hidden, dtype, gain, rms):
    return dict(kind=kind, rows=rows, hidden=hidden, dtype=dtype, gain=gain, rms=rms)


def listed():
    cases = [
        # One layer of the smallest model, without its table: ten tensors, the call's latency counts.
        ("clip_1x512_f32", _clip(1, 512, 1376, 0, "f32", "f32", 0.1)),
        # The whole smallest model in fp32, with embedding and head.
        ("clip_8x512_f32", _clip(8, 512, 1376, 32000, "f32", "f32", 0.1)),
        # The 24-layer model with the odd MLP width, bf16: the largest list, far beyond L2.
        ("clip_24x2048_bf16", _clip(24, 2048, 5461, 32000, "bf16", "bf16", 0.1)),
        # Gradients of several micro-batches summed in fp32, clipped into the bf16 that the step reads.
        ("clip_8x1024_f32_to_bf16", _clip(8, 1024, 2736, 32000, "f32", "bf16", 0.1)),
        # The lookup of one short sequence, and of a batch of 512 sequences of 256 tokens.
        ("lookup_1x256_512_f32", _tokens("lookup", 1, 256, 512, 32000, "f32", "f32", "i64", 0.0, 1.0)),
        ("lookup_512x256_1024_bf16", _tokens("lookup", 512, 256, 1024, 32000, "bf16", "bf16", "i64", 0.1, 32.0)),
        # The table's gradient of a micro-batch (its zero rows are most of what is written), and of a whole batch.
        ("lookup_grad_16x256_512_f32", _tokens("lookup_grad", 16, 256, 512, 32000, "f32", "f32", "i64", 0.0, 1.0)),
        ("lookup_grad_512x256_2048_bf16", _tokens("lookup_grad", 512, 256, 2048, 32000, "bf16", "bf16", "i64", 0.1, 1.0)),
        # Layer norm of one short sequence; the form without mean over the tokens of a micro-batch of the largest model.
        ("norm_256x512_f32", _norm("norm", 256, 512, "f32", "f32", False)),
        ("norm_rms_32768x4096_bf16", _norm("norm", 32768, 4096, "bf16", "bf16", True)),
        # Their backward passes: an odd width with bias and fp32 gains; the largest model's.
        ("norm_grad_4096x1707_bf16", _norm("norm_grad", 4096, 1707, "bf16", "f32", False)),
        ("norm_grad_rms_32768x4096_bf16", _norm("norm_grad", 32768, 4096, "bf16", "bf16", True)),
    ]
    return [dict(name=name, **case) for name, case in cases]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _near(rng, x, multiple):
    """x itself or, more often, the multiple nearest to it."""
    return x if rng.random() < 0.4 else max(multiple, x // multiple * multiple)


def draw(rng):
    kind = rng.choice(["clip", "clip", "grad_norm", "lookup", "lookup_grad", "lookup_grad", "norm", "norm_grad", "norm_grad"])
    dtype = rng.choice(["f32", "bf16"])
    if kind in ("clip", "grad_norm"):
        hidden = _near(rng, _log(rng, 24, 4096), 64)
        mlp = _near(rng, int(hidden * rng.uniform(2.0, 3.5)), 16)
        per_layer = 4 * hidden * hidden + 3 * hidden * mlp
        layers = max(1, min(_log(rng, 1, 32), 500_000_000 // per_layer))
        vocab = rng.choice([0, _near(rng, _log(rng, 50, 64000), 64)])
        out = dtype if kind == "grad_norm" or rng.random() < 0.6 else rng.choice(["f32", "bf16"])
        return _clip(layers, hidden, mlp, vocab, dtype, out, rng.choice([0.01, 0.1, 0.9, 2.0]), kind)
    if kind in ("lookup", "lookup_grad"):
        length = _near(rng, _log(rng, 1, 4096), 32)
        batch = max(1, min(_log(rng, 1, 512), 131072 // length))
        hidden = _near(rng, _log(rng, 16, 4096), 64)
        out = dtype if kind == "lookup" or rng.random() < 0.7 else "f32"
        return _tokens(kind, batch, length, hidden, _near(rng, _log(rng, 50, 128000), 64), dtype, out,
                       rng.choice(["i32", "i64"]), rng.choice([0.0, 0.1, 0.5]), rng.choice([1.0, round(math.sqrt(hidden), 3)]))
    hidden = _near(rng, _log(rng, 16, 12000), 64)
    rows = max(1, min(_log(rng, 1, 65536), 134_000_000 // hidden))
    return _norm(kind, rows, hidden, dtype, rng.choice([dtype, "f32"]), rng.random() < 0.5)


# ------------------------------------------------------------------------------------------ inputs
def _shapes(case):
    h, f = case["hidden"], case["mlp"]
    per_layer = [(h, h)] * 4 + [(h, f)] * 2 + [(f, h)] + [(h,)] * 2
    return per_layer * case["layers"] + [(h,)] + ([(case["vocab"], h)] * 2 if case["vocab"] else [])


def _places(shapes):
    """Where each tensor lies in one buffer (each starts on a 256-byte boundary), and the buffer's length."""
    places, total = [], 0
    for shape in shapes:
        places.append((total, shape))
        total += (math.prod(shape) + 127) // 128 * 128
    return places, total


def _views(flat, places):
    return [flat[at:at + math.prod(shape)].view(shape) for at, shape in places]


def _zipf(u, vocab):
    """Token ids from uniform numbers: the inverse of the distribution function, log-linear."""
    return (ZIPF * ((vocab + ZIPF) / ZIPF) ** u - ZIPF).long().clamp_(0, vocab - 1)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, dt = case["kind"], TORCH[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    if kind in ("clip", "grad_norm"):
        places, total = _places(_shapes(case))
        flat = torch.zeros(total, dtype=dt, device="cuda")
        G = _views(flat, places)
        squares = 0.0
        for g in G:                            # one scale per column, and one per tensor
            c = torch.exp(0.5 * normal(g.shape[-1])) * (1e-3 * math.exp(0.5 * math.sin(len(g) + g.shape[-1])))
            g.copy_(normal(*g.shape).mul_(c))
            squares = squares + g.shape[0] * c.square().sum() if g.dim() == 2 else squares + c.square().sum()
        expected = float(torch.sqrt(squares))
        state = dict(case=case, G=G, max_norm=case["limit"] * expected, flat=flat)
        if kind == "clip":
            state["flat_out"] = torch.zeros(total, dtype=TORCH[case["out"]], device="cuda")
            state["out"] = _views(state["flat_out"], places)
        return state
    if kind in ("lookup", "lookup_grad"):
        b, s, h, v = case["batch"], case["length"], case["hidden"], case["vocab"]
        tokens = _zipf(torch.rand(b, s, generator=gen, device="cuda", dtype=torch.float64), v)
        if case["padding"]:                    # the sequences end between (1 - 2 padding) of the length and all of it
            ends = s - (torch.rand(b, 1, generator=gen, device="cuda") * (2 * case["padding"] * s)).long()
            tokens = torch.where(torch.arange(s, device="cuda") < ends, tokens, -1)
        tokens = tokens.to(TORCH[case["index"]])
        if kind == "lookup":
            return dict(case=case, tokens=tokens, table=normal(v, h).mul_(0.02).to(dt))
        return dict(case=case, tokens=tokens, dY=normal(b, s, h).mul_(1e-3).to(dt),
                    G=torch.empty(v, h, dtype=TORCH[case["out"]], device="cuda"))
    rows, h, gt = case["rows"], case["hidden"], TORCH[case["gain"]]
    # the residual stream: channels of unequal size, an offset per row
    x = normal(rows, h).mul_(torch.exp(0.7 * normal(h))).add_(0.3 * normal(rows, 1)).to(dt)
    gain = (1.0 + 0.2 * normal(h)).to(gt)
    bias = None if case["rms"] else (0.1 * normal(h)).to(gt)
    if kind == "norm":
        return dict(case=case, x=x, gain=gain, bias=bias)
    y, mean, rstd = _plain_norm(x, gain, bias, case["rms"])
    return dict(case=case, x=x, gain=gain, mean=mean, rstd=rstd, dY=normal(rows, h).mul_(1e-3).to(dt))


EPS = 1e-6


def _plain_norm(x, gain, bias, rms):
    u = x.float()
    mean = None if rms else u.mean(dim=1)
    if not rms:
        u = u - mean[:, None]
    rstd = torch.rsqrt(u.square().mean(dim=1) + EPS)
    y = u * rstd[:, None] * gain.float()
    if bias is not None:
        y = y + bias.float()
    return y.to(x.dtype), mean, rstd


def _plain(state):
    case = state["case"]
    kind = case["kind"]
    if kind in ("clip", "grad_norm"):
        norm = torch.stack([g.float().square().sum(dtype=torch.float64) for g in state["G"]]).sum().sqrt()
        if kind == "grad_norm":
            return dict(norm=norm.float())
        scale = torch.where(torch.isfinite(norm), state["max_norm"] / norm.clamp_min(state["max_norm"]), 1.0).float()
        [o.copy_(g.float() * scale) for g, o in zip(state["G"], state["out"])]
        return dict(out=state["flat_out"], norm=norm.float(), scale=scale)
    if kind == "lookup":
        tokens = state["tokens"].long()
        rows = state["table"][tokens.clamp_min(0)].float() * case["scale"]
        return dict(Y=torch.where((tokens >= 0)[..., None], rows, 0.0).to(state["table"].dtype))
    if kind == "lookup_grad":
        tokens = state["tokens"].reshape(-1).long()
        rows = torch.where((tokens >= 0)[:, None], state["dY"].reshape(-1, case["hidden"]).float(), 0.0)
        G = torch.zeros(case["vocab"], case["hidden"], device=rows.device).index_add_(0, tokens.clamp_min(0), rows)
        state["G"].copy_(G * case["scale"])
        return dict(G=state["G"])
    if kind == "norm":
        y, mean, rstd = _plain_norm(state["x"], state["gain"], state["bias"], case["rms"])
        return dict(Y=y, mean=mean, rstd=rstd)
    x, dY, rstd = state["x"].float(), state["dY"].float(), state["rstd"][:, None]
    xh = (x if case["rms"] else x - state["mean"][:, None]) * rstd
    q = dY * state["gain"].float()
    dx = q - xh * (q * xh).mean(dim=1, keepdim=True)
    if not case["rms"]:
        dx = dx - q.mean(dim=1, keepdim=True)
    out = dict(dX=(dx * rstd).to(state["x"].dtype), dgain=(dY * xh).sum(dim=0).to(state["gain"].dtype))
    if not case["rms"]:
        out["dbias"] = dY.sum(dim=0).to(state["gain"].dtype)
    return out


def run(state):
    if not own:
        return _plain(state)
    from paper_2410_01623_b200 import binding as fb
    case = state["case"]
    kind = case["kind"]
    if kind == "grad_norm":
        return dict(norm=fb.grad_norm(state["G"]))
    if kind == "clip":
        norm, scale = fb.clip_grads(state["G"], state["max_norm"], out=state["out"])
        return dict(out=state["flat_out"], norm=norm, scale=scale)
    if kind == "lookup":
        return dict(Y=fb.embedding(state["table"], state["tokens"], scale=case["scale"]))
    if kind == "lookup_grad":
        return dict(G=fb.embedding_grad(state["tokens"], state["dY"], case["vocab"], scale=case["scale"], out=state["G"]))
    if kind == "norm":
        y, mean, rstd = fb.layer_norm(state["x"], state["gain"], state["bias"], eps=EPS, rms=case["rms"])
        return dict(Y=y, mean=mean, rstd=rstd)
    dx, dgain, dbias = fb.layer_norm_grad(state["dY"], state["x"], state["gain"], state["mean"], state["rstd"],
                                          rms=case["rms"])
    out = dict(dX=dx, dgain=dgain)
    if not case["rms"]:
        out["dbias"] = dbias
    return out


# ------------------------------------------------------------------------------------------ what the cases are held to
def _distinct(case):
    """The expected number of different tokens in the batch, and the number of positions that hold one."""
    n = case["batch"] * case["length"] * (1 - case["padding"])
    v = torch.arange(case["vocab"], dtype=torch.float64)
    p = torch.log((v + 1 + ZIPF) / (v + ZIPF)) / math.log((case["vocab"] + ZIPF) / ZIPF)
    return float((1 - torch.exp(n * torch.log1p(-p.clamp_max(1 - 1e-12)))).sum()), n


def work(case):
    kind, es = case["kind"], SIZE[case["dtype"]]
    if kind in ("clip", "grad_norm"):
        n = sum(math.prod(shape) for shape in _shapes(case))
        return {"bytes": n * es + (n * SIZE[case["out"]] if kind == "clip" else 0), "flops": (3 if kind == "clip" else 2) * n}
    h = case["hidden"]
    if kind in ("lookup", "lookup_grad"):
        n = case["batch"] * case["length"]
        distinct, valid = _distinct(case)
        if kind == "lookup":
            return {"bytes": n * SIZE[case["index"]] + distinct * h * es + n * h * es, "flops": valid * h}
        return {"bytes": n * SIZE[case["index"]] + valid * h * es + case["vocab"] * h * SIZE[case["out"]], "flops": valid * h + distinct * h}
    rows, stats = case["rows"], 4 if case["rms"] else 8
    if kind == "norm":
        return {"bytes": 2 * rows * h * es + rows * stats, "flops": (5 if case["rms"] else 8) * rows * h}
    return {"bytes": 3 * rows * h * es + rows * stats, "flops": (10 if case["rms"] else 13) * rows * h}


def exact(case, seed):
    """The same outputs from the definitions, in 64 bits."""
    state = prepare(case, seed)
    kind, f64 = case["kind"], torch.float64
    if kind in ("clip", "grad_norm"):
        G = state["flat"].to(f64)              # what lies between the tensors is zero
        norm = float(torch.dot(G, G)) ** 0.5
        if kind == "grad_norm":
            return dict(norm=torch.tensor(norm, dtype=f64))
        scale = min(1.0, state["max_norm"] / norm)
        return dict(out=G.mul_(scale), norm=torch.tensor(norm, dtype=f64), scale=torch.tensor(scale, dtype=f64))
    if kind == "lookup":
        padded = torch.cat([state["table"].to(f64), torch.zeros(1, case["hidden"], dtype=f64, device="cuda")])
        return dict(Y=padded[state["tokens"].long()] * case["scale"])           # -1: the last row
    if kind == "lookup_grad":
        tokens = state["tokens"].long().reshape(-1)
        order = torch.argsort(tokens, stable=True)
        G = torch.zeros(case["vocab"], case["hidden"], dtype=f64, device="cuda")
        width = max(1, 400_000_000 // max(1, len(tokens)))
        dY = state["dY"].reshape(len(tokens), -1)
        count = torch.bincount(tokens + 1, minlength=case["vocab"] + 1)
        ends = torch.cumsum(count, 0)
        for a in range(0, case["hidden"], width):                               # differences of running sums
            sums = torch.cat([torch.zeros(1, min(width, case["hidden"] - a), dtype=f64, device="cuda"),
                              torch.cumsum(dY[:, a:a + width].to(f64)[order], 0)])
            G[:, a:a + width] = (sums[ends[1:]] - sums[ends[:-1]]) * case["scale"]
        return dict(G=G)
    x, gain = state["x"].to(f64), state["gain"].to(f64)
    mean = torch.zeros_like(x[:, :1]) if case["rms"] else x.sum(1, keepdim=True) / case["hidden"]
    x -= mean
    rstd = 1.0 / torch.sqrt((x * x).sum(1, keepdim=True) / case["hidden"] + EPS)
    x *= rstd
    if kind == "norm":
        y = x * gain + (0.0 if case["rms"] else state["bias"].to(f64))
        return dict(Y=y, mean=None if case["rms"] else mean[:, 0], rstd=rstd[:, 0])
    dY = state["dY"].to(f64)
    out = dict(dgain=torch.einsum("rh,rh->h", dY, x))
    if not case["rms"]:
        out["dbias"] = torch.einsum("rh->h", dY)
    along = ((dY * gain) * x).sum(1, keepdim=True) / case["hidden"]
    level = 0.0 if case["rms"] else (dY * gain).sum(1, keepdim=True) / case["hidden"]
    out["dX"] = rstd * (dY * gain - level - along * x)
    return out
