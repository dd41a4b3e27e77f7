"""The calls whose speed the model operators are judged by: the embedding lookup and its gradient,
the norms of queries and keys with the position rotation and their gradient, and distillation from a
teacher's top logits (loss, gradient, and both in one pass).

Where `own` is false `run` computes the operators in elementary torch operations in 32 bits, where it
is true through the public binding.  Token ids follow a Zipf-Mandelbrot law (the few most frequent
tokens make up a large share of a text, most of the vocabulary does not occur), activations and
gradients are N(0, s^2), logits are N(0, 2.5^2) raised at the teacher's entries.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "i32": torch.int32, "i64": torch.int64}
BYTES = {"f32": 4, "bf16": 2, "i32": 4, "i64": 8}
EPS = 1e-6
_OPS = None


def _ops():
    global _OPS
    if _OPS is None:
        from paper_2608_05088_gb300 import model_ops
        _OPS = model_ops
    return _OPS


# ------------------------------------------------------------------ the cases

def _embed(op, tokens, dim, vocab, src, dst, ids="i64", scale=1.0, pad=0.0, accumulate=False):
    return {"op": op, "tokens": tokens, "dim": dim, "vocab": vocab, "src": src, "dst": dst, "ids": ids,
            "scale": scale, "pad": pad, "accumulate": accumulate}


def _qk(op, batch, seq, heads, kv_heads, dim, rot, dtype, interleaved=False, fused=True, block=1024):
    return {"op": op, "batch": batch, "seq": seq, "heads": heads, "kv_heads": kv_heads, "dim": dim, "rot": rot,
            "dtype": dtype, "interleaved": interleaved, "fused": fused, "block": block}


def _distill(op, rows, vocab, topk, dtype, tau=1.0, short=0.0, masked=0.0):
    return {"op": op, "rows": rows, "vocab": vocab, "topk": topk, "dtype": dtype, "tau": tau, "short": short,
            "masked": masked}


def listed():
    return [
        # One new token for each of 16 sequences of a GPT-2 Large model: a launch and its latency.
        dict(_embed("embed", 16, 1280, 50304, "bf16", "bf16"), name="embed_16_tokens"),
        # The lookup of a training step of GPT-2 Large, 40 sequences of 1024 tokens (fp32 residual stream).
        dict(_embed("embed", 40960, 1280, 50304, "bf16", "f32", scale=35.78), name="embed_gpt2_large"),
        # The embedding's gradient of a step of 16 sequences: the whole table's gradient is written.
        dict(_embed("embed_grad", 16384, 1280, 50304, "bf16", "f32"), name="embed_grad_gpt2_large"),
        # A tied table of odd sizes: added to what the head's gradient left there, ragged text with padding.
        dict(_embed("embed_grad", 4999, 501, 32003, "f32", "f32", ids="i32", scale=22.38, pad=0.07, accumulate=True),
             name="embed_grad_tied_odd"),
        # Queries and keys of one new token for each of 16 sequences.
        dict(_qk("qk_norm", 16, 1, 20, 20, 64, 64, "bf16"), name="qk_norm_16_tokens"),
        # One layer of a training step of GPT-2 Large, read out of the fused qkv activations.
        dict(_qk("qk_norm", 16, 1024, 20, 20, 64, 64, "bf16"), name="qk_norm_gpt2_large"),
        # The same layer's backward pass.
        dict(_qk("qk_norm_grad", 16, 1024, 20, 20, 64, 64, "bf16"), name="qk_norm_grad_gpt2_large"),
        # Fewer key heads than query heads, a head of 80 of which 40 are rotated in neighbouring pairs, fp32, odd lengths.
        dict(_qk("qk_norm_grad", 3, 1021, 24, 6, 80, 40, "f32", interleaved=True, fused=False), name="qk_norm_grad_odd"),
        # Scoring a few positions against stored teacher logits.
        dict(_distill("distill_loss", 24, 50304, 16, "f32"), name="distill_loss_24_rows"),
        # Loss and gradient of 8 sequences of 1024 tokens, prompts masked.
        dict(_distill("distill_loss_grad", 8192, 50304, 64, "bf16", tau=2.0, masked=0.1), name="distill_gpt2"),
        # The gradient alone, from the forward pass's row statistics: unpadded vocabulary (odd rows), short teacher lists.
        dict(_distill("distill_grad", 1531, 50257, 100, "f32", tau=1.5, short=0.3, masked=0.05), name="distill_grad_odd"),
        # A large vocabulary, which no single SM's shared memory holds a row of.
        dict(_distill("distill_loss_grad", 2048, 131072, 32, "bf16"), name="distill_large_vocab"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _uneven(rng, n, steps):
    """n rounded down to one of the steps, 1 among them."""
    step = rng.choice(steps)
    return max(1, n // step * step) if n >= step else n


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "embed_grad", "qk_norm", "qk_norm_grad", "distill_loss",
                     "distill_loss_grad", "distill_grad"])
    if op.startswith("embed"):
        tokens = _uneven(rng, _log_int(rng, 1, 40960), [64, 64, 8, 1, 1])
        dim = _uneven(rng, _log_int(rng, 64, 1600), [64, 64, 8, 1])
        vocab = _uneven(rng, _log_int(rng, 300, 50304), [64, 8, 1])
        types = rng.choice([("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
        accumulate = op == "embed_grad" and types[1] == "f32" and rng.random() < 0.4
        return _embed(op, tokens, dim, vocab, types[0], types[1], ids=rng.choice(["i32", "i64"]),
                      scale=rng.choice([1.0, round(math.sqrt(dim), 2)]),
                      pad=rng.choice([0.0, 0.05, 0.3]) if tokens >= 64 else 0.0, accumulate=accumulate)
    if op.startswith("qk"):
        seq = _uneven(rng, _log_int(rng, 1, 4096), [64, 8, 1])
        batch = max(1, min(64, _log_int(rng, 1, 16384) // seq))
        kv = rng.choice([1, 2, 4, 5, 8, 12, 20])
        dim = rng.choice([32, 48, 64, 64, 80, 96, 128, 128])
        rot = rng.choice([dim, dim, dim // 2])
        return _qk(op, batch, seq, kv * rng.choice([1, 1, 2, 4] if kv <= 5 else [1]), kv, dim, rot,
                   rng.choice(["bf16", "bf16", "f32"]), interleaved=rng.random() < 0.4, fused=rng.random() < 0.6,
                   block=max(1024, seq))
    vocab = _uneven(rng, _log_int(rng, 1000, 200000), [64, 64, 8, 1])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    rows = _uneven(rng, min(_log_int(rng, 1, 16384), 400_000_000 // (vocab * BYTES[dtype])), [64, 1])
    return _distill(op, rows, vocab, min(rng.choice([1, 5, 16, 50, 64, 128, 256]), vocab // 2), dtype,
                    tau=rng.choice([1.0, 1.0, 1.5, 2.0, 4.0]), short=rng.choice([0.0, 0.2]),
                    masked=rng.choice([0.0, 0.1, 0.5]) if rows >= 16 else 0.0)


# ----------------------------------------------------------------- the inputs

def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _normal(g, shape, dtype, std=1.0):
    return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(0.0, std, generator=g).to(DTYPES[dtype])


def _zipf(vocab):
    """Probabilities of the ids: 1 / (rank + 2.7)."""
    p = 1.0 / (np.arange(vocab, dtype=np.float64) + 2.7)
    return p / p.sum()


def _prepare_embed(c, g):
    cdf = torch.from_numpy(np.cumsum(_zipf(c["vocab"]))).to(DEV)
    u = torch.rand(c["tokens"], generator=g, device=DEV, dtype=torch.float64)
    ids = torch.searchsorted(cdf, u).clamp_(max=c["vocab"] - 1)
    if c["pad"]:
        ids[torch.rand(c["tokens"], generator=g, device=DEV) < c["pad"]] = -1
    s = {"ids": ids.to(DTYPES[c["ids"]])}
    if c["op"] == "embed":
        s["table"] = _normal(g, (c["vocab"], c["dim"]), c["src"], 0.02)
    else:
        s["dout"] = _normal(g, (c["tokens"], c["dim"]), c["src"], 1e-3)
        if c["accumulate"]:
            s["dtable"] = _normal(g, (c["vocab"], c["dim"]), c["dst"], 1e-3)
    return s


def _prepare_qk(c, g):
    b, n, h, k, d = c["batch"], c["seq"], c["heads"], c["kv_heads"], c["dim"]

    def pair():
        if c["fused"]:      # the q and k parts of one [batch, seq, (h + 2 k) d] activation
            x = _normal(g, (b, n, (h + 2 * k) * d), c["dtype"])
            return x[..., :h * d].view(b, n, h, d), x[..., h * d:(h + k) * d].view(b, n, k, d)
        return _normal(g, (b, n, h, d), c["dtype"]), _normal(g, (b, n, k, d), c["dtype"])

    s = {}
    s["q"], s["k"] = pair()
    s["q_gain"] = 1.0 + _normal(g, (d,), "f32", 0.1)
    s["k_gain"] = 1.0 + _normal(g, (d,), "f32", 0.1)
    half = c["rot"] // 2
    angle = torch.arange(c["block"], device=DEV, dtype=torch.float64)[:, None] * torch.pow(
        10000.0, -torch.arange(half, device=DEV, dtype=torch.float64) / half)[None, :]
    s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    start = torch.randint(0, c["block"] - n + 1, (b, 1), generator=g, device=DEV)
    s["positions"] = start + torch.arange(n, device=DEV)[None, :]
    if c["op"] == "qk_norm_grad":
        s["dq_out"] = _normal(g, (b, n, h, d), c["dtype"], 1e-2)
        s["dk_out"] = _normal(g, (b, n, k, d), c["dtype"], 1e-2)
    return s


def _prepare_distill(c, g):
    n, v, k = c["rows"], c["vocab"], c["topk"]
    step = torch.randint(1, max(2, v // k), (n, 1), generator=g, device=DEV)
    first = torch.randint(0, v, (n, 1), generator=g, device=DEV)
    idx = (first + step * torch.arange(k, device=DEV)[None, :]) % v
    fall = torch.empty((n, k), device=DEV).exponential_(generator=g).mul_(4.0 / math.sqrt(k)).cumsum(1)
    top = 14.0 - fall
    x = torch.empty((n, v), device=DEV).normal_(0.0, 2.5, generator=g)
    x.scatter_add_(1, idx, 0.7 * top)
    s = {"logits": x.to(DTYPES[c["dtype"]]), "top_logits": top}
    if c["short"]:          # teachers that kept fewer entries for some rows
        keep = torch.randint(1, k + 1, (n, 1), generator=g, device=DEV)
        few = torch.rand((n, 1), generator=g, device=DEV) < c["short"]
        idx = torch.where(few & (torch.arange(k, device=DEV)[None, :] >= keep), torch.full_like(idx, -1), idx)
    s["top_ids"] = idx.to(torch.int32)
    weight = (torch.rand(n, generator=g, device=DEV) >= c["masked"]).float()
    s["weight"] = weight / n
    if c["op"] == "distill_grad":       # what the forward pass keeps: a row's maximum and sum of exponentials
        y = s["logits"].float()
        m = y.amax(1)
        s["stats"] = torch.stack([m, ((y - m[:, None]) / c["tau"]).exp().sum(1)], 1)
        s["dloss"] = 1.0 + 0.1 * torch.randn(n, generator=g, device=DEV)
    return s


def prepare(case, seed):
    g = _generator(seed)
    make = _prepare_embed if case["op"].startswith("embed") else _prepare_qk if case["op"].startswith("qk") \
        else _prepare_distill
    s = make(case, g)
    s["case"] = case
    return s


# ------------------------------------------------------------------- the calls

def _run_own(s, c):
    ops = _ops()
    op = c["op"]
    if op == "embed":
        return {"out": ops.embed(s["table"], s["ids"], scale=c["scale"], dtype=DTYPES[c["dst"]])}
    if op == "embed_grad":
        if c["accumulate"]:
            return {"dtable": ops.embed_grad(s["dout"], s["ids"], c["vocab"], scale=c["scale"], out=s["dtable"],
                                             accumulate=True)}
        return {"dtable": ops.embed_grad(s["dout"], s["ids"], c["vocab"], scale=c["scale"], dtype=DTYPES[c["dst"]])}
    if op.startswith("qk"):
        args = (s["q"], s["k"], s["q_gain"], s["k_gain"], s["cos"], s["sin"])
        how = dict(positions=s["positions"], eps=EPS, interleaved=c["interleaved"])
        if op == "qk_norm":
            q, k = ops.qk_norm(*args, **how)
            return {"q": q, "k": k}
        dq, dk, dqg, dkg = ops.qk_norm_grad(s["dq_out"], s["dk_out"], *args, **how)
        return {"dq": dq, "dk": dk, "dq_gain": dqg, "dk_gain": dkg}
    args = (s["logits"], s["top_ids"], s["top_logits"])
    how = dict(weight=s["weight"], temperature=c["tau"])
    if op == "distill_loss":
        loss, stats = ops.distill_loss(*args, **how)
        return {"loss": loss, "stats": stats}
    if op == "distill_grad":
        return {"dlogits": ops.distill_grad(*args, s["stats"], dloss=s["dloss"], **how)}
    loss, dlogits = ops.distill_loss_grad(*args, **how)
    return {"loss": loss, "dlogits": dlogits}


def _plain_embed(s, c):
    ids = s["ids"].long()
    here = ids >= 0
    at = ids.clamp(min=0)
    if c["op"] == "embed":
        rows = s["table"][at].float() * c["scale"]
        return {"out": torch.where(here[:, None], rows, torch.zeros_like(rows)).to(DTYPES[c["dst"]])}
    d = s["dout"].float() * c["scale"]
    d = torch.where(here[:, None], d, torch.zeros_like(d))
    if c["accumulate"]:
        return {"dtable": s["dtable"].index_add_(0, at, d)}
    out = torch.zeros((c["vocab"], c["dim"]), device=d.device)
    return {"dtable": out.index_add_(0, at, d).to(DTYPES[c["dst"]])}


def _turn(x, cos, sin, rot, interleaved):
    """Pairs of the first rot entries of x turned by the angles."""
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_qk(s, c):
    cos, sin = s["cos"][s["positions"]][:, :, None, :], s["sin"][s["positions"]][:, :, None, :]
    dt = DTYPES[c["dtype"]]

    def forward(x, gain):
        x = x.float()
        n = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain
        return _turn(n, cos, sin, c["rot"], c["interleaved"]).to(dt)

    def backward(dy, x, gain):
        x = x.float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        dn = _turn(dy.float(), cos, -sin, c["rot"], c["interleaved"])
        xr = x * r
        u = dn * gain
        dx = r * (u - xr * (u * xr).mean(-1, keepdim=True))
        return dx.to(dt), (dn * xr).sum((0, 1, 2))

    if c["op"] == "qk_norm":
        return {"q": forward(s["q"], s["q_gain"]), "k": forward(s["k"], s["k_gain"])}
    dq, dqg = backward(s["dq_out"], s["q"], s["q_gain"])
    dk, dkg = backward(s["dk_out"], s["k"], s["k_gain"])
    return {"dq": dq, "dk": dk, "dq_gain": dqg, "dk_gain": dkg}


def _plain_distill(s, c):
    tau, idx = c["tau"], s["top_ids"].long()
    here, at = idx >= 0, idx.clamp(min=0)
    on = (s["weight"] != 0) & here.any(1)
    w = torch.where(on, s["weight"], torch.zeros_like(s["weight"]))
    x = s["logits"].float()
    t = torch.where(here, s["top_logits"].float() / tau, torch.full_like(s["top_logits"], -float("inf")))
    t = t - t.amax(1, keepdim=True)
    e = t.exp()
    p = e / e.sum(1, keepdim=True)
    if c["op"] == "distill_grad":
        m, total = s["stats"][:, :1], s["stats"][:, 1:]
        w = w * s["dloss"]
        z = ((x - m) / tau).exp()
    else:
        m = x.amax(1, keepdim=True)
        z = ((x - m) / tau).exp()
        total = z.sum(1, keepdim=True)
        log_p = t - e.sum(1, keepdim=True).log()
        log_q = (x.gather(1, at) - m) / tau - total.log()
        loss = w * tau * tau * torch.where(here, p * (log_p - log_q), torch.zeros_like(p)).sum(1)
        if c["op"] == "distill_loss":
            return {"loss": loss, "stats": torch.cat([m, total], 1) * on[:, None]}
    grad = z.mul_(1.0 / total).scatter_add_(1, at, -p).mul_((w * tau)[:, None]).to(s["logits"].dtype)
    return {"dlogits": grad} if c["op"] == "distill_grad" else {"loss": loss, "dlogits": grad}


def run(state):
    c = state["case"]
    if own:
        return _run_own(state, c)
    if c["op"].startswith("embed"):
        return _plain_embed(state, c)
    if c["op"].startswith("qk"):
        return _plain_qk(state, c)
    return _plain_distill(state, c)


# -------------------------------------------------------------------- the work

def _distinct(c):
    """Expected number of distinct ids among the case's tokens."""
    n = c["tokens"] * (1.0 - c["pad"])
    return float(-np.expm1(n * np.log1p(-_zipf(c["vocab"]))).sum())


def work(case):
    c = case
    if c["op"].startswith("embed"):
        n, d = c["tokens"], c["dim"]
        src, dst, rows = BYTES[c["src"]], BYTES[c["dst"]], _distinct(c)
        if c["op"] == "embed":
            moved = rows * d * src + n * d * dst
        else:
            moved = n * (1.0 - c["pad"]) * d * src + (2 * rows if c["accumulate"] else c["vocab"]) * d * dst
        return {"bytes": moved + n * BYTES[c["ids"]], "flops": n * d}
    if c["op"].startswith("qk"):
        tokens, heads = c["batch"] * c["seq"], c["heads"] + c["kv_heads"]
        x = tokens * heads * c["dim"]
        grad = c["op"] == "qk_norm_grad"
        small = tokens * 8 + min(c["block"], tokens) * c["rot"] * 4 + c["dim"] * (16 if grad else 8)
        return {"bytes": (3 if grad else 2) * x * BYTES[c["dtype"]] + small, "flops": (16 if grad else 8) * x}
    n, v, k = c["rows"], c["vocab"], c["topk"]
    live = n * (1.0 - c["masked"])
    size = live * v * BYTES[c["dtype"]]
    small = n * 4 + live * k * 8
    if c["op"] == "distill_loss":
        return {"bytes": size + small + 12 * n, "flops": 4 * live * v}
    return {"bytes": size + n * v * BYTES[c["dtype"]] + small + (12 if c["op"] == "distill_grad" else 4) * n,
            "flops": (4 if c["op"] == "distill_grad" else 8) * live * v}


# ----------------------------------------------------------- values in 64 bits

def _exact_embed(s, c):
    ids = s["ids"].long()
    keep = torch.nonzero(ids >= 0).squeeze(1)
    if c["op"] == "embed":
        out = torch.zeros((c["tokens"], c["dim"]), dtype=torch.float64, device=DEV)
        out[keep] = s["table"].double()[ids[keep]] * c["scale"]
        return {"out": out}
    order = torch.argsort(ids[keep], stable=True)
    rows = s["dout"].double()[keep[order]]
    total = torch.cat([torch.zeros((1, c["dim"]), dtype=torch.float64, device=DEV), rows.cumsum(0)])
    end = torch.searchsorted(ids[keep[order]], torch.arange(c["vocab"], device=DEV), right=True)
    begin = torch.cat([torch.zeros_like(end[:1]), end[:-1]])
    d = (total[end] - total[begin]) * c["scale"]
    return {"dtable": d + s["dtable"].double() if c["accumulate"] else d}


def _exact_qk(s, c):
    rot, half = c["rot"], c["rot"] // 2
    first = torch.arange(half, device=DEV) * (2 if c["interleaved"] else 1)
    second = first + (1 if c["interleaved"] else half)
    theta = torch.complex(s["cos"].double(), s["sin"].double())[s["positions"]].unsqueeze(2)

    def unit(x):
        x = x.double()
        return x, (x.square().sum(-1, keepdim=True) / c["dim"] + EPS).sqrt()

    def turned(x, by):
        z = torch.complex(x[..., first], x[..., second]) * by
        y = x.clone()
        y[..., first], y[..., second] = z.real, z.imag
        return y

    def gradient(dy, x, gain):
        x, norm = unit(x)
        dn = turned(dy.double(), theta.conj())
        dgain = torch.einsum("bthd,bthd->d", dn, x / norm)
        u = dn * gain.double()
        along = torch.einsum("bthd,bthd->bth", u, x).unsqueeze(-1)
        return u / norm - x * along / (c["dim"] * norm ** 3), dgain

    def forward(x, gain):
        x, norm = unit(x)
        return turned(x / norm * gain.double(), theta)

    if c["op"] == "qk_norm":
        return {"q": forward(s["q"], s["q_gain"]), "k": forward(s["k"], s["k_gain"])}
    dq, dqg = gradient(s["dq_out"], s["q"], s["q_gain"])
    dk, dkg = gradient(s["dk_out"], s["k"], s["k_gain"])
    return {"dq": dq, "dk": dk, "dq_gain": dqg, "dk_gain": dkg}


def _exact_distill(s, c):
    tau = float(c["tau"])
    z = s["logits"].double()
    ids = s["top_ids"].long()
    at = ids.clamp(min=0)
    w = s["weight"].double() * (ids >= 0).any(1)
    on = (w != 0)[:, None]
    t = (s["top_logits"].double() / tau).masked_fill(on & (ids < 0), float("-inf"))
    log_p = torch.log_softmax(t, 1)
    p = log_p.exp().masked_fill(ids < 0, 0.0)
    log_q = torch.log_softmax(z / tau, 1)
    gap = (log_p - log_q.gather(1, at)).masked_fill(ids < 0, 0.0)
    loss = w * tau ** 2 * (p * gap).sum(1)
    if c["op"] == "distill_loss":
        m = z.max(1).values
        stats = torch.stack([m, torch.exp((z - m[:, None]) / tau).sum(1)], 1)
        return {"loss": loss, "stats": stats * on}
    if c["op"] == "distill_grad":
        w = w * s["dloss"].double()
    grad = log_q.exp_().scatter_add_(1, at, -p).mul_((w * tau)[:, None])
    return {"dlogits": grad} if c["op"] == "distill_grad" else {"loss": loss, "dlogits": grad}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("embed"):
        return _exact_embed(s, case)
    return _exact_qk(s, case) if case["op"].startswith("qk") else _exact_distill(s, case)
