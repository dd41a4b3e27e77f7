"""The calls whose speed the operators at the end of a training step are judged by: the RMS norm with the
residual's addition (16 or 32 bits, or 8 bits with scales) and its gradient, an output head's cross entropy
without its logits (loss, gradients, and both), and AdamW on many tensors with states in 8 bits.

Where `own` is false `run` computes the operators in elementary torch operations in 32 bits (64 where a value
decides between two codes), where it is true through the public binding.  Activations and gradients are
N(0, s^2), labels follow a Zipf-Mandelbrot law and their logits are raised, as a trained head's are.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "i32": torch.int32, "i64": torch.int64}
BYTES = {"f32": 4, "bf16": 2, "i32": 4, "i64": 8}
EPS = 1e-6
GROUP = 128             # entries of a row that share a scale (8-bit norms)
BLOCK = 256             # entries of a tensor that share a scale (8-bit states)
ADAM = {"lr": 9e-4, "betas": (0.9, 0.95), "eps": 1e-8}
SEED = 20


# ------------------------------------------------------------------ the cases

def _norm(op, tokens, dim, x, stream, y, residual=True):
    return {"op": op, "tokens": tokens, "dim": dim, "x": x, "stream": stream, "y": y, "residual": residual}


def _head(op, rows, dim, vocab, hidden, table, labels="i64", masked=0.0, accumulate=False):
    return {"op": op, "rows": rows, "dim": dim, "vocab": vocab, "hidden": hidden, "table": table, "labels": labels,
            "masked": masked, "accumulate": accumulate}


def _adamw(vocab, positions, dim, layers, grad, copy):
    return {"op": "adamw8", "vocab": vocab, "positions": positions, "dim": dim, "layers": layers, "grad": grad,
            "copy": copy}


def listed():
    return [
        # One new token for each of 16 sequences: a launch and its latency.
        dict(_norm("rms_norm", 16, 1280, "bf16", "bf16", "bf16"), name="rms_norm_16_tokens"),
        # One norm of a training step of GPT-2 Large's size: a sublayer's output added to an fp32 stream.
        dict(_norm("rms_norm", 16384, 1280, "bf16", "f32", "bf16"), name="rms_norm_gpt2_large"),
        # The same with the normalised rows in 8 bits, for a matrix product that takes those.
        dict(_norm("rms_norm_8bit", 16384, 1280, "bf16", "bf16", "e4m3"), name="rms_norm_8bit_gpt2_large"),
        # The backward pass of the second.
        dict(_norm("rms_norm_grad", 16384, 1280, "bf16", "f32", "bf16"), name="rms_norm_grad_gpt2_large"),
        # Rows of odd length, fp32, no stream to add.
        dict(_norm("rms_norm_grad", 4999, 501, "f32", "f32", "f32", residual=False), name="rms_norm_grad_odd"),
        # Scoring a few positions: the table has to be read once.
        dict(_head("head_loss", 24, 1280, 50304, "bf16", "bf16"), name="head_loss_24_rows"),
        # Loss and gradients of 8 sequences of 1024 tokens, prompts masked.
        dict(_head("head_loss_grad", 8192, 1280, 50304, "bf16", "bf16", masked=0.1), name="head_gpt2_large"),
        # The gradients alone in fp32 from the forward pass's statistics, odd sizes, added to a tied table's.
        dict(_head("head_grad", 1531, 501, 32003, "f32", "f32", labels="i32", masked=0.05, accumulate=True),
             name="head_grad_odd"),
        # A large vocabulary.
        dict(_head("head_loss_grad", 2048, 1024, 131072, "bf16", "bf16"), name="head_large_vocab"),
        # A small model's vectors and short table: launches and their latency.
        dict(_adamw(512, 64, 64, 2, "f32", False), name="adamw8_small"),
        # All that AdamW updates of GPT-2 Large: 443 tensors, bf16 gradients and copies.
        dict(_adamw(50304, 1024, 1280, 36, "bf16", True), name="adamw8_gpt2_large"),
        # Odd sizes, fp32 gradients.
        dict(_adamw(32003, 257, 501, 7, "f32", True), name="adamw8_odd"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _uneven(rng, n, steps):
    """n rounded down to one of the steps, 1 among them."""
    step = rng.choice(steps)
    return max(1, n // step * step) if n >= step else n


def draw(rng):
    kind = rng.choice(["rms_norm", "rms_norm_8bit", "rms_norm_grad", "head_loss", "head_loss_grad", "head_grad",
                       "adamw8"])
    if kind.startswith("rms"):
        dim = _uneven(rng, _log_int(rng, 64, 8192), [64, 64, 8, 1])
        tokens = _uneven(rng, min(_log_int(rng, 1, 32768), 21_000_000 // dim), [64, 8, 1])
        x, stream = rng.choice([("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
        y = "e4m3" if kind == "rms_norm_8bit" else rng.choice(["bf16", stream])
        residual = stream != x or rng.random() < 0.7
        return _norm(kind, tokens, dim, x, stream, y, residual=residual)
    if kind.startswith("head"):
        hidden, table = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16")])
        dim = _uneven(rng, _log_int(rng, 64, 1600), [64, 64, 8, 1])
        vocab = _uneven(rng, _log_int(rng, 500, 131072), [64, 8, 1])
        most = 5.2e11 if hidden == "bf16" else 8e10
        rows = _uneven(rng, max(1, min(_log_int(rng, 1, 8192), int(most / (dim * vocab)), 400_000_000 // vocab)),
                       [64, 8, 1])
        return _head(kind, rows, dim, vocab, hidden, table, labels=rng.choice(["i32", "i64"]),
                     masked=rng.choice([0.0, 0.1, 0.5]) if rows >= 16 else 0.0,
                     accumulate=kind != "head_loss" and table == "f32" and rng.random() < 0.4)
    dim = _uneven(rng, _log_int(rng, 40, 1280), [64, 8, 1])
    vocab = _uneven(rng, _log_int(rng, 100, 50304), [64, 8, 1])
    return _adamw(vocab, _log_int(rng, 1, 1024), dim, rng.randint(1, 36), rng.choice(["bf16", "f32"]),
                  rng.random() < 0.7)


# ----------------------------------------------------------------- the inputs

def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _normal(g, shape, dtype, std=1.0):
    return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(0.0, std, generator=g).to(DTYPES[dtype])


def _prepare_norm(c, g):
    n, d = c["tokens"], c["dim"]
    s = {"gain": 1.0 + _normal(g, (d,), "f32", 0.1)}
    if c["op"] == "rms_norm_grad":
        s["h"] = _normal(g, (n, d), c["stream"], 2.0)
        s["dy"] = _normal(g, (n, d), c["y"], 1e-2)
        s["dh"] = _normal(g, (n, d), c["stream"], 1e-2) if c["residual"] else None
    else:
        s["x"] = _normal(g, (n, d), c["x"])
        s["residual"] = _normal(g, (n, d), c["stream"], 2.0) if c["residual"] else None
    return s


def _prepare_head(c, g):
    n, d, v = c["rows"], c["dim"], c["vocab"]
    s = {"table": _normal(g, (v, d), c["table"], 0.05)}
    p = 1.0 / (np.arange(v, dtype=np.float64) + 2.7)
    cdf = torch.from_numpy(np.cumsum(p / p.sum())).to(DEV)
    u = torch.rand(n, generator=g, device=DEV, dtype=torch.float64)
    labels = torch.searchsorted(cdf, u).clamp_(max=v - 1)
    # Hidden rows of a trained model: their label's logit stands some eight units out.
    raised = torch.empty((n, d), device=DEV).normal_(0.0, 1.0, generator=g)
    raised += s["table"][labels].float() * (8.0 / (0.0025 * d))
    s["hidden"] = raised.to(DTYPES[c["hidden"]])
    labels[torch.rand(n, generator=g, device=DEV) < c["masked"]] = -1
    s["labels"] = labels.to(DTYPES[c["labels"]])
    s["weight"] = torch.full((n,), 1.0 / n, device=DEV)
    if c["op"] == "head_grad":      # what the forward pass keeps: a row's maximum and sum of exponentials
        x = s["hidden"].float() @ s["table"].float().t()
        m = x.amax(1)
        stats = torch.stack([m, (x - m[:, None]).exp_().sum(1)], 1)
        s["stats"] = stats * (labels >= 0)[:, None]
        s["dloss"] = 1.0 + 0.1 * torch.randn(n, generator=g, device=DEV)
    if c["accumulate"]:
        s["dtable"] = _normal(g, (v, d), c["table"], 1e-3)
    return s


def _sizes(c):
    """(entries, weight decay) of the tensors: token and position tables, per layer two gains, four biases,
    the last gain."""
    d = c["dim"]
    layer = [(d, 0.0), (3 * d, 0.0), (d, 0.0), (d, 0.0), (4 * d, 0.0), (d, 0.0)]
    return [(c["vocab"] * d, 0.1), (c["positions"] * d, 0.1)] + c["layers"] * layer + [(d, 0.0)]


def _blocks(c):
    return [-(-n // BLOCK) for n, _ in _sizes(c)]


def _prepare_adamw(c, g):
    sizes, blocks = _sizes(c), _blocks(c)
    total = sum(blocks)
    # Every tensor starts on a block of one flat buffer; what lies between two of them is zero.
    count = torch.tensor(blocks, device=DEV)
    s = {"tensor": torch.repeat_interleave(torch.arange(len(sizes), device=DEV), count)}
    first = torch.cumsum(count, 0) - count
    s["at"] = (torch.arange(total, device=DEV) - first[s["tensor"]]) * BLOCK
    length = torch.tensor([n for n, _ in sizes], device=DEV)
    here = s["at"][:, None] + torch.arange(BLOCK, device=DEV)[None, :] < length[s["tensor"]][:, None]
    s["decay"] = torch.tensor([wd for _, wd in sizes], dtype=torch.float32, device=DEV)[s["tensor"]][:, None]
    # Gradients of rows that differ by orders of magnitude, states as of some steps.
    scale = torch.empty((total, 1), device=DEV).normal_(-8.0, 1.5, generator=g).exp_()
    s["g"] = (_normal(g, (total, BLOCK), "f32") * scale * here).to(DTYPES[c["grad"]])
    s["w"] = _normal(g, (total, BLOCK), "f32", 0.02) * here
    s["copy"] = s["w"].to(torch.bfloat16) if c["copy"] else None
    for name, value, codes in (("m", _normal(g, (total, BLOCK), "f32", 0.3), _m_codes),
                               ("v", _normal(g, (total, BLOCK), "f32", 0.3).exp_(), _v_codes)):
        value = value * scale * here
        s[name + "_scale"] = _exponent(value)
        s[name] = codes(value, s[name + "_scale"], torch.full_like(value, 32768, dtype=torch.int32), value)
    s["t"] = 100
    if own:
        from paper_2608_05088_gb300 import malt
        w, gr, m, v = (s[k].view(-1) for k in ("w", "g", "m", "v"))
        copy = s["copy"].view(-1) if c["copy"] else None
        params, b = [], 0
        for (n, wd), k in zip(sizes, blocks):
            a = b * BLOCK
            params.append((w[a:a + n], None if copy is None else copy[a:a + n], gr[a:a + n], m[a:a + n],
                           s["m_scale"][b:b + k], v[a:a + n], s["v_scale"][b:b + k], wd))
            b += k
        kept = {k: s[k].clone() for k in ("m", "m_scale", "v", "v_scale")}
        s["optimizer"] = malt.AdamW8(params, seed=SEED)     # zeroes the states
        for k, t in kept.items():
            s[k].copy_(t)
        s["optimizer"].set_step(s["t"])
        s["hparams"] = malt.adamw_hparams(**ADAM)
    return s


def prepare(case, seed):
    g = _generator(seed)
    make = _prepare_norm if case["op"].startswith("rms") else _prepare_head if case["op"].startswith("head") \
        else _prepare_adamw
    s = make(case, g)
    s["case"] = case
    return s


# -------------------------------------------------------------- codes of states

def _power(e):
    """2^e, e an int32 tensor from -126 to 127."""
    return ((e + 127) << 23).view(torch.float32)


def _exponent(value):
    """Per block the byte e with the largest |value| at most 1.9375 2^(e - 127), from 27 up."""
    bits = value.abs().amax(1).view(torch.int32)
    return ((bits + 0x7ffff) >> 23).clamp_(min=27).to(torch.uint8)


def _scaled(value, scale):
    """Bits of |value| 2^(127 - e) 2^-120: the float's exponent field is the code's."""
    z = value.abs() * _power(127 - scale.int())[:, None] * 2.0 ** -120
    return z.view(torch.int32)


def _m_codes(value, scale, random, _):
    """Sign, 3 bits of exponent, 4 of mantissa, the rest rounded up where it and 16 random bits carry."""
    code = (_scaled(value, scale) + (random << 3)) >> 19
    return (code | (value.view(torch.int32) >> 24 & 0x80)).to(torch.uint8)


def _v_codes(root, scale, random, second):
    """3 bits of exponent, 5 of mantissa; only zero has code 0."""
    code = (_scaled(root, scale) + (random << 2)) >> 18
    return torch.where((code == 0) & (second > 0), torch.ones_like(code), code).to(torch.uint8)


def _m_values(code, scale):
    c = code.int()
    x = ((c & 0x7f) << 19).view(torch.float32) * 2.0 ** 120 * _power(scale.int() - 127)[:, None]
    return torch.where(c >= 0x80, -x, x)


def _v_values(code, scale):
    return (code.int() << 18).view(torch.float32) * 2.0 ** 120 * _power(scale.int() - 127)[:, None]


def _mix(x):
    """A hash of 32 bits (in int64)."""
    x = ((x ^ x >> 16) * 0x6A09E667) & 0xffffffff
    x = ((x ^ x >> 15) * 0xBB67AE85) & 0xffffffff
    return x ^ x >> 16


def _random(s, t):
    """32 random bits per entry: of seed, step, tensor and the entry's place in it."""
    key = _mix(_mix(_mix(torch.full_like(s["tensor"], SEED)) ^ t) ^ s["tensor"])
    return _mix((s["at"][:, None] + torch.arange(BLOCK, device=DEV)[None, :]) ^ _mix(key)[:, None])


# ------------------------------------------------------------------- the calls

def _run_own(s, c):
    op = c["op"]
    if op == "adamw8":
        s["optimizer"].step(s["hparams"])
        m, root = s["optimizer"].moments(dtype=torch.bfloat16)
        out = {"w": s["w"], "m": m, "root": root}
        return dict(out, copy=s["copy"]) if c["copy"] else out
    from paper_2608_05088_gb300 import model_ops as ops
    if op == "rms_norm":
        y, h = ops.rms_norm(s["x"], s["gain"], residual=s["residual"], eps=EPS, dtype=DTYPES[c["y"]])
        return {"y": y, "h": h} if c["residual"] else {"y": y}
    if op == "rms_norm_8bit":
        codes, scales, h = ops.rms_norm_8bit(s["x"], s["gain"], residual=s["residual"], eps=EPS)
        return _out_8bit(codes, scales, h, c)
    if op == "rms_norm_grad":
        dx, dgain = ops.rms_norm_grad(s["dy"], s["h"], s["gain"], dh=s["dh"], eps=EPS)
        return {"dx": dx, "dgain": dgain}
    args = (s["hidden"], s["table"], s["labels"])
    if op == "head_loss":
        loss, stats = ops.head_loss(*args, weight=s["weight"])
        return {"loss": loss, "stats": stats}
    into = dict(dtable=s["dtable"], accumulate=True) if c["accumulate"] else {}
    if op == "head_grad":
        dhidden, dtable = ops.head_grad(*args, s["stats"], dloss=s["dloss"], weight=s["weight"], **into)
        return {"dhidden": dhidden, "dtable": dtable}
    loss, dhidden, dtable = ops.head_loss_grad(*args, weight=s["weight"], **into)
    return {"loss": loss, "dhidden": dhidden, "dtable": dtable}


def _out_8bit(codes, scales, h, c):
    """The values that the codes stand for, in 16 bits, and the scales."""
    pad = scales.shape[1] * GROUP - codes.shape[1]
    q = torch.nn.functional.pad(codes.to(torch.bfloat16), (0, pad)).view(codes.shape[0], -1, GROUP)
    out = {"y": (q * scales[:, :, None]).to(torch.bfloat16), "scales": scales}
    return dict(out, h=h) if c["residual"] else out


def _plain_norm(s, c):
    if c["op"] == "rms_norm_grad":
        h = s["h"].float()
        r = torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS)
        hr, dy = h * r, s["dy"].float()
        u = dy * s["gain"]
        dx = r * (u - hr * (u * hr).mean(-1, keepdim=True))
        if s["dh"] is not None:
            dx = dx + s["dh"].float()
        return {"dx": dx.to(s["h"].dtype), "dgain": (dy * hr).double().sum(0).float()}
    h = s["x"]
    if s["residual"] is not None:
        h = (s["x"].float() + s["residual"].float()).to(s["residual"].dtype)
    x = h.float()
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * s["gain"]
    if c["op"] == "rms_norm":
        y = y.to(DTYPES[c["y"]])
        return {"y": y, "h": h} if c["residual"] else {"y": y}
    n, d = y.shape
    groups = -(-d // GROUP)
    a = torch.nn.functional.pad(y, (0, groups * GROUP - d)).view(n, groups, GROUP)
    scales = a.abs().amax(-1).clamp(min=1e-30) / 448.0
    codes = (a / scales[:, :, None]).to(torch.float8_e4m3fn).view(n, -1)[:, :d]
    return _out_8bit(codes, scales, h, c)


def _plain_head(s, c):
    labels = s["labels"].long()
    on, at = labels >= 0, labels.clamp(min=0)
    w = torch.where(on, s["weight"], torch.zeros_like(s["weight"]))
    h = torch.where(on[:, None], s["hidden"].float(), torch.zeros((), device=DEV))
    table = s["table"].float()
    x = h @ table.t()
    if c["op"] == "head_grad":
        m, total = s["stats"][:, :1], torch.where(on, s["stats"][:, 1], torch.ones_like(w))[:, None]
        w = w * s["dloss"]
    else:
        m = x.amax(1, keepdim=True)
        of_label = x.gather(1, at[:, None])
    x.sub_(m).exp_()
    if c["op"] != "head_grad":
        total = x.sum(1, keepdim=True)
        loss = w * (total.log() + (m - of_label))[:, 0]
        if c["op"] == "head_loss":
            return {"loss": loss, "stats": torch.cat([m, total], 1) * on[:, None]}
    x.mul_(w[:, None] / total)
    x.scatter_add_(1, at[:, None], -w[:, None])
    dhidden = (x @ table).to(s["hidden"].dtype)
    dtable = x.t() @ h
    dtable = s["dtable"].add_(dtable) if c["accumulate"] else dtable.to(s["table"].dtype)
    out = {"dhidden": dhidden, "dtable": dtable}
    return out if c["op"] == "head_grad" else dict(out, loss=loss)


def _fma(a, b, c):
    """a b + c rounded once."""
    return (a.double() * b + c).float()


def _plain_adamw(s, c):
    f = np.float32
    lr, b1, b2, eps = (f(v) for v in (ADAM["lr"], *ADAM["betas"], ADAM["eps"]))
    s["t"] += 1
    t = s["t"]
    step = float(f(float(lr) / (1.0 - float(b1) ** t)))
    root_scale = float(f(1.0 / math.sqrt(1.0 - float(b2) ** t)))
    g = s["g"].float()
    m = _fma(_m_values(s["m"], s["m_scale"]), float(b1), g * float(f(1) - b1))
    v = _v_values(s["v"], s["v_scale"])
    v = _fma(v * v, float(b2), g * float(f(1) - b2) * g)
    root = v.sqrt()
    decay = 1.0 - float(lr) * s["decay"]
    s["w"].copy_(s["w"] * decay - step * (m / (root * root_scale + float(eps))))
    bits = _random(s, t)
    s["m_scale"].copy_(_exponent(m))
    s["v_scale"].copy_(_exponent(root))
    s["m"].copy_(_m_codes(m, s["m_scale"], (bits >> 16).int(), m))
    s["v"].copy_(_v_codes(root, s["v_scale"], (bits & 0xffff).int(), v))
    out = {"w": s["w"], "m": _m_values(s["m"], s["m_scale"]).view(-1).to(torch.bfloat16),
           "root": _v_values(s["v"], s["v_scale"]).view(-1).to(torch.bfloat16)}
    if c["copy"]:
        out["copy"] = s["copy"].copy_(s["w"])
    return out


def run(state):
    c = state["case"]
    if own:
        return _run_own(state, c)
    if c["op"].startswith("rms"):
        return _plain_norm(state, c)
    return _plain_head(state, c) if c["op"].startswith("head") else _plain_adamw(state, c)


# -------------------------------------------------------------------- the work

def work(case):
    c = case
    if c["op"].startswith("rms"):
        n, x = c["dim"], c["tokens"] * c["dim"]
        stream = BYTES[c["stream"]]
        if c["op"] == "rms_norm_grad":
            each = BYTES[c["y"]] + stream * (3 if c["residual"] else 2)
            return {"bytes": x * each + 8 * n, "flops": 10 * x}
        each = BYTES[c["x"]] + (2 * stream if c["residual"] else 0) + (1 if c["y"] == "e4m3" else BYTES[c["y"]])
        scales = c["tokens"] * -(-n // GROUP) * 4 if c["y"] == "e4m3" else 0
        return {"bytes": x * each + scales + 4 * n, "flops": 5 * x}
    if c["op"].startswith("head"):
        d, v = c["dim"], c["vocab"]
        live = c["rows"] * (1.0 - c["masked"])
        hidden, table = live * d * BYTES[c["hidden"]], v * d * BYTES[c["table"]]
        one = 2.0 * live * v * d
        small = c["rows"] * (BYTES[c["labels"]] + 4)
        if c["op"] == "head_loss":
            return {"bytes": hidden + table + small + 12 * c["rows"], "flops": one}
        moved = hidden + table * (3 if c["accumulate"] else 2) + c["rows"] * d * BYTES[c["hidden"]] + small
        return {"bytes": moved + (12 if c["op"] == "head_grad" else 4) * c["rows"], "flops": 3 * one}
    n, blocks = sum(k for k, _ in _sizes(c)), sum(_blocks(c))
    # weights and codes read and written, gradients read, copies written, and the states' values read out
    each = 8 + 4 + BYTES[c["grad"]] + (2 if c["copy"] else 0) + 4
    return {"bytes": n * each + 4 * blocks, "flops": 30 * n}


# ----------------------------------------------------------- values in 64 bits

def _exact_norm(s, c):
    gain = s["gain"].double()
    if c["op"] == "rms_norm_grad":
        h, dy = s["h"].double(), s["dy"].double()
        norm = (h.square().sum(-1, keepdim=True) / c["dim"] + EPS).sqrt()
        u = dy * gain
        along = torch.einsum("td,td->t", u, h)[:, None]
        dx = u / norm - h * along / (c["dim"] * norm ** 3)
        if c["residual"]:
            dx += s["dh"].double()
        return {"dx": dx, "dgain": torch.einsum("td,td->d", dy, h / norm)}
    full = h = s["x"].double()
    if c["residual"]:
        full = h + s["residual"].double()
        h = full.to(s["residual"].dtype).double()       # the norm is that of the stream as it is kept
    y = h / (h.square().sum(-1, keepdim=True) / c["dim"] + EPS).sqrt() * gain
    out = {"h": full} if c["residual"] else {}
    if c["op"] == "rms_norm":
        return dict(out, y=y)
    n, d = y.shape
    groups = -(-d // GROUP)
    grouped = torch.zeros((n, groups * GROUP), dtype=torch.float64, device=DEV)
    grouped[:, :d] = y
    grouped = grouped.view(n, groups, GROUP)
    scales = grouped.abs().max(-1).values.clamp(min=1e-30) / 448.0
    q = grouped / scales[:, :, None]
    step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
    return dict(out, y=torch.round(q / step) * step * scales[:, :, None], scales=scales)


def _exact_head(s, c):
    labels = s["labels"].long()
    live = torch.nonzero(labels >= 0).squeeze(1)
    w = s["weight"].double()[live]
    h, table = s["hidden"].double()[live], s["table"].double()
    logits = h @ table.t()
    rows = torch.arange(len(live), device=DEV)
    m = logits.max(1).values
    lse = torch.logsumexp(logits, 1)

    def spread(values):
        out = torch.zeros((c["rows"], *values.shape[1:]), dtype=torch.float64, device=DEV)
        out[live] = values
        return out

    loss = spread(w * (lse - logits[rows, labels[live]]))
    if c["op"] == "head_loss":
        return {"loss": loss, "stats": spread(torch.stack([m, (lse - m).exp()], 1))}
    if c["op"] == "head_grad":
        w = w * s["dloss"].double()[live]
    dlogits = torch.softmax(logits, 1)
    dlogits[rows, labels[live]] -= 1.0
    dlogits *= w[:, None]
    dtable = dlogits.t() @ h
    out = {"dhidden": spread(dlogits @ table), "dtable": dtable + s["dtable"].double() if c["accumulate"] else dtable}
    return out if c["op"] == "head_grad" else dict(out, loss=loss)


def _exact_adamw(s, c):
    lr, b1, b2, eps = (float(np.float32(v)) for v in (ADAM["lr"], *ADAM["betas"], ADAM["eps"]))
    t = s["t"] + 1
    g = s["g"].double()

    def value(code, bits):      # (1 + mantissa) 2^(exponent - 7), without the leading one at exponent 0
        e, f = code >> bits, (code & (1 << bits) - 1).double() / (1 << bits)
        return torch.where(e > 0, (1.0 + f) * torch.exp2(e.double() - 7.0), f * 2.0 ** -6)

    def unit(scale):
        return torch.exp2(scale.double() - 127.0)[:, None]

    def code_value(x, random, bits):
        largest = x.max(1, keepdim=True).values.clamp(min=2.0 ** -101)
        e = torch.floor(torch.log2(largest))
        e = torch.where(largest > 1.9375 * torch.exp2(e), e + 1.0, e).clamp(min=-100.0)
        y = x / torch.exp2(e)
        step = torch.exp2(torch.floor(torch.log2(y.clamp(min=2.0 ** -6))) - bits)
        k = torch.floor(y / step + random.double() / 65536.0)
        return torch.where((k == 0) & (x > 0) & (bits == 5), torch.ones_like(k), k) * step * torch.exp2(e)

    code = s["m"].long()
    m = value(code & 0x7f, 4) * unit(s["m_scale"]) * torch.where(code >= 0x80, -1.0, 1.0).double()
    m = b1 * m + (1.0 - b1) * g
    v = b2 * (value(s["v"].long(), 5) * unit(s["v_scale"])).square() + (1.0 - b2) * g.square()
    w = (1.0 - lr * s["decay"].double()) * s["w"].double()
    w -= lr * (m / (1.0 - b1 ** t)) / ((v / (1.0 - b2 ** t)).sqrt() + eps)
    bits = _random(s, t)
    out = {"w": w, "m": (code_value(m.abs(), bits >> 16, 4) * m.sign()).view(-1),
           "root": code_value(v.sqrt(), bits & 0xffff, 5).view(-1)}
    return dict(out, copy=w) if c["copy"] else out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("rms"):
        return _exact_norm(s, case)
    return _exact_head(s, case) if case["op"].startswith("head") else _exact_adamw(s, case)
