"""The model operators against their fp64 oracle, element by element, and their bounds:
u is half an fp32 ulp, h half a bf16 one; a sum of n terms is off by at most n u times the
sum of their sizes, whatever its order, and a result by a few u per operation before it.
Every output lies between canary margins."""
import numpy as np
import pytest

from oracle import model_ops_ref as ref
from tests.gpu_harness import canaries_intact, guarded

pytestmark = pytest.mark.gpu

U, H = 2.0 ** -24, 2.0 ** -8
TINY = 1e-37            # below it fp32 and bf16 lose bits to underflow


def torch_and_ops():
    import torch
    from paper_2608_05088_gb300 import model_ops
    return torch, model_ops


def host(t):
    return t.detach().double().cpu().numpy()


def out_bound(value, bound, dtype):
    """The bound of a result rounded once to its type."""
    return bound + np.abs(value) * (H * 1.01 if "bfloat16" in str(dtype) else 0.0) + TINY


def check(got, want, bound, what):
    got = host(got).reshape(want.shape)
    want = np.where(np.abs(want) > np.finfo(np.float32).max, np.copysign(np.inf, want), want)    # past fp32
    with np.errstate(invalid="ignore"):
        off = np.abs(got - want)
    bad = ~(off <= bound) & ~(np.isnan(got) & np.isnan(want)) & ~(got == want)
    assert not bad.any(), (what, int(bad.sum()), got[bad][:4], want[bad][:4], np.broadcast_to(bound, want.shape)[bad][:4])


def placed(values, dtype, ld=None, shift=0):
    """values as a CUDA matrix of row stride ld, `shift` elements past an aligned address."""
    import torch
    rows, cols = values.shape
    ld = cols if ld is None else ld
    buf = torch.full((rows * ld + shift + 8,), float("nan"), dtype=dtype, device="cuda")
    t = buf[shift:shift + rows * ld].view(rows, ld)[:, :cols]
    t.copy_(torch.as_tensor(values))
    return t


def margins(rows, cols, dtype, ld=None, shift=0):
    """An output matrix between canaries: (matrix, whole buffer, check)."""
    import torch
    ld = cols if ld is None else ld
    flat, buf = guarded((rows * ld + shift,), dtype, "cuda")
    flat.fill_(-7.625e7)
    t = flat[shift:].view(rows, ld)[:, :cols]

    def intact():
        hole = flat[shift:].view(rows, ld)[:, cols:]
        return canaries_intact(buf) and bool((flat[:shift] == -7.625e7).all()) and bool((hole == -7.625e7).all())

    return t, intact


# ------------------------------------------------------------------ embedding

def some_ids(rng, tokens, vocab, kind):
    if kind == "same":
        return np.full(tokens, vocab // 2)
    if kind == "few":
        return rng.integers(0, min(vocab, 3), tokens)
    if kind == "zipf":
        return np.minimum((vocab + 1) ** rng.random(tokens) - 1, vocab - 1).astype(np.int64)
    ids = rng.integers(0, vocab, tokens)
    if kind == "padded":
        ids[rng.random(tokens) < 0.4] = -1
        ids[rng.random(tokens) < 0.05] = vocab + 3
        ids[:1] = -(2 ** 31)
    return ids


EMBED = [
    # tokens, vocab, dim, table, rows, ids, kind, ld pads, shift
    (1, 1, 1, "f32", "f32", "i64", "any", 0, 0),
    (1, 7, 64, "bf16", "bf16", "i32", "any", 0, 0),
    (33, 50, 8, "f32", "bf16", "i64", "few", 0, 0),
    (65, 11, 127, "bf16", "f32", "i32", "padded", 0, 0),
    (300, 1000, 129, "f32", "f32", "i64", "zipf", 3, 1),
    (257, 500, 768, "bf16", "bf16", "i64", "padded", 8, 0),
    (97, 300, 1280, "bf16", "f32", "i64", "zipf", 0, 4),
    (513, 64, 260, "f32", "f32", "i32", "same", 4, 0),
    (3000, 2, 24, "bf16", "bf16", "i32", "same", 1, 1),
    (5000, 400, 36, "f32", "f32", "i64", "zipf", 0, 0),
    (2048, 400000, 4, "f32", "f32", "i32", "any", 0, 0),
    (70001, 40, 9, "bf16", "f32", "i64", "zipf", 0, 0),
    (70001, 40, 16, "f32", "f32", "i32", "same", 0, 0),
    (40, 12, 5000, "bf16", "f32", "i64", "few", 0, 0),
]


def embed_case(case):
    torch, _ = torch_and_ops()
    tokens, vocab, dim, table, rows, ids, kind, pad, shift = case
    types = {"f32": torch.float32, "bf16": torch.bfloat16, "i32": torch.int32, "i64": torch.int64}
    rng = np.random.default_rng(tokens + 31 * vocab + dim)
    at = some_ids(rng, tokens, vocab, kind)
    return (tokens, vocab, dim, types[table], types[rows], torch.as_tensor(at).to("cuda", types[ids]), at, dim + pad,
            shift, rng)


@pytest.mark.parametrize("case", EMBED)
def test_embed(case):
    torch, ops = torch_and_ops()
    tokens, vocab, dim, tt, rt, ids, at, ld, shift, rng = embed_case(case)
    table = placed(rng.standard_normal((vocab, dim)), tt, ld, shift)
    out, intact = margins(tokens, dim, rt, ld, shift)
    ops.embed(table, ids, scale=1.75, out=out)
    want = ref.embed(host(table), at, 1.75)
    # 1.75 times a value is rounded in fp32 first, then to the output's type
    check(out, want, out_bound(want, U * np.abs(want), rt), "out")
    assert intact()
    assert torch.equal(ops.embed(table, ids, scale=1.75, dtype=rt).nan_to_num(7.0), out.nan_to_num(7.0))


@pytest.mark.parametrize("accumulate", (False, True))
@pytest.mark.parametrize("case", EMBED)
def test_embed_gradient(case, accumulate):
    torch, ops = torch_and_ops()
    tokens, vocab, dim, tt, rt, ids, at, ld, shift, rng = embed_case(case)
    values = rng.standard_normal((tokens, dim))
    outside = (at < 0) | (at >= vocab)
    values[outside] = np.nan            # what padding's gradient holds does not count
    dout = placed(values, rt, ld, shift)
    out, intact = margins(vocab, dim, tt, ld, shift)
    old = np.zeros((vocab, dim))
    if accumulate:
        out.copy_(torch.as_tensor(rng.standard_normal((vocab, dim))))
        old = host(out)
    again = out.clone()
    ops.embed_grad(dout, ids, vocab, scale=0.375, out=out, accumulate=accumulate)
    d = host(dout)
    d[outside] = 0.0
    new = ref.embed_grad(d, at, vocab, 0.375)
    count = np.bincount(at[~outside], minlength=vocab)[:, None]
    size = ref.embed_grad(np.abs(d), at, vocab, 0.375)
    want = old + new
    bound = (count + 2) * U * size + 2 * U * np.abs(want)
    check(out, want, np.where(count > 0, out_bound(want, bound, tt), 0.0), "dtable")
    assert intact()
    twice = torch.empty_like(out) if not accumulate else again
    ops.embed_grad(dout, ids, vocab, scale=0.375, out=twice, accumulate=accumulate)
    assert torch.equal(twice, out)      # no sum depends on timing


def test_embed_without_tokens():
    torch, ops = torch_and_ops()
    ids = torch.empty((2, 0), dtype=torch.int64, device="cuda")
    assert ops.embed(torch.ones(3, 8, device="cuda"), ids).shape == (2, 0, 8)
    dout = torch.empty((2, 0, 8), device="cuda")
    assert not ops.embed_grad(dout, ids, 3).any()
    keep = torch.ones(3, 8, device="cuda")
    assert bool((ops.embed_grad(dout, ids, 3, out=keep, accumulate=True) == 1).all())


def test_embed_gradient_matches_differences():
    """Along a random direction of the table the lookup, linear in it, moves by what the
    gradient says."""
    torch, ops = torch_and_ops()
    g = torch.Generator(device="cuda").manual_seed(4)
    table, step = (torch.randn(50, 24, device="cuda", generator=g) for _ in range(2))
    ids = torch.randint(-1, 50, (200,), device="cuda", generator=g)
    dout = torch.randn(200, 24, device="cuda", generator=g)
    grad = ops.embed_grad(dout, ids, 50, scale=3.0)
    up, down = (ops.embed(table + h * step, ids, scale=3.0).double() for h in (1.0, -1.0))
    diff = ((up - down) / 2 * dout.double()).sum()
    # table + step and its output are rounded: 3 u of each of the 4800 terms' sizes at most
    size = (3.0 * (table.abs().amax() + step.abs().amax()) * dout.abs().sum()).double()
    assert abs(diff - (grad.double() * step.double()).sum()) < 6 * U * size


# ------------------------------------------------- norms of queries and keys

QK = [
    # batch, seq, heads, kv, dim, rot, dtype, interleaved, layout, gains
    (1, 1, 1, 1, 2, 2, "f32", False, "plain", "f32"),
    (1, 1, 20, 20, 64, 64, "bf16", False, "plain", "f32"),
    (3, 7, 4, 2, 64, 64, "bf16", False, "fused", "f32"),
    (2, 33, 3, 1, 64, 32, "bf16", True, "fused", "bf16"),
    (2, 19, 5, 5, 80, 80, "bf16", False, "heads", "f32"),
    (1, 130, 6, 2, 96, 48, "f32", False, "plain", None),
    (2, 65, 8, 8, 128, 128, "bf16", True, "plain", "f32"),
    (2, 65, 8, 4, 128, 128, "f32", False, "heads", "f32"),
    (1, 9, 2, 2, 256, 256, "bf16", False, "plain", "f32"),
    (1, 9, 2, 1, 512, 128, "f32", True, "plain", "f32"),
    (1, 5, 1, 1, 1024, 1024, "f32", False, "plain", "f32"),
    (2, 11, 3, 3, 7, 4, "f32", False, "plain", "f32"),
    (2, 11, 3, 3, 65, 0, "bf16", False, "plain", "f32"),
    (1, 40, 12, 12, 32, 32, "bf16", True, "odd", "f32"),
    (1, 40, 12, 0, 48, 24, "f32", False, "odd", "f32"),
    (5, 301, 20, 20, 64, 64, "bf16", False, "fused", "f32"),
    (4, 257, 24, 6, 80, 40, "f32", True, "plain", "f32"),
    (1, 1000, 1, 1, 16, 16, "bf16", False, "plain", "f32"),
]


def heads_view(values, dtype, layout, shift=None):
    """values [batch, seq, heads, dim] on the GPU in a layout: plain, a slice of a wider activation
    (fused), heads before tokens (heads), or from an odd address with odd strides (odd)."""
    import torch
    b, s, h, d = values.shape
    if layout == "heads":
        t = torch.empty((b, h, s, d), dtype=dtype, device="cuda").transpose(1, 2)
    elif layout == "fused":
        t = torch.full((b, s, 3 * h * d + 16), float("nan"), dtype=dtype, device="cuda")
        t = t[..., 8:8 + h * d].view(b, s, h, d) if h else t.new_empty((b, s, 0, d))
    elif layout == "odd":
        t = torch.full((b * s * (h * (d + 1) + 3) + 1,), float("nan"), dtype=dtype, device="cuda")[1:]
        t = t.as_strided((b, s, h, d), (s * (h * (d + 1) + 3), h * (d + 1) + 3, d + 1, 1), 1)
    else:
        t = torch.empty((b, s, h, d), dtype=dtype, device="cuda")
    t.copy_(torch.as_tensor(values))
    return t


class QKCase:
    def __init__(self, case, seed=0):
        import torch
        (self.b, self.s, self.h, self.kv, self.d, self.rot, dt, self.inter, layout, gains) = case
        self.dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dt]
        rng = self.rng = np.random.default_rng(seed + self.d + 7 * self.s)
        shape = lambda h: (self.b, self.s, h, self.d)
        scale = np.exp(rng.standard_normal((self.b, self.s, 1, 1)))
        self.q, self.k = (heads_view(rng.standard_normal(shape(h)) * scale, self.dt, layout) for h in (self.h, self.kv))
        self.dq_out, self.dk_out = (heads_view(rng.standard_normal(shape(h)), self.dt, layout)
                                    for h in (self.h, self.kv))
        gt = {"f32": torch.float32, "bf16": torch.bfloat16}.get(gains)
        self.gains = [None if gains is None else torch.as_tensor(rng.uniform(0.5, 1.5, self.d)).to("cuda", gt)
                      for _ in range(2)]
        block = self.s + 5
        angle = rng.uniform(0, 6.3, (block, self.rot // 2))
        self.cos, self.sin = (torch.as_tensor(f(angle)).to("cuda", torch.float32) for f in (np.cos, np.sin))
        self.positions = torch.as_tensor(rng.integers(0, block, (self.b, self.s))).to("cuda")
        self.eps = float(np.float32(1e-5))

    def args(self):
        return (self.q, self.k, *self.gains, self.cos, self.sin)

    def angles(self, positions):
        at = np.broadcast_to(host(positions).astype(np.int64), (self.b, self.s))
        return host(self.cos)[at][:, :, None, :], host(self.sin)[at][:, :, None, :]

    def rolled(self, x, cos, sin):
        """Sizes of the terms of a rotation of x."""
        y = np.abs(x)
        a, b = ref._pairs(self.rot, self.inter)
        c, s = np.abs(cos), np.abs(sin)
        out = y.copy()
        out[..., a] = y[..., a] * c + y[..., b] * s
        out[..., b] = y[..., b] * c + y[..., a] * s
        return out

    def check_forward(self, q, k, positions):
        cos, sin = self.angles(positions)
        for got, x, gain in ((q, self.q, self.gains[0]), (k, self.k, self.gains[1])):
            x = host(x)
            g = np.ones(self.d) if gain is None else host(gain)
            want = ref.qk_norm(x, g, cos, sin, self.eps, self.inter)
            r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + self.eps)
            size = self.rolled(x * r * g, cos, sin)
            check(got, want, out_bound(want, (self.d / 2 + 16) * U * size, self.dt), "y")

    def check_backward(self, grads, positions):
        cos, sin = self.angles(positions)
        dq, dk, dqg, dkg = grads
        for dx, dg, dy, x, gain in ((dq, dqg, self.dq_out, self.q, self.gains[0]),
                                    (dk, dkg, self.dk_out, self.k, self.gains[1])):
            x, dy = host(x), host(dy)
            g = np.ones(self.d) if gain is None else host(gain)
            want, want_g = ref.qk_norm_grad(dy, x, g, cos, sin, self.eps, self.inter)
            r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + self.eps)
            dn = self.rolled(dy, cos, sin)
            size = r * (dn * g + np.abs(x) * r * r * (dn * g * np.abs(x)).mean(-1, keepdims=True))
            check(dx, want, out_bound(want, (self.d + 32) * U * size, self.dt), "dx")
            if gain is not None:
                rows = max(1, x[..., 0].size)
                size_g = (dn * np.abs(x) * r).reshape(-1, self.d).sum(0)
                check(dg, want_g, (rows + self.d + 32) * U * size_g + TINY, "dgain")
            else:
                assert dg is None


@pytest.mark.parametrize("case", QK)
def test_qk_norm(case):
    torch, ops = torch_and_ops()
    c = QKCase(case)
    how = dict(eps=c.eps, interleaved=c.inter)
    q, k = ops.qk_norm(*c.args(), positions=c.positions, **how)
    c.check_forward(q, k, c.positions)
    # 32-bit positions, shared positions, none, and a layout of the outputs' own
    q2, k2 = ops.qk_norm(*c.args(), positions=c.positions.int(), **how)
    assert torch.equal(q, q2) and torch.equal(k, k2)
    c.check_forward(*ops.qk_norm(*c.args(), positions=c.positions[0], **how), c.positions[:1])
    c.check_forward(*ops.qk_norm(*c.args(), positions=c.positions[:1].expand(c.b, c.s), **how), c.positions[:1])
    c.check_forward(*ops.qk_norm(*c.args(), **how), torch.arange(c.s)[None])
    odd = [heads_view(np.zeros(t.shape), c.dt, "odd") for t in (c.q, c.k)]
    ops.qk_norm(*c.args(), positions=c.positions, q_out=odd[0], k_out=odd[1], **how)
    c.check_forward(*odd, c.positions)
    if c.b == 1:
        flat = [t[0] for t in (c.q, c.k)]
        q3, k3 = ops.qk_norm(*flat, *c.args()[2:], positions=c.positions[0], **how)
        assert torch.equal(q3, q[0]) and torch.equal(k3, k[0])
    # in place
    ops.qk_norm(*c.args(), positions=c.positions, q_out=c.q, k_out=c.k, **how)
    assert torch.equal(c.q, q) and torch.equal(c.k, k)


@pytest.mark.parametrize("case", QK)
def test_qk_norm_gradient(case):
    torch, ops = torch_and_ops()
    c = QKCase(case, seed=1)
    how = dict(positions=c.positions, eps=c.eps, interleaved=c.inter)
    grads = ops.qk_norm_grad(c.dq_out, c.dk_out, *c.args(), **how)
    c.check_backward(grads, c.positions)
    again = ops.qk_norm_grad(c.dq_out, c.dk_out, *c.args(), **how)
    for a, b in zip(grads, again):
        assert (a is None and b is None) or torch.equal(a, b)
    # into the incoming gradients' own buffers
    dy = c.dq_out.clone(), c.dk_out.clone()
    place = ops.qk_norm_grad(c.dq_out, c.dk_out, *c.args(), dq=c.dq_out, dk=c.dk_out, **how)
    assert torch.equal(place[0], grads[0]) and torch.equal(place[1], grads[1])
    # and into the inputs'
    place = ops.qk_norm_grad(*dy, *c.args(), dq=c.q, dk=c.k, **how)
    assert torch.equal(place[0], grads[0]) and torch.equal(place[1], grads[1])


def test_qk_norm_output_margins():
    torch, ops = torch_and_ops()
    c = QKCase((2, 37, 6, 3, 48, 48, "bf16", False, "plain", "f32"))
    outs = [margins(1, t.numel(), c.dt) for t in (c.q, c.k, c.q, c.k)]
    views = [o.view(t.shape) for (o, _), t in zip(outs, (c.q, c.k, c.q, c.k))]
    ops.qk_norm(*c.args(), positions=c.positions, eps=c.eps, q_out=views[0], k_out=views[1])
    ops.qk_norm_grad(c.dq_out, c.dk_out, *c.args(), positions=c.positions, eps=c.eps, dq=views[2], dk=views[3])
    assert all(intact() for _, intact in outs)


@pytest.mark.parametrize("dim", (64, 20))
def test_qk_norm_positions_outside_the_tables_and_empty_rows(dim):
    torch, ops = torch_and_ops()
    c = QKCase((2, 9, 2, 2, dim, 8, "f32", False, "plain", "f32"))
    c.positions[0, 3] = -1
    c.positions[1, 8] = c.cos.shape[0]
    c.q[1, 2] = 0.0
    q, k = ops.qk_norm(*c.args(), positions=c.positions, eps=c.eps)
    bad = torch.zeros(2, 9, dtype=torch.bool)
    bad[0, 3] = bad[1, 8] = True
    assert bool(q[bad][..., :8].isnan().all()) and bool(q[bad][..., 8:].isfinite().all())
    assert bool(q[~bad].isfinite().all()) and bool(k[~bad].isfinite().all()) and not q[1, 2].any()
    dq, dk, dqg, _ = ops.qk_norm_grad(c.dq_out, c.dk_out, *c.args(), positions=c.positions, eps=c.eps)
    assert bool(dq[bad].isnan().all()) and bool(dq[~bad].isfinite().all()) and bool(dqg[:8].isnan().all())
    none = ops.qk_norm_grad(c.dq_out[:, :0], c.dk_out[:, :0], c.q[:, :0], c.k[:, :0], *c.args()[2:])
    assert none[0].shape == (2, 0, 2, dim) and not none[2].any() and not none[3].any()


def test_qk_norm_gradient_matches_differences():
    torch, ops = torch_and_ops()
    c = QKCase((2, 21, 4, 4, 64, 64, "f32", False, "plain", "f32"), seed=5)
    how = dict(positions=c.positions, eps=c.eps)
    dq, _, dqg, _ = ops.qk_norm_grad(c.dq_out, c.dk_out, *c.args(), **how)
    step = torch.randn(c.q.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    gstep = torch.randn(64, device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    h = 2.0 ** -7

    def value(sign):
        y, _ = ops.qk_norm(c.q + sign * h * step, c.k, c.gains[0] + sign * h * gstep, *c.args()[3:], **how)
        return (y.double() * c.dq_out.double()).sum()

    diff = (value(1) - value(-1)) / (2 * h)
    want = (dq.double() * step.double()).sum() + (dqg.double() * gstep.double()).sum()
    # the third derivative's term, h^2 / 6 of values of order 1 a piece (10752 of random sign, rows of
    # rms down to 0.1 making it a thousand times that), and 32 u / h of rounding for each
    n = c.q.numel()
    assert abs(diff - want) < (h * h / 6 * 1000 + 32 * U / h) * np.sqrt(n) * 4


# --------------------------------------------------------------- distillation

DISTILL = [
    # rows, vocab, top, dtype, teacher, ids, tau, kind, ld pad, shift, grad ld pad, grad shift
    (1, 1, 1, "f32", "f32", "i32", 1.0, "any", 0, 0, 0, 0),
    (3, 7, 2, "bf16", "f32", "i64", 1.0, "any", 0, 0, 0, 0),
    (5, 100, 0, "f32", "f32", "i32", 1.0, "any", 0, 0, 0, 0),
    (17, 513, 5, "f32", "bf16", "i64", 2.0, "short", 0, 0, 0, 0),
    (16, 1000, 16, "bf16", "f32", "i32", 0.5, "masked", 8, 0, 8, 0),
    (9, 999, 16, "bf16", "f32", "i32", 1.5, "short", 3, 1, 3, 1),
    (9, 999, 16, "f32", "f32", "i32", 1.5, "short", 0, 0, 1, 2),
    (6, 2001, 33, "f32", "f32", "i64", 4.0, "twice", 0, 3, 0, 3),
    (4, 1500, 1024, "bf16", "bf16", "i32", 1.0, "twice", 0, 0, 0, 0),
    (200, 257, 8, "f32", "f32", "i32", 1.0, "masked", 0, 0, 0, 0),
    (2, 50304, 64, "bf16", "f32", "i32", 2.0, "any", 0, 0, 0, 0),
    (3, 50257, 64, "f32", "f32", "i64", 1.0, "short", 0, 0, 0, 0),
    (41, 9001, 20, "bf16", "f32", "i32", 1.0, "hidden", 0, 0, 0, 0),
    (2, 131072, 10, "f32", "f32", "i32", 0.25, "hidden", 0, 0, 0, 0),
    (7, 4096, 12, "f32", "f32", "i32", 3.0, "lowest", 0, 0, 0, 0),
    (300, 5000, 3, "bf16", "f32", "i32", 1.0, "lowest", 0, 0, 0, 0),
    (2, 300001, 100, "bf16", "f32", "i32", 1.0, "any", 0, 0, 0, 0),
]


class DistillCase:
    def __init__(self, case):
        import torch
        (self.n, self.v, self.k, dt, teacher, ids, self.tau, kind, pad, shift, self.gpad, self.gshift) = case
        types = {"f32": torch.float32, "bf16": torch.bfloat16, "i32": torch.int32, "i64": torch.int64}
        self.dt = types[dt]
        rng = self.rng = np.random.default_rng(self.n * 1000 + self.v + self.k)
        x = rng.standard_normal((self.n, self.v)) * 2.5
        top = np.stack([rng.choice(self.v, self.k, replace=self.k > self.v) for _ in range(self.n)]) \
            if self.k else np.zeros((self.n, 0), np.int64)
        t = rng.standard_normal((self.n, self.k)) * 2
        self.weight = rng.uniform(0.5, 1.5, self.n).astype(np.float32)
        self.dloss = rng.standard_normal(self.n).astype(np.float32)
        if kind == "short":         # absent entries: negative, past the vocabulary, or a teacher's -inf
            top[rng.random(top.shape) < 0.3] = -1
            top[rng.random(top.shape) < 0.1] = self.v
            t[rng.random(top.shape) < 0.1] = -np.inf
            top[0] = -1
            t[-1] = -np.inf
        elif kind == "masked":      # rows that do not count hold what they like
            off = rng.random(self.n) < 0.4
            self.weight[off] = 0.0
            x[off] = np.nan
            t[off] = np.inf
        elif kind == "twice":
            top[:, 1::2] = top[:, 0:-1:2] if self.k % 2 == 0 else top[:, 0:-2:2]
        elif kind == "hidden":      # entries of the vocabulary that are switched off
            x[rng.random(x.shape) < 0.5] = -np.inf
            x[:, : self.v // 3] = -np.inf
            np.put_along_axis(x, top, rng.standard_normal(top.shape), 1)
        elif kind == "lowest":
            low = float(torch.finfo(self.dt).min)
            x[rng.random(x.shape) < 0.5] = low
            x[0] = low              # a row of nothing else is a uniform one
            t[1 % self.n] = float(torch.finfo(torch.float32).min)
        self.ids_np = top
        self.x = placed(x, self.dt, self.v + pad, shift)
        self.top_ids = torch.as_tensor(top).to("cuda", types[ids])
        self.t = torch.as_tensor(t).to("cuda", types[teacher])
        self.w = torch.as_tensor(self.weight).to("cuda")

    def oracle(self, dloss=None):
        return ref.distill(host(self.x), self.ids_np, host(self.t), self.weight, self.tau, dloss)

    def bounds(self, dloss=None):
        """(loss, stats, gradient) bounds.  Half an ulp of every value that goes into an exponent is an
        error relative to its size; a sum of the vocabulary takes at most v / 512 + 32 additions in a row."""
        x, t, n = host(self.x), host(self.t), self.n
        with np.errstate(all="ignore"):
            on = (self.weight != 0) & ((self.ids_np >= 0) & (self.ids_np < self.v) & (t != -np.inf)).any(1)
            m = np.where(on, np.nanmax(np.where(np.isnan(x), -np.inf, x), 1), 0.0)[:, None]
            depth = np.where(on[:, None], (m - x) / self.tau, 0.0)
            q = np.where(on[:, None], np.exp(-depth), 0.0)
            s = np.maximum(q.sum(1), 1e-30)
            q /= s[:, None]
            mean_depth = (q * np.where(q > 0, depth, 0.0)).sum(1)
            rel_s = (self.v / 512 + 64 + 8 * mean_depth) * U        # relative error of the sum
            listed = (self.ids_np >= 0) & (self.ids_np < self.v) & (t != -np.inf) & on[:, None]
            tt = np.where(listed, t / self.tau, -np.inf)
            tt = np.where(listed, tt - np.where(on, tt.max(1, initial=-np.inf), 0.0)[:, None], -np.inf)
            p = np.where(listed, np.exp(tt), 0.0)
            p /= np.maximum(p.sum(1), 1e-30)[:, None]
            x_at = np.take_along_axis(depth, np.clip(self.ids_np, 0, self.v - 1).astype(np.int64), 1) if self.k else p
            size = np.where(p > 0, p * (4 + np.where(p > 0, np.abs(tt), 0) + x_at + np.log(self.v) + np.log(self.k + 1)), 0)
            w = self.weight.astype(np.float64)
            loss = w * self.tau ** 2 * (rel_s + ((self.k + 32) * U) * size.sum(1)) + TINY
            f = np.abs(w * (1 if dloss is None else dloss)) * self.tau
            err_p = np.where(p > 0, p * (self.k + 32 + 4 * np.abs(np.where(p > 0, tt, 0))) * U, 0.0)
            grad = q * (rel_s[:, None] + (16 + 8 * np.where(q > 0, depth, 0.0)) * U)
            target = np.zeros_like(q)
            for i in range(n):
                np.add.at(target[i], np.clip(self.ids_np[i], 0, self.v - 1).astype(np.int64), err_p[i])
            grad = f[:, None] * (grad + target)
            # exponentials below fp32's smallest normal are 0
            grad = grad + f[:, None] * 2.0 ** -126 + TINY
        return loss, np.stack([np.zeros(n), rel_s * s], 1) + TINY, grad


@pytest.mark.parametrize("case", DISTILL)
def test_distill_loss(case):
    torch, ops = torch_and_ops()
    c = DistillCase(case)
    loss, stats = ops.distill_loss(c.x, c.top_ids, c.t, weight=c.w, temperature=c.tau)
    want, want_stats, _ = c.oracle()
    bound, bound_stats, _ = c.bounds()
    check(loss, want, bound, "loss")
    check(stats, want_stats, bound_stats, "stats")
    again, _ = ops.distill_loss(c.x, c.top_ids, c.t, weight=c.w, temperature=c.tau)
    assert torch.equal(loss, again)


@pytest.mark.parametrize("case", DISTILL)
def test_distill_gradient(case):
    torch, ops = torch_and_ops()
    c = DistillCase(case)
    args, how = (c.x, c.top_ids, c.t), dict(weight=c.w, temperature=c.tau)
    loss, stats = ops.distill_loss(*args, **how)
    out, intact = margins(c.n, c.v, c.dt, c.v + c.gpad, c.gshift)
    both, got = ops.distill_loss_grad(*args, dlogits=out, **how)
    want_loss, _, want = c.oracle()
    bound_loss, _, bound = c.bounds()
    check(got, want, out_bound(want, bound, c.dt), "dlogits")
    check(both, want_loss, bound_loss, "loss")
    assert intact()
    assert torch.equal(ops.distill_loss_grad(*args, **how)[1], got)
    # from the statistics, with the gradient of each loss
    dloss = torch.as_tensor(c.dloss).cuda()
    dloss[c.n // 2] = 0.0
    _, _, want = c.oracle(host(dloss))
    _, _, bound = c.bounds(host(dloss))
    out2, intact2 = margins(c.n, c.v, c.dt, c.v + c.gpad, c.gshift)
    ops.distill_grad(*args, stats, dloss=dloss, dlogits=out2, **how)
    check(out2, want, out_bound(want, bound, c.dt), "dlogits of dloss")
    assert intact2()
    plain = ops.distill_grad(*args, stats, **how)
    # in place of the logits
    keep = c.x.clone()
    ops.distill_grad(*args, stats, dlogits=c.x, **how)
    assert torch.equal(c.x, plain)
    c.x.copy_(keep)
    ops.distill_loss_grad(*args, dlogits=c.x, **how)
    assert torch.equal(c.x, got)


@pytest.mark.parametrize("dtype", ("f32", "bf16"))
@pytest.mark.parametrize("tau", (1e-2, 1e-4, 1e-7, 1e-12))
def test_distill_at_cold_temperatures(tau, dtype):
    """Exponents of any size: s / T reaches 1e14, and softmax is all but the largest entry."""
    torch, ops = torch_and_ops()
    c = DistillCase((6, 2500, 20, dtype, "f32", "i32", tau, "any", 0, 0, 0, 0))
    loss, dx = ops.distill_loss_grad(c.x, c.top_ids, c.t, weight=c.w, temperature=c.tau)
    want_loss, want_stats, want = c.oracle()
    bound_loss, bound_stats, bound = c.bounds()
    check(loss, want_loss, bound_loss, "loss")
    check(dx, want, out_bound(want, bound, c.dt), "dlogits")
    again, stats = ops.distill_loss(c.x, c.top_ids, c.t, weight=c.w, temperature=c.tau)
    check(stats, want_stats, bound_stats, "stats")
    assert torch.equal(ops.distill_grad(c.x, c.top_ids, c.t, stats, weight=c.w, temperature=c.tau), dx)


def test_distill_of_any_weight_and_shape():
    torch, ops = torch_and_ops()
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(2, 3, 50, device="cuda", generator=g)
    t, ids = x.topk(4, dim=-1)
    loss, dx = ops.distill_loss_grad(x, ids, t)
    flat, dflat = ops.distill_loss_grad(x.view(6, 50), ids.view(6, 4), t.view(6, 4), weight=torch.ones(6, device="cuda"))
    assert loss.shape == (2, 3) and torch.equal(loss.view(6), flat) and torch.equal(dx.view(6, 50), dflat)
    # a teacher that lists the whole vocabulary and agrees with the student
    t, ids = x.sort(dim=-1)
    loss, dx = ops.distill_loss_grad(x, ids, t)
    assert loss.abs().max() < 60 * U * 8 and dx.abs().max() < 60 * U


@pytest.mark.parametrize("value", (float("nan"), float("inf")))
def test_distill_propagates_what_counts(value):
    torch, ops = torch_and_ops()
    x = torch.zeros(3, 5000, device="cuda")
    x[1, 4321] = value
    x[2] = -float("inf")
    ids = torch.tensor([[7, 8]] * 3, device="cuda")
    loss, dx = ops.distill_loss_grad(x, ids, torch.zeros(3, 2, device="cuda"))
    assert bool(loss[0].isfinite()) and bool(dx[0].isfinite().all())
    assert bool(loss[1:].isnan().all()) and bool(dx[2].isnan().all()) and bool(dx[1].isnan().any())


def test_distill_gradient_matches_differences():
    torch, ops = torch_and_ops()
    g = torch.Generator(device="cuda").manual_seed(9)
    x, step = (torch.randn(12, 700, device="cuda", generator=g) for _ in range(2))
    t, ids = torch.randn(12, 700, device="cuda", generator=g).topk(9, dim=1)
    _, dx = ops.distill_loss_grad(x, ids, t, temperature=1.5)
    h = 2.0 ** -6
    up, down = (ops.distill_loss(x + s * h * step, ids, t, temperature=1.5)[0].double().sum() for s in (1, -1))
    # third derivatives of order 1 along the step, 12 rows; losses below 32 to 16 u each
    assert abs((up - down) / (2 * h) - (dx.double() * step.double()).sum()) < 12 * (h * h + 16 * U * 32 / h)


def test_operators_on_another_stream():
    """Inputs made and outputs read on a side stream, with the work of the current one unfinished."""
    torch, ops = torch_and_ops()
    side = torch.cuda.Stream()
    x = torch.randn(64, 4000, device="cuda")
    t, ids = x.topk(8, dim=1)
    table = torch.randn(4000, 64, device="cuda")
    want = ops.distill_loss_grad(x, ids, t)[1], ops.embed_grad(table[:64], ids[:, 0].contiguous(), 4000)
    first = ids[:, 0].contiguous()
    torch.cuda.synchronize()
    for _ in range(3):
        got = (ops.distill_loss_grad(x, ids, t, stream=side)[1], ops.embed_grad(table[:64], first, 4000, stream=side))
        junk = [torch.full((64, 4000), 3.0, device="cuda") for _ in range(4)]
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and len(junk) == 4


def test_the_binding_refuses():
    torch, ops = torch_and_ops()
    f = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype, device="cuda")
    i = lambda *s, dtype=torch.int64: torch.zeros(s, dtype=dtype, device="cuda")
    half = torch.float16
    bad = [
        lambda: ops.embed(f(8), i(4)),
        lambda: ops.embed(f(8, 4, dtype=half), i(4)),
        lambda: ops.embed(f(8, 4), i(4, dtype=torch.int16)),
        lambda: ops.embed(f(8, 4), i(4, 2)[:, 0]),
        lambda: ops.embed(f(4, 8).t(), i(4)),
        lambda: ops.embed(f(8, 4), i(4), out=f(4, 5)),
        lambda: ops.embed(f(8, 4), i(4), out=f(1, 4).expand(4, 4)),
        lambda: ops.embed(f(8, 4), torch.zeros(4, dtype=torch.int64)),
        lambda: ops.embed_grad(f(5, 4), i(4), 8),
        lambda: ops.embed_grad(f(4, 4), i(4), 8, accumulate=True),
        lambda: ops.embed_grad(f(4, 4), i(4), 8, out=f(7, 4)),
        lambda: ops.embed_grad(f(1, 4).expand(4, 4), i(4), 8),
        lambda: ops.qk_norm(f(2, 3, 4, 8), f(2, 3, 4, 6), None, None, f(5, 4), f(5, 4)),
        lambda: ops.qk_norm(f(2, 3, 4, 8), f(2, 2, 4, 8), None, None, f(5, 4), f(5, 4)),
        lambda: ops.qk_norm(f(2, 3, 4, 8), f(2, 3, 4, 8), f(7), None, f(5, 4), f(5, 4)),
        lambda: ops.qk_norm(f(2, 3, 4, 8), f(2, 3, 4, 8), f(8), f(8, dtype=torch.bfloat16), f(5, 4), f(5, 4)),
        lambda: ops.qk_norm(f(2, 3, 4, 8), f(2, 3, 4, 8), None, None, f(5, 4), f(5, 3)),
        lambda: ops.qk_norm(f(2, 3, 4, 8), f(2, 3, 4, 8), None, None, f(5, 4), f(5, 4), positions=i(2, 4)),
        lambda: ops.qk_norm(f(2, 3, 4, 8), f(2, 3, 4, 8), None, None, f(5, 4), f(5, 4), q_out=f(2, 3, 4, 7)),
        lambda: ops.qk_norm(f(2, 3, 8, 4).transpose(2, 3), f(2, 3, 4, 8), None, None, f(5, 4), f(5, 4)),
        lambda: ops.qk_norm_grad(f(2, 3, 4, 8), f(2, 3, 3, 8), f(2, 3, 4, 8), f(2, 3, 4, 8), None, None, f(5, 4), f(5, 4)),
        lambda: ops.distill_loss(f(4, 9), i(4, 2), f(4, 3)),
        lambda: ops.distill_loss(f(4, 9), i(3, 2), f(3, 2)),
        lambda: ops.distill_loss(f(4, 9), f(4, 2), f(4, 2)),
        lambda: ops.distill_loss(f(4, 9, dtype=half), i(4, 2), f(4, 2)),
        lambda: ops.distill_loss(f(9, 4).t(), i(4, 2), f(4, 2)),
        lambda: ops.distill_loss(f(4, 9), i(4, 2), f(4, 2), weight=f(3)),
        lambda: ops.distill_grad(f(4, 9), i(4, 2), f(4, 2), f(4)),
        lambda: ops.distill_grad(f(4, 9), i(4, 2), f(4, 2), f(4, 2), dloss=f(3)),
        lambda: ops.distill_loss_grad(f(4, 9), i(4, 2), f(4, 2), dlogits=f(4, 8)),
    ]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    from paper_2608_05088_gb300 import malt
    with pytest.raises(malt.MaltError, match="-1"):
        ops.distill_loss(f(4, 9), i(4, 2), f(4, 2), temperature=0.0)
    with pytest.raises(malt.MaltError, match="-2"):
        ops.qk_norm(f(1, 1, 1, 1026), f(1, 1, 1, 1026), None, None, f(1, 2), f(1, 2))
