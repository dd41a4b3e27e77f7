"""The model operators where sizes, values, streams or types are at an edge."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("per_warp", (40, 64, 65, 300))
@pytest.mark.parametrize("rows", (1, 2, 3, 7, 31))
def test_every_token_of_crowded_rows_is_placed_once(per_warp, rows):
    """A few rows of one ordering block take most tokens, each row from lanes that differ from
    one group of 32 to the next.  Whole numbers, whose sums fp32 holds: a token that took
    another's place changes the result."""
    import torch
    from paper_2608_05088_gb300 import model_ops as ops
    tokens, vocab, dim = 32 * per_warp, 1024 * 4, 12
    g = torch.Generator().manual_seed(per_warp * 100 + rows)
    own = 5 + 128 * torch.randint(0, rows, (tokens,), generator=g)      # rows of one block of 128
    ids = torch.where(torch.rand(tokens, generator=g) < 0.8, own, torch.randint(-1, vocab, (tokens,), generator=g))
    dout = torch.randint(-8, 9, (tokens, dim), generator=g).float()
    want = torch.zeros(vocab, dim).index_add_(0, ids.clamp(min=0), dout * (ids >= 0)[:, None])
    for dtype in (torch.int32, torch.int64):
        at = ids.to("cuda", dtype)
        assert torch.equal(ops.embed_grad(dout.cuda(), at, vocab).cpu(), want)
        added = torch.ones(vocab, dim, device="cuda")
        ops.embed_grad(dout.cuda(), at, vocab, out=added, accumulate=True)
        assert torch.equal(added.cpu(), want + 1)


@pytest.mark.parametrize("dim", (128, 1280, 77))
def test_parts_of_long_rows_are_this_calls(dim):
    """Rows over many windows, gradients of changing whole numbers in memory that the call before
    left full of other parts: a part read too early changes a sum."""
    import torch
    from paper_2608_05088_gb300 import model_ops as ops
    tokens = 6000
    g = torch.Generator().manual_seed(dim)
    ids = torch.randint(0, 5, (tokens,), generator=g).cuda()
    douts = [torch.randint(-8, 9, (tokens, dim), generator=g).float().cuda() for _ in range(2)]
    want = [torch.zeros(5, dim, device="cuda", dtype=torch.float64).index_add_(0, ids, d.double()) for d in douts]
    for i in range(20):
        assert torch.equal(ops.embed_grad(douts[i % 2], ids, 5).double(), want[i % 2])


def _stream_calls(seed):
    """Every operator on inputs of one seed: calls that take a stream and return a list of results."""
    import torch
    from paper_2608_05088_gb300 import model_ops as ops
    g = torch.Generator("cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g)
    table, ids = normal(4000, 64), torch.randint(0, 40, (900,), device="cuda", generator=g)
    dout = normal(900, 64)
    q, k, dq, dk = (normal(2, 150, h, 64) for h in (8, 4, 8, 4))
    gain, cs = normal(64), normal(150, 32)
    x = normal(64, 4000)
    t, top = normal(64, 4000).topk(8, dim=1)
    stats = ops.distill_loss(x, top, t)[1]
    torch.cuda.synchronize()
    return [lambda s: [ops.embed(table, ids, stream=s)],
            lambda s: [ops.embed_grad(dout, ids, 4000, stream=s)],
            lambda s: list(ops.qk_norm(q, k, gain, gain, cs, cs, stream=s)),
            lambda s: list(ops.qk_norm_grad(dq, dk, q, k, gain, gain, cs, cs, stream=s)),
            lambda s: list(ops.distill_loss(x, top, t, stream=s)),
            lambda s: [ops.distill_grad(x, top, t, stats, stream=s)],
            lambda s: list(ops.distill_loss_grad(x, top, t, stream=s))]


@pytest.mark.parametrize("op", range(7))
def test_memory_of_a_call_on_another_stream(op):
    """Blocks that the current stream freed, its work on them still queued, are of the sizes that
    the call allocates; and a result dropped while the current stream has yet to read it is not
    handed to the next call."""
    import torch
    from paper_2608_05088_gb300 import malt
    first, second = _stream_calls(1)[op], _stream_calls(2)[op]
    want = first(None)
    side, here = torch.cuda.Stream(), torch.cuda.current_stream()
    sizes = [t.numel() * t.element_size() for t in want]
    sizes += [malt.load().malt_embed_workspace_bytes(900, 64), malt.load().malt_qk_norm_workspace_bytes(64)]
    for _ in range(3):
        freed = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(4)]
        torch.cuda.synchronize()
        torch.cuda._sleep(20_000_000)
        for t in freed:
            t.fill_(0x55)       # behind the sleep
        del freed, t
        got = first(side)
        side.synchronize()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        here.wait_stream(side)
        torch.cuda._sleep(20_000_000)
        kept = [t.clone() for t in got]         # behind the sleep
        del got
        other = second(side)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(kept, want)) and len(other) == len(want)


_LARGE_TABLES = """
import sys, torch
sys.path.insert(0, {root!r})
from paper_2608_05088_gb300 import model_ops as ops
vocab, dim = {vocab}, {dim}
ids = torch.randint(0, vocab, (300,), generator=torch.Generator().manual_seed(vocab))
dout = torch.randint(-8, 9, (300, dim), generator=torch.Generator().manual_seed(1)).float()
want = torch.zeros(vocab, dim).index_add_(0, ids, dout)
for index in (torch.int32, torch.int64):
    for table in (torch.float32, torch.bfloat16):
        got = ops.embed_grad(dout.cuda(), ids.to("cuda", index), vocab, dtype=table)
        assert torch.equal(got.float().cpu(), want), (index, table)
"""


@pytest.mark.parametrize("dim", (8, 5))
@pytest.mark.parametrize("vocab", (38400, 38401, 40478, 46208, 46209, 131072, 131073))
def test_embedding_gradient_of_any_vocabulary_alone(vocab, dim):
    """In a process of its own: nothing that a call of another size left behind helps this one."""
    import pathlib
    import subprocess
    import sys
    root = str(pathlib.Path(__file__).resolve().parent.parent)
    r = subprocess.run([sys.executable, "-c", _LARGE_TABLES.format(root=root, vocab=vocab, dim=dim)],
                       capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr[-2000:]


@pytest.mark.parametrize("teacher", ("float32", "bfloat16"))
@pytest.mark.parametrize("top", (1, 5, 40))
def test_a_teacher_of_nan_is_listed(top, teacher):
    """Rows: finite entries; one NaN among them; all NaN; NaN where nothing is listed."""
    import torch
    from paper_2608_05088_gb300 import model_ops as ops
    g = torch.Generator("cuda").manual_seed(top)
    x = torch.randn(4, 3000, device="cuda", generator=g)
    ids = torch.rand(4, 3000, device="cuda", generator=g).topk(top, dim=1).indices
    t = torch.randn(4, top, device="cuda", generator=g)
    t[1, top // 2] = t[2] = t[3] = float("nan")
    ids[3] = -1
    t = t.to(getattr(torch, teacher))
    loss, stats = ops.distill_loss(x, ids, t)
    both, dx = ops.distill_loss_grad(x, ids, t)
    alone = ops.distill_grad(x, ids, t, stats)
    for got in (loss, both):
        assert got.isnan().tolist() == [False, True, True, False] and got[3] == 0
    assert bool((stats[:3] > 0).all()) and not stats[3].any()
    listed = torch.zeros(4, 3000, dtype=torch.bool, device="cuda")
    listed[1:3].scatter_(1, ids[1:3], True)
    for got in (dx, alone):
        assert torch.equal(got.isnan(), listed) and not got[3].any() and bool((got[1:3][~listed[1:3]] > 0).all())


@pytest.mark.parametrize("rows,vocab", ((24, 2503), (24, 60000), (160, 1500), (160, 2503), (160, 6000), (160, 20000)))
@pytest.mark.parametrize("sign", (1, -1))
@pytest.mark.parametrize("tau", (1.085e-5, 3e-4, 1e-7))
def test_sums_where_the_maximum_crosses_the_exponents_range(tau, sign, rows, vocab):
    """Rows of two values a few ulps apart, s / T log2(e) of one below 2^20 in size and of the other
    not, the lower one first in every thread's order.  Bounds: u for each of the additions in a row
    (vocab / 512 + 64 at most) and a few of each exponent, which are below 1."""
    import numpy as np
    import torch
    from paper_2608_05088_gb300 import model_ops as ops
    u, f = 2.0 ** -24, np.float32
    rng = np.random.default_rng(vocab)
    tau = float(f(tau))
    c = f(1.4426950408889634) / f(tau)

    def step(v, n):
        for _ in range(abs(n)):
            v = np.nextafter(v, f(np.inf if n > 0 else -np.inf))
        return v

    edge = f(2.0 ** 20) / c
    while edge * c < f(2.0 ** 20):
        edge = step(edge, 1)
    while step(edge, -1) * c >= f(2.0 ** 20):
        edge = step(edge, -1)       # the first value past the range
    x = np.empty((rows, vocab), f)
    cut = rng.integers(vocab // 3, vocab // 2, rows)
    for i in range(rows):
        inside, past = step(edge, -int(rng.integers(1, 5))), step(edge, int(rng.integers(0, 4)))
        low, high = (inside, past) if sign > 0 else (-past, -inside)
        x[i, :cut[i]], x[i, cut[i]:] = low, high
    wide = x.astype(np.float64)
    m = wide.max(1, keepdims=True)
    e = np.exp((wide - m) / tau)
    total = e.sum(1)
    ids = np.tile([3, vocab - 2], (rows, 1))
    log_q = (np.take_along_axis(wide, ids, 1) - m) / tau - np.log(total)[:, None]
    want_loss = tau ** 2 * (0.5 * (np.log(0.5) - log_q)).sum(1)
    want = e / total[:, None]
    np.put_along_axis(want, ids, np.take_along_axis(want, ids, 1) - 0.5, 1)
    rel = (vocab / 512 + 64 + 8) * u

    args = (torch.from_numpy(x).cuda(), torch.from_numpy(ids).cuda(), torch.zeros(rows, 2, device="cuda"))
    loss, stats = ops.distill_loss(*args, temperature=tau)
    both, dx = ops.distill_loss_grad(*args, temperature=tau)
    alone = ops.distill_grad(*args, stats, temperature=tau)
    host = lambda t: t.double().cpu().numpy()
    assert (host(stats)[:, 0] == m[:, 0]).all()
    assert (np.abs(host(stats)[:, 1] / total - 1) <= rel).all()
    for got in (loss, both):
        assert (np.abs(host(got) - want_loss) <= tau ** 2 * (rel + 34 * u * (5 + np.abs(log_q).max()))).all()
    for got in (dx, alone):
        assert (np.abs(host(got) / tau - want) <= (rel + 24 * u) * e / total[:, None] + 34 * u * (want < 0)).all()


def test_autograd_sees_given_outputs_change():
    """A tensor that a call writes counts as modified, so a backward pass that has kept it refuses;
    what the call allocates belongs to no graph."""
    import torch
    from paper_2608_05088_gb300 import model_ops as ops
    new = lambda *s: torch.randn(*s, device="cuda")
    ids = torch.arange(6, device="cuda")
    q, gain, cs = new(1, 6, 2, 64), torch.ones(64, device="cuda"), new(6, 32)
    x = new(6, 100)
    t, top = x.topk(4, dim=1)
    stats = ops.distill_loss(x, top, t)[1]
    calls = [((6, 8), lambda out: ops.embed(new(9, 8), ids, out=out)),
             ((9, 8), lambda out: ops.embed_grad(new(6, 8), ids, 9, out=out)),
             ((9, 8), lambda out: ops.embed_grad(new(6, 8), ids, 9, out=out, accumulate=True)),
             (q.shape, lambda out: ops.qk_norm(q, q, gain, gain, cs, cs, q_out=out)),
             (q.shape, lambda out: ops.qk_norm(q, q, gain, gain, cs, cs, k_out=out)),
             (q.shape, lambda out: ops.qk_norm_grad(q, q, q, q, gain, gain, cs, cs, dq=out)),
             (q.shape, lambda out: ops.qk_norm_grad(q, q, q, q, gain, gain, cs, cs, dk=out)),
             (x.shape, lambda out: ops.distill_grad(x, top, t, stats, dlogits=out)),
             (x.shape, lambda out: ops.distill_loss_grad(x, top, t, dlogits=out)),
             (x.shape, lambda out: ops.distill_loss_grad(out, top, t, dlogits=out)),
             (x.shape, lambda out: ops.distill_loss_grad(x, top, t, dlogits=out, stream=torch.cuda.Stream()))]
    for shape, call in calls:
        y = new(*shape).requires_grad_().sigmoid()          # its gradient is made from y itself
        torch.cuda.synchronize()
        call(y.detach())
        torch.cuda.synchronize()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.sum().backward()
        with torch.inference_mode():
            call(new(*shape))
    table = new(9, 8).requires_grad_()
    assert not ops.embed(table, ids).requires_grad


def test_rows_of_a_wider_activation():
    """[batch, tokens, entries] views whose rows lie at one stride (a padded vocabulary's logits, a slice
    of an activation) are matrices like any other; views whose rows do not are refused.

    A distillation sum's order goes by its row's alignment, which the views do not share with their
    copies: two sums of 101 terms differ by twice 64 u and 8 u for each unit of depth (16 here at most),
    a loss also by (k + 32) u of |log p| + |log q| (32 at most), a gradient by 32 u more and as much of p."""
    import torch
    from paper_2608_05088_gb300 import model_ops as ops
    x = torch.randn(3, 7, 112, device="cuda")
    logits, wide = x[..., :101], torch.zeros(3, 7, 104, device="cuda")
    t, top = logits.topk(6, dim=-1)
    u = 2.0 ** -24
    same_loss = lambda a, b: bool(((a - b).abs() <= 2 * u * (64 + 128 + 38 * 32)).all())
    same_grad = lambda a, b: bool(((a - b).abs() <= 2 * u * (64 + 128 + 32 + 38)).all())
    loss, dx = ops.distill_loss_grad(logits.contiguous(), top, t)
    got, dgot = ops.distill_loss_grad(logits, top[..., :6], t, dlogits=wide[..., :101])
    assert same_loss(got, loss) and same_grad(dgot, dx) and not wide[..., 101:].any()
    assert same_grad(ops.distill_loss_grad(logits, top, t)[1], dx)
    few = ops.distill_loss(logits.contiguous(), top[..., :2].contiguous(), t[..., :2].contiguous())
    assert same_loss(ops.distill_loss(logits, top[..., :2], t[..., :2])[0], few[0])
    one = ops.distill_loss_grad(logits[1:2, 3:4], top[1:2, 3:4], t[1:2, 3:4])
    assert same_grad(one[1], dx[1:2, 3:4])
    table, ids = torch.randn(50, 24, device="cuda"), torch.randint(0, 50, (3, 7), device="cuda")
    out = torch.zeros(3, 7, 40, device="cuda")
    assert torch.equal(ops.embed(table, ids, out=out[..., 8:32]), table[ids]) and not out[..., :8].any()
    assert torch.equal(ops.embed_grad(out[..., 8:32], ids, 50), ops.embed_grad(table[ids], ids, 50))
    for bad in (x[:, :-1], x[:, ::2], x[..., ::2], x.transpose(0, 1), x[:1].expand(3, 7, 112), x.transpose(1, 2)):
        rows = torch.zeros(*bad.shape[:-1], 2, device="cuda")
        with pytest.raises(ValueError, match="stride|contiguous|overlapping"):
            ops.distill_loss(bad, rows.long(), rows)
