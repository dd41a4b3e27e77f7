"""The output head at its edges: operands in one matrix, sums in parts, rows of few entries, views of a table whose
rows are no whole 16 bytes."""
import numpy as np
import pytest

from oracle import model_ops_ref as ref
from tests.test_gpu_head import BF16, F32, bounds, case
from tests.test_gpu_model_ops import U, check, out_bound, placed, torch_and_ops

pytestmark = pytest.mark.gpu


def test_columns_of_one_matrix():
    """Hidden rows and their gradient, table and its gradient side by side."""
    torch, ops = torch_and_ops()
    hidden, table, labels, weight = case(300, 64, 500, BF16, BF16)
    X, W = torch.as_tensor(hidden).bfloat16().cuda(), torch.as_tensor(table).bfloat16().cuda()
    Y, C = torch.as_tensor(labels).cuda(), torch.as_tensor(weight).cuda()
    want = ops.head_loss_grad(X, W, Y, weight=C)
    both, tables = torch.zeros(300, 128, device="cuda").bfloat16(), torch.zeros(500, 160, device="cuda").bfloat16()
    both[:, :64], tables[:, 64:128] = X, W
    loss, dh, dw = ops.head_loss_grad(both[:, :64], tables[:, 64:128], Y, weight=C, dhidden=both[:, 64:], dtable=tables[:, :64])
    assert torch.equal(loss, want[0]) and torch.equal(both[:, 64:], want[1]) and torch.equal(tables[:, :64], want[2])
    assert torch.equal(both[:, :64], X) and torch.equal(tables[:, 64:128], W) and not bool(tables[:, 128:].any())
    for bad in (dict(dhidden=both[:, 56:120]), dict(dtable=tables[:, 8:72]), dict(dhidden=X), dict(dtable=W)):
        args = (X, W) if bad.get("dhidden") is X or bad.get("dtable") is W else (both[:, :64], tables[:, 64:128])
        with pytest.raises(ops.malt.MaltError):
            ops.head_loss_grad(*args, Y, weight=C, **bad)


# What fills several parts: logits of more than 2048 entries (turned, and not); dtable of more than 1024 rows that
# count, as boxes and element by element; dhidden of pieces of more than 1024 entries.
@pytest.mark.parametrize("rows,dim,vocab", [(24, 2200, 300), (300, 2200, 600), (1500, 132, 700), (1500, 101, 700),
                                            (1531, 501, 32003)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_fp32_sums_in_parts(rows, dim, vocab, accumulate):
    """Against fp64 products.  A sum's parts lose what a sum of 32 or 16 slices of 64 does, so that relative 2-norms stay
    where those of one part are: with random signs some 1e-6; a part lost or taken twice is off by its share."""
    torch, ops = torch_and_ops()
    g = torch.Generator(device="cuda").manual_seed(rows + dim)
    W = torch.randn(vocab, dim, generator=g, device="cuda") * 1.5 / dim ** 0.5
    Y = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    X = torch.randn(rows, dim, generator=g, device="cuda") + 2 * W[Y]
    Y[torch.rand(rows, generator=g, device="cuda") < 0.1] = -1
    old = torch.randn(vocab, dim, generator=g, device="cuda") * 0.1
    dtable = old.clone() if accumulate else None
    loss, dh, dw = ops.head_loss_grad(X, W, Y, dtable=dtable, accumulate=accumulate)
    _, stats = ops.head_loss(X, W, Y)
    on = Y >= 0
    x, w = X.double()[on], W.double()
    l = x @ w.t()
    m = l.max(1).values
    lse = torch.logsumexp(l, 1)
    at = torch.arange(len(x), device="cuda")
    p = torch.exp(l - lse[:, None])
    p[at, Y[on]] -= 1
    near = lambda a, b, tol: float((a.double() - b).norm() / b.norm()) < tol
    assert near(loss[on], lse - l[at, Y[on]], 1e-5) and near(stats[on, 0], m, 3e-6)
    assert near(stats[on, 1], (lse - m).exp(), 1e-5)
    assert near(dh[on], p @ w, 5e-6) and float(dh[~on].abs().sum()) == 0
    want = p.t() @ x
    assert near(dw.double() - old if accumulate else dw, want, 5e-6)


@pytest.mark.parametrize("rows,dim,vocab", [(24, 2200, 300), (128, 4099, 520), (300, 2200, 600), (520, 4160, 700)])
@pytest.mark.parametrize("table_type", [BF16, F32])
def test_bf16_logits_in_parts(rows, dim, vocab, table_type):
    """Loss and gradients of bf16 rows longer than a part; element by element, within the bounds of their sums."""
    torch, ops = torch_and_ops()
    exact = table_type == F32
    hidden, table, labels, weight = case(rows, dim, vocab, BF16, table_type, seed=dim)
    X, W = torch.as_tensor(hidden).bfloat16().cuda(), torch.as_tensor(table).to(getattr(torch, table_type)).cuda()
    Y, C = torch.as_tensor(labels).cuda(), torch.as_tensor(weight).cuda()
    loss, m, s, dhidden, dtable = ref.head(hidden, table, labels, weight)
    b_loss, b_m, b_s, b_dh, b_dt = bounds(hidden, table, labels, weight, np.ones(rows), exact)
    got, stats = ops.head_loss(X, W, Y, weight=C)
    check(got, loss, b_loss, "loss")
    check(stats[:, 0], m, b_m + U * np.abs(m), "m")
    check(stats[:, 1], s, s * (b_s + b_m), "s")
    both, dh, dw = ops.head_loss_grad(X, W, Y, weight=C, dtype=torch.float32)
    assert torch.equal(both, got)
    check(dh, dhidden, out_bound(dhidden, b_dh, dh.dtype), "dhidden")
    check(dw, dtable, out_bound(dtable, b_dt, dw.dtype), "dtable")
    dh2, dw2 = ops.head_grad(X, W, Y, stats, weight=C, dtype=torch.float32)
    assert torch.equal(dh2, dh) and torch.equal(dw2, dw)
    # far below the bounds: dl's and the result's rounding
    near = lambda a, b, tol: float(np.linalg.norm(a.double().cpu().numpy() - b) / np.linalg.norm(b)) < tol
    assert near(got, loss, 1e-5) and near(dh, dhidden, 2.0 ** -8) and near(dw, dtable, 5e-6 if exact else 2.0 ** -8)


def test_views_of_a_table_with_odd_rows():
    """Rows whose last 16 bytes are shared with what lies behind them: it is not read into the logits."""
    torch, ops = torch_and_ops()
    for rows in (40, 300):
        for dim, ld in ((21, 24), (45, 48), (61, 72), (129, 136)):
            hidden, table, labels, weight = case(rows, dim, 700, BF16, BF16, seed=dim)
            X, Y, C = torch.as_tensor(hidden).bfloat16().cuda(), torch.as_tensor(labels).cuda(), torch.as_tensor(weight).cuda()
            W = placed(table, torch.bfloat16, ld)         # NaN behind every row
            want = ops.head_loss_grad(X, W.contiguous(), Y, weight=C)
            got = ops.head_loss_grad(X, W, Y, weight=C)
            assert all(bool(t.isfinite().all()) for t in got)
            assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("rows", [1, 24, 100, 300])
@pytest.mark.parametrize("dim", [1280, 4096])
def test_rows_of_one_entry(rows, dim):
    """A logit that is a single product is that product."""
    torch, ops = torch_and_ops()
    g = torch.Generator(device="cuda").manual_seed(rows)
    W = torch.randn(800, dim, generator=g, device="cuda").bfloat16()
    X = torch.zeros(rows, dim, device="cuda").bfloat16()
    k = torch.randint(0, dim, (rows,), generator=g, device="cuda")
    X[torch.arange(rows, device="cuda"), k] = 3.0
    Y = torch.randint(0, 800, (rows,), generator=g, device="cuda")
    for x, w in ((X, W), (X.float(), W), (X, W.float())):
        stats = ops.head_loss(x, w, Y)[1]
        assert torch.equal(stats[:, 0], (W.float()[:, k] * 3).max(0).values)


@pytest.mark.parametrize("rows", [24, 100, 300])
@pytest.mark.parametrize("dim,filled", [(1280, 1280), (1600, 800), (4096, 4096), (4096, 2048), (8200, 8200)])
def test_long_sums_of_one_sign(rows, dim, filled):
    """What a tensor core's cut-off sums lose on the average is put back, for as many terms as there are.

    A sum of n steps of 16 terms of one sign loses half an ulp of its partial sum a step, 0.36 n 2^-24 of the result:
    1.7e-6 at 1280, 2.7e-6 at 2048.  The mean over the rows' maxima is within 7e-7 of none: a quarter of that, and
    what is lost beside it (the spread of 80 to 256 steps, 3 ulp of 1.2e-7 over the root of 24 rows)."""
    torch, ops = torch_and_ops()
    g = torch.Generator(device="cuda").manual_seed(dim)
    W = (torch.rand(600, dim, generator=g, device="cuda") + 0.5).bfloat16()
    X = (torch.rand(rows, dim, generator=g, device="cuda") + 0.5).bfloat16()
    X[:, filled:] = 0
    Y = torch.full((rows,), 1, device="cuda")
    W[1] = 0                                    # (a label's logit is exact: not the largest)
    stats = ops.head_loss(X, W, Y)[1]
    want = (X.double() @ W.double().t()).max(1).values
    off = stats[:, 0].double() / want - 1
    assert abs(float(off.mean())) < 7e-7, float(off.mean())


@pytest.mark.parametrize("rows,dim,vocab", [(300, 739, 964), (300, 1600, 3000), (300, 4096, 2000)])
def test_gradients_on_statistics_from_elsewhere(rows, dim, vocab):
    """The gradient is that of the given statistics, here those of torch's fp32 products, to what logits of our own
    are off by: parts of 512 terms, of which each loses about two ulp of a partial sum of some units (2.4e-7 each)
    beside what is put back, eight of them 1.4e-6; a row's dl is as much of itself off, of which 2e-6 is the bound."""
    torch, ops = torch_and_ops()
    g = torch.Generator(device="cuda").manual_seed(dim)
    W = torch.randn(vocab, dim, generator=g, device="cuda") * 0.05
    Y = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    X = torch.randn(rows, dim, generator=g, device="cuda") + W[Y] * (8.0 / (0.0025 * dim))
    x = X @ W.t()
    m = x.amax(1)
    stats = torch.stack([m, (x - m[:, None]).exp().sum(1)], 1)
    dh, dw = ops.head_grad(X, W, Y, stats)
    p = torch.exp(X.double() @ W.double().t() - stats[:, :1].double()) / stats[:, 1:].double()
    p[torch.arange(rows, device="cuda"), Y] -= 1
    for got, want in ((dh, p @ W.double()), (dw, p.t() @ X.double())):
        assert float((got.double() - want).norm() / want.norm()) < 2e-6
