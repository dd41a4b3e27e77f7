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
