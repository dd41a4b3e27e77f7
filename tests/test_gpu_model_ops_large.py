"""The model operators past 2^31 elements (offsets of 64 bits), at their limits on sizes
that fit the GPU, and replayed from a CUDA graph."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def free_memory():
    import torch
    yield
    torch.cuda.empty_cache()


def test_embedding_of_a_table_past_32_bits():
    import torch
    from paper_2608_05088_gb300 import model_ops as ops
    vocab, dim = 1_100_000, 2048            # 2.25e9 elements
    table = torch.zeros(vocab, dim, dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([vocab - 1, 0, vocab - 2, vocab // 2, vocab - 1, -1, vocab], device="cuda")
    rows = torch.randn(5, dim, device="cuda").bfloat16()
    table[ids[:5]] = rows
    rows[0] = rows[4]                       # the same row twice
    table[vocab - 1] = rows[4]
    out = ops.embed(table, ids)
    assert torch.equal(out[:5], rows) and not out[5].any() and bool(out[6].isnan().all())
    del out
    table.fill_(5.0)
    d = torch.randn(7, dim, device="cuda").bfloat16()
    ops.embed_grad(d, ids, vocab, out=table)
    want = (d[0].float() + d[4].float()).bfloat16()
    assert torch.equal(table[vocab - 1], want)
    assert torch.equal(table[0], d[1]) and torch.equal(table[vocab - 2], d[2]) and torch.equal(table[vocab // 2], d[3])
    table[ids[:5]] = 0.0
    assert not table.any()                  # every other row was written as zero


def test_query_norms_of_tensors_past_32_bits():
    import torch
    from paper_2608_05088_gb300 import model_ops as ops
    shape, apart = (3, 3, 2), (1_100_000_000, 262144, 128, 1)      # the last batch starts at 2.2e9
    for dtype, dim in ((torch.bfloat16, 64), (torch.float32, 20)):     # aligned rows, and any
        storage = torch.empty(2_202_000_000, dtype=dtype, device="cuda")
        q = storage.as_strided((*shape, dim), apart)
        q.copy_(torch.randn(*shape, dim, device="cuda"))
        small = q.contiguous()
        cs = torch.rand(8, dim // 2, device="cuda")
        a = ops.qk_norm(q, q, None, None, cs, cs)
        b = ops.qk_norm(small, small, None, None, cs, cs)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        dy = torch.randn(*shape, dim, device="cuda").to(dtype)
        far = storage.as_strided((*shape, dim), apart, 64 * 4096)
        ops.qk_norm_grad(dy, dy, q, q, None, None, cs, cs, dq=far)
        assert torch.equal(far, ops.qk_norm_grad(dy, dy, small, small, None, None, cs, cs)[0])
        del storage, q, far


def test_distillation_of_logits_past_32_bits():
    import torch
    from paper_2608_05088_gb300 import model_ops as ops
    rows, vocab = 44_000, 50304             # 2.2e9 logits
    x = torch.empty(rows, vocab, dtype=torch.bfloat16, device="cuda").normal_()
    ids = torch.randint(0, vocab, (rows, 4), device="cuda")
    top = torch.randn(rows, 4, device="cuda")
    weight = torch.zeros(rows, device="cuda")
    weight[-3:] = 1.0
    weight[0] = 1.0
    keep = [0, rows - 3, rows - 2, rows - 1]
    loss, stats = ops.distill_loss(x, ids, top, weight=weight)
    want, dwant = ops.distill_loss_grad(x[keep].clone(), ids[keep], top[keep])
    assert torch.allclose(loss[keep], want, rtol=1e-5) and not loss[1:-3].any()
    ops.distill_grad(x, ids, top, stats, weight=weight, dlogits=x)      # in place
    assert torch.allclose(x[keep].float(), dwant.float(), rtol=2.0 ** -7, atol=1e-7)
    assert not x[1:-3].any()


def test_replayed_from_a_graph():
    import torch
    from paper_2608_05088_gb300 import model_ops as ops
    x = torch.randn(40, 3000, device="cuda")
    top, ids = x.topk(8, dim=1)
    q = torch.randn(2, 9, 4, 64, device="cuda")
    gain = torch.ones(64, device="cuda")
    cs = torch.rand(9, 32, device="cuda")
    table = torch.randn(3000, 64, device="cuda")
    tokens = ids[:, 0].contiguous()

    def work():
        a = ops.distill_loss_grad(x, ids, top)[1]
        b = ops.qk_norm_grad(q, q, q, q, gain, gain, cs, cs)
        c = ops.embed_grad(ops.embed(table, tokens), tokens, 3000)
        return (a, *b, c)

    want = [t.clone() for t in work()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = work()
    for _ in range(3):
        for t in got:
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
