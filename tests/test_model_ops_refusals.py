"""Arguments that the model operators refuse, on the host and without a GPU: the C entry
points by status code, the binding by ValueError."""
import pytest
import torch

from paper_2608_05088_gb300 import build, malt, model_ops

F32, BF16, I32, I64 = malt.MALT_F32, malt.MALT_BF16, malt.MALT_I32, malt.MALT_I64
A = 1 << 20         # an aligned address that nothing reads: every call here fails before a launch


@pytest.fixture(scope="module")
def lib():
    build.build()
    return malt.load()


def embed(**kw):
    f = dict(ids=A, ids_dtype=I32, table_dtype=F32, rows_dtype=F32, scale=1.0, tokens=4, vocab=8, dim=16, table=A,
             table_ld=16, rows=A, rows_ld=16)
    f.update(kw)
    return model_ops._EMBED.pack(*f.values())


EMBED_BAD = [
    (dict(tokens=-1), malt.MALT_ERR_INVALID_ARG), (dict(vocab=-1), malt.MALT_ERR_INVALID_ARG),
    (dict(dim=-1), malt.MALT_ERR_INVALID_ARG), (dict(scale=float("nan")), malt.MALT_ERR_INVALID_ARG),
    (dict(ids=0), malt.MALT_ERR_INVALID_ARG), (dict(table=0), malt.MALT_ERR_INVALID_ARG),
    (dict(rows=0), malt.MALT_ERR_INVALID_ARG), (dict(table_ld=15), malt.MALT_ERR_INVALID_ARG),
    (dict(rows_ld=15), malt.MALT_ERR_INVALID_ARG), (dict(ids_dtype=F32), malt.MALT_ERR_UNSUPPORTED),
    (dict(table_dtype=I32), malt.MALT_ERR_UNSUPPORTED), (dict(rows_dtype=7), malt.MALT_ERR_UNSUPPORTED),
    (dict(tokens=1 << 31), malt.MALT_ERR_UNSUPPORTED), (dict(vocab=1 << 31), malt.MALT_ERR_UNSUPPORTED),
    (dict(dim=1 << 31, table_ld=1 << 31, rows_ld=1 << 31), malt.MALT_ERR_UNSUPPORTED),
    (dict(ids=A + 2), malt.MALT_ERR_MISALIGNED), (dict(ids=A + 4, ids_dtype=I64), malt.MALT_ERR_MISALIGNED),
    (dict(table=A + 2), malt.MALT_ERR_MISALIGNED), (dict(rows=A + 1, rows_dtype=BF16), malt.MALT_ERR_MISALIGNED),
]


@pytest.mark.parametrize("bad,code", EMBED_BAD)
def test_embed_refuses(lib, bad, code):
    assert lib.malt_embed_forward(embed(**bad), None) == code
    assert lib.malt_embed_backward(embed(**bad), 0, A, 1 << 40, None) == code


def test_embed_workspace_and_empty_calls(lib):
    need = lib.malt_embed_workspace_bytes(4, 16)
    assert need > 0 and lib.malt_embed_workspace_bytes(-1, 16) == 0
    assert lib.malt_embed_backward(embed(), 0, A, need - 1, None) == malt.MALT_ERR_INVALID_ARG
    assert lib.malt_embed_backward(embed(), 0, None, need, None) == malt.MALT_ERR_INVALID_ARG
    assert lib.malt_embed_backward(embed(), 0, A + 8, need, None) == malt.MALT_ERR_MISALIGNED
    assert lib.malt_embed_forward(None, None) == malt.MALT_ERR_INVALID_ARG
    # nothing to do: no launch
    assert lib.malt_embed_forward(embed(tokens=0, ids=0, rows=0), None) == malt.MALT_OK
    assert lib.malt_embed_backward(embed(tokens=0, ids=0, rows=0), 1, A, 1 << 20, None) == malt.MALT_OK
    assert lib.malt_embed_backward(embed(vocab=0, table=0), 0, A, 1 << 20, None) == malt.MALT_OK


def qk(**kw):
    f = dict(dtype=BF16, gain_dtype=F32, head_dim=64, rot_dim=64, interleaved=0, eps=1e-6, batch=2, seq=3, positions=0,
             positions_dtype=0, pad=0, stride=0, cos=A, sin=A, table_rows=8, q_gain=A, k_gain=A)
    f.update(kw)
    return model_ops._QK.pack(*f.values())


def heads(data=A, heads=4, batch_stride=3 * 256, seq_stride=256, head_stride=64):
    return model_ops._HEADS.pack(data, heads, batch_stride, seq_stride, head_stride)


QK_BAD = [
    (dict(dtype=I32), malt.MALT_ERR_UNSUPPORTED), (dict(gain_dtype=3), malt.MALT_ERR_UNSUPPORTED),
    (dict(head_dim=0), malt.MALT_ERR_UNSUPPORTED), (dict(head_dim=1025), malt.MALT_ERR_UNSUPPORTED),
    (dict(rot_dim=63), malt.MALT_ERR_INVALID_ARG), (dict(rot_dim=66), malt.MALT_ERR_INVALID_ARG),
    (dict(rot_dim=-2), malt.MALT_ERR_INVALID_ARG), (dict(eps=-1.0), malt.MALT_ERR_INVALID_ARG),
    (dict(eps=float("nan")), malt.MALT_ERR_INVALID_ARG), (dict(batch=-1), malt.MALT_ERR_INVALID_ARG),
    (dict(batch=1 << 16, seq=1 << 15), malt.MALT_ERR_UNSUPPORTED), (dict(cos=0), malt.MALT_ERR_INVALID_ARG),
    (dict(table_rows=-1), malt.MALT_ERR_INVALID_ARG), (dict(positions=A, positions_dtype=F32), malt.MALT_ERR_UNSUPPORTED),
    (dict(positions=A + 4, positions_dtype=I64), malt.MALT_ERR_MISALIGNED), (dict(sin=A + 2), malt.MALT_ERR_MISALIGNED),
    (dict(k_gain=A + 2), malt.MALT_ERR_MISALIGNED),
]


@pytest.mark.parametrize("bad,code", QK_BAD)
def test_qk_norm_refuses(lib, bad, code):
    h = heads()
    assert lib.malt_qk_norm_forward(qk(**bad), h, h, h, h, None) == code
    assert lib.malt_qk_norm_backward(qk(**bad), h, h, h, h, h, h, A, A, A, 1 << 40, None) == code


@pytest.mark.parametrize("bad,code", [
    (None, malt.MALT_ERR_INVALID_ARG), (dict(data=0), malt.MALT_ERR_INVALID_ARG),
    (dict(heads=5), malt.MALT_ERR_INVALID_ARG), (dict(heads=-1), malt.MALT_ERR_INVALID_ARG),
    (dict(data=A + 1), malt.MALT_ERR_MISALIGNED)])
def test_qk_norm_refuses_heads(lib, bad, code):
    h, b = heads(), None if bad is None else heads(**bad)
    for i in range(4):
        args = [b if j == i else h for j in range(4)]
        assert lib.malt_qk_norm_forward(qk(), *args, None) == code
    for i in range(6):
        args = [b if j == i else h for j in range(6)]
        assert lib.malt_qk_norm_backward(qk(), *args, A, A, A, 1 << 40, None) == code


def test_qk_norm_workspace_and_empty_calls(lib):
    h = heads()
    need = lib.malt_qk_norm_workspace_bytes(64)
    assert need > 0 and lib.malt_qk_norm_workspace_bytes(0) == 0
    assert lib.malt_qk_norm_backward(qk(), h, h, h, h, h, h, A, A, A, need - 1, None) == malt.MALT_ERR_INVALID_ARG
    assert lib.malt_qk_norm_backward(qk(), h, h, h, h, h, h, A, A, A + 8, need, None) == malt.MALT_ERR_MISALIGNED
    assert lib.malt_qk_norm_forward(qk(seq=0), h, h, h, h, None) == malt.MALT_OK
    n = heads(data=0, heads=0)
    assert lib.malt_qk_norm_forward(qk(), n, n, n, n, None) == malt.MALT_OK


def distill(**kw):
    f = dict(logits=A, ld=100, rows=4, vocab=100, dtype=F32, ids_dtype=I32, top_ids=A, top_ids_ld=8, top_logits=A,
             top_logits_ld=8, top=8, weight=A, top_dtype=F32, temperature=1.0)
    f.update(kw)
    return model_ops._DISTILL.pack(*f.values())


DISTILL_BAD = [
    (dict(rows=-1), malt.MALT_ERR_INVALID_ARG), (dict(vocab=0), malt.MALT_ERR_INVALID_ARG),
    (dict(top=-1), malt.MALT_ERR_INVALID_ARG), (dict(temperature=0.0), malt.MALT_ERR_INVALID_ARG),
    (dict(temperature=-1.0), malt.MALT_ERR_INVALID_ARG), (dict(temperature=float("nan")), malt.MALT_ERR_INVALID_ARG),
    (dict(temperature=float("inf")), malt.MALT_ERR_INVALID_ARG), (dict(ld=99), malt.MALT_ERR_INVALID_ARG),
    (dict(top_ids_ld=7), malt.MALT_ERR_INVALID_ARG), (dict(top_logits_ld=7), malt.MALT_ERR_INVALID_ARG),
    (dict(logits=0), malt.MALT_ERR_INVALID_ARG), (dict(top_ids=0), malt.MALT_ERR_INVALID_ARG),
    (dict(top_logits=0), malt.MALT_ERR_INVALID_ARG), (dict(dtype=I32), malt.MALT_ERR_UNSUPPORTED),
    (dict(ids_dtype=F32), malt.MALT_ERR_UNSUPPORTED), (dict(top_dtype=9), malt.MALT_ERR_UNSUPPORTED),
    (dict(top=1025, top_ids_ld=1025, top_logits_ld=1025), malt.MALT_ERR_UNSUPPORTED),
    (dict(rows=1 << 27), malt.MALT_ERR_UNSUPPORTED), (dict(vocab=1 << 31, ld=1 << 31), malt.MALT_ERR_UNSUPPORTED),
    (dict(logits=A + 2), malt.MALT_ERR_MISALIGNED), (dict(top_ids=A + 4, ids_dtype=I64), malt.MALT_ERR_MISALIGNED),
    (dict(weight=A + 2), malt.MALT_ERR_MISALIGNED),
]


@pytest.mark.parametrize("bad,code", DISTILL_BAD)
def test_distill_refuses(lib, bad, code):
    d = distill(**bad)
    ld = max(100, bad.get("ld", 0))
    assert lib.malt_distill_forward(d, A, A, None) == code
    assert lib.malt_distill_backward(d, A, A, A, ld, None) == code
    assert lib.malt_distill_forward_backward(d, A, A, A, ld, None) == code


def test_distill_refuses_outputs(lib):
    d = distill()
    assert lib.malt_distill_forward(d, None, A, None) == malt.MALT_ERR_INVALID_ARG
    assert lib.malt_distill_forward(d, A + 2, A, None) == malt.MALT_ERR_MISALIGNED
    assert lib.malt_distill_backward(d, None, A, A, 100, None) == malt.MALT_ERR_INVALID_ARG
    assert lib.malt_distill_backward(d, A, A, None, 100, None) == malt.MALT_ERR_INVALID_ARG
    assert lib.malt_distill_backward(d, A, A, A, 99, None) == malt.MALT_ERR_INVALID_ARG
    assert lib.malt_distill_backward(d, A, A, A + 2, 100, None) == malt.MALT_ERR_MISALIGNED
    assert lib.malt_distill_forward_backward(d, None, None, A, 100, None) == malt.MALT_ERR_INVALID_ARG
    empty = distill(rows=0, logits=0, top_ids=0, top_logits=0, weight=0)
    assert lib.malt_distill_forward_backward(empty, None, None, None, 100, None) == malt.MALT_OK


def test_the_binding_refuses_host_tensors():
    t, ids = torch.zeros(8, 16), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="CUDA"):
        model_ops.embed(t, ids)
    with pytest.raises(ValueError, match="CUDA"):
        model_ops.embed_grad(torch.zeros(4, 16), ids, 8)
    q, cs = torch.zeros(2, 3, 4, 16), torch.zeros(8, 8)
    with pytest.raises(ValueError, match="CUDA"):
        model_ops.qk_norm(q, q, None, None, cs, cs)
    with pytest.raises(ValueError, match="CUDA"):
        model_ops.qk_norm_grad(q, q, q, q, None, None, cs, cs)
    x = torch.zeros(4, 100)
    top = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="CUDA"):
        model_ops.distill_loss(x, top.long(), top)
    with pytest.raises(ValueError, match="CUDA"):
        model_ops.distill_grad(x, top.long(), top, torch.zeros(4, 2))
    with pytest.raises(ValueError, match="CUDA"):
        model_ops.distill_loss_grad(x, top.long(), top)
