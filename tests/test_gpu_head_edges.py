"""The output head at its edges: operands in one matrix."""
import numpy as np
import pytest

from tests.test_gpu_head import BF16, case
from tests.test_gpu_model_ops import torch_and_ops

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
