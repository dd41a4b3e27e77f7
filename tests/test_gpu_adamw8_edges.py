"""AdamW with 8-bit moments at its edges: zeros of both signs, read-outs beside steps, tensors whose memory
is another one than at construction."""
import numpy as np
import pytest

from oracle import adamw8_ref as ref
from tests.test_gpu_adamw8 import make, state_of

pytestmark = pytest.mark.gpu


def test_roots_of_negative_zero():
    """-0 is zero: code 0, and its neighbours keep theirs."""
    import torch
    malt, params, intact = make([1000, 77], torch.float32)
    opt = malt.AdamW8(params)
    g = torch.Generator(device="cuda").manual_seed(2)
    root = torch.rand(opt.moments()[0].shape, generator=g, device="cuda") + 0.1
    m = torch.randn(root.shape, generator=g, device="cuda")
    root[::2] = -0.0
    root[5:40:7] = -0.0
    m[3::11] = -0.0
    opt.set_moments(m, root)
    for p, (a, b) in zip(params, opt.spans()):
        want = ref.encode(m[a:b].cpu().numpy(), root[a:b].cpu().numpy(), np.full(b - a, 0x80008000, np.uint64))
        got = state_of(p)
        assert all((x == y).all() for x, y in zip(got[1:], want[1:]))
        assert all((x == y).all() for x, y in zip(ref.values(*got), ref.values(*want)))
    assert intact()
    opt.close()
