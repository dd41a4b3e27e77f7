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


def test_reading_moments_beside_steps():
    """A read-out on another stream changes nothing of a step, and the count waits for the steps."""
    import torch
    malt, params, _ = make([300_000] * 8 + [7] * 30, torch.bfloat16)
    twin = make([300_000] * 8 + [7] * 30, torch.bfloat16)[1]
    read, alone = malt.AdamW8(params, seed=1), malt.AdamW8(twin, seed=1)
    hp = malt.adamw_hparams(lr=1e-2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda._sleep(100_000_000)              # cycles: the steps below wait for it, the read-outs do not
    read.step(hp)
    read.moments(stream=side)
    assert read.get_step() == 1
    alone.step(hp)
    for _ in range(300):
        read.step(hp)
        read.moments(dtype=torch.bfloat16, stream=side)
        alone.step(hp)
    torch.cuda.synchronize()
    for p, q in zip(params, twin):
        assert all(torch.equal(x, y) for x, y in zip(p[:7], q[:7]) if x is not None)
    read.close()
    alone.close()
