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
    steps = torch.cuda.Stream()
    steps.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(steps):              # (a stream that the default one does not wait for)
        torch.cuda._sleep(100_000_000)
        read.step(hp)
    read.moments(stream=side)
    assert read.get_step() == 2
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


def test_tensors_that_move():
    """A step and a read-out follow tensors to other memory, and refuse what no longer holds them."""
    import torch
    malt, params, _ = make([3000, 500, 40], torch.float32)
    twin = make([3000, 500, 40], torch.float32)[1]
    a, b = malt.AdamW8(params, seed=6), malt.AdamW8(twin, seed=6)
    hp = malt.adamw_hparams(lr=1e-2)
    old = []
    for k in range(7):
        for p in params:
            if p[k] is not None:
                old.append((p[k].data, p[k].clone()))
                p[k].data = p[k].clone()
        for opt in (a, b):
            opt.step(hp)
        assert all(torch.equal(x, y) for x, y in zip(a.moments(), b.moments()))
        for p, q in zip(params, twin):
            assert all(torch.equal(x, y) for x, y in zip(p[:7], q[:7]) if x is not None)
        moved = {t.data_ptr() for p in params for t in p[:7] if t is not None}
        assert all(torch.equal(x, y) for x, y in old if x.data_ptr() not in moved)
        old.clear()
    # moments that are set go to the codes' new memory
    m, root = a.moments()
    for p in params:
        p[5].data = torch.zeros_like(p[5])
    a.set_moments(m, root)
    assert all(torch.equal(x, y) for x, y in zip(a.moments(), (m, root)))
    # other tensors for one step are for one step
    others = [(*p[:2], torch.zeros_like(p[2]), *p[3:]) for p in params]
    a.step(hp, params=others)
    b.step(hp, params=[(*q[:2], torch.zeros_like(q[2]), *q[3:]) for q in twin])
    for opt in (a, b):
        opt.step(hp)
    for p, q in zip(params, twin):
        assert all(torch.equal(x, y) for x, y in zip(p[:7], q[:7]) if x is not None)
    a.close()
    b.close()


def test_tensors_whose_memory_is_gone():
    """Refused on the host, before anything is launched; given memory again, they are stepped."""
    import torch
    from paper_2608_05088_gb300 import malt
    w, g = torch.ones(1000, device="cuda"), torch.ones(1100, device="cuda")[100:]
    opt = malt.AdamW8([(w, None, g, *malt.adamw8_states(w), 0.0)])
    hp = malt.adamw_hparams(lr=1e-2)
    torch.cuda.synchronize()
    bytes_of = g.untyped_storage().nbytes()
    g.untyped_storage().resize_(0)
    for _ in range(2):
        with pytest.raises(ValueError, match="resized"):
            opt.step(hp)
    g.untyped_storage().resize_(bytes_of)
    g.fill_(1.0)
    opt.step(hp)
    assert opt.get_step() == 1 and bool((w < 1).all())
    for bad in (torch.ones(1000, 2, device="cuda")[:, 0], w.half(), w[:500].clone()):
        kept = w.data
        w.data = bad
        with pytest.raises((ValueError, malt.MaltError)):
            opt.step(hp)
        w.data = kept
    opt.step(hp)
    assert opt.get_step() == 2
    opt.close()
