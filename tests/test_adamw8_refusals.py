"""Tensors that AdamW with 8-bit moments refuses, on the host and without a GPU."""
import pytest
import torch

from paper_2608_05088_gb300 import build, malt


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()


def entry(n=300, g_dtype=torch.float32):
    w = torch.zeros(n)
    return (w, w.bfloat16(), w.to(g_dtype, copy=True), *malt.adamw8_states(w), 0.1)


def test_tensors_on_another_device(monkeypatch):
    """A state is made on the current device; its tensors have to be there, then and at every step."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 1)
    for make in (lambda: malt.AdamW8([entry()]), lambda: malt.malt_adamw8_init_state([entry()]),
                 lambda: malt.WholeOptimizer([], [entry()], moment_bits=8)):
        with monkeypatch.context() as m:
            m.setattr(malt, "malt_init_state", lambda params, stream=None: None)
            with pytest.raises(ValueError, match="current CUDA device"):
                make()
    opt = malt.AdamW8.__new__(malt.AdamW8)
    opt._address = torch.Tensor.data_ptr
    opt.state, opt.params, opt._device, opt._on = None, (entry(),), 0, torch.device("cuda", 0)
    with pytest.raises(ValueError, match="where the state is"):
        opt.step(malt.adamw_hparams(), params=[entry()])
    opt._tensors, opt._codes, opt._at, opt._codes_at = [opt.params[0][0]], [opt.params[0][3]], [0], [0]
    for call in (lambda: opt.step(malt.adamw_hparams()), lambda: opt.moments(), lambda: opt.set_moments(None, None)):
        with pytest.raises(ValueError, match="where the state is"):
            call()


def test_tensors_that_overlap():
    """By any byte, of one entry or of two; neighbours do not."""
    buf, raw = torch.zeros(2000), torch.zeros(4000, dtype=torch.uint8)
    low = torch.zeros(4000, dtype=torch.bfloat16)

    def two(w=(0, 512), copy=(0, 1024), g=(1100, 1400), m=(0, 300), v=(600, 900), ms=(1200, 1202), vs=(1204, 1206)):
        """Two entries of 300 elements, from these places of shared buffers on."""
        at = lambda t, i, k=300: t[i:i + k]
        return [(at(buf, w[i]), at(low, copy[i]), at(buf, g[i]), at(raw, m[i]), at(raw, ms[i], 2), at(raw, v[i]),
                 at(raw, vs[i], 2), 0.0) for i in range(2)]

    assert len(malt.adamw8_params_array(two(w=(0, 300), g=(600, 900), m=(0, 300), v=(600, 900)))) == 2
    assert len(malt.adamw8_params_array(two(g=(1100, 1100)))) == 2        # gradients are read
    assert len(malt.adamw8_params_array(two(g=(1100, 1250)))) == 2
    assert len(malt.adamw8_params_array(two())) == 2
    for bad in (dict(w=(0, 256)), dict(w=(4, 0)), dict(copy=(0, 299)), dict(m=(0, 256)), dict(v=(600, 256)),
                dict(m=(0, 901)), dict(ms=(1200, 1201)), dict(vs=(1204, 1203)), dict(ms=(1200, 899))):
        with pytest.raises(ValueError, match="share memory"):
            malt.adamw8_params_array(two(**bad))
    for bad in (dict(g=(4, 1100)), dict(g=(1100, 212 + 300 - 1)), dict(g=(811, 1200)), dict(g=(1200, 0))):
        with pytest.raises(ValueError, match="share memory"):
            malt.adamw8_params_array(two(**bad))
    w = torch.zeros(300)
    for part in (w, w.view(torch.bfloat16)[100:400]):                   # a gradient in its own weights
        with pytest.raises(ValueError, match="share memory"):
            malt.adamw8_params_array([(w, None, part, *malt.adamw8_states(w), 0.0)])
