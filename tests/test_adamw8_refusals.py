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
    opt.state, opt.params, opt._device, opt._on = None, (entry(),), 0, torch.device("cuda", 0)
    with pytest.raises(ValueError, match="where the state is"):
        opt.step(malt.adamw_hparams(), params=[entry()])
    opt._tensors, opt._codes, opt._at, opt._codes_at = [opt.params[0][0]], [opt.params[0][3]], [0], [0]
    for call in (lambda: opt.step(malt.adamw_hparams()), lambda: opt.moments(), lambda: opt.set_moments(None, None)):
        with pytest.raises(ValueError, match="where the state is"):
            call()
