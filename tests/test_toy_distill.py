"""The small distilled language model: its gradients against torch's own of the plain
model, and that training lowers the loss."""
import math

import pytest

pytestmark = pytest.mark.gpu


def plain_loss(torch, cfg, weights, cos, sin, tokens, ids, top):
    """The model of toy_distill in elementary torch operations, in 64 bits."""
    b, n = tokens.shape
    d, hd = cfg.dim, cfg.dim // cfg.heads
    h = weights["table"][tokens] * math.sqrt(d)
    rows = (h @ weights["qkv"].t()).view(b, n, 3, cfg.heads, hd)

    def turned(x, gain):
        x = x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt() * gain
        a, c = x[..., :hd // 2], x[..., hd // 2:]
        co, si = cos[None, :, None], sin[None, :, None]
        return torch.cat([a * co - c * si, c * co + a * si], -1)

    q, k = turned(rows[:, :, 0], weights["q_gain"]), turned(rows[:, :, 1], weights["k_gain"])
    score = torch.einsum("bihd,bjhd->bhij", q, k) / math.sqrt(hd)
    score = score.masked_fill(torch.ones(n, n, dtype=torch.bool, device=h.device).triu(1), float("-inf"))
    h = h + torch.einsum("bhij,bjhd->bihd", score.softmax(-1), rows[:, :, 2]).reshape(b, n, d) @ weights["out"].t()
    h = h + torch.relu(h @ weights["up"].t()).square() @ weights["down"].t()
    log_q = torch.log_softmax(h.reshape(b * n, d) @ weights["table"].t() / cfg.temperature, 1)
    log_p = torch.log_softmax(top / cfg.temperature, 1)
    kl = (log_p.exp() * (log_p - log_q.gather(1, ids.long()))).sum(1) * cfg.temperature ** 2
    keep = (torch.arange(n, device=h.device) >= cfg.prompt).repeat(b)
    return kl[keep].mean()


def test_gradients_of_a_step_are_the_plain_models():
    """fp32 products of this size are off by about sqrt(512) * 2^-24 = 1.3e-6 of their result a
    layer; a dozen of them in a row, some cancelling, stay within 1e-4 of a gradient's norm."""
    import torch
    from paper_2608_05088_gb300 import toy_distill as toy
    before = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    try:
        cfg = toy.Config(dtype=torch.float32, batch=3, seq=21)
        teacher, model = toy.Teacher(cfg), toy.Model(cfg)
        tokens = torch.randint(0, cfg.vocab, (cfg.batch, cfg.seq), generator=torch.Generator().manual_seed(7)).cuda()
        loss = model.loss_and_gradients(tokens, teacher)
        weights = {n: w.double().requires_grad_() for n, w in (model.matrices | model.others).items()}
        ids, top = teacher.entries(tokens)
        want = plain_loss(torch, cfg, weights, model.cos.double(), model.sin.double(), tokens, ids, top.double())
        grads = torch.autograd.grad(want, list(weights.values()))
        assert abs(float(loss) / float(want.detach()) - 1) < 1e-5
        for name, g in zip(weights, grads):
            assert float((model.grads[name].double() - g).norm() / g.norm()) < 1e-4, name
        model.optimizer.close()
    finally:
        torch.backends.cuda.matmul.allow_tf32 = before


def test_training_lowers_the_loss():
    from paper_2608_05088_gb300 import toy_distill as toy
    trace = toy.train(steps=60)
    assert all(math.isfinite(x) for x in trace)
    assert sum(trace[-5:]) < 0.6 * sum(trace[:5])
