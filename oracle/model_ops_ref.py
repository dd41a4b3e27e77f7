"""fp64 oracle of the model operators (test infrastructure only): the formulas of
include/malt.h in NumPy, each forward pass and its gradient."""
from __future__ import annotations

import numpy as np


def embed(table, ids, scale=1.0):
    """scale * table[ids]; zero rows for negative ids, NaN rows for ids past the table."""
    table, ids = np.asarray(table, np.float64), np.asarray(ids).reshape(-1)
    out = np.zeros((ids.size, table.shape[1]))
    inside = (ids >= 0) & (ids < table.shape[0])
    out[inside] = scale * table[ids[inside]]
    out[ids >= table.shape[0]] = np.nan
    return out


def embed_grad(dout, ids, vocab, scale=1.0):
    dout, ids = np.asarray(dout, np.float64), np.asarray(ids).reshape(-1)
    d = np.zeros((vocab, dout.shape[1]))
    inside = (ids >= 0) & (ids < vocab)
    np.add.at(d, ids[inside], scale * dout[inside])
    return d


def _pairs(rot, interleaved):
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, rot // 2 + i)


def rotate(n, cos, sin, interleaved, back=False):
    """Pairs of n's first 2 * cos.shape[-1] entries turned by the angles (or back)."""
    a, b = _pairs(2 * cos.shape[-1], interleaved)
    s = -sin if back else sin
    y = np.array(n, np.float64)
    y[..., a] = n[..., a] * cos - n[..., b] * s
    y[..., b] = n[..., b] * cos + n[..., a] * s
    return y


def qk_norm(x, gain, cos, sin, eps, interleaved=False):
    """x [..., heads, dim]; cos, sin [..., 1, pairs]: the angles of each token."""
    x = np.asarray(x, np.float64)
    r = 1.0 / np.sqrt(np.mean(x * x, -1, keepdims=True) + eps)
    return rotate(x * r * gain, cos, sin, interleaved)


def qk_norm_grad(dy, x, gain, cos, sin, eps, interleaved=False):
    """(dx, dgain) of qk_norm."""
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    r = 1.0 / np.sqrt(np.mean(x * x, -1, keepdims=True) + eps)
    dn = rotate(dy, cos, sin, interleaved, back=True)
    u = dn * gain
    dx = r * (u - x * r * r * np.mean(u * x, -1, keepdims=True))
    return dx, (dn * x * r).reshape(-1, x.shape[-1]).sum(0)


def _targets(top_ids, top_logits, vocab, temperature):
    """Listed entries of a row and their probabilities and log-probabilities."""
    listed = (top_ids >= 0) & (top_ids < vocab) & (top_logits != -np.inf)
    t = top_logits[listed] / temperature
    log_p = t - t.max() if t.size else t
    log_p = log_p - np.log(np.exp(log_p).sum()) if t.size else t
    return top_ids[listed].astype(np.int64), np.exp(log_p), log_p


def distill(logits, top_ids, top_logits, weight=None, temperature=1.0, dloss=None):
    """(loss [rows], stats [rows, 2], dlogits [rows, vocab])."""
    logits = np.asarray(logits, np.float64)
    top_logits = np.asarray(top_logits, np.float64)
    n, vocab = logits.shape
    weight = np.ones(n) if weight is None else np.asarray(weight, np.float64)
    dloss = np.ones(n) if dloss is None else np.asarray(dloss, np.float64)
    loss, stats, grad = np.zeros(n), np.zeros((n, 2)), np.zeros((n, vocab))
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        for i in range(n):
            ids, p, log_p = _targets(np.asarray(top_ids[i]), top_logits[i], vocab, temperature)
            if weight[i] == 0 or ids.size == 0:
                continue
            m = logits[i].max()
            e = np.exp((logits[i] - m) / temperature)
            stats[i] = m, e.sum()
            log_q = (logits[i] - m) / temperature - np.log(e.sum())
            terms = np.where(p == 0, 0.0, p * (log_p - log_q[ids]))
            loss[i] = weight[i] * temperature ** 2 * terms.sum()
            if dloss[i] != 0:
                g = e / e.sum()
                np.subtract.at(g, ids, p)
                grad[i] = weight[i] * dloss[i] * temperature * g
    return loss, stats, grad
