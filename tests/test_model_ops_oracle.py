"""The oracle of the model operators: its gradients against central differences of its
own forward passes (CPU only)."""
import numpy as np
import pytest

from oracle import model_ops_ref as ref

H = 1e-5        # step of the differences: error about H^2, rounding about 1e-16 / H
TOL = 1e-7      # a hundred times their sum for values of order 1


def differences(f, x):
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        keep = x[i]
        x[i] = keep + H
        up = f(x)
        x[i] = keep - H
        g[i] = (up - f(x)) / (2 * H)
        x[i] = keep
    return g


def test_embed_gradient_is_the_difference():
    rng = np.random.default_rng(1)
    ids = np.array([2, 0, 2, -1, 4, 2])
    dout = rng.standard_normal((6, 3))
    table = rng.standard_normal((5, 3))
    got = ref.embed_grad(dout, ids, 5, 1.7)
    want = differences(lambda t: float((ref.embed(t, ids, 1.7) * dout).sum()), table)
    assert np.abs(got - want).max() < TOL


@pytest.mark.parametrize("interleaved", (False, True))
@pytest.mark.parametrize("dim,pairs", ((6, 3), (7, 2), (4, 0)))
def test_qk_norm_gradient_is_the_difference(dim, pairs, interleaved):
    rng = np.random.default_rng(2)
    x, dy = rng.standard_normal((2, 3, 2, dim))
    gain = rng.standard_normal(dim)
    angle = rng.uniform(0, 6, (3, 1, pairs))
    cos, sin = np.cos(angle), np.sin(angle)
    dx, dgain = ref.qk_norm_grad(dy, x, gain, cos, sin, 1e-3, interleaved)

    def value(x, gain):
        return float((ref.qk_norm(x, gain, cos, sin, 1e-3, interleaved) * dy).sum())

    assert np.abs(dx - differences(lambda v: value(v, gain), x)).max() < TOL
    assert np.abs(dgain - differences(lambda v: value(x, v), gain)).max() < TOL


def test_distill_gradient_is_the_difference():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((4, 9))
    ids = np.array([[0, 3, 8], [2, -1, 5], [7, 7, 1], [4, 9, -1]])
    t = rng.standard_normal((4, 3))
    t[0, 1] = -np.inf
    weight = np.array([0.5, 1.5, 0.25, 2.0])
    dloss = np.array([1.0, -0.5, 2.0, 0.0])
    _, _, got = ref.distill(x, ids, t, weight, 1.7, dloss)
    want = differences(lambda v: float((ref.distill(v, ids, t, weight, 1.7)[0] * dloss).sum()), x)
    assert np.abs(got - want).max() < TOL


def test_distill_rows_without_a_teacher():
    x = np.full((3, 4), np.nan)
    loss, stats, grad = ref.distill(x, np.array([[-1], [1], [2]]), np.array([[0.0], [0.0], [-np.inf]]),
                                    np.array([1.0, 0.0, 1.0]))
    assert not loss.any() and not stats.any() and not grad.any()
