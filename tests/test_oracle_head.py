"""The fp64 oracle of the residual norm and of the distillation loss (CPU): gradients against central
differences, and the properties that fix each definition."""
import numpy as np
import pytest

from oracle import operators as O


def _fd(f, x, direction, h=1e-6):
    return (f(x + h * direction) - f(x - h * direction)) / (2 * h)


def test_rms_norm_gradient_against_differences():
    rng = np.random.default_rng(1)
    h, g, w, ds = rng.normal(size=(5, 24)), 1 + 0.1 * rng.normal(size=24), rng.normal(size=(5, 24)), rng.normal(size=(5, 24))
    run = lambda a, b: (O.rms_norm(a, b) * w).sum() + (a * ds).sum()  # noqa: E731
    dx, dg, mag, gmag = O.rms_norm_backward(w, h, g, ds)
    for _ in range(3):
        v, u = rng.normal(size=h.shape), rng.normal(size=24)
        assert np.isclose(_fd(lambda a: run(a, g), h, v), (dx * v).sum(), rtol=1e-6)
        assert np.isclose(_fd(lambda b: run(h, b), g, u), (dg * u).sum(), rtol=1e-6)
    assert (mag >= np.abs(dx) - 1e-12).all() and (gmag >= np.abs(dg) - 1e-12).all()


def test_rms_norm_has_unit_mean_square():
    h = np.random.default_rng(2).normal(size=(3, 40)) * 7
    assert np.allclose((O.rms_norm(h, np.ones(40), 1e-12) ** 2).mean(-1), 1)


@pytest.mark.parametrize("alpha", [0.0, 0.3, 1.0])
@pytest.mark.parametrize("tau", [1.0, 2.0, 0.7])
def test_distillation_gradient_against_differences(alpha, tau):
    rng = np.random.default_rng(3)
    T, V, K = 6, 17, 5
    z = rng.normal(size=(T, V)) * 2
    ids = np.stack([rng.permutation(V)[:K] for _ in range(T)])
    ids[1, 2:] = -1           # fewer entries
    ids[2] = -1               # none
    ids[3, 1] = ids[3, 0]     # one twice
    ids[4, 0] = V + 3         # no token
    t, labels = rng.normal(size=(T, K)) * 3, rng.integers(0, V, T)
    labels[2], labels[5] = -100, V
    w = rng.normal(size=T)
    run = lambda a: (O.distill(a, ids, t, labels, alpha, tau)[0] * w).sum()  # noqa: E731
    loss, grad, size = O.distill(z, ids, t, labels, alpha, tau)
    for _ in range(4):
        v = rng.normal(size=z.shape)
        assert np.isclose(_fd(run, z, v), (grad * w[:, None] * v).sum(), rtol=1e-5, atol=1e-8)
    assert loss[2] == 0 and not grad[2].any()
    assert np.allclose(grad.sum(1), 0, atol=1e-12)
    assert (size["loss"] >= np.abs(loss) * 0.2).all()


def test_a_student_that_is_the_teacher_has_no_divergence():
    rng = np.random.default_rng(4)
    z = rng.normal(size=(3, 9))
    ids = np.tile(np.arange(9), (3, 1))
    loss, grad, _ = O.distill(z, ids, z, alpha=1.0, tau=3.0)
    assert np.allclose(loss, 0, atol=1e-14) and np.allclose(grad, 0, atol=1e-14)


def test_labels_alone_are_the_cross_entropy():
    z = np.log(np.array([[0.2, 0.5, 0.3]]))
    loss, grad, _ = O.distill(z, labels=[1], alpha=0.0)
    assert np.allclose(loss, -np.log(0.5)) and np.allclose(grad, [[0.2, -0.5, 0.3]])
