"""The fp64 oracle of the operators around the blocks (CPU): gradients against central
differences, and the properties that fix each definition."""
import numpy as np
import pytest

from oracle import operators as O


def _fd(f, x, direction, h=1e-6):
    return (f(x + h * direction) - f(x - h * direction)) / (2 * h)


def test_embedding_gradient_is_the_adjoint_of_the_lookup():
    rng = np.random.default_rng(1)
    ids = np.array([3, 7, -1, 3, 99, 5, 3, 12])
    table, dy = rng.normal(size=(8, 5)), rng.normal(size=(8, 5))
    y = O.embedding(ids, table, 1.7, first=3)
    assert not y[[2, 4, 7]].any() and np.array_equal(y[0], 1.7 * table[0]) and np.array_equal(y[1], 1.7 * table[4])
    g, mag, count = O.embedding_backward(ids, dy, 8, 1.7, first=3)
    assert np.isclose((y * dy).sum(), (g * table).sum(), rtol=1e-12)
    assert count.tolist() == [3, 0, 1, 0, 1, 0, 0, 0] and (mag >= np.abs(g)).all()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rope", [0, 16, 32])
def test_qk_gradient_against_differences(rope, interleaved):
    rng = np.random.default_rng(2)
    T, q, kv, d = 5, 4, 2, 32
    qkv, w = rng.normal(size=(T, q + 2 * kv, d)), rng.normal(size=(T, q + 2 * kv, d))
    gq, gk = 1 + 0.1 * rng.normal(size=d), 1 + 0.1 * rng.normal(size=d)
    cs = O.rope_table(50, rope)[rng.integers(0, 50, T)] if rope else None
    run = lambda x, a, b: (O.qk_norm_rope(x, a, b, cs, q, kv, rope, interleaved) * w).sum()  # noqa: E731
    dx, dgq, dgk = O.qk_norm_rope_backward(w, qkv, gq, gk, cs, q, kv, rope, interleaved)
    for _ in range(3):
        v, u = rng.normal(size=qkv.shape), rng.normal(size=d)
        assert np.isclose(_fd(lambda x: run(x, gq, gk), qkv, v), (dx * v).sum(), rtol=1e-6)
        assert np.isclose(_fd(lambda a: run(qkv, a, gk), gq, u), (dgq * u).sum(), rtol=1e-6)
        assert np.isclose(_fd(lambda b: run(qkv, gq, b), gk, u), (dgk * u).sum(), rtol=1e-6)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotated_scores_depend_on_the_distance_only(interleaved):
    rng = np.random.default_rng(3)
    d, table = 32, O.rope_table(200, 32)
    row = rng.normal(size=(1, 3, d))
    one = np.ones(d)

    def score(pq, pk):
        z = lambda p: O.qk_norm_rope(row, one, one, table[[p]], 1, 1, d, interleaved)[0]  # noqa: E731
        return z(pq)[0] @ z(pk)[1]
    assert np.isclose(score(20, 13), score(120, 113), rtol=1e-10)
    out = O.qk_norm_rope(row, one, one, table[[77]], 1, 1, d, interleaved)
    assert np.allclose((out[0, :2] ** 2).mean(-1), 1.0, atol=1e-5) and np.array_equal(out[0, 2], row[0, 2])


def test_e4m3_codes():
    v = O.e4m3_values()
    assert v[0] == 0 and v[1] == 2.0 ** -9 and v[8] == 2.0 ** -6 and v[126] == 448.0 and np.isnan(v[127])
    assert np.array_equal(v[128:255], -v[:127])
    torch = pytest.importorskip("torch")
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(t, v, equal_nan=True)


def test_checkpoint_rounding():
    rng = np.random.default_rng(4)
    x = rng.normal(size=(40, 96)) * 10.0 ** rng.integers(-8, 9, size=(40, 1))
    x[0] = 0.0
    x[1, :32] = 448.0
    x[2, :32] = 449.0
    x[3, 5], x[3, 40] = np.inf, np.nan
    q, s = O.act8_save(x)
    r = O.act8_restore(q, s)
    bad = ~np.isfinite(x)
    assert np.isnan(r[bad]).all() and np.isfinite(r[~bad]).all() and not r[0].any()
    assert s[1, 0] == 127 and s[2, 0] == 128 and s[0, 0] == 10
    step = np.repeat(2.0 ** (s.astype(float) - 127.0), 32, axis=1)
    bound = np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * step)
    assert (np.abs(r - x)[~bad] <= bound[~bad]).all()
    again = O.act8_save(np.where(bad, 0.0, r))
    assert np.array_equal(O.act8_restore(*again)[~bad], r[~bad])  # restored values keep their value


def test_gelu_parts_against_differences():
    u = np.linspace(-12, 12, 481)
    g, slope = O.gelu_parts(u)
    h = 1e-5
    assert np.allclose((O.gelu_parts(u + h)[0] - O.gelu_parts(u - h)[0]) / (2 * h), slope, atol=1e-8)
    assert np.allclose(g - O.gelu_parts(-u)[0], u, atol=1e-12)
