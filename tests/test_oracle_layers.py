"""Pins of the invariant layers' oracle: gradients against central differences,
closed forms, and the 8-bit checkpoint's bounds and edge values."""
import numpy as np
import pytest

from oracle import layers as ol


def _rng(seed=0):
    return np.random.default_rng(seed)


@pytest.mark.parametrize("name", ol.ACTIVATIONS)
def test_dense_gradients_equal_differences(name):
    rng = _rng(1)
    x, W, b, res, dy = (rng.standard_normal(s) for s in ((5, 7), (7, 6), (6,), (5, 6), (5, 6)))
    f = lambda x, W, b: (ol.dense_fwd(x, W, b, res, name)[0] * dy).sum()  # noqa: E731
    z = ol.dense_fwd(x, W, b, res, name)[1]
    assert np.abs(z).min() > 1e-3                # no relu kink within a step
    dx, dW, db = ol.dense_bwd(x, W, dy, z, name)
    h = 1e-5
    for got, at in ((dx, 0), (dW, 1), (db, 2)):
        for i in np.ndindex(got.shape):
            p, m = [x, W, b], [x, W, b]
            p[at], m[at] = p[at].copy(), m[at].copy()
            p[at][i] += h
            m[at][i] -= h
            assert abs((f(*p) - f(*m)) / (2 * h) - got[i]) < 1e-8 * max(1.0, abs(got[i]) * 10)


def test_layer_norm_gradients_equal_differences():
    rng = _rng(2)
    x, g, b, dy = (rng.standard_normal(s) for s in ((4, 9), (9,), (9,), (4, 9)))
    f = lambda x, g, b: (ol.layer_norm_fwd(x, g, b)[0] * dy).sum()  # noqa: E731
    _, mean, rstd = ol.layer_norm_fwd(x, g, b)
    grads = ol.layer_norm_bwd(x, g, dy, mean, rstd)
    h = 1e-5
    for at, got in enumerate(grads):
        for i in np.ndindex(got.shape):
            p, m = [x, g, b], [x, g, b]
            p[at], m[at] = p[at].copy(), m[at].copy()
            p[at][i] += h
            m[at][i] -= h
            assert abs((f(*p) - f(*m)) / (2 * h) - got[i]) < 1e-7


def test_layer_norm_closed_form():
    y, mean, rstd = ol.layer_norm_fwd([[1.0, 3.0], [5.0, 5.0]], eps=0.25)
    assert np.allclose(mean, [2, 5]) and np.allclose(rstd, [1 / np.sqrt(1.25), 2])
    assert np.allclose(y, [[-1 / np.sqrt(1.25), 1 / np.sqrt(1.25)], [0, 0]])


def test_activations_far_out():
    z = np.array([-1e4, -40.0, 40.0, 1e4])
    for name in ("silu", "gelu", "relu"):
        y, d = ol.act(name, z)
        assert np.allclose(y, [0, 0, 40, 1e4], atol=1e-12) and np.allclose(d, [0, 0, 1, 1], atol=1e-12)


def test_checkpoint_error_is_at_most_half_a_step():
    rng = _rng(3)
    x = (rng.standard_normal((50, 100)) * np.exp(3 * rng.standard_normal((50, 1)))).astype(np.float32)
    q, c = ol.pack8(x)
    assert q.min() >= -127 and q.max() <= 127 and c.shape == (50, 4)
    v = ol.unpack8(q, c)
    step = np.ldexp(1.0, np.repeat(c.astype(int) - 127, 32, 1)[:, :100])
    assert (np.abs(v - x) <= step / 2).all()
    # the step is the smallest power of two for which that holds
    top = np.abs(np.pad(x, ((0, 0), (0, 28)))).reshape(50, 4, 32).max(-1)
    assert (top >= 63.5 * np.ldexp(1.0, c.astype(int) - 127)).all()
    assert (top < 127.5 * np.ldexp(1.0, c.astype(int) - 127)).all()
    assert np.array_equal(ol.unpack8(*ol.pack8(v)), v)        # packing again changes nothing


@pytest.mark.parametrize("top,q,e", [(1.0, 64, -6), (127.0, 127, 0), (127.49, 127, 0), (127.5, 64, 1), (128.0, 64, 1),
                                     (2.0**-126, 1, -126), (3.4028235e38, 127, 121), (2.0**-121, 64, -127)])
def test_checkpoint_edges(top, q, e):
    got, c = ol.pack8(np.array([[top, -top, 0.0]]))
    if top == 2.0**-126:                          # the step does not go below 2^-127
        q, e = 2, -127
    assert got.tolist() == [[q, -q, 0]] and int(c[0, 0]) - 127 == e


def test_checkpoint_of_zeros_and_non_finite_groups():
    x = np.zeros((3, 65))
    x[1, 40] = np.inf
    x[2, 64] = np.nan
    q, c = ol.pack8(x)
    assert c.tolist() == [[0, 0, 0], [0, 255, 0], [0, 0, 255]] and not q.any()
    v = ol.unpack8(q, c)
    assert np.isnan(v[1, 32:64]).all() and np.isnan(v[2, 64]) and np.nansum(np.abs(v)) == 0
