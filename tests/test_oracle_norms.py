"""The 64-bit definition of normed and turned heads against differences and against itself."""
import numpy as np
import pytest

from oracle import layer as ol


def parts(seed, rows=4, heads=3, size=10, pairs=3):
    g = np.random.default_rng(seed)
    return (g.normal(size=(rows, heads, size)), g.normal(size=size), g.integers(0, 50, rows), 10.0 ** -np.arange(pairs), g.normal(size=(rows, heads, size)))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("weighed", [False, True])
def test_gradients_are_those_of_differences(interleaved, weighed):
    x, w, pos, f, dout = parts(1)
    w = w if weighed else None
    loss = lambda x, w: float((ol.norm_rotate(x, w, pos, f, 1e-3, interleaved, 1.3) * dout).sum())
    dx, dw = ol.norm_rotate(x, w, pos, f, 1e-3, interleaved, 1.3, dout)
    step = 1e-6
    for at in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[at] += step
        down[at] -= step
        assert abs((loss(up, w) - loss(down, w)) / (2 * step) - dx[at]) < 1e-7 * (1 + abs(dx[at])) * 10
    base = np.ones(x.shape[2]) if w is None else w
    for e in range(x.shape[2]):
        up, down = base.copy(), base.copy()
        up[e] += step
        down[e] -= step
        assert abs((loss(x, up) - loss(x, down)) / (2 * step) - dw[e]) < 1e-6 * (1 + abs(dw[e]))


def test_a_head_has_the_length_that_the_norm_gives_it():
    x, _, pos, f, _ = parts(2)
    out = ol.norm_rotate(x * 1e3, None, pos, f, 1e-9)
    np.testing.assert_allclose((out ** 2).mean(-1), 1.0, rtol=1e-12)
    np.testing.assert_allclose(ol.norm_rotate(np.zeros_like(x), None, pos, f, 1e-6), 0.0)
    np.testing.assert_allclose(ol.norm_rotate(x, None, pos, f, 1e-6), ol.rotate(ol.norm_rotate(x, None, pos, f[:0], 1e-6), pos, f), rtol=1e-13, atol=1e-13)
