"""The 64-bit definitions of the layer operators against what can be worked out by hand, and their gradients against differences."""
import numpy as np
import pytest

from oracle import layer as ol


def test_one_key_is_its_value_and_none_is_nothing():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((3, 2, 8)), rng.standard_normal((3, 1, 8)), rng.standard_normal((3, 1, 8))
    out, lse = ol.attention(q, k, v, [0, 2, 3], [0, 1, 3], causal=True)
    # two rows on one key: the first stands before it
    assert np.all(out[0] == 0) and np.all(lse[:, 0] == -np.inf)
    assert np.allclose(out[1], v[0]) and np.allclose(lse[0, 1], 8 ** -0.5 * q[1, 0] @ k[0, 0])


def test_masks_by_hand():
    assert ol.visible(3, 4, 1, causal=True).tolist() == [[True, True, False, False], [True, True, True, False], [True] * 4]
    assert ol.visible(2, 4, 0, causal=True, prefix=3).tolist() == [[True, True, True, False]] * 2
    d = np.array([1, -1, 1])
    assert ol.visible(3, 3, 0, q_docs=d, k_docs=d).tolist() == [[True, False, True], [False] * 3, [True, False, True]]


@pytest.mark.parametrize("cap", [0.0, 2.0])
def test_attention_gradients_against_differences(cap):
    rng = np.random.default_rng(1)
    q, k, v, g = (rng.standard_normal(s) for s in ((5, 4, 8), (7, 2, 8), (7, 2, 8), (5, 4, 8)))
    how = dict(q_offsets=[0, 3, 5], k_offsets=[0, 4, 7], causal=True, prefix=[0, 2], slopes=np.array([0.1, 0.2, 0.3, 0.4]), cap=cap)
    grads = ol.attention(q, k, v, dout=g, **how)[2:]
    h = 1e-5                                   # error h^2 / 6 of the third derivative, rounding 1e-16 / h
    for t, grad in zip((q, k, v), grads):
        for _ in range(12):
            i = tuple(rng.integers(0, n) for n in t.shape)
            was = t[i]
            sides = []
            for x in (was + h, was - h):
                t[i] = x
                sides.append(np.sum(ol.attention(q, k, v, **how)[0] * g))
            t[i] = was
            assert abs((sides[0] - sides[1]) / (2 * h) - grad[i]) < 1e-8


def test_rotation_keeps_lengths_and_turns_back():
    rng = np.random.default_rng(2)
    x, pos, f = rng.standard_normal((4, 2, 10)), np.array([0, 1, 77, -3]), np.array([1.0, 0.1, 0.01])
    for interleaved in (False, True):
        y = ol.rotate(x, pos, f, interleaved, 1.5)
        assert np.allclose(y[0, :, :6], 1.5 * x[0, :, :6]) and np.array_equal(y[..., 6:], x[..., 6:])
        assert np.allclose(np.linalg.norm(y[..., :6], axis=-1), 1.5 * np.linalg.norm(x[..., :6], axis=-1))
        assert np.allclose(ol.rotate(y, pos, f, interleaved, 1 / 1.5, inverse=True), x)
        # the gradient is the turn back with the same magnitude: <R x, y> = <x, R^T y>
        w = rng.standard_normal(x.shape)
        assert np.isclose(np.sum(y[..., :6] * w[..., :6]), np.sum(x[..., :6] * ol.rotate(w, pos, f, interleaved, 1.5, True)[..., :6]))
    a, b = x[1, 0, 0], x[1, 0, 3]
    assert np.allclose(ol.rotate(x, pos, f)[1, 0, [0, 3]], [a * np.cos(1) - b * np.sin(1), a * np.sin(1) + b * np.cos(1)])


def test_philox_known_answers():
    """The vectors that the generator was published with."""
    f = 0xFFFFFFFF
    for counter, key, want in (
            ((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
            ((f, f, f, f), (f, f), (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
            ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0), (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))):
        assert tuple(int(v) for v in ol.philox(counter, key)) == want


def test_dropout_rates_and_extremes():
    x = np.ones((400, 250))
    for p in (0.0, 0.1, 0.5, 1.0):
        y = ol.dropout(x, None, None, 12345, 6, p)
        n = np.count_nonzero(y == 0)
        assert abs(n - p * x.size) <= 5 * np.sqrt(x.size * p * (1 - p)) + 1
        if p < 1:
            assert np.allclose(y[y != 0], 1 / (1 - p), rtol=1e-4)
    a, b = ol.kept(8, 40, 1, 0, 0.5)[0], ol.kept(8, 33, 1, 0, 0.5)[0]
    assert np.array_equal(a[:, :33], b)                        # a mask does not depend on the width
    assert not np.array_equal(a, ol.kept(8, 40, 1, 1, 0.5)[0]) and not np.array_equal(a, ol.kept(8, 40, 2, 0, 0.5)[0])
    dx, db = ol.dropout_gradients(x, 12345, 6, 0.1)
    assert np.array_equal(dx, ol.dropout(x, None, None, 12345, 6, 0.1)) and np.allclose(db, dx.sum(0))
