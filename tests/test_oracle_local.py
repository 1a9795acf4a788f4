"""The 64-bit definitions of windows, first keys and the learned bias, by hand and against differences; what the library makes of buckets."""
import os

import numpy as np
import pytest

from oracle import layer as ol
from paper_2504_03702_amd import binding as ps


def test_windows_by_hand():
    see = lambda *a, **k: ["".join("x" if t else "." for t in row) for row in ol.visible(*a, **k)]
    assert see(4, 6, 2, left=1, right=0) == [".xx...", "..xx..", "...xx.", "....xx"]
    assert see(4, 6, 2, left=1, right=0, sinks=1) == ["xxx...", "x.xx..", "x..xx.", "x...xx"]
    assert see(2, 5, 0, left=0, right=1, sinks=4) == ["xxxx.", "xxxx."]              # the first keys are seen from in front of them too
    assert see(2, 5, 0, causal=True, left=0, right=3, sinks=4) == ["x....", "xx..."]
    assert see(2, 5, 1, causal=True, prefix=4, right=1) == ["xxx..", "xxxx."]        # a prefix inside the window
    assert see(1, 3, -9, left=2, right=2, sinks=1) == ["x.."] and see(1, 3, 9, left=2, right=2) == ["..."]


def test_bias_gradient_is_that_of_differences():
    g = np.random.default_rng(4)
    q, k, v, dout = g.normal(size=(7, 2, 5)), g.normal(size=(9, 1, 5)), g.normal(size=(9, 1, 5)), g.normal(size=(7, 2, 5))
    where, bias = np.array([2, 0, -1, 1, 3, 1, 0]), g.normal(size=(4, 2))
    run = lambda b, **k_: ol.attention(q, k, v, [0, 3, 7], [0, 5, 9], buckets=where, bias=b, left=3, right=2, sinks=1, cap=2.0, **k_)
    got = run(bias, dout=dout)[5]
    for at in np.ndindex(bias.shape):
        up, down = bias.copy(), bias.copy()
        up[at] += 1e-6
        down[at] -= 1e-6
        assert abs((run(up)[0] * dout).sum() - (run(down)[0] * dout).sum() - 2e-6 * got[at]) < 1e-14 + 2e-6 * 1e-7
    assert np.abs(got.sum(0)).max() > 1e-3                           # (distances without a bucket have the rest)


@pytest.mark.parametrize("n,reach,both", [(32, 128, True), (32, 128, False), (64, 512, True), (8, 17, True), (8, 1000, False), (4, 1, True), (2, 1, False),
                                          (16, 4, True), (64, 65536, True), (32, 100, True), (10, 37, True)])
def test_buckets(n, reach, both):
    if not os.path.exists(ps.LIB_PATH):
        from paper_2504_03702_amd import build
        build.build_library(verbose=False)
    got = ps.ps_bias_buckets(n, reach, both).numpy()
    # (the whole numbers of the far ones are long: every distance near, some far ones)
    some = np.r_[0:min(2 * reach + 1, 40), reach - min(reach, 600):reach + min(reach, 600) + 1, 2 * reach - min(reach, 40):2 * reach + 1]
    if reach <= 1000:
        np.testing.assert_array_equal(got, ol.buckets(n, reach, both))
    assert got[reach] == 0 and got.min() == 0 and got.max() == n - 1 - (reach == 0) and len(got) == 2 * reach + 1
    left = got[:reach + 1][::-1]
    assert np.all(np.diff(left) >= 0) and np.all(got[some] < n)
    assert np.all(got[reach + 1:] == (left[1:] + n // 2 if both else 0))


@pytest.mark.parametrize("a", [(0, 10), (65, 100), (3, 10), (2, 10), (32, 7), (32, 65537), (32, -1)])
def test_buckets_refuse(a):
    with pytest.raises(ps.PsError):
        ps.ps_bias_buckets(*a)
