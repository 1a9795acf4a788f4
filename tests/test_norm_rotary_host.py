"""What the calls of normed and turned heads decide on the host.  No kernel runs, no GPU is needed."""
import ctypes
import os

import pytest
import torch

from paper_2504_03702_amd import binding as ps

EINVAL, EWORKSPACE, EUNSUPPORTED = -1, -5, -6


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ps.LIB_PATH):
        from paper_2504_03702_amd import build
        build.build_library(verbose=False)
    return ps.load_library()


def desc(change):
    d = ps.ps_norm_rotary_desc(1, 64, 32, 0, 4, 2, 1.0, 1e-6, 5)
    for n in ("x", "out", "dout", "dx"):
        setattr(d, n, ps.ps_strides(256, 64))
        setattr(d, n + "2", ps.ps_strides(128, 64))
    for n, v in change.items():
        if n.startswith("d_"):
            setattr(d, n[2:], v)
    return d


def forward(lib, **change):
    p = dict(x=256, weight=256, out=512, x2=1024, weight2=256, out2=2048, positions=256, frequencies=256)
    p.update({n: v for n, v in change.items() if not n.startswith("d_")})
    return lib.ps_norm_rotary_forward(ctypes.byref(desc(change)), *p.values(), None)


def backward(lib, **change):
    p = dict(x=256, weight=256, dout=512, dx=768, dweight=256, x2=1024, weight2=256, dout2=2048, dx2=4096, dweight2=256, positions=256,
             frequencies=256, ws=256, nbytes=1 << 24)
    p.update({n: v for n, v in change.items() if not n.startswith("d_")})
    return lib.ps_norm_rotary_backward(ctypes.byref(desc(change)), *p.values(), None)


BOTH = [dict(d_dtype=2), dict(d_dtype=-1), dict(d_head_dim=0), dict(d_n_pairs=33), dict(d_n_pairs=-1), dict(d_heads=0), dict(d_heads2=-1), dict(d_heads2=0),
        dict(d_n_rows=-1), dict(d_interleaved=2), dict(d_eps=0.0), dict(d_eps=-1.0), dict(d_eps=1e-40), dict(d_eps=float("nan")), dict(d_eps=float("inf")),
        dict(x=None), dict(x2=None), dict(positions=None), dict(frequencies=None), dict(x=257), dict(weight=257), dict(weight2=257),
        dict(d_x=ps.ps_strides(-1, 64)), dict(d_x2=ps.ps_strides(128, -1))]


@pytest.mark.parametrize("change", BOTH + [dict(out=None), dict(out2=None), dict(out=513), dict(d_out=ps.ps_strides(256, 32)), dict(d_out2=ps.ps_strides(0, 64)),
                                           dict(out=256, d_x=ps.ps_strides(512, 64)), dict(out2=1024, d_x2=ps.ps_strides(512, 64))])
def test_forward_refuses(lib, change):
    assert forward(lib, **change) == EINVAL


@pytest.mark.parametrize("change", BOTH + [dict(dout=None), dict(dx=None), dict(dout2=None), dict(dx2=None), dict(dx=769), dict(dweight=258), dict(dweight2=258),
                                           dict(d_dx=ps.ps_strides(256, 32)), dict(d_dout=ps.ps_strides(-256, 64)), dict(dx=512, d_dx=ps.ps_strides(512, 64)),
                                           dict(dx=256, d_dx=ps.ps_strides(512, 64)), dict(dx2=2048, d_dx2=ps.ps_strides(512, 64))])
def test_backward_refuses(lib, change):
    assert backward(lib, **change) == EINVAL


def test_what_is_not_supported(lib):
    for call in (forward, backward):
        assert call(lib, d_head_dim=520) == EUNSUPPORTED and call(lib, d_n_rows=1 << 31) == EUNSUPPORTED and call(lib, d_heads=1 << 22) == EUNSUPPORTED
    assert backward(lib, ws=None) == EWORKSPACE and backward(lib, ws=128) == EWORKSPACE and backward(lib, nbytes=1000) == EWORKSPACE
    assert forward(lib, d_n_rows=0) == 0
    size = ps.ps_norm_rotary_workspace_bytes
    assert size(-1, 4, 2, 64) == size(1 << 31, 4, 2, 64) == size(5, 0, 2, 64) == size(5, 4, -1, 64) == size(5, 4, 2, 0) == size(5, 4, 2, 520) == 0
    assert 0 < size(0, 1, 0, 1) and size(5, 4, 2, 64) <= 1 << 20


def test_the_binding_refuses():
    x = torch.zeros(4, 2, 8)
    for bad in (dict(x=None), dict(x=x[0]), dict(x=x), dict(x=x, x2=x)):
        a = dict(x=None, weight=None, positions=None, frequencies=None, out=x)
        a.update(bad)
        with pytest.raises((TypeError, ValueError)):
            ps.ps_norm_rotary_forward(**a)
    with pytest.raises((TypeError, ValueError)):
        ps.ps_norm_rotary_backward(x, None, None, None, x, x, None, x)


def test_workspace_of_heads_that_the_calls_refuse(lib):
    size = ps.ps_norm_rotary_workspace_bytes
    assert size(5, 1 << 20, 0, 64) > 0 and size(5, 1 << 19, 1 << 19, 64) > 0
    assert size(5, (1 << 20) + 1, 0, 64) == size(5, 1, 1 << 20, 64) == size(5, (1 << 31) - 1, (1 << 31) - 1, 1) == 0
