"""What the calls of local attention decide on the host: refusals and workspace sizes.  No kernel runs, no GPU is needed."""
import ctypes
import os

import pytest
import torch

from paper_2504_03702_amd import binding as ps
from paper_2504_03702_amd import layers

EINVAL, EWORKSPACE, EUNSUPPORTED = -1, -5, -6


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ps.LIB_PATH):
        from paper_2504_03702_amd import build
        build.build_library(verbose=False)
    return ps.load_library()


def desc(**change):
    d = ps.ps_attention_desc(1, 2, 4, 2, 64, 10, 12, 0, 20, 24, 0.125, 0.0)
    for n in ("q", "out", "dout", "dq"):
        setattr(d, n, ps.ps_strides(256, 64))
    for n in ("k", "v", "dk", "dv"):
        setattr(d, n, ps.ps_strides(128, 64))
    for n, v in change.items():
        setattr(d, n, v)
    return d


def local(**change):
    l = ps.ps_attention_local(5, 3, 1, 8, 4, 256, 256)
    for n, v in change.items():
        setattr(l, n, v)
    return l


def forward(lib, d=None, l=None, **change):
    a = dict(seqs=ps.ps_attention_seqs(256, 256), q=256, k=256, v=256, out=256, lse=256, rest=None, ws=256, n=1 << 24)
    a.update(change)
    s = a.pop("seqs")
    return lib.ps_local_attention_forward(ctypes.byref(d or desc()), ctypes.byref(s) if s else None, ctypes.byref(l) if l else None, *a.values(), None, None)


def backward(lib, d=None, l=None, **change):
    a = dict(seqs=ps.ps_attention_seqs(256, 256), q=256, k=256, v=256, out=256, lse=256, rest=None, dout=256, dq=256, dk=256, dv=256, dbias=256, ws=256, n=1 << 24)
    a.update(change)
    s = a.pop("seqs")
    return lib.ps_local_attention_backward(ctypes.byref(d or desc()), ctypes.byref(s) if s else None, ctypes.byref(l) if l else None, *a.values(), None, None)


@pytest.mark.parametrize("call", [forward, backward])
def test_refusals(lib, call):
    assert call(lib, l=None) == EINVAL and call(lib, l=local(), seqs=None) == EINVAL
    for change in (dict(sinks=-1), dict(n_buckets=-1), dict(reach=-1), dict(buckets=None), dict(bias=None), dict(buckets=258), dict(bias=257)):
        assert call(lib, l=local(**change)) == EINVAL, change
    for change in (dict(n_buckets=65), dict(reach=65537)):
        assert call(lib, l=local(**change)) == EUNSUPPORTED, change
    assert call(lib, desc(heads=66, kv_heads=2, head_dim=8), local()) == EUNSUPPORTED
    assert call(lib, desc(heads=65536, kv_heads=65536), local()) == call(lib, desc(heads=16384, kv_heads=16384), local(reach=65536)) == EUNSUPPORTED
    for change in (dict(dtype=2), dict(heads=3), dict(scale=0.0), dict(causal=2), dict(q=ps.ps_strides(256, 60))):
        assert call(lib, desc(**change), local()) == EINVAL, change
    assert call(lib, desc(head_dim=136), local()) == EUNSUPPORTED
    for change in (dict(q=None), dict(k=None), dict(v=264), dict(out=None), dict(rest=264), dict(lse=258)):
        assert call(lib, l=local(), **change) == EINVAL, change
    assert call(lib, l=local(), ws=None) == EWORKSPACE and call(lib, l=local(), ws=128) == EWORKSPACE and call(lib, l=local(), n=100) == EWORKSPACE


def test_a_gradient_goes_with_a_bias(lib):
    assert backward(lib, l=local(n_buckets=0)) == EINVAL and backward(lib, l=local(), dbias=258) == EINVAL
    for n in ("dout", "dq", "dk", "dv"):
        assert backward(lib, l=local(), **{n: None}) == EINVAL, n
    assert backward(lib, desc(n_seq=0), local(), dbias=None) == 0 and forward(lib, desc(n_seq=0), local()) == 0


def test_workspace(lib):
    size = lambda *a, **k: ps.ps_local_attention_workspace_bytes(*a, **k)
    bf16 = torch.bfloat16
    assert size(1, 8, 8, 8, 8, 4, 4, 64, bf16, sinks=-1) == size(1, 8, 8, 8, 8, 4, 4, 64, bf16, n_buckets=65, reach=4) == 0
    assert size(1, 8, 8, 8, 8, 4, 4, 64, bf16, reach=65537) == size(1, 8, 8, 8, 8, 3, 4, 64, bf16) == 0
    assert lib.ps_local_attention_workspace_bytes(ctypes.byref(desc()), None, 0) == 0
    # without anything local as much as the other call's
    for shape in ((1, 8, 8, 8, 8, 4, 4, 64, bf16), (1, 1, 8192, 1, 8192, 16, 4, 128, bf16), (4, 4096, 4096, 1024, 1024, 8, 8, 64, torch.float32)):
        for back in (False, True):
            assert size(*shape, back) == ps.ps_attention_workspace_bytes(*shape, back)
    # of a long cache a window leaves shares of its own keys: 4100 and a block's rows are 138 tiles at most, in shares of 16 tiles or more 9, of 128 and 2 floats
    # for each of 1024 rows, however long the cache; besides, 8 bytes for 64 tokens (documents)
    for longest in (32768, 1 << 20):
        assert size(32, 32, 32 * longest, 1, longest, 32, 8, 128, bf16, left=4095, right=0, sinks=4) <= 9 * 1024 * 130 * 4 + 8 * (32 * longest // 64) + 4096
    # the largest windows, numbers that come near the end of theirs, nothing at all
    top = 2 ** 31 - 1
    for how in (dict(left=top, right=top, sinks=top), dict(left=0, right=0, sinks=top), dict(left=top, right=0, sinks=5)):
        assert 0 < size(3, 3000, 3000, 1000, 1000, 4, 2, 64, bf16, True, **how) < 1 << 30
    assert size(0, 0, 0, 0, 0, 4, 2, 64, bf16, True, left=1, sinks=3, n_buckets=4, reach=3) > 0
    assert size(1, 1 << 20, 1 << 20, 1 << 20, 1 << 20, 8, 8, 64, bf16, True, left=1023, right=0, sinks=4) < 1 << 30
    assert size(1, 1 << 20, 1 << 20, 1 << 20, 1 << 20, 8, 8, 64, bf16, True, left=1023, right=0, sinks=1 << 20) < 1 << 31


# Bounds that leave no blocks of keys or rows, beside windows that are shorter than what is left; blocks whose number does not fit 32 bits.
@pytest.mark.parametrize("n_seq,n_q,n_k,max_q,max_k", [(1, 1000, 33, 1000, 0), (1000, 1000, 100000, 1 << 20, 0), (0, 4096, 1 << 20, 1 << 20, 127), (2, 33, 1 << 20, 0, 1 << 20),
                                                       (100000, 4096, 0, 1 << 20, 1000)])
@pytest.mark.parametrize("how", [dict(left=1, right=0, sinks=1), dict(left=0), dict(left=100, right=100, sinks=1000, n_buckets=8, reach=16)])
def test_workspace_without_blocks(lib, n_seq, n_q, n_k, max_q, max_k, how):
    for heads, dtype in ((10, torch.bfloat16), (2, torch.float32)):
        for back in (False, True):
            assert 0 < ps.ps_local_attention_workspace_bytes(n_seq, n_q, n_k, max_q, max_k, heads, 2, 64, dtype, back, **how) < 1 << 30


def test_the_binding_refuses():
    t = torch.zeros(4, 2, 8)
    with pytest.raises((TypeError, ValueError)):
        ps.ps_local_attention_forward(t, t, t, t, t, 4, 4, t, None, t)
    for how in (dict(buckets=torch.zeros(3)), dict(bias=torch.zeros(3, 2)), dict(buckets=torch.zeros(4), bias=torch.zeros(3, 2)), dict(buckets=torch.zeros(3), bias=torch.zeros(3, 3)),
                dict(buckets=torch.zeros(3), bias=torch.zeros(6))):
        with pytest.raises(ValueError):
            ps._local("a call", 2, -1, -1, 0, how.get("buckets"), how.get("bias"))
    with pytest.raises(ValueError):
        ps._local("a call", 2, -1, -1, 0, None, None, torch.zeros(3, 2))


def test_layer_function_refuses():
    q = torch.zeros(4, 2, 8)
    seqs = layers.Sequences(torch.tensor([0, 4]), torch.tensor([0, 4]), 4, 4)
    with pytest.raises(ValueError):
        layers.attention(q, q, q, seqs, slopes=torch.zeros(2, requires_grad=True), window=(1, 1))
    for how in (dict(bias=torch.zeros(3, 2)), dict(buckets=torch.zeros(3, dtype=torch.int32))):
        with pytest.raises(ValueError):
            layers.attention(q, q, q, seqs, **how)
