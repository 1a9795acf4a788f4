"""What the layer operators decide on the host: refusals, workspace sizes, frequencies.  No kernel runs, no GPU is needed."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

from paper_2504_03702_amd import binding as ps

from tests.test_kernel_resources import kernels, workgroups_a_unit  # noqa: F401  (a fixture)

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


def seqs(**change):
    s = ps.ps_attention_seqs(256, 256)
    for n, v in change.items():
        setattr(s, n, v)
    return s


def forward(lib, d, s, q=256, k=256, v=256, out=256, lse=256, rest=None, ws=256, nbytes=1 << 20):
    return lib.ps_attention_forward(ctypes.byref(d), ctypes.byref(s) if s else None, q, k, v, out, lse, rest, ws, nbytes, None, None)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=2), EINVAL), (dict(n_seq=-1), EINVAL), (dict(heads=0), EINVAL), (dict(heads=3), EINVAL), (dict(kv_heads=0), EINVAL),
    (dict(head_dim=0), EINVAL), (dict(head_dim=12), EUNSUPPORTED), (dict(head_dim=136), EUNSUPPORTED), (dict(max_q=-1), EINVAL),
    (dict(max_k=-1), EINVAL), (dict(n_q=-1), EINVAL), (dict(n_k=1 << 31), EINVAL), (dict(causal=2), EINVAL), (dict(scale=0.0), EINVAL),
    (dict(scale=-1.0), EINVAL), (dict(scale=float("nan")), EINVAL), (dict(softcap=-1.0), EINVAL), (dict(softcap=float("nan")), EINVAL),
    (dict(q=ps.ps_strides(-256, 64)), EINVAL), (dict(k=ps.ps_strides(128, 60)), EINVAL), (dict(out=ps.ps_strides(256, 0)), EINVAL),
    (dict(out=ps.ps_strides(0, 64)), EINVAL), (dict(heads=256, kv_heads=1, max_q=1 << 20), EUNSUPPORTED)])
def test_attention_refuses_descriptors(lib, change, code):
    assert forward(lib, desc(**change), seqs()) == code
    assert code == EINVAL or lib.ps_attention_workspace_bytes(ctypes.byref(desc(**change)), 1) == 0


@pytest.mark.parametrize("change,code", [
    (dict(s=None), EINVAL), (dict(s=seqs(q_offsets=None)), EINVAL), (dict(s=seqs(q_docs=256)), EINVAL), (dict(q=None), EINVAL),
    (dict(k=None), EINVAL), (dict(v=264), EINVAL), (dict(out=None), EINVAL), (dict(lse=258), EINVAL), (dict(rest=264), EINVAL),
    (dict(ws=None), EWORKSPACE), (dict(ws=128), EWORKSPACE), (dict(nbytes=0), EWORKSPACE)])
def test_attention_refuses_pointers(lib, change, code):
    assert forward(lib, desc(), **{"s": seqs(), **change}) == code


def test_a_rest_is_for_bf16(lib):
    assert forward(lib, desc(dtype=0), seqs(), rest=256) == EINVAL


@pytest.mark.parametrize("n", [(1 << 30) + 1, (1 << 31) - 1])
def test_sequences_whose_places_would_not_fit_are_refused(lib, n):
    assert forward(lib, desc(max_k=n, n_k=n), seqs()) == EUNSUPPORTED
    assert forward(lib, desc(heads=2, max_q=n, n_q=n), seqs()) == EUNSUPPORTED
    assert lib.ps_attention_workspace_bytes(ctypes.byref(desc(max_k=n, n_k=n)), 1) == 0


def test_backward_refuses(lib):
    def call(d, **change):
        a = dict(q=256, k=256, v=256, out=256, lse=256, rest=None, dout=256, dq=256, dk=256, dv=256, ws=256, n=1 << 20)
        a.update(change)
        return lib.ps_attention_backward(ctypes.byref(d), ctypes.byref(seqs()), *list(a.values())[:10], a["ws"], a["n"], None, None)

    for n in ("q", "k", "v", "out", "lse", "dout", "dq", "dk", "dv"):
        assert call(desc(), **{n: None}) == EINVAL, n
    assert call(desc(dk=ps.ps_strides(128, 32))) == EINVAL and call(desc(dq=ps.ps_strides(64, 64))) == EINVAL
    assert call(desc(), ws=None) == EWORKSPACE and call(desc(), n=100) == EWORKSPACE
    assert call(desc(n_seq=0)) == 0


def test_workspace_grows_with_what_is_shared_out(lib):
    size = lambda *a, **k: ps.ps_attention_workspace_bytes(*a, **k)
    bf16 = torch.bfloat16
    assert 0 < size(1, 8, 8, 8, 8, 4, 4, 64, bf16) <= 4096
    # rows of 128 floats, twice as many shares of a cache twice as long, up to where shares grow instead
    a, b = size(1, 1, 4096, 1, 4096, 16, 4, 128, bf16), size(1, 1, 8192, 1, 8192, 16, 4, 128, bf16)
    assert 1.5 * a < b < 2.5 * a
    assert size(64, 64, 64 << 20, 1, 1 << 20, 32, 8, 128, bf16) < 1 << 29
    # one long sequence among many short ones
    assert size(500, 600, 600 + (1 << 20), 100, 1 << 20, 1, 1, 128, bf16, backward=True) < 1 << 31
    assert size(4, 4096, 4096, 1024, 1024, 8, 8, 64, bf16, backward=True) >= size(4, 4096, 4096, 1024, 1024, 8, 8, 64, bf16)


def test_frequencies():
    i = np.arange(32)
    plain = 10000.0 ** (-i / 32)
    close = lambda a, b: np.testing.assert_allclose(a.numpy(), b, rtol=2 ** -23)
    close(ps.ps_rotary_frequencies(32), plain)
    close(ps.ps_rotary_frequencies(32, scaling=ps.PS_ROTARY_LINEAR, factor=4.0), plain / 4)
    based = ps.ps_rotary_frequencies(32, scaling=ps.PS_ROTARY_BASE, factor=4.0).numpy()
    assert based[0] == 1.0 and abs(based[31] * 4 / plain[31] - 1) < 1e-6 and np.all(based[1:] < plain[1:])
    turns = 4096 * plain / (2 * np.pi)
    kept = np.clip((turns - 1) / 31, 0, 1)
    close(ps.ps_rotary_frequencies(32, scaling=ps.PS_ROTARY_PARTS, factor=4.0, trained_len=4096), plain / 4 * (1 - kept) + plain * kept)
    assert np.any(kept == 0) and np.any(kept == 1)
    for bad in (dict(n_pairs=0), dict(n_pairs=4, base=0.0), dict(n_pairs=4, scaling=7), dict(n_pairs=4, scaling=1, factor=0.0),
                dict(n_pairs=1, scaling=2, factor=2.0), dict(n_pairs=4, scaling=3, factor=2.0, trained_len=0),
                dict(n_pairs=4, scaling=3, factor=2.0, trained_len=8, slow=4.0, fast=4.0)):
        with pytest.raises(ps.PsError):
            ps.ps_rotary_frequencies(**bad)


def test_rotary_and_dropout_refuse(lib):
    def turn(**change):
        d = ps.ps_rotary_desc(1, 64, 32, 0, 0, 2, 0, 1.0, 5)
        d.x = d.out = ps.ps_strides(128, 64)
        p = dict(x=256, out=256, x2=None, out2=None, positions=256, frequencies=256)
        for n, v in change.items():
            p.update({n: v}) if n in p else setattr(d, n[2:] if n.startswith("d_") else n, v)
        return lib.ps_rotary(ctypes.byref(d), *p.values(), None)

    for change in (dict(dtype=3), dict(n_pairs=33), dict(n_pairs=-1), dict(heads=0), dict(interleaved=2), dict(inverse=2), dict(n_rows=-1),
                   dict(x=None), dict(out=None), dict(positions=None), dict(frequencies=None), dict(x2=256), dict(x=257), dict(d_out=ps.ps_strides(128, 0)),
                   dict(d_x=ps.ps_strides(-1, 64)), dict(d_x=ps.ps_strides(256, 64))):
        assert turn(**change) == EINVAL, change
    assert turn(head_dim=8192) == EUNSUPPORTED and turn(n_rows=0) == 0
    drop = lambda x=256, ld=16, rng=256, p=0.1, dtype=0, rows=4, cols=16, out=512, ld_out=16: lib.ps_dropout_forward(
        x, ld, None, None, 0, rng, p, dtype, rows, cols, out, ld_out, None)
    for change in (dict(x=None), dict(rng=None), dict(out=None), dict(ld=15), dict(ld_out=15), dict(p=-0.1), dict(p=1.1), dict(p=float("nan")),
                   dict(dtype=2), dict(rows=-1), dict(cols=-1), dict(x=258), dict(rng=260), dict(out=256, ld_out=24)):
        assert drop(**change) == EINVAL, change
    assert drop(rows=1 << 31) == EUNSUPPORTED and drop(cols=(1 << 20) + 1) == EUNSUPPORTED and drop(rows=0) == 0 and drop(cols=0) == 0
    back = lambda dbias=256, ws=256, n=1 << 20: lib.ps_dropout_backward(256, 16, 256, 0.1, 0, 4, 16, 512, 16, dbias, ws, n, None)
    assert back(ws=None) == EWORKSPACE and back(ws=128) == EWORKSPACE and back(n=0) == EWORKSPACE
    assert lib.ps_dropout_workspace_bytes(-1, 4) == 0 and lib.ps_dropout_workspace_bytes(65536, 1024) >= 4 * 1024


def test_hot_kernels_leave_room_for_two_workgroups(kernels):  # noqa: F811
    """Registers that do not fit are reloaded behind a tile on its way from memory, and waited for with it."""
    hot = {n: k for n, k in kernels.items() if re.match(r"(attend|query_gradients|key_gradients)_kernel<(__bf16|bool _Accum|DF16b)", n) or
           ("attend_kernelIDF16b" in n or "gradients_kernelIDF16b" in n)}
    assert len(hot) >= 9
    assert {n: k for n, k in hot.items() if k["vgpr_spill_count"]} == {}
    assert {n: workgroups_a_unit(k) for n, k in hot.items() if workgroups_a_unit(k) < 2} == {}
