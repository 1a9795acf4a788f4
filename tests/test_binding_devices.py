"""Tensors of another GPU than the current one are refused, by the binding's own checks and by the extension's: the stream is the current device's."""
import importlib.machinery
import importlib.util
import shutil
import types

import pytest
import torch

from paper_2504_03702_amd import binding as ps

F32, I32, I64, U8 = torch.float32, torch.int32, torch.int64, torch.uint8


def stand_in(index, shape=(4, 2, 8), dtype=F32):
    """What the checks ask of a tensor on cuda:index, without one."""
    strides = [1]
    for n in reversed(shape[1:]):
        strides.insert(0, strides[0] * n)
    t = torch.empty(shape, dtype=dtype)
    made = types.SimpleNamespace(is_cuda=True, dtype=dtype, shape=t.shape, device=types.SimpleNamespace(index=index), is_contiguous=lambda: True, data_ptr=lambda: 256,
                                 numel=t.numel, dim=t.dim, stride=lambda i: strides[i])
    return made


def test_the_checks(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    assert ps._ptr(stand_in(0), F32, "x") == 256 and ps._ptr(None, F32, "x") is None
    with pytest.raises(ValueError, match="cuda:1"):
        ps._ptr(stand_in(1), F32, "x")
    with pytest.raises(ValueError, match="cuda:1"):
        ps._sized_ptr(stand_in(1), F32, 64, "x")
    for check, shape in ((ps._heads_ptr, (4, 2, 8)), (ps._rows_ptr, (4, 8))):
        monkeypatch.setattr(torch, "Tensor", types.SimpleNamespace)
        assert check(stand_in(0, shape), shape, F32, "x")[0] == 256
        with pytest.raises(ValueError, match="cuda:1"):
            check(stand_in(1, shape), shape, F32, "x")
        monkeypatch.undo()
        monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)


def calls():
    """Each of the calls, as (name in the extension, function, arguments)."""
    dev = "cuda:0"
    new = lambda *s, t=F32: torch.zeros(s, dtype=t, device=dev)
    x, w, f, pos = new(4, 2, 8), new(8), new(4), new(4, t=I32)
    off, ws = torch.tensor([0, 4], dtype=I32, device=dev), ps.alloc_workspace(1 << 22, dev)
    lse, rng, rows = new(2, 4), new(2, t=I64), new(4, 8)
    return [("rotary", ps.ps_rotary, (x, pos, f, x.clone())), ("dropout_forward", ps.ps_dropout_forward, (rows, None, None, rng, 0.5, rows.clone())),
            ("dropout_backward", ps.ps_dropout_backward, (rows, rng, 0.5, rows.clone(), None, None)),
            ("attention_forward", ps.ps_attention_forward, (x, x, x, off, off, 4, 4, x.clone(), lse, ws)),
            ("attention_backward", ps.ps_attention_backward, (x, x, x, x, lse, x, off, off, 4, 4, x.clone(), x.clone(), x.clone(), ws)),
            ("norm_rotary_forward", ps.ps_norm_rotary_forward, (x, w, pos, f, x.clone())),
            ("norm_rotary_backward", ps.ps_norm_rotary_backward, (x, w, pos, f, x, x.clone(), w.clone(), ws)),
            ("local_attention_forward", ps.ps_local_attention_forward, (x, x, x, off, off, 4, 4, x.clone(), lse, ws, 1, 1)),
            ("local_attention_backward", ps.ps_local_attention_backward, (x, x, x, x, lse, x, off, off, 4, 4, x.clone(), x.clone(), x.clone(), ws, 1, 1)),
            ("anticipate", ps.ps_anticipate, (pos, pos, pos, None, 2, 8, new(16, t=I32), None, ws)),
            ("scaler_scan", ps.ps_scaler_scan, (new(16, t=I32), new(2, t=I32), 2, 8, 4, *[new(2, t=I32) for _ in range(4)], new(1, t=torch.float64)))]


@pytest.mark.gpu
def test_every_call_by_ctypes(monkeypatch):
    made = calls()
    for _, call, args in made:
        call(*args)
    monkeypatch.setattr(ps, "_made", lambda name, *a: False)
    for _, call, args in made:
        call(*args)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for name, call, args in made:
        with pytest.raises(ValueError, match="current device is cuda:1"):
            call(*args)


@pytest.mark.gpu
def test_every_call_by_the_extension(monkeypatch, tmp_path):
    """A second copy of it, loaded where the current device is another (its stream: the default one)."""
    made = calls()
    lib, seen = ps.load_library(), {}
    real = ps._native
    monkeypatch.setattr(ps, "_made", lambda name, *a: seen.setdefault(name, a) is not None and getattr(real, name)(*a) == 0)
    for _, call, args in made:
        call(*args)
    assert set(seen) == {name for name, _, _ in made}
    path = tmp_path / "copy" / real.__file__.rsplit("/", 1)[1]
    path.parent.mkdir()
    shutil.copy(real.__file__, path)
    copies = []
    for device in (0, 1):
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda device=device: device)
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0)
        own = path.with_name(f"{device}_{path.name}")
        shutil.copy(path, own)
        loader = importlib.machinery.ExtensionFileLoader("_marshal", str(own))
        copies.append(importlib.util.module_from_spec(importlib.util.spec_from_loader("_marshal", loader)))
        addresses = [getattr(lib, "ps_" + n) for n in ("predict_load", "anticipate", "anticipate_static", "lookahead_update", "scaler_scan", "route", "forecast",
                                                       "attention_forward", "attention_backward", "rotary", "dropout_forward", "dropout_backward", "norm_rotary_forward",
                                                       "norm_rotary_backward", "local_attention_forward", "local_attention_backward")]
        copies[-1].bind(*[ps.ctypes.cast(a, ps.ctypes.c_void_p).value for a in addresses])
    for name, args in seen.items():
        assert getattr(copies[0], name)(*args) == 0, name
        assert getattr(copies[1], name)(*args) is NotImplemented, name
    monkeypatch.undo()
    torch.cuda.synchronize()
