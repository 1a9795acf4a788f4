"""Thin ctypes binding over the C-ABI library (``include/preserve.h``), same names as the C calls.

Argument marshalling only: tensors supply device pointers, ``torch.cuda.current_stream()`` the
stream; every step of the path runs in the library's HIP kernels.  There is no fallback: if the
library is missing or there is no GPU the calls raise.  The calls with nothing to object to are
marshalled by an extension module (``csrc/marshal.cpp``); what it hands back is marshalled here,
with the checks that say what is wrong, and so is every call where the module is not built."""
from __future__ import annotations

import ctypes
import importlib
import os
import warnings
from typing import Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpreserve.so")

PS_OK = 0
PS_ERRORS = {-1: "PS_EINVAL", -2: "PS_EIO", -3: "PS_EFORMAT", -4: "PS_ENOMEM", -5: "PS_EWORKSPACE",
             -6: "PS_EUNSUPPORTED", -7: "PS_EHIP"}
PS_ST_BAD_TOKEN, PS_ST_BAD_LENGTH, PS_ST_NAN, PS_ST_BAD_RECORD, PS_ST_RANGE = 0x01, 0x02, 0x04, 0x10, 0x20

EXPORTS = ["ps_model_load", "ps_model_free", "ps_model_get_info", "ps_workspace_bytes", "ps_predict_load",
           "ps_anticipate_workspace_bytes", "ps_anticipate", "ps_anticipate_static", "ps_status_read", "ps_strerror",
           "ps_profile_enable", "ps_profile_read", "ps_profile_clock", "ps_profile_stream_read",
           "ps_lookahead_workspace_bytes", "ps_lookahead_update", "ps_scaler_scan", "ps_route", "ps_forecast",
           "ps_attention_workspace_bytes", "ps_attention_forward", "ps_attention_backward", "ps_rotary", "ps_rotary_frequencies",
           "ps_dropout_workspace_bytes", "ps_dropout_forward", "ps_dropout_backward",
           "ps_norm_rotary_workspace_bytes", "ps_norm_rotary_forward", "ps_norm_rotary_backward",
           "ps_local_attention_workspace_bytes", "ps_local_attention_forward", "ps_local_attention_backward", "ps_bias_buckets"]
PS_FAMILIES = ["embed", "gemm", "attention", "layernorm", "head", "refine"]


class PsError(RuntimeError):
    def __init__(self, code: int, where: str):
        super().__init__(f"{where}: {PS_ERRORS.get(code, code)}")
        self.code = code


class ps_model_info(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("layers", "hidden", "heads", "ffn", "vocab", "max_pos",
                                              "n_soft", "head_hidden", "dtype", "d_max")]


class ps_strides(ctypes.Structure):
    _fields_ = [("row", ctypes.c_int64), ("head", ctypes.c_int64)]


class ps_attention_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "n_seq", "heads", "kv_heads", "head_dim", "max_q", "max_k", "causal")] + \
        [("n_q", ctypes.c_int64), ("n_k", ctypes.c_int64), ("scale", ctypes.c_float), ("softcap", ctypes.c_float)] + \
        [(n, ps_strides) for n in ("q", "k", "v", "out", "dout", "dq", "dk", "dv")]


class ps_attention_seqs(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q_offsets", "k_offsets", "k_lengths", "q_start", "prefix", "q_docs", "k_docs", "slopes")]


class ps_attention_local(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("left", "right", "sinks", "n_buckets", "reach")] + \
        [("buckets", ctypes.c_void_p), ("bias", ctypes.c_void_p)]


class ps_rotary_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "head_dim", "n_pairs", "interleaved", "inverse", "heads", "heads2")] + \
        [("magnitude", ctypes.c_float), ("n_rows", ctypes.c_int64)] + [(n, ps_strides) for n in ("x", "out", "x2", "out2")]


class ps_norm_rotary_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "head_dim", "n_pairs", "interleaved", "heads", "heads2")] + \
        [("magnitude", ctypes.c_float), ("eps", ctypes.c_float), ("n_rows", ctypes.c_int64)] + \
        [(n, ps_strides) for n in ("x", "out", "x2", "out2", "dout", "dx", "dout2", "dx2")]


class ps_status(ctypes.Structure):
    _fields_ = [("flags", ctypes.c_int32), ("reserved", ctypes.c_int32), ("first_bad", ctypes.c_int64)]


_lib = None
_native = None          # the extension module, bound to the loaded library; None where there is none


def load_library() -> ctypes.CDLL:
    """Load ``libpreserve.so`` (built in-tree by ``build.py``) and declare its entry points."""
    global _lib, _native
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(f"{LIB_PATH} is not built; run paper_2504_03702_amd/build.py")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    lib.ps_model_load.restype = ctypes.c_int
    lib.ps_model_load.argtypes = [ctypes.c_char_p, ctypes.c_int, ctypes.POINTER(vp)]
    lib.ps_model_free.restype = None
    lib.ps_model_free.argtypes = [vp]
    lib.ps_model_get_info.restype = ctypes.c_int
    lib.ps_model_get_info.argtypes = [vp, ctypes.POINTER(ps_model_info)]
    lib.ps_workspace_bytes.restype = sz
    lib.ps_workspace_bytes.argtypes = [vp, i64, i32]
    lib.ps_predict_load.restype = ctypes.c_int
    lib.ps_predict_load.argtypes = [vp, vp, vp, vp, i32, i64, vp, vp, vp, sz, vp, vp]
    lib.ps_anticipate_workspace_bytes.restype = sz
    lib.ps_anticipate_workspace_bytes.argtypes = [i64, i32, i32]
    lib.ps_anticipate.restype = ctypes.c_int
    lib.ps_anticipate.argtypes = [vp, vp, vp, vp, i64, i32, i32, vp, vp, vp, sz, vp, vp]
    lib.ps_anticipate_static.restype = ctypes.c_int
    lib.ps_anticipate_static.argtypes = [vp, vp, vp, vp, i64, i32, i32, vp, vp, vp, vp]
    lib.ps_lookahead_workspace_bytes.restype = sz
    lib.ps_lookahead_workspace_bytes.argtypes = [i64, i32, i32]
    lib.ps_lookahead_update.restype = ctypes.c_int
    lib.ps_lookahead_update.argtypes = [vp, vp, vp, vp, vp, vp, i64, i32, i32, vp, vp, vp, vp, vp, sz, vp, vp]
    lib.ps_scaler_scan.restype = ctypes.c_int
    lib.ps_scaler_scan.argtypes = [vp, vp, i32, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp]
    lib.ps_route.restype = ctypes.c_int
    lib.ps_route.argtypes = [vp, vp, i32, i32, i32, vp, vp, vp, vp, i32, i32, vp, vp, vp, vp]
    lib.ps_forecast.restype = ctypes.c_int
    lib.ps_forecast.argtypes = [vp, i32, vp, vp, i32, i32, vp, vp, vp]
    lib.ps_status_read.restype = ctypes.c_int
    lib.ps_status_read.argtypes = [vp, vp, ctypes.POINTER(ps_status)]
    lib.ps_profile_enable.restype = ctypes.c_int
    lib.ps_profile_enable.argtypes = [vp, ctypes.c_int]
    lib.ps_profile_read.restype = ctypes.c_int
    lib.ps_profile_read.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64)]
    lib.ps_profile_clock.restype = ctypes.c_int
    lib.ps_profile_clock.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_double)]
    lib.ps_profile_stream_read.restype = ctypes.c_int
    lib.ps_profile_stream_read.argtypes = [vp, ctypes.c_int64, vp, vp]
    desc, seqs = ctypes.POINTER(ps_attention_desc), ctypes.POINTER(ps_attention_seqs)
    lib.ps_attention_workspace_bytes.restype = sz
    lib.ps_attention_workspace_bytes.argtypes = [desc, ctypes.c_int]
    lib.ps_attention_forward.restype = ctypes.c_int
    lib.ps_attention_forward.argtypes = [desc, seqs, vp, vp, vp, vp, vp, vp, vp, sz, vp, vp]
    lib.ps_attention_backward.restype = ctypes.c_int
    lib.ps_attention_backward.argtypes = [desc, seqs, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp, vp]
    lib.ps_rotary.restype = ctypes.c_int
    lib.ps_rotary.argtypes = [ctypes.POINTER(ps_rotary_desc), vp, vp, vp, vp, vp, vp, vp]
    dbl = ctypes.c_double
    lib.ps_rotary_frequencies.restype = ctypes.c_int
    lib.ps_rotary_frequencies.argtypes = [i32, dbl, ctypes.c_int, dbl, i32, dbl, dbl, ctypes.POINTER(ctypes.c_float)]
    lib.ps_dropout_workspace_bytes.restype = sz
    lib.ps_dropout_workspace_bytes.argtypes = [i64, i32]
    lib.ps_dropout_forward.restype = ctypes.c_int
    lib.ps_dropout_forward.argtypes = [vp, i64, vp, vp, i64, vp, ctypes.c_float, i32, i64, i32, vp, i64, vp]
    lib.ps_dropout_backward.restype = ctypes.c_int
    lib.ps_dropout_backward.argtypes = [vp, i64, vp, ctypes.c_float, i32, i64, i32, vp, i64, vp, vp, sz, vp]
    norm = ctypes.POINTER(ps_norm_rotary_desc)
    lib.ps_norm_rotary_workspace_bytes.restype = sz
    lib.ps_norm_rotary_workspace_bytes.argtypes = [i64, i32, i32, i32]
    lib.ps_norm_rotary_forward.restype = ctypes.c_int
    lib.ps_norm_rotary_forward.argtypes = [norm, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.ps_norm_rotary_backward.restype = ctypes.c_int
    lib.ps_norm_rotary_backward.argtypes = [norm, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    local = ctypes.POINTER(ps_attention_local)
    lib.ps_local_attention_workspace_bytes.restype = sz
    lib.ps_local_attention_workspace_bytes.argtypes = [desc, local, ctypes.c_int]
    lib.ps_local_attention_forward.restype = ctypes.c_int
    lib.ps_local_attention_forward.argtypes = [desc, seqs, local, vp, vp, vp, vp, vp, vp, vp, sz, vp, vp]
    lib.ps_local_attention_backward.restype = ctypes.c_int
    lib.ps_local_attention_backward.argtypes = [desc, seqs, local, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp, vp]
    lib.ps_bias_buckets.restype = ctypes.c_int
    lib.ps_bias_buckets.argtypes = [i32, i32, ctypes.c_int, ctypes.POINTER(i32)]
    lib.ps_strerror.restype = ctypes.c_char_p
    lib.ps_strerror.argtypes = [ctypes.c_int]
    _native = _extension()
    if _native is not None:
        _native.bind(*[ctypes.cast(getattr(lib, "ps_" + name), vp).value for name in (
            "predict_load", "anticipate", "anticipate_static", "lookahead_update", "scaler_scan", "route", "forecast",
            "attention_forward", "attention_backward", "rotary", "dropout_forward", "dropout_backward", "norm_rotary_forward",
            "norm_rotary_backward", "local_attention_forward", "local_attention_backward")])
    _lib = lib
    return lib


def _extension():
    """The extension module, None if it is not there or does not load (built for another torch): calls then take some
    microseconds more."""
    try:
        return importlib.import_module("._marshal", __package__)
    except ModuleNotFoundError:
        return None
    except ImportError as e:
        warnings.warn(f"calls go by ctypes: {e}")
        return None


def _on_current_device(t: torch.Tensor, name: str) -> None:
    """The stream is the current device's: tensors of another would be read by a kernel of the wrong one."""
    here = torch.cuda.current_device()
    if t.device.index != here:
        raise ValueError(f"{name}: is on cuda:{t.device.index}, the current device is cuda:{here}")


def _ptr(t: Optional[torch.Tensor], dtype: torch.dtype, name: str) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise TypeError(f"{name}: need a contiguous {dtype} tensor on the GPU")
    _on_current_device(t, name)
    return t.data_ptr()


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _made(name: str, *args) -> bool:
    """Whether the extension module has made the call; False before the library is loaded and for arguments with
    anything to object to."""
    if _native is None:
        return False
    code = getattr(_native, name)(*args)
    if code is NotImplemented:
        return False
    if code != PS_OK:
        raise PsError(code, "ps_" + name)
    return True


def _check(code: int, where: str) -> None:
    if code != PS_OK:
        raise PsError(code, where)


class Model:
    """Owner of a ``ps_model*``."""

    def __init__(self, handle: int, device: int):
        self.handle, self.device = handle, device
        info = ps_model_info()
        _check(load_library().ps_model_get_info(handle, ctypes.byref(info)), "ps_model_get_info")
        self.info = info

    def close(self) -> None:
        if self.handle:
            load_library().ps_model_free(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def ps_model_load(path: str, device: int = 0) -> Model:
    if not torch.cuda.is_available():
        raise RuntimeError("ps_model_load needs a GPU")
    out = ctypes.c_void_p()
    _check(load_library().ps_model_load(os.fsencode(path), device, ctypes.byref(out)), "ps_model_load")
    return Model(out.value, device)


def ps_profile_enable(model: Model, on: bool) -> None:
    _check(load_library().ps_profile_enable(model.handle, int(on)), "ps_profile_enable")


def ps_profile_read(model: Model) -> dict:
    """{family: (milliseconds, launches)} since the last read; waits for the current stream."""
    n = len(PS_FAMILIES)
    ms, cnt = (ctypes.c_double * n)(), (ctypes.c_int64 * n)()
    _check(load_library().ps_profile_read(model.handle, _stream(), ms, cnt), "ps_profile_read")
    return {f: (float(ms[i]), int(cnt[i])) for i, f in enumerate(PS_FAMILIES)}


def ps_profile_clock(model: Model) -> float:
    """Core clock (GHz) sustained during the last large GEMM launched while profiling was on; 0 if none."""
    ghz = ctypes.c_double(0.0)
    _check(load_library().ps_profile_clock(model.handle, _stream(), ctypes.byref(ghz)), "ps_profile_clock")
    return float(ghz.value)


def ps_profile_stream_read(data: torch.Tensor, sink: torch.Tensor, nbytes: Optional[int] = None) -> None:
    """Enqueue the read-only yardstick kernel over the first nbytes of `data` (all of it by default); the XOR
    of its 64-bit words is accumulated into sink[0] (int64 / uint64 device tensor)."""
    n = data.numel() * data.element_size() if nbytes is None else int(nbytes)
    _check(load_library().ps_profile_stream_read(data.data_ptr(), n, sink.data_ptr(), _stream()),
           "ps_profile_stream_read")


def ps_workspace_bytes(model: Model, max_tokens: int, max_req: int) -> int:
    return int(load_library().ps_workspace_bytes(model.handle, max_tokens, max_req))


def new_status(device="cuda") -> torch.Tensor:
    """A zeroed device ps_status block (two int64 words)."""
    return torch.zeros(2, dtype=torch.int64, device=device)


def ps_status_read(status: torch.Tensor) -> Tuple[int, int]:
    """(flags, first_bad) after waiting for the current stream."""
    out = ps_status()
    _check(load_library().ps_status_read(_ptr(status, torch.int64, "status"), _stream(), ctypes.byref(out)),
           "ps_status_read")
    return int(out.flags), int(out.first_bad)


def ps_predict_load(model: Model, token_ids: torch.Tensor, offsets: torch.Tensor,
                    lengths: Optional[torch.Tensor], pred_f: torch.Tensor, pred_tokens: torch.Tensor,
                    workspace: torch.Tensor, status: Optional[torch.Tensor] = None) -> None:
    if _made("predict_load", model.handle, token_ids, offsets, lengths, pred_f, pred_tokens, workspace, status):
        return
    n_req = offsets.numel() - 1
    _check(load_library().ps_predict_load(
        model.handle, _ptr(token_ids, torch.int32, "token_ids"), _ptr(offsets, torch.int32, "offsets"),
        _ptr(lengths, torch.int32, "lengths"), n_req, token_ids.numel(),
        _ptr(pred_f, torch.float32, "pred_f"), _ptr(pred_tokens, torch.int32, "pred_tokens"),
        _ptr(workspace, torch.uint8, "workspace"), workspace.numel(),
        _ptr(status, torch.int64, "status"), _stream()), "ps_predict_load")


def ps_anticipate_workspace_bytes(n_req: int, n_inst: int, horizon: int) -> int:
    return int(load_library().ps_anticipate_workspace_bytes(n_req, n_inst, horizon))


def ps_anticipate(pred_tokens: torch.Tensor, instance_id: torch.Tensor, arrival_bucket: torch.Tensor,
                  rate: Optional[torch.Tensor], n_inst: int, horizon: int, load: torch.Tensor,
                  overflow: Optional[torch.Tensor], workspace: torch.Tensor,
                  status: Optional[torch.Tensor] = None) -> None:
    if _made("anticipate", pred_tokens, instance_id, arrival_bucket, rate, n_inst, horizon, load, overflow, workspace, status):
        return
    if load.numel() != n_inst * horizon or (overflow is not None and overflow.numel() != n_inst) or \
            (rate is not None and rate.numel() != n_inst) or \
            instance_id.numel() != pred_tokens.numel() or arrival_bucket.numel() != pred_tokens.numel():
        raise ValueError("ps_anticipate: array sizes do not match n_req / n_inst / horizon")
    _check(load_library().ps_anticipate(
        _ptr(pred_tokens, torch.int32, "pred_tokens"), _ptr(instance_id, torch.int32, "instance_id"),
        _ptr(arrival_bucket, torch.int32, "arrival_bucket"), _ptr(rate, torch.int32, "rate"),
        pred_tokens.numel(), n_inst, horizon, _ptr(load, torch.int32, "load"),
        _ptr(overflow, torch.int64, "overflow"), _ptr(workspace, torch.uint8, "workspace"),
        workspace.numel(), _ptr(status, torch.int64, "status"), _stream()), "ps_anticipate")


PS_ANTICIPATE_STATIC_BYTES = 8 << 20


def ps_anticipate_static(pred_tokens: torch.Tensor, instance_id: torch.Tensor, arrival_bucket: torch.Tensor,
                         rate: Optional[torch.Tensor], n_inst: int, horizon: int, load: torch.Tensor,
                         overflow: Optional[torch.Tensor], status: Optional[torch.Tensor] = None) -> None:
    """ps_anticipate without a workspace argument: the library's own fixed device array holds the partial curves."""
    if _made("anticipate_static", pred_tokens, instance_id, arrival_bucket, rate, n_inst, horizon, load, overflow, status):
        return
    if load.numel() != n_inst * horizon or (overflow is not None and overflow.numel() != n_inst) or \
            (rate is not None and rate.numel() != n_inst) or \
            instance_id.numel() != pred_tokens.numel() or arrival_bucket.numel() != pred_tokens.numel():
        raise ValueError("ps_anticipate_static: array sizes do not match n_req / n_inst / horizon")
    _check(load_library().ps_anticipate_static(
        _ptr(pred_tokens, torch.int32, "pred_tokens"), _ptr(instance_id, torch.int32, "instance_id"),
        _ptr(arrival_bucket, torch.int32, "arrival_bucket"), _ptr(rate, torch.int32, "rate"),
        pred_tokens.numel(), n_inst, horizon, _ptr(load, torch.int32, "load"),
        _ptr(overflow, torch.int64, "overflow"), _ptr(status, torch.int64, "status"), _stream()),
        "ps_anticipate_static")


def ps_lookahead_workspace_bytes(n_rec: int, n_inst: int, map_len: int) -> int:
    return int(load_library().ps_lookahead_workspace_bytes(n_rec, n_inst, map_len))


def ps_lookahead_update(instance_id: torch.Tensor, start_iter: torch.Tensor, prompt_tokens: torch.Tensor,
                        i_begin: torch.Tensor, i_end: torch.Tensor, sign: torch.Tensor, n_inst: int, map_len: int,
                        kv_tokens: torch.Tensor, overflow: Optional[torch.Tensor], workspace: torch.Tensor,
                        capacity: Optional[torch.Tensor] = None, fraction: Optional[torch.Tensor] = None,
                        status: Optional[torch.Tensor] = None) -> None:
    if _made("lookahead_update", instance_id, start_iter, prompt_tokens, i_begin, i_end, sign, n_inst, map_len, kv_tokens,
             overflow, workspace, capacity, fraction, status):
        return
    cols = (instance_id, start_iter, prompt_tokens, i_begin, i_end, sign)
    n = instance_id.numel()
    if any(c.numel() != n for c in cols) or kv_tokens.numel() != n_inst * map_len or \
            (overflow is not None and overflow.numel() != n_inst) or \
            (capacity is not None and capacity.numel() != n_inst) or \
            (fraction is not None and fraction.numel() != n_inst * map_len):
        raise ValueError("ps_lookahead_update: array sizes do not match n_rec / n_inst / map_len")
    names = ("instance_id", "start_iter", "prompt_tokens", "i_begin", "i_end", "sign")
    _check(load_library().ps_lookahead_update(
        *[_ptr(c, torch.int32, nm) for c, nm in zip(cols, names)], n, n_inst, map_len,
        _ptr(kv_tokens, torch.int32, "kv_tokens"), _ptr(overflow, torch.int64, "overflow"),
        _ptr(capacity, torch.int32, "capacity"), _ptr(fraction, torch.float32, "fraction"),
        _ptr(workspace, torch.uint8, "workspace"), workspace.numel(), _ptr(status, torch.int64, "status"),
        _stream()), "ps_lookahead_update")


def ps_scaler_scan(kv_tokens: torch.Tensor, capacity: torch.Tensor, n_inst: int, map_len: int, window: int,
                   over_count: torch.Tensor, peak_tokens: torch.Tensor, overloaded: torch.Tensor,
                   summary: torch.Tensor, scale_down: torch.Tensor, over_pct: int = 95, share_pct: int = 10,
                   idle_pct: int = 30) -> None:
    if _made("scaler_scan", kv_tokens, capacity, n_inst, map_len, window, over_count, peak_tokens, overloaded, summary,
             scale_down, over_pct, share_pct, idle_pct):
        return
    if kv_tokens.numel() != n_inst * map_len or capacity.numel() != n_inst or summary.numel() != 2 or \
            scale_down.numel() != 1 or any(t.numel() != n_inst for t in (over_count, peak_tokens, overloaded)):
        raise ValueError("ps_scaler_scan: array sizes do not match n_inst / map_len")
    _check(load_library().ps_scaler_scan(
        _ptr(kv_tokens, torch.int32, "kv_tokens"), _ptr(capacity, torch.int32, "capacity"), n_inst, map_len, window,
        over_pct, share_pct, idle_pct, _ptr(over_count, torch.int32, "over_count"),
        _ptr(peak_tokens, torch.int32, "peak_tokens"), _ptr(overloaded, torch.int32, "overloaded"),
        _ptr(summary, torch.int32, "summary"), _ptr(scale_down, torch.float64, "scale_down"), _stream()),
        "ps_scaler_scan")


def ps_route(prompt_tokens: torch.Tensor, pred_tokens: torch.Tensor, n_inst: int, window: int,
             window_tokens: Optional[torch.Tensor], capacity: torch.Tensor, queued_p: torch.Tensor,
             current_d: torch.Tensor, assigned: torch.Tensor, score100: torch.Tensor, t_mem_pct: int = 80,
             beta: int = 1, status: Optional[torch.Tensor] = None) -> None:
    if _made("route", prompt_tokens, pred_tokens, n_inst, window, window_tokens, capacity, queued_p, current_d, assigned, score100,
             t_mem_pct, beta, status):
        return
    n = prompt_tokens.numel()
    if pred_tokens.numel() != n or assigned.numel() != n or score100.numel() != n or capacity.numel() != n_inst or \
            queued_p.numel() != n_inst or current_d.numel() != n_inst or \
            (window_tokens is not None and window_tokens.numel() != n_inst * window):
        raise ValueError("ps_route: array sizes do not match n_req / n_inst / window")
    _check(load_library().ps_route(
        _ptr(prompt_tokens, torch.int32, "prompt_tokens"), _ptr(pred_tokens, torch.int32, "pred_tokens"), n, n_inst,
        window, _ptr(window_tokens, torch.int32, "window_tokens"), _ptr(capacity, torch.int32, "capacity"),
        _ptr(queued_p, torch.int64, "queued_p"), _ptr(current_d, torch.int64, "current_d"), t_mem_pct, beta,
        _ptr(assigned, torch.int32, "assigned"), _ptr(score100, torch.int64, "score100"),
        _ptr(status, torch.int64, "status"), _stream()), "ps_route")


def ps_forecast(weights: torch.Tensor, hidden: int, hist_p: torch.Tensor, hist_d: torch.Tensor, n_services: int,
                k: int, mu: torch.Tensor, out: torch.Tensor) -> None:
    if _made("forecast", weights, hidden, hist_p, hist_d, n_services, k, mu, out):
        return
    if weights.numel() != n_services * 2 * (5 * hidden * hidden + 10 * hidden + 1) or hist_p.numel() != n_services * k or \
            hist_d.numel() != n_services * k or mu.numel() != 3 * n_services or out.numel() != 5 * n_services:
        raise ValueError("ps_forecast: array sizes do not match n_services / hidden / k")
    _check(load_library().ps_forecast(
        _ptr(weights, torch.float32, "weights"), hidden, _ptr(hist_p, torch.float32, "hist_p"),
        _ptr(hist_d, torch.float32, "hist_d"), n_services, k, _ptr(mu, torch.float32, "mu"),
        _ptr(out, torch.float32, "out"), _stream()), "ps_forecast")


# ---- operators of a layer that is fine-tuned, or takes long prompts -------------------------------------------------------
_DTYPES = {torch.float32: 0, torch.bfloat16: 1}


def _heads_ptr(t: torch.Tensor, shape: Tuple[int, int, int], dtype: torch.dtype, name: str) -> Tuple[int, ps_strides]:
    """Address and strides of a tensor [rows, heads, head_dim] whose last dimension is dense."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype != dtype:
        raise TypeError(f"{name}: need a {dtype} tensor on the GPU")
    _on_current_device(t, name)
    if tuple(t.shape) != shape:
        raise ValueError(f"{name}: has shape {tuple(t.shape)}, not {shape}")
    if t.shape[2] > 1 and t.stride(2) != 1:
        raise ValueError(f"{name}: a head's elements have to be neighbours")
    # (torch keeps any stride for dimensions of one)
    return t.data_ptr(), ps_strides(*[t.stride(i) if t.shape[i] > 1 else shape[2] for i in (0, 1)])


def _dtype_code(dtype: torch.dtype, where: str) -> int:
    if dtype not in _DTYPES:
        raise TypeError(f"{where}: takes float32 and bfloat16, not {dtype}")
    return _DTYPES[dtype]


def _sized_ptr(t: Optional[torch.Tensor], dtype: torch.dtype, n: int, name: str) -> Optional[int]:
    p = _ptr(t, dtype, name)
    if t is not None and t.numel() != n:
        raise ValueError(f"{name}: has {t.numel()} elements, not {n}")
    return p


def ps_attention_workspace_bytes(n_seq: int, n_q: int, n_k: int, max_q: int, max_k: int, heads: int, kv_heads: int, head_dim: int,
                                 dtype: torch.dtype, backward: bool = False) -> int:
    d = ps_attention_desc(_dtype_code(dtype, "ps_attention_workspace_bytes"), n_seq, heads, kv_heads, head_dim, max_q, max_k, 0, n_q,
                          n_k, 1.0, 0.0)
    return int(load_library().ps_attention_workspace_bytes(ctypes.byref(d), int(backward)))


def _attention(where, q, k, q_offsets, k_offsets, max_q, max_k, scale, softcap, causal, k_lengths, q_start, prefix, slopes, q_docs,
               k_docs, tensors):
    """The call's descriptor, its sequences and the addresses of `tensors` ({name: (tensor, whether it has k's shape)})."""
    if not isinstance(q, torch.Tensor) or not isinstance(k, torch.Tensor) or q.dim() != 3 or k.dim() != 3:
        raise TypeError(f"{where}: q and k are tensors of rows, heads and elements")
    n_seq, (n_q, heads, size), (n_k, kv_heads, _) = q_offsets.numel() - 1, q.shape, k.shape
    if n_seq < 0 or k_offsets.numel() != n_seq + 1 or (q_docs is None) != (k_docs is None):
        raise ValueError(f"{where}: offsets of n_seq + 1 elements, and documents of both queries and keys or of neither")
    d = ps_attention_desc(_dtype_code(q.dtype, where), n_seq, heads, kv_heads, size, max_q, max_k, int(causal), n_q, n_k,
                          size ** -0.5 if scale is None else scale, softcap)
    at = {}
    for name, (t, keys) in tensors.items():
        at[name], strides = _heads_ptr(t, (n_k, kv_heads, size) if keys else (n_q, heads, size), q.dtype, name)
        setattr(d, name, strides)
    i32 = torch.int32
    seqs = ps_attention_seqs(_ptr(q_offsets, i32, "q_offsets"), _ptr(k_offsets, i32, "k_offsets"),
                             _sized_ptr(k_lengths, i32, n_seq, "k_lengths"), _sized_ptr(q_start, i32, n_seq, "q_start"),
                             _sized_ptr(prefix, i32, n_seq, "prefix"), _sized_ptr(q_docs, i32, n_q, "q_docs"),
                             _sized_ptr(k_docs, i32, n_k, "k_docs"), _sized_ptr(slopes, torch.float32, heads, "slopes"))
    return d, seqs, at, heads * n_q


def ps_attention_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q_offsets: torch.Tensor, k_offsets: torch.Tensor,
                         max_q: int, max_k: int, out: torch.Tensor, lse: Optional[torch.Tensor], workspace: torch.Tensor,
                         scale: Optional[float] = None, softcap: float = 0.0, causal: bool = False,
                         k_lengths: Optional[torch.Tensor] = None, q_start: Optional[torch.Tensor] = None,
                         prefix: Optional[torch.Tensor] = None, slopes: Optional[torch.Tensor] = None,
                         q_docs: Optional[torch.Tensor] = None, k_docs: Optional[torch.Tensor] = None,
                         status: Optional[torch.Tensor] = None, out_rest: Optional[torch.Tensor] = None) -> None:
    """q, out [n_q, heads, head_dim]; k, v [n_k, kv_heads, head_dim]; lse [heads, n_q] float32; scale: head_dim ** -0.5 for None;
    out_rest [n_q, heads, head_dim], in bfloat16 calls whose gradients are wanted, for ps_attention_backward()."""
    if _made("attention_forward", q, k, v, q_offsets, k_offsets, max_q, max_k, out, lse, workspace, scale, softcap, causal, k_lengths,
             q_start, prefix, slopes, q_docs, k_docs, status, out_rest):
        return
    d, seqs, at, n_lse = _attention("ps_attention_forward", q, k, q_offsets, k_offsets, max_q, max_k, scale, softcap, causal, k_lengths,
                                    q_start, prefix, slopes, q_docs, k_docs,
                                    {"q": (q, False), "k": (k, True), "v": (v, True), "out": (out, False)})
    _check(load_library().ps_attention_forward(
        ctypes.byref(d), ctypes.byref(seqs), at["q"], at["k"], at["v"], at["out"], _sized_ptr(lse, torch.float32, n_lse, "lse"),
        _sized_ptr(out_rest, torch.bfloat16, q.numel(), "out_rest"), _ptr(workspace, torch.uint8, "workspace"), workspace.numel(), _ptr(status, torch.int64, "status"), _stream()),
        "ps_attention_forward")


def ps_attention_backward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, lse: torch.Tensor, dout: torch.Tensor,
                          q_offsets: torch.Tensor, k_offsets: torch.Tensor, max_q: int, max_k: int, dq: torch.Tensor, dk: torch.Tensor,
                          dv: torch.Tensor, workspace: torch.Tensor, scale: Optional[float] = None, softcap: float = 0.0,
                          causal: bool = False, k_lengths: Optional[torch.Tensor] = None, q_start: Optional[torch.Tensor] = None,
                          prefix: Optional[torch.Tensor] = None, slopes: Optional[torch.Tensor] = None,
                          q_docs: Optional[torch.Tensor] = None, k_docs: Optional[torch.Tensor] = None,
                          status: Optional[torch.Tensor] = None, out_rest: Optional[torch.Tensor] = None) -> None:
    """Arguments as of ps_attention_forward(), which has left `out`, `lse` and `out_rest`; dq like q, dk and dv like k."""
    if _made("attention_backward", q, k, v, out, lse, dout, q_offsets, k_offsets, max_q, max_k, dq, dk, dv, workspace, scale, softcap,
             causal, k_lengths, q_start, prefix, slopes, q_docs, k_docs, status, out_rest):
        return
    d, seqs, at, n_lse = _attention("ps_attention_backward", q, k, q_offsets, k_offsets, max_q, max_k, scale, softcap, causal, k_lengths,
                                    q_start, prefix, slopes, q_docs, k_docs,
                                    {"q": (q, False), "k": (k, True), "v": (v, True), "out": (out, False), "dout": (dout, False),
                                     "dq": (dq, False), "dk": (dk, True), "dv": (dv, True)})
    _check(load_library().ps_attention_backward(
        ctypes.byref(d), ctypes.byref(seqs), at["q"], at["k"], at["v"], at["out"], _sized_ptr(lse, torch.float32, n_lse, "lse"),
        _sized_ptr(out_rest, torch.bfloat16, q.numel(), "out_rest"), at["dout"], at["dq"], at["dk"], at["dv"], _ptr(workspace, torch.uint8, "workspace"), workspace.numel(),
        _ptr(status, torch.int64, "status"), _stream()), "ps_attention_backward")


PS_ROTARY_PLAIN, PS_ROTARY_LINEAR, PS_ROTARY_BASE, PS_ROTARY_PARTS = 0, 1, 2, 3


def ps_rotary_frequencies(n_pairs: int, base: float = 10000.0, scaling: int = PS_ROTARY_PLAIN, factor: float = 1.0,
                          trained_len: int = 0, slow: float = 1.0, fast: float = 32.0) -> torch.Tensor:
    """[n_pairs] float32 on the host."""
    out = torch.empty(max(n_pairs, 0), dtype=torch.float32)
    _check(load_library().ps_rotary_frequencies(n_pairs, base, scaling, factor, trained_len, slow, fast,
                                                ctypes.cast(out.data_ptr(), ctypes.POINTER(ctypes.c_float))), "ps_rotary_frequencies")
    return out


def ps_rotary(x: torch.Tensor, positions: torch.Tensor, frequencies: torch.Tensor, out: torch.Tensor, x2: Optional[torch.Tensor] = None,
              out2: Optional[torch.Tensor] = None, interleaved: bool = False, magnitude: float = 1.0, inverse: bool = False) -> None:
    """x, out [n_rows, heads, head_dim] and, turned by the same angles, x2, out2 [n_rows, heads2, head_dim]; out may be x."""
    if _made("rotary", x, positions, frequencies, out, x2, out2, interleaved, magnitude, inverse):
        return
    if not isinstance(x, torch.Tensor) or x.dim() != 3 or (x2 is None) != (out2 is None) or (x2 is not None and x2.dim() != 3):
        raise TypeError("ps_rotary: x and x2 are tensors of rows, heads and elements, each with its out")
    n, heads, size = x.shape
    d = ps_rotary_desc(_dtype_code(x.dtype, "ps_rotary"), size, frequencies.numel(), int(interleaved), int(inverse), heads,
                       0 if x2 is None else x2.shape[1], magnitude, n)
    at = {}
    for name, t in (("x", x), ("out", out), ("x2", x2), ("out2", out2)):
        if t is None:
            at[name] = None
            continue
        at[name], strides = _heads_ptr(t, (n, x2.shape[1] if name.endswith("2") else heads, size), x.dtype, name)
        setattr(d, name, strides)
    _check(load_library().ps_rotary(ctypes.byref(d), at["x"], at["out"], at["x2"], at["out2"], _sized_ptr(positions, torch.int32, n, "positions"),
                                    _ptr(frequencies, torch.float32, "frequencies"), _stream()), "ps_rotary")


def _rows_ptr(t: Optional[torch.Tensor], shape: Tuple[int, int], dtype: torch.dtype, name: str) -> Tuple[Optional[int], int]:
    """Address of a tensor [rows, cols] whose rows are dense, and how far they are apart."""
    if t is None:
        return None, 0
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype != dtype:
        raise TypeError(f"{name}: need a {dtype} tensor on the GPU")
    _on_current_device(t, name)
    if tuple(t.shape) != shape or (shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name}: need shape {shape} and dense rows")
    return t.data_ptr(), t.stride(0) if shape[0] > 1 else shape[1]


def ps_dropout_workspace_bytes(rows: int, cols: int) -> int:
    return int(load_library().ps_dropout_workspace_bytes(rows, cols))


def ps_dropout_forward(x: torch.Tensor, bias: Optional[torch.Tensor], residual: Optional[torch.Tensor], rng: torch.Tensor, p: float,
                       out: torch.Tensor) -> None:
    """out = residual + dropout(x + bias) of tensors [rows, cols]; rng: two int64 on the GPU, seed and number of the call."""
    if _made("dropout_forward", x, bias, residual, rng, p, out):
        return
    if not isinstance(x, torch.Tensor) or x.dim() != 2:
        raise TypeError("ps_dropout_forward: x is a tensor of rows and columns")
    shape, code = tuple(x.shape), _dtype_code(x.dtype, "ps_dropout_forward")
    xp, res, to = (_rows_ptr(t, shape, x.dtype, name) for t, name in ((x, "x"), (residual, "residual"), (out, "out")))
    if out is None:
        raise TypeError("out: need a tensor")
    _check(load_library().ps_dropout_forward(*xp, _sized_ptr(bias, x.dtype, shape[1], "bias"), *res, _sized_ptr(rng, torch.int64, 2, "rng"),
                                             p, code, *shape, *to, _stream()), "ps_dropout_forward")


def ps_dropout_backward(dout: torch.Tensor, rng: torch.Tensor, p: float, dx: torch.Tensor, dbias: Optional[torch.Tensor],
                        workspace: Optional[torch.Tensor]) -> None:
    """dx of dropout's x and, unless it is None, dbias ([cols] float32) from dout; rng and p as forwards."""
    if _made("dropout_backward", dout, rng, p, dx, dbias, workspace):
        return
    if not isinstance(dout, torch.Tensor) or dout.dim() != 2 or dx is None:
        raise TypeError("ps_dropout_backward: dout and dx are tensors of rows and columns")
    shape, code = tuple(dout.shape), _dtype_code(dout.dtype, "ps_dropout_backward")
    g, to = (_rows_ptr(t, shape, dout.dtype, name) for t, name in ((dout, "dout"), (dx, "dx")))
    _check(load_library().ps_dropout_backward(
        *g, _sized_ptr(rng, torch.int64, 2, "rng"), p, code, *shape, *to, _sized_ptr(dbias, torch.float32, shape[1], "dbias"),
        _ptr(workspace, torch.uint8, "workspace"), 0 if workspace is None else workspace.numel(), _stream()), "ps_dropout_backward")


def ps_norm_rotary_workspace_bytes(n_rows: int, heads: int, heads2: int, head_dim: int) -> int:
    return int(load_library().ps_norm_rotary_workspace_bytes(n_rows, heads, heads2, head_dim))


def _norm_rotary(where, x, x2, positions, frequencies, eps, interleaved, magnitude, tensors):
    """The call's descriptor and the addresses of `tensors` ({name: tensor}; names that end in 2 have x2's shape)."""
    if not isinstance(x, torch.Tensor) or x.dim() != 3 or (x2 is not None and (not isinstance(x2, torch.Tensor) or x2.dim() != 3)):
        raise TypeError(f"{where}: x and x2 are tensors of rows, heads and elements")
    (n, heads, size), heads2 = x.shape, 0 if x2 is None else x2.shape[1]
    if frequencies is not None and positions is None:
        raise TypeError(f"{where}: frequencies go with positions")
    d = ps_norm_rotary_desc(_dtype_code(x.dtype, where), size, 0 if frequencies is None else frequencies.numel(), int(interleaved), heads, heads2,
                            magnitude, eps, n)
    at = {}
    for name, t in tensors.items():
        second = name.endswith("2")
        if t is None and second and x2 is None:
            at[name] = None
            continue
        at[name], strides = _heads_ptr(t, (n, heads2 if second else heads, size), x.dtype, name)
        setattr(d, name, strides)
    return d, at, _sized_ptr(positions, torch.int32, n, "positions"), _ptr(frequencies, torch.float32, "frequencies"), size


def ps_norm_rotary_forward(x: torch.Tensor, weight: Optional[torch.Tensor], positions: Optional[torch.Tensor], frequencies: Optional[torch.Tensor],
                           out: torch.Tensor, x2: Optional[torch.Tensor] = None, weight2: Optional[torch.Tensor] = None,
                           out2: Optional[torch.Tensor] = None, eps: float = 1e-6, interleaved: bool = False, magnitude: float = 1.0) -> None:
    """x, out [n_rows, heads, head_dim]; weight [head_dim] of the same type, None: ones; x2, weight2, out2: a second tensor's, turned by the same
    angles.  out may be x.  frequencies None: no rotation."""
    if _made("norm_rotary_forward", x, weight, positions, frequencies, out, x2, weight2, out2, eps, interleaved, magnitude):
        return
    d, at, pos, freq, size = _norm_rotary("ps_norm_rotary_forward", x, x2, positions, frequencies, eps, interleaved, magnitude,
                                          {"x": x, "out": out, "x2": x2, "out2": out2})
    _check(load_library().ps_norm_rotary_forward(
        ctypes.byref(d), at["x"], _sized_ptr(weight, x.dtype, size, "weight"), at["out"], at["x2"], _sized_ptr(weight2, x.dtype, size, "weight2"),
        at["out2"], pos, freq, _stream()), "ps_norm_rotary_forward")


def ps_norm_rotary_backward(x: torch.Tensor, weight: Optional[torch.Tensor], positions: Optional[torch.Tensor], frequencies: Optional[torch.Tensor],
                            dout: torch.Tensor, dx: torch.Tensor, dweight: Optional[torch.Tensor], workspace: torch.Tensor,
                            x2: Optional[torch.Tensor] = None, weight2: Optional[torch.Tensor] = None, dout2: Optional[torch.Tensor] = None,
                            dx2: Optional[torch.Tensor] = None, dweight2: Optional[torch.Tensor] = None, eps: float = 1e-6,
                            interleaved: bool = False, magnitude: float = 1.0) -> None:
    """dx like x and, unless they are None, dweight and dweight2 ([head_dim] float32), from dout; the rest as forwards.  dx may be dout or x."""
    if _made("norm_rotary_backward", x, weight, positions, frequencies, dout, dx, dweight, workspace, x2, weight2, dout2, dx2, dweight2, eps,
             interleaved, magnitude):
        return
    d, at, pos, freq, size = _norm_rotary("ps_norm_rotary_backward", x, x2, positions, frequencies, eps, interleaved, magnitude,
                                          {"x": x, "dout": dout, "dx": dx, "x2": x2, "dout2": dout2, "dx2": dx2})
    f32 = torch.float32
    _check(load_library().ps_norm_rotary_backward(
        ctypes.byref(d), at["x"], _sized_ptr(weight, x.dtype, size, "weight"), at["dout"], at["dx"], _sized_ptr(dweight, f32, size, "dweight"),
        at["x2"], _sized_ptr(weight2, x.dtype, size, "weight2"), at["dout2"], at["dx2"], _sized_ptr(dweight2, f32, size, "dweight2"), pos, freq,
        _ptr(workspace, torch.uint8, "workspace"), workspace.numel(), _stream()), "ps_norm_rotary_backward")


def ps_bias_buckets(n_buckets: int, reach: int, both_sides: bool = True) -> torch.Tensor:
    """[2 reach + 1] int32 on the host: the bucket of a key `reach` in front of its row, ..., `reach` behind it."""
    out = torch.empty(max(2 * reach + 1, 1), dtype=torch.int32)
    _check(load_library().ps_bias_buckets(n_buckets, reach, int(both_sides), ctypes.cast(out.data_ptr(), ctypes.POINTER(ctypes.c_int32))),
           "ps_bias_buckets")
    return out


def ps_local_attention_workspace_bytes(n_seq: int, n_q: int, n_k: int, max_q: int, max_k: int, heads: int, kv_heads: int, head_dim: int,
                                       dtype: torch.dtype, backward: bool = False, left: int = -1, right: int = -1, sinks: int = 0,
                                       n_buckets: int = 0, reach: int = 0) -> int:
    """n_buckets, reach: of the learned bias, 0 without one."""
    d = ps_attention_desc(_dtype_code(dtype, "ps_local_attention_workspace_bytes"), n_seq, heads, kv_heads, head_dim, max_q, max_k, 0, n_q,
                          n_k, 1.0, 0.0)
    return int(load_library().ps_local_attention_workspace_bytes(ctypes.byref(d), ctypes.byref(ps_attention_local(left, right, sinks, n_buckets, reach)),
                                                                 int(backward)))


def _local(where, heads, left, right, sinks, buckets, bias, dbias=None):
    if (buckets is None) != (bias is None) or (dbias is not None and bias is None):
        raise ValueError(f"{where}: a bias goes with its buckets")
    if bias is None:
        return ps_attention_local(left, right, sinks)
    if bias.dim() != 2 or bias.shape[1] != heads or buckets.dim() != 1 or buckets.numel() % 2 == 0:
        raise ValueError(f"{where}: need a bias of buckets and {heads} heads, and a bucket for each of 2 reach + 1 distances")
    return ps_attention_local(left, right, sinks, bias.shape[0], buckets.numel() // 2, _ptr(buckets, torch.int32, "buckets"),
                              _ptr(bias, torch.float32, "bias"))


def ps_local_attention_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q_offsets: torch.Tensor, k_offsets: torch.Tensor,
                               max_q: int, max_k: int, out: torch.Tensor, lse: Optional[torch.Tensor], workspace: torch.Tensor,
                               left: int = -1, right: int = -1, sinks: int = 0, buckets: Optional[torch.Tensor] = None,
                               bias: Optional[torch.Tensor] = None, scale: Optional[float] = None, softcap: float = 0.0, causal: bool = False,
                               k_lengths: Optional[torch.Tensor] = None, q_start: Optional[torch.Tensor] = None,
                               prefix: Optional[torch.Tensor] = None, slopes: Optional[torch.Tensor] = None,
                               q_docs: Optional[torch.Tensor] = None, k_docs: Optional[torch.Tensor] = None,
                               status: Optional[torch.Tensor] = None, out_rest: Optional[torch.Tensor] = None) -> None:
    """ps_attention_forward() of rows that see the keys from `left` in front of them to `right` behind (-1: without end) and the first
    `sinks`, with bias [n_buckets, heads] (float32) by the distance's bucket, buckets [2 reach + 1] (int32)."""
    if _made("local_attention_forward", q, k, v, q_offsets, k_offsets, max_q, max_k, out, lse, workspace, left, right, sinks, buckets, bias,
             scale, softcap, causal, k_lengths, q_start, prefix, slopes, q_docs, k_docs, status, out_rest):
        return
    where = "ps_local_attention_forward"
    d, seqs, at, n_lse = _attention(where, q, k, q_offsets, k_offsets, max_q, max_k, scale, softcap, causal, k_lengths, q_start, prefix, slopes,
                                    q_docs, k_docs, {"q": (q, False), "k": (k, True), "v": (v, True), "out": (out, False)})
    local = _local(where, q.shape[1], left, right, sinks, buckets, bias)
    _check(load_library().ps_local_attention_forward(
        ctypes.byref(d), ctypes.byref(seqs), ctypes.byref(local), at["q"], at["k"], at["v"], at["out"], _sized_ptr(lse, torch.float32, n_lse, "lse"),
        _sized_ptr(out_rest, torch.bfloat16, q.numel(), "out_rest"), _ptr(workspace, torch.uint8, "workspace"), workspace.numel(),
        _ptr(status, torch.int64, "status"), _stream()), where)


def ps_local_attention_backward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, lse: torch.Tensor, dout: torch.Tensor,
                                q_offsets: torch.Tensor, k_offsets: torch.Tensor, max_q: int, max_k: int, dq: torch.Tensor, dk: torch.Tensor,
                                dv: torch.Tensor, workspace: torch.Tensor, left: int = -1, right: int = -1, sinks: int = 0,
                                buckets: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                                dbias: Optional[torch.Tensor] = None, scale: Optional[float] = None, softcap: float = 0.0,
                                causal: bool = False, k_lengths: Optional[torch.Tensor] = None, q_start: Optional[torch.Tensor] = None,
                                prefix: Optional[torch.Tensor] = None, slopes: Optional[torch.Tensor] = None,
                                q_docs: Optional[torch.Tensor] = None, k_docs: Optional[torch.Tensor] = None,
                                status: Optional[torch.Tensor] = None, out_rest: Optional[torch.Tensor] = None) -> None:
    """Arguments as of ps_local_attention_forward(), which has left `out`, `lse` and `out_rest`; dq like q, dk and dv like k, dbias like bias or
    None."""
    if _made("local_attention_backward", q, k, v, out, lse, dout, q_offsets, k_offsets, max_q, max_k, dq, dk, dv, workspace, left, right, sinks,
             buckets, bias, dbias, scale, softcap, causal, k_lengths, q_start, prefix, slopes, q_docs, k_docs, status, out_rest):
        return
    where = "ps_local_attention_backward"
    d, seqs, at, n_lse = _attention(where, q, k, q_offsets, k_offsets, max_q, max_k, scale, softcap, causal, k_lengths, q_start, prefix, slopes,
                                    q_docs, k_docs, {"q": (q, False), "k": (k, True), "v": (v, True), "out": (out, False), "dout": (dout, False),
                                                     "dq": (dq, False), "dk": (dk, True), "dv": (dv, True)})
    local = _local(where, q.shape[1], left, right, sinks, buckets, bias, dbias)
    _check(load_library().ps_local_attention_backward(
        ctypes.byref(d), ctypes.byref(seqs), ctypes.byref(local), at["q"], at["k"], at["v"], at["out"], _sized_ptr(lse, torch.float32, n_lse, "lse"),
        _sized_ptr(out_rest, torch.bfloat16, q.numel(), "out_rest"), at["dout"], at["dq"], at["dk"], at["dv"],
        None if dbias is None else _sized_ptr(dbias, torch.float32, bias.numel(), "dbias"), _ptr(workspace, torch.uint8, "workspace"),
        workspace.numel(), _ptr(status, torch.int64, "status"), _stream()), where)


def alloc_workspace(nbytes: int, device="cuda") -> torch.Tensor:
    """Uninitialised device scratch; torch's allocator hands out 512-byte aligned blocks."""
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)
