"""ctypes binding of libtwinkv.so (C ABI in include/twinkv.h).

Argument marshalling only: torch supplies device memory and the current HIP stream;
every step of the computation runs in the library's HIP kernels.  The library must have
been built (``python -m paper_2608_27128_amd.build``); a missing build raises.

Shapes: keys (n_heads, T, d) or (T, d) with the channel dimension contiguous, bfloat16 or
float32, on a GPU; retained / outputs (n_heads, T).  ``cu_seqlens`` (host sequence of
n_seqs + 1 ints) splits T into sequences; the default is one sequence of length T.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtwinkv.so")

TWINKV_OK = 0
TWINKV_BF16, TWINKV_F32 = 0, 1
OP_NN_SCORES, OP_REPAIR, OP_REPAIR_FROM_SCORES, OP_TWIN_COUNTS, OP_SCORE_EVICT, OP_COMPACT = range(6)
MAX_TAUS = 32
MAX_LEVELS = 4
PROBLEM_OK, PROBLEM_BUDGET_MISMATCH, PROBLEM_NONFINITE = 0, 1, 2
NOALLOC_MAX_SEQS = 2048

_lib = None

_VP = ctypes.c_void_p
_I = ctypes.c_int
_I64 = ctypes.c_int64
_F = ctypes.c_float
_PI64 = ctypes.POINTER(ctypes.c_int64)

SIGNATURES = {
    "twinkv_workspace_bytes": (_I64, [_I, _I, _I, _I, _I, _PI64]),
    "twinkv_nn_scores": (_I, [_VP, _I, _I, _I, _I, _PI64, _I64, _I64, _VP, _I,
                              _VP, _VP, _VP, _VP, _VP, _VP, _I64, _VP]),
    "twinkv_repair": (_I, [_VP, _I, _I, _I, _I, _PI64, _I64, _I64, _VP, _VP, _PI64, _F, _I, _I, _I,
                           _VP, _VP, _VP, _VP, _VP, _VP, _I64, _VP]),
    "twinkv_repair_from_scores": (_I, [_VP, _VP, _VP, _I, _I, _PI64, _PI64, _F, _I, _I, _VP,
                                       _VP, _I64, _VP]),
    "twinkv_repair_from_scores_noalloc": (_I, [_VP, _VP, _VP, _I, _I, _PI64, _PI64, _F, _I, _I,
                                               _VP, _VP]),
    "twinkv_twin_counts": (_I, [_VP, _I, _I, _I, _I, _PI64, _I64, _I64, _F, _I, _VP, _VP, _VP,
                                _I64, _VP]),
    "twinkv_score_evict": (_I, [_VP, _I, _I, _I, _I, _PI64, _I64, _I64, _PI64, _F, _I, _I, _I,
                                _VP, _VP, _VP, _VP, _VP, _I64, _VP]),
    "twinkv_prevalence": (_I, [_VP, _I, _I, _PI64, ctypes.POINTER(ctypes.c_float), _I, _VP, _VP,
                               _I64, _VP]),
    "twinkv_select_topk": (_I, [_VP, _I, _I, _PI64, _PI64, _I, _I, _VP, _VP, _VP, _I64, _VP]),
    "twinkv_nn_scores_levels": (_I, [_VP, _I, _I, _I, _I, _PI64, _I64, _I64, _VP, _I, _I, _VP,
                                     _VP, _VP, _VP, _VP, _VP, _I64, _VP]),
    "twinkv_levels_workspace_bytes": (_I64, [_I, _I, _I, _I, _PI64, _I, _I]),
    "twinkv_compact": (_I, [_VP, _VP, _I, _I, _I, _I, _PI64, _I64, _I64, _I64, _I64, _VP, _PI64,
                            _VP, _VP, _VP, _VP, _VP, _I64, _VP]),
    "twinkv_qk_norm_rope": (_I, [_VP, _VP, _I, _I, _I, _I, _I64, _I64, _I64, _I64, _I64, _VP, _VP, _F,
                                 _VP, _I64, _VP, _VP, _I64, _I64, _VP, _I64, _I64, _VP]),
    "twinkv_attention_workspace_bytes": (_I64, [_I, _I, _I, _I, _I, _PI64, _PI64, _I64, _I64]),
    "twinkv_sink_attention": (_I, [_VP, _VP, _VP, _I, _I, _I, _I, _I, _PI64, _PI64, _I64, _I64, _I64,
                                   _I64, _I64, _I64, _I64, _I64, _F, _VP, _I64, _I64, _VP, _VP, _I64,
                                   _VP]),
    "twinkv_cache4_workspace_bytes": (_I64, [_I]),
    "twinkv_cache4_compact": (_I, [_VP, _VP, _I, _PI64, _I64, _I64, _I64, _I64, _VP, _VP, _VP, _VP, _VP,
                                   _VP, _I64, _VP]),
    "twinkv_cache4_append": (_I, [_VP, _VP, _I, _PI64, _I64, _I64, _I64, _I64, _VP, _VP, _VP, _VP, _VP,
                                  _I64, _VP]),
    "twinkv_cache4_read": (_I, [_VP, _VP, _VP, _I, _PI64, _VP, _VP, _VP, _I64, _VP]),
    "twinkv_cache4_attention": (_I, [_VP, _I, _I, _PI64, _I64, _I64, _VP, _VP, _F, _VP, _I64, _I64, _VP,
                                     _VP, _I64, _VP]),
    "twinkv_mass_workspace_bytes": (_I64, [_I, _I, _I, _I, _I, _PI64, _PI64, _I64, _I64]),
    "twinkv_attention_mass": (_I, [_VP, _VP, _I, _I, _I, _I, _I, _PI64, _PI64, _I64, _I64, _I64, _I64, _I64,
                                   _I64, _F, _VP, _VP, _VP, _VP, _I64, _VP]),
    "twinkv_cache8_workspace_bytes": (_I64, [_I]),
    "twinkv_cache8_compact": (_I, [_VP, _VP, _I, _PI64, _I64, _I64, _I64, _I64, _VP, _VP, _VP, _VP, _VP, _VP,
                                   _VP, _VP, _I64, _VP]),
    "twinkv_cache8_append": (_I, [_VP, _VP, _I, _PI64, _I64, _I64, _I64, _I64, _VP, _VP, _VP, _VP, _VP, _I64,
                                  _VP]),
    "twinkv_cache8_read": (_I, [_VP, _VP, _VP, _I, _PI64, _VP, _VP, _VP, _I64, _VP]),
    "twinkv_cache8_attention": (_I, [_VP, _I, _I, _PI64, _I64, _I64, _VP, _VP, _F, _VP, _I64, _I64, _VP, _VP,
                                     _VP, _VP, _I64, _VP]),
    "twinkv_cache8_attention_workspace_bytes": (_I64, [_I, _I, _I, _I, _I, _PI64, _PI64, _I]),
    "twinkv_cache8_evict": (_I, [_VP, _VP, _VP, _VP, _PI64, _I, _I, _VP, _VP, _VP, _VP, _VP, _I64, _VP]),
    "twinkv_status_string": (ctypes.c_char_p, [_I]),
    "twinkv_version": (_I, []),
    "twinkv_profile_sim_events": (None, [_VP, _VP]),
}


class TwinKVError(RuntimeError):
    def __init__(self, fn: str, code: int):
        super().__init__(f"{fn} failed: {status_string(code)} (code {code})")
        self.code = code


def lib() -> ctypes.CDLL:
    """The loaded library (loads it on first use; raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2608_27128_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def status_string(code: int) -> str:
    return lib().twinkv_status_string(int(code)).decode()


def version() -> int:
    return int(lib().twinkv_version())


def _i64_array(values) -> ctypes.Array:
    arr = np.ascontiguousarray(np.asarray(values, dtype=np.int64))
    return (ctypes.c_int64 * len(arr))(*arr.tolist())


def workspace_bytes(op: int, dtype: int, d: int, n_heads: int, cu_seqlens) -> int:
    cu = _i64_array(cu_seqlens)
    n = int(lib().twinkv_workspace_bytes(op, dtype, d, n_heads, len(cu) - 1, cu))
    if n < 0:
        raise TwinKVError("twinkv_workspace_bytes", -n)
    return n


def levels_workspace_bytes(dtype: int, d: int, n_heads: int, cu_seqlens, n_levels: int,
                           want_all: bool) -> int:
    cu = _i64_array(cu_seqlens)
    n = int(lib().twinkv_levels_workspace_bytes(dtype, d, n_heads, len(cu) - 1, cu,
                                                int(n_levels), 1 if want_all else 0))
    if n < 0:
        raise TwinKVError("twinkv_levels_workspace_bytes", -n)
    return n


def _event_handle(e):
    if e is None:
        return None
    if isinstance(e, ctypes.c_void_p):
        return e.value
    return int(e)


def profile_sim_events(start=None, stop=None) -> None:
    """Record two hipEvent_t handles (ints or c_void_p) around the similarity kernel of later
    calls on this thread (None, None stops)."""
    lib().twinkv_profile_sim_events(_event_handle(start), _event_handle(stop))


def _torch():
    import torch
    return torch


def _prep_keys(keys):
    torch = _torch()
    if keys.dim() == 2:
        keys = keys.unsqueeze(0)
    if keys.dim() != 3:
        raise ValueError("keys must be (n_heads, T, d) or (T, d)")
    if keys.dtype == torch.bfloat16:
        dt = TWINKV_BF16
    elif keys.dtype == torch.float32:
        dt = TWINKV_F32
    else:
        raise ValueError(f"unsupported key dtype {keys.dtype}")
    return keys, dt


def _on_gpu(t, name: str):
    """Device check, after the shape and offset checks (which need no GPU)."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be on a GPU")
    if t.dim() == 3 and t.stride(2) != 1:
        t = t.contiguous()
    return t


def _vec2d(x, name: str):
    """A float32 (n_heads, T) or (T,) tensor, before the device check."""
    torch = _torch()
    if x.dim() == 1:
        x = x.unsqueeze(0)
    if x.dim() != 2 or x.dtype != torch.float32:
        raise ValueError(f"{name} must be a float32 (n_heads, T) tensor")
    return x


def _cu(cu_seqlens, T: int):
    """The sequence offsets as int64, checked against the tensors' token count T: the library
    lays every [n_heads][T] buffer out from cu_seqlens, so an offset list that ends anywhere
    but T would make its kernels read or write outside the tensors."""
    if cu_seqlens is None:
        return np.array([0, T], dtype=np.int64)
    cu = np.asarray(cu_seqlens, dtype=np.int64)
    if cu.ndim != 1 or len(cu) < 2:
        raise ValueError("cu_seqlens must list n_seqs + 1 >= 2 offsets")
    if cu[0] != 0 or np.any(np.diff(cu) < 0):
        raise ValueError("cu_seqlens must start at 0 and never decrease")
    if cu[-1] != T:
        raise ValueError(f"cu_seqlens[-1] = {int(cu[-1])} must equal T = {T}")
    return cu


def _check_outputs(out: dict, spec: dict, fn: str) -> dict:
    """Buffers passed back through ``outputs``: each present entry must have the shape, dtype
    and device the call writes (``spec``: name -> (shape, dtype, device, required))."""
    got = dict(out)
    for name, (shape, dtype, dev, required) in spec.items():
        t = got.get(name)
        if t is None:
            if required:
                raise ValueError(f"{fn}: outputs[{name!r}] is required")
            continue
        if tuple(t.shape) != tuple(shape) or t.dtype != dtype or t.device != dev:
            raise ValueError(f"{fn}: outputs[{name!r}] must be {tuple(shape)} {dtype} on {dev}, "
                             f"got {tuple(t.shape)} {t.dtype} on {t.device}")
        if not t.is_contiguous():
            raise ValueError(f"{fn}: outputs[{name!r}] must be contiguous")
    return got


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(device) -> int:
    # the handle alone, where torch has it (the name is not of its documented interface): building its stream
    # object costs a small call more than its launch
    torch = _torch()
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return torch.cuda.current_stream(device).cuda_stream if raw is None else raw(device.index)


def _mask(x, n_heads, T, device, name):
    torch = _torch()
    if x is None:
        return None
    if x.dim() == 1:
        x = x.unsqueeze(0)
    if tuple(x.shape) != (n_heads, T):
        raise ValueError(f"{name} must have shape ({n_heads}, {T})")
    if x.dtype == torch.bool:
        x = x.to(torch.uint8)
    if x.dtype != torch.uint8:
        raise ValueError(f"{name} must be uint8 or bool")
    if x.device != device:
        raise ValueError(f"{name} must be on {device}")
    return x.contiguous()


def _launch(dev, name: str, *args) -> None:
    """Call the library entry point ``name`` with the tensors' device current: the library
    enqueues on the given stream of the current device and keeps its per-device state there."""
    torch = _torch()
    fn = getattr(_lib or lib(), name)
    if torch.cuda.current_device() == dev.index:
        rc = fn(*args)
    else:
        with torch.cuda.device(dev):
            rc = fn(*args)
    if rc != TWINKV_OK:
        raise TwinKVError(name, rc)


def _nbytes(t) -> int:
    return t.numel() * t.element_size()


def _workspace(workspace, nbytes: int, dev):
    """The caller's workspace when it is large enough (a contiguous tensor on the call's
    device; its byte count is what is compared), else a fresh uint8 buffer of nbytes."""
    torch = _torch()
    if workspace is not None:
        if workspace.device != dev or not workspace.is_contiguous():
            raise ValueError(f"workspace must be a contiguous tensor on {dev}")
        if _nbytes(workspace) >= nbytes:
            return workspace
    return torch.empty((nbytes,), dtype=torch.uint8, device=dev)


def nn_scores(keys, retained=None, w: int = 32, cu_seqlens=None, *, want_arg: bool = True,
              workspace=None) -> dict:
    """Best twin of every token: best_all/arg_all over all keys, best_ret/arg_ret (Eq. 4 b_i(S0))
    over the retained set when ``retained`` is given, and a per-problem status."""
    torch = _torch()
    keys, dt = _prep_keys(keys)
    H, T, d = keys.shape
    cu = _cu(cu_seqlens, T)
    keys = _on_gpu(keys, "keys")
    dev = keys.device
    ret = _mask(retained, H, T, dev, "retained")
    out = {
        "best_all": torch.empty((H, T), dtype=torch.float32, device=dev),
        "arg_all": torch.empty((H, T), dtype=torch.int32, device=dev) if want_arg else None,
        "status": torch.empty((H * (len(cu) - 1),), dtype=torch.int32, device=dev),
    }
    if ret is not None:
        out["best_ret"] = torch.empty((H, T), dtype=torch.float32, device=dev)
        out["arg_ret"] = torch.empty((H, T), dtype=torch.int32, device=dev) if want_arg else None
    ws = _workspace(workspace, workspace_bytes(OP_NN_SCORES, dt, d, H, cu), dev)
    _launch(dev, "twinkv_nn_scores",
        keys.data_ptr(), dt, d, H, len(cu) - 1, _i64_array(cu), keys.stride(0), keys.stride(1),
        _ptr(ret), int(w), _ptr(out["best_all"]), _ptr(out["arg_all"]),
        _ptr(out.get("best_ret")), _ptr(out.get("arg_ret")), _ptr(out["status"]),
        ws.data_ptr(), _nbytes(ws), _stream(dev))
    return {k: v for k, v in out.items() if v is not None}


def nn_scores_levels(keys, level, n_levels: int, w: int = 32, cu_seqlens=None, *,
                     want_all: bool = False, want_arg: bool = True, workspace=None,
                     outputs: Optional[dict] = None) -> dict:
    """b_i(S_k) (Sec. 3.4 Eq. 4) for nested retained sets S_1 within ... within S_L given as a
    level array (n_heads, T) uint8 (k = the smallest set holding the token, 0 = none):
    best_lvl / arg_lvl of shape (n_levels, n_heads, T), and best_all / arg_all when
    ``want_all``.  ``outputs`` may pass back the dict of an earlier call."""
    torch = _torch()
    keys, dt = _prep_keys(keys)
    H, T, d = keys.shape
    cu = _cu(cu_seqlens, T)
    n_seqs = len(cu) - 1
    if level is None:
        raise ValueError("level is required")
    if not 1 <= int(n_levels) <= MAX_LEVELS:
        raise ValueError(f"n_levels must be in [1, {MAX_LEVELS}]")
    keys = _on_gpu(keys, "keys")
    dev = keys.device
    lv = _mask(level, H, T, dev, "level")
    f32, i32 = torch.float32, torch.int32
    spec = {
        "best_lvl": ((n_levels, H, T), f32, dev, True),
        "arg_lvl": ((n_levels, H, T), i32, dev, False),
        "best_all": ((H, T), f32, dev, False),
        "arg_all": ((H, T), i32, dev, False),
        "status": ((H * n_seqs,), i32, dev, True),
    }
    if outputs is None:
        out = {
            "best_lvl": torch.empty((n_levels, H, T), dtype=f32, device=dev),
            "arg_lvl": torch.empty((n_levels, H, T), dtype=i32, device=dev) if want_arg else None,
            "best_all": torch.empty((H, T), dtype=f32, device=dev) if want_all else None,
            "arg_all": torch.empty((H, T), dtype=i32, device=dev) if (want_all and want_arg) else None,
            "status": torch.empty((H * n_seqs,), dtype=i32, device=dev),
        }
    else:
        out = _check_outputs(outputs, spec, "nn_scores_levels")
        want_all = out.get("best_all") is not None or out.get("arg_all") is not None
    ws = _workspace(workspace, levels_workspace_bytes(dt, d, H, cu, n_levels, want_all), dev)
    _launch(dev, "twinkv_nn_scores_levels",
        keys.data_ptr(), dt, d, H, n_seqs, _i64_array(cu), keys.stride(0), keys.stride(1),
        lv.data_ptr(), int(n_levels), int(w), _ptr(out.get("best_all")), _ptr(out.get("arg_all")),
        out["best_lvl"].data_ptr(), _ptr(out.get("arg_lvl")), _ptr(out["status"]),
        ws.data_ptr(), _nbytes(ws), _stream(dev))
    return {k: v for k, v in out.items() if v is not None}


def _budget(budget, n_seqs: int):
    return np.broadcast_to(np.asarray(budget, dtype=np.int64), (n_seqs,)).copy()


def repair(keys, retained, budget, tau: float, w: int = 32, n_sink: int = 4, n_recent: int = 64,
           cu_seqlens=None, *, want_all: bool = True, want_arg: bool = True, out_mask=None,
           workspace=None, outputs: Optional[dict] = None) -> dict:
    """The repair pass of Sec. 3.4: S1 (uint8 mask), stats (|O|, |D|, m, status) per problem,
    and the scores it was computed from (best_ret = b; best_all/arg_all when want_all).

    ``outputs`` may pass back the dict of an earlier call with the same shapes to reuse its
    buffers (the entries it holds decide what is computed); ``out_mask`` may be ``retained``
    itself for an in-place update."""
    torch = _torch()
    keys, dt = _prep_keys(keys)
    H, T, d = keys.shape
    cu = _cu(cu_seqlens, T)
    n_seqs = len(cu) - 1
    if retained is None:
        raise ValueError("retained is required")
    bud = _budget(budget, n_seqs)
    keys = _on_gpu(keys, "keys")
    dev = keys.device
    ret = _mask(retained, H, T, dev, "retained")
    f32, i32 = torch.float32, torch.int32
    if outputs is None:
        out = {
            "s1": torch.empty((H, T), dtype=torch.uint8, device=dev),
            "stats": torch.empty((H * n_seqs, 4), dtype=i32, device=dev),
            "best_ret": torch.empty((H, T), dtype=f32, device=dev),
            "arg_ret": torch.empty((H, T), dtype=i32, device=dev) if want_arg else None,
            "best_all": torch.empty((H, T), dtype=f32, device=dev) if want_all else None,
            "arg_all": torch.empty((H, T), dtype=i32, device=dev) if (want_all and want_arg) else None,
        }
    else:
        spec = {
            "s1": ((H, T), torch.uint8, dev, out_mask is None),
            "stats": ((H * n_seqs, 4), i32, dev, True),
            "best_ret": ((H, T), f32, dev, False),
            "arg_ret": ((H, T), i32, dev, False),
            "best_all": ((H, T), f32, dev, False),
            "arg_all": ((H, T), i32, dev, False),
        }
        out = _check_outputs(outputs, spec, "repair")
    if out_mask is not None:
        m = _mask(out_mask, H, T, dev, "out_mask")
        if m.data_ptr() != out_mask.data_ptr():
            raise ValueError("out_mask must be a contiguous uint8 (n_heads, T) tensor")
        out["s1"] = out_mask
    ws = _workspace(workspace, workspace_bytes(OP_REPAIR, dt, d, H, cu), dev)
    _launch(dev, "twinkv_repair",
        keys.data_ptr(), dt, d, H, n_seqs, _i64_array(cu), keys.stride(0), keys.stride(1),
        ret.data_ptr(), out["s1"].data_ptr(), _i64_array(bud), float(tau), int(w), int(n_sink),
        int(n_recent), out["stats"].data_ptr(), _ptr(out.get("best_all")), _ptr(out.get("arg_all")),
        _ptr(out.get("best_ret")), _ptr(out.get("arg_ret")), ws.data_ptr(), _nbytes(ws), _stream(dev))
    return {k: v for k, v in out.items() if v is not None}


def repair_from_scores(b, retained, budget, tau: float, n_sink: int = 4, n_recent: int = 64,
                       cu_seqlens=None, *, out_mask=None) -> dict:
    """Classification, ranking and swap of Sec. 3.4 from given scores b (n_heads, T) float32."""
    torch = _torch()
    b = _vec2d(b, "b")
    H, T = b.shape
    cu = _cu(cu_seqlens, T)
    n_seqs = len(cu) - 1
    if retained is None:
        raise ValueError("retained is required")
    bud = _budget(budget, n_seqs)
    b = _on_gpu(b, "b").contiguous()
    dev = b.device
    ret = _mask(retained, H, T, dev, "retained")
    if out_mask is not None:
        s1 = _mask(out_mask, H, T, dev, "out_mask")
        if s1.data_ptr() != out_mask.data_ptr():
            raise ValueError("out_mask must be a contiguous uint8 (n_heads, T) tensor")
    else:
        s1 = torch.empty((H, T), dtype=torch.uint8, device=dev)
    stats = torch.empty((H * n_seqs, 4), dtype=torch.int32, device=dev)
    ws = _workspace(None, workspace_bytes(OP_REPAIR_FROM_SCORES, 0, 64, H, cu), dev)
    _launch(dev, "twinkv_repair_from_scores",
        b.data_ptr(), ret.data_ptr(), s1.data_ptr(), H, n_seqs, _i64_array(cu), _i64_array(bud),
        float(tau), int(n_sink), int(n_recent), stats.data_ptr(), ws.data_ptr(), _nbytes(ws),
        _stream(dev))
    return {"s1": s1, "stats": stats}


def repair_from_scores_noalloc(b, retained, budget, tau: float, n_sink: int = 4,
                               n_recent: int = 64, cu_seqlens=None, *, outputs: dict) -> dict:
    """repair_from_scores through the entry point that allocates nothing: the caller passes
    the output buffers (``outputs`` with "s1" uint8 (n_heads, T) and "stats" int32
    (n_heads * n_seqs, 4)), and the library's static scratch holds the sequence table (at
    most NOALLOC_MAX_SEQS sequences).  Calls overlapping on one GPU race."""
    torch = _torch()
    b = _vec2d(b, "b")
    H, T = b.shape
    cu = _cu(cu_seqlens, T)
    n_seqs = len(cu) - 1
    if retained is None:
        raise ValueError("retained is required")
    bud = _budget(budget, n_seqs)
    b = _on_gpu(b, "b")
    if not b.is_contiguous():
        raise ValueError("b must be contiguous (the call may not allocate a copy)")
    dev = b.device
    if retained.dim() == 1:
        retained = retained.unsqueeze(0)
    if (tuple(retained.shape) != (H, T) or retained.dtype != torch.uint8 or retained.device != dev
            or not retained.is_contiguous()):
        raise ValueError(f"retained must be a contiguous uint8 ({H}, {T}) tensor on {dev}")
    spec = {"s1": ((H, T), torch.uint8, dev, True), "stats": ((H * n_seqs, 4), torch.int32, dev, True)}
    out = _check_outputs(outputs, spec, "repair_from_scores_noalloc")
    _launch(dev, "twinkv_repair_from_scores_noalloc",
        b.data_ptr(), retained.data_ptr(), out["s1"].data_ptr(), H, n_seqs, _i64_array(cu),
        _i64_array(bud), float(tau), int(n_sink), int(n_recent), out["stats"].data_ptr(),
        _stream(dev))
    return out


def twin_counts(keys, tau: float, w: int = 32, cu_seqlens=None, *, workspace=None) -> dict:
    """Eq. 2 twin counts r_i (int32, (n_heads, T)) and a per-problem status."""
    torch = _torch()
    keys, dt = _prep_keys(keys)
    H, T, d = keys.shape
    cu = _cu(cu_seqlens, T)
    keys = _on_gpu(keys, "keys")
    dev = keys.device
    counts = torch.empty((H, T), dtype=torch.int32, device=dev)
    status = torch.empty((H * (len(cu) - 1),), dtype=torch.int32, device=dev)
    ws = _workspace(workspace, workspace_bytes(OP_TWIN_COUNTS, dt, d, H, cu), dev)
    _launch(dev, "twinkv_twin_counts",
        keys.data_ptr(), dt, d, H, len(cu) - 1, _i64_array(cu), keys.stride(0), keys.stride(1),
        float(tau), int(w), counts.data_ptr(), status.data_ptr(), ws.data_ptr(), _nbytes(ws),
        _stream(dev))
    return {"counts": counts, "status": status}


def score_evict(keys, budget, tau: float, w: int = 32, n_sink: int = 4, n_recent: int = 64,
                cu_seqlens=None, *, want_scores: bool = True, workspace=None,
                outputs: Optional[dict] = None) -> dict:
    """The standalone scorer of Sec. 3.2: counts (Eq. 2), scores (Eq. 3), the kept set of the
    `budget` highest scores (uint8) and per-problem stats {kept, count at cut, status, 0}.
    ``outputs`` may pass back the dict of an earlier call with the same shapes."""
    torch = _torch()
    keys, dt = _prep_keys(keys)
    H, T, d = keys.shape
    cu = _cu(cu_seqlens, T)
    n_seqs = len(cu) - 1
    bud = _budget(budget, n_seqs)
    keys = _on_gpu(keys, "keys")
    dev = keys.device
    if outputs is None:
        out = {
            "retained": torch.empty((H, T), dtype=torch.uint8, device=dev),
            "counts": torch.empty((H, T), dtype=torch.int32, device=dev),
            "scores": torch.empty((H, T), dtype=torch.float32, device=dev) if want_scores else None,
            "stats": torch.empty((H * n_seqs, 4), dtype=torch.int32, device=dev),
        }
    else:
        spec = {
            "retained": ((H, T), torch.uint8, dev, True),
            "counts": ((H, T), torch.int32, dev, True),
            "scores": ((H, T), torch.float32, dev, False),
            "stats": ((H * n_seqs, 4), torch.int32, dev, True),
        }
        out = _check_outputs(outputs, spec, "score_evict")
        out.setdefault("scores", None)
    ws = _workspace(workspace, workspace_bytes(OP_SCORE_EVICT, dt, d, H, cu), dev)
    _launch(dev, "twinkv_score_evict",
        keys.data_ptr(), dt, d, H, n_seqs, _i64_array(cu), keys.stride(0), keys.stride(1),
        _i64_array(bud), float(tau), int(w), int(n_sink), int(n_recent),
        out["retained"].data_ptr(), out["counts"].data_ptr(), _ptr(out["scores"]),
        out["stats"].data_ptr(), ws.data_ptr(), _nbytes(ws), _stream(dev))
    return {k: v for k, v in out.items() if v is not None}


def select_topk(scores, budget, n_sink: int = 4, n_recent: int = 64, cu_seqlens=None, *,
                workspace=None, outputs: Optional[dict] = None) -> dict:
    """A score-based policy's retained set (Sec. 3.1 / 3.2): per problem the ``budget[s]``
    positions first in the order protected, higher score, lower position (NaN last).
    scores: float32 (n_heads, T) on the GPU.  Returns retained uint8 (n_heads, T) and
    stats int32 (n_heads * n_seqs, 4) = {kept, NaN scores, 0, 0}."""
    torch = _torch()
    scores = _vec2d(scores, "scores")
    H, T = scores.shape
    cu = _cu(cu_seqlens, T)
    n_seqs = len(cu) - 1
    bud = _budget(budget, n_seqs)
    scores = _on_gpu(scores, "scores").contiguous()
    dev = scores.device
    if outputs is None:
        out = {
            "retained": torch.empty((H, T), dtype=torch.uint8, device=dev),
            "stats": torch.empty((H * n_seqs, 4), dtype=torch.int32, device=dev),
        }
    else:
        spec = {"retained": ((H, T), torch.uint8, dev, True),
                "stats": ((H * n_seqs, 4), torch.int32, dev, True)}
        out = _check_outputs(outputs, spec, "select_topk")
    ws = _workspace(workspace, workspace_bytes(OP_REPAIR_FROM_SCORES, 0, 64, H, cu), dev)
    _launch(dev, "twinkv_select_topk",
        scores.data_ptr(), H, n_seqs, _i64_array(cu), _i64_array(bud), int(n_sink),
        int(n_recent), out["retained"].data_ptr(), _ptr(out["stats"]), ws.data_ptr(),
        _nbytes(ws), _stream(dev))
    return out


def prevalence(best_all, taus, cu_seqlens=None) -> "torch.Tensor":
    """Tokens with at least one twin (best_all > tau) per problem and threshold:
    int32 (n_heads * n_seqs, len(taus))."""
    torch = _torch()
    best_all = _vec2d(best_all, "best_all")
    H, T = best_all.shape
    cu = _cu(cu_seqlens, T)
    n_seqs = len(cu) - 1
    tv = np.ascontiguousarray(np.asarray(taus, dtype=np.float32).reshape(-1))
    if not 1 <= len(tv) <= MAX_TAUS:
        raise ValueError(f"between 1 and {MAX_TAUS} thresholds")
    best_all = _on_gpu(best_all, "best_all").contiguous()
    dev = best_all.device
    out = torch.empty((H * n_seqs, len(tv)), dtype=torch.int32, device=dev)
    ws = _workspace(None, workspace_bytes(OP_REPAIR_FROM_SCORES, 0, 64, H, cu), dev)
    _launch(dev, "twinkv_prevalence",
        best_all.data_ptr(), H, n_seqs, _i64_array(cu),
        tv.ctypes.data_as(ctypes.POINTER(ctypes.c_float)), len(tv), out.data_ptr(),
        ws.data_ptr(), _nbytes(ws), _stream(dev))
    return out


def compact(keys, retained, capacity, values=None, cu_seqlens=None, *, want_pos: bool = True,
            workspace=None, outputs: Optional[dict] = None) -> dict:
    """KV compaction (Sec. 3.1): the rows of the retained positions of every problem, in
    position order, in its ``capacity[s]`` reserved rows: keys (and values) (n_heads, C, d),
    positions (n_heads, C) int32 (-1 on unused rows) and stats {kept, capacity, status, 0}.
    ``values`` must have the dtype and shape of ``keys``.  ``outputs`` may pass back the dict
    of an earlier call with the same shapes to reuse its buffers."""
    torch = _torch()
    keys, dt = _prep_keys(keys)
    H, T, d = keys.shape
    if values is not None:
        if values.dim() == 2:
            values = values.unsqueeze(0)
        if values.dtype != keys.dtype or tuple(values.shape) != (H, T, d):
            raise ValueError("values must match keys in dtype and shape")
    cu = _cu(cu_seqlens, T)
    n_seqs = len(cu) - 1
    if retained is None:
        raise ValueError("retained is required")
    cap = _budget(capacity, n_seqs)
    C = int(cap.sum())
    keys = _on_gpu(keys, "keys")
    dev = keys.device
    if values is not None:
        values = _on_gpu(values, "values")
        if values.device != dev:
            raise ValueError("values must be on the keys' device")
    ret = _mask(retained, H, T, dev, "retained")
    if outputs is None:
        out = {
            "keys": torch.empty((H, C, d), dtype=keys.dtype, device=dev),
            "values": torch.empty((H, C, d), dtype=keys.dtype, device=dev) if values is not None else None,
            "pos": torch.empty((H, C), dtype=torch.int32, device=dev) if want_pos else None,
            "stats": torch.empty((H * n_seqs, 4), dtype=torch.int32, device=dev),
        }
    else:
        spec = {
            "keys": ((H, C, d), keys.dtype, dev, True),
            "values": ((H, C, d), keys.dtype, dev, values is not None),
            "pos": ((H, C), torch.int32, dev, False),
            "stats": ((H * n_seqs, 4), torch.int32, dev, True),
        }
        out = _check_outputs(outputs, spec, "compact")
        out.setdefault("values", None)
        out.setdefault("pos", None)
        if values is None:
            out["values"] = None
    ws = _workspace(workspace, workspace_bytes(OP_COMPACT, dt, d, H, cu), dev)
    vs = (values.stride(0), values.stride(1)) if values is not None else (0, 0)
    _launch(dev, "twinkv_compact",
        keys.data_ptr(), _ptr(values), dt, d, H, n_seqs, _i64_array(cu), keys.stride(0),
        keys.stride(1), vs[0], vs[1], ret.data_ptr(), _i64_array(cap), out["keys"].data_ptr(),
        _ptr(out["values"]), _ptr(out["pos"]), out["stats"].data_ptr(), ws.data_ptr(), _nbytes(ws),
        _stream(dev))
    return {k: v for k, v in out.items() if v is not None}


# ---------------------------------------------------------------- the layer around the cache

def _offsets(cu, T: int, name: str):
    """Host offsets as (C array over an int64 copy of them, sequences), checked to end at T: what the tensors
    hold.  That they start at 0 and never decrease the library checks, before anything is enqueued."""
    arr = np.array((0, T) if cu is None else cu, dtype=np.int64)
    if arr.ndim != 1 or arr.size < 2:
        raise ValueError(f"{name} must list n_seqs + 1 >= 2 offsets")
    if arr[-1] != T:
        raise ValueError(f"{name}[-1] = {int(arr[-1])} must equal T = {T}")
    return (ctypes.c_int64 * arr.size).from_buffer(arr), arr.size - 1


def _rows(x, name: str, dtype=None, d=None, dev=None):
    """A (heads, T, d) tensor (or (T, d)) of a supported type, as the library addresses it: any head
    and token strides of a multiple of 16 bytes, channels contiguous; others are copied.  Returns it with
    its dtype code."""
    torch = _torch()
    if x.dim() == 2:
        x = x.unsqueeze(0)
    if x.dim() != 3:
        raise ValueError(f"{name} must be (heads, T, d) or (T, d)")
    if x.dtype == torch.bfloat16:
        dt = TWINKV_BF16
    elif x.dtype == torch.float32:
        dt = TWINKV_F32
    else:
        raise ValueError(f"unsupported {name} dtype {x.dtype}")
    if dtype is not None and x.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {x.dtype}")
    if d is not None and x.shape[2] != d:
        raise ValueError(f"{name} must have {d} channels, got {x.shape[2]}")
    if dev is not None and x.device != dev:
        raise ValueError(f"{name} must be on {dev}")
    if not x.is_cuda:
        raise ValueError(f"{name} must be on a GPU")
    h, t, c = x.stride()
    lanes = 16 // x.element_size()
    if c != 1 or t % lanes or h % lanes or t < x.shape[2] or x.data_ptr() % 16:
        x = x.clone(memory_format=torch.contiguous_format)
    return x, dt


def _rows_overlap(heads: int, T: int, h: int, t: int, d: int) -> bool:
    """Whether two of the rows of d channels at head * h + token * t (t >= d) share a place."""
    if heads < 2:
        return False
    if h < d:
        return True
    if T < 2 or h >= (T - 1) * t + d or t >= (heads - 1) * h + d:
        return False
    for at in range(h, min(heads * h, (T - 1) * t + d), h):  # the distance of two heads, against that of tokens
        token = min(at // t, T - 1)
        if at - token * t < d or (token < T - 1 and (token + 1) * t - at < d):
            return True
    return False


def _out_rows(out, shape, like, name: str):
    """The caller's output rows (written in place, so they must be addressable as they are), or new ones."""
    if out is None:
        return like.new_empty(shape)
    if tuple(out.shape) != tuple(shape) or out.dtype != like.dtype or out.device != like.device:
        raise ValueError(f"{name} must be {tuple(shape)} {like.dtype} on {like.device}, got "
                         f"{tuple(out.shape)} {out.dtype} on {out.device}")
    h, t, c = out.stride()
    lanes = 16 // out.element_size()
    if c != 1 or t % lanes or h % lanes or t < shape[2] or out.data_ptr() % 16 or _rows_overlap(shape[0], shape[1], h, t, shape[2]):
        raise ValueError(f"{name} must have contiguous channels, strides of multiples of 16 bytes and no overlap")
    return out


def _no_gradient(fn: str, *tensors) -> None:
    """These calls return tensors that torch's autograd does not know of: where it would record one, the
    gradient would be lost without a word."""
    for x in tensors:
        if x is not None and x.requires_grad and _torch().is_grad_enabled():
            raise ValueError(f"{fn} has no gradient: call it under torch.no_grad(), or on detached tensors")


def _small(x, shape, dtype, dev, name: str):
    """A contiguous, 16-byte aligned operand of one exact shape and type (None stays None)."""
    if x is None:
        return None
    if x.shape != shape or x.dtype != dtype or x.device != dev:
        raise ValueError(f"{name} must be {shape} {dtype} on {dev}, got {tuple(x.shape)} {x.dtype} on {x.device}")
    if x.is_contiguous() and x.data_ptr() % 16 == 0:
        return x
    return x.clone(memory_format=_torch().contiguous_format)


def _scratch(workspace, nbytes: int, dev, fn: str):
    """(tensor, pointer, bytes) of a workspace; nothing where nothing is needed."""
    if nbytes < 0:
        raise TwinKVError(fn, -nbytes)
    if nbytes == 0 and workspace is None:
        return None, None, 0
    ws = _workspace(workspace, nbytes, dev)
    return ws, ws.data_ptr(), _nbytes(ws)


def qk_norm_rope(q, k, q_weight=None, k_weight=None, eps: float = 1e-6, rope=None, positions=None, *,
                 q_out=None, k_out=None) -> dict:
    """RMS norm of each head of q (Hq, T, d) and k (Hk, T, d) (a weight (d,) float32 each; None: not
    normalised) and the rotary embedding by ``rope`` (n_pos, d) float32 (cos of the d/2 pairs, then
    sin; None: no rotation) at ``positions`` (T,) int32.  Channel c turns with c + d/2; a token whose position
    is no row of the table gets NaN.  A projection's token-major output goes in as its (H, T, d) view.  q or k
    may be None.  The outputs may be the inputs.  There is no gradient: inputs that require one are refused
    (torch.no_grad() lifts that)."""
    torch = _torch()
    some = q if q is not None else k
    if some is None:
        raise ValueError("q or k is required")
    _no_gradient("qk_norm_rope", q, k, q_weight, k_weight, rope, q_out, k_out)
    dt = T = d = None
    if q is not None:
        q, dt = _rows(q, "q")
        _, T, d = q.shape
    if k is not None:
        k, dt = _rows(k, "k", some.dtype, d, some.device)
        if T is not None and k.shape[1] != T:
            raise ValueError(f"k must have {T} tokens, got {k.shape[1]}")
        _, T, d = k.shape
    dev = some.device
    f32 = torch.float32
    q_weight = _small(q_weight, (d,), f32, dev, "q_weight")
    k_weight = _small(k_weight, (d,), f32, dev, "k_weight")
    if rope is not None:
        if positions is None:
            raise ValueError("positions is required with rope")
        rope = _small(rope, (rope.shape[0], d), f32, dev, "rope")
        positions = _small(positions, (T,), torch.int32, dev, "positions")
    n_pos = 0 if rope is None else rope.shape[0]
    # a table without rows has no address, and none is the library's "no rotation"
    table = torch.empty((1, d), dtype=f32, device=dev) if rope is not None and n_pos == 0 else rope
    out = {}
    args = {"q": (None, 0, 0, 0, None, 0, 0), "k": (None, 0, 0, 0, None, 0, 0)}
    for name, x, to in (("q", q, q_out), ("k", k, k_out)):
        if x is None:
            continue
        if to is not None and to.dim() == 2:
            to = to.unsqueeze(0)
        o = out[name] = _out_rows(to, x.shape, x, f"{name}_out")
        args[name] = (x.data_ptr(), x.shape[0], x.stride(0), x.stride(1), o.data_ptr(), o.stride(0), o.stride(1))
    qa, ka = args["q"], args["k"]
    _launch(dev, "twinkv_qk_norm_rope", qa[0], ka[0], dt, d, qa[1], ka[1], T, qa[2], qa[3], ka[2], ka[3],
            _ptr(q_weight), _ptr(k_weight), float(eps), _ptr(table), n_pos,
            None if rope is None else positions.data_ptr(), qa[4], qa[5], qa[6], ka[4], ka[5], ka[6], _stream(dev))
    return out


def attention_workspace_bytes(dtype: int, d: int, n_heads: int, group: int, cu_q, cu_k, window: int,
                              n_sink: int) -> int:
    cq, n_seqs = _offsets(cu_q, int(cu_q[-1]), "cu_q")
    ck, n_k = _offsets(cu_k, int(cu_k[-1]), "cu_k")
    if n_k != n_seqs:
        raise ValueError("cu_q and cu_k must list the same number of sequences")
    n = int(lib().twinkv_attention_workspace_bytes(dtype, d, n_heads, group, n_seqs, cq, ck, int(window), int(n_sink)))
    if n < 0:
        raise TwinKVError("twinkv_attention_workspace_bytes", -n)
    return n


def _group(n_q: int, n_heads: int) -> int:
    if n_heads == 0 or n_q % n_heads or n_q == 0:
        raise ValueError(f"{n_q} query heads do not divide over {n_heads} KV heads")
    return n_q // n_heads


def sink_attention(q, k, v, window: int, n_sink: int = 4, scale: Optional[float] = None, cu_q=None, cu_k=None,
                   *, want_lse: bool = False, out=None, workspace=None) -> dict:
    """Causal attention over a sliding window and the first ``n_sink`` tokens.  q (Hq, Tq, d) are the
    last tokens of each sequence, k and v (H, Tk, d) all of its tokens; query head h reads KV head
    h // (Hq // H).  A query at position p sees j <= p with p - j < window or j < n_sink.  scale defaults to
    1 / sqrt(d).  Returns out, and lse (Hq, Tq) float32 with ``want_lse``.  For bfloat16 the softmax weights are
    rounded to bfloat16 for the product with v, for float32 nothing is.  There is no gradient: inputs that
    require one are refused (torch.no_grad() lifts that)."""
    torch = _torch()
    _no_gradient("sink_attention", q, k, v, out)
    q, dt = _rows(q, "q")
    Hq, Tq, d = q.shape
    dev = q.device
    k, _ = _rows(k, "k", q.dtype, d, dev)
    v, _ = _rows(v, "v", q.dtype, d, dev)
    H, Tk, _ = k.shape
    if tuple(v.shape) != (H, Tk, d):
        raise ValueError("v must match k in shape")
    group = _group(Hq, H)
    cq, n_seqs = _offsets(cu_q, Tq, "cu_q")
    ck, n_k = _offsets(cu_k, Tk, "cu_k")
    if n_k != n_seqs:
        raise ValueError("cu_q and cu_k must list the same number of sequences")
    if window < 0 or n_sink < 0:
        raise ValueError("window and n_sink must not be negative")
    res = {"out": _out_rows(out, (Hq, Tq, d), q, "out")}
    if want_lse:
        res["lse"] = torch.empty((Hq, Tq), dtype=torch.float32, device=dev)
    o = res["out"]
    window, n_sink = min(int(window), 1 << 62), min(int(n_sink), 1 << 62)
    nb = lib().twinkv_attention_workspace_bytes(dt, d, H, group, n_seqs, cq, ck, window, n_sink)
    ws, wp, wn = _scratch(workspace, int(nb), dev, "twinkv_attention_workspace_bytes")
    _launch(dev, "twinkv_sink_attention", q.data_ptr(), k.data_ptr(), v.data_ptr(), dt, d, H, group, n_seqs, cq, ck,
            q.stride(0), q.stride(1), k.stride(0), k.stride(1), v.stride(0), v.stride(1), window, n_sink,
            float(d ** -0.5 if scale is None else scale), o.data_ptr(), o.stride(0), o.stride(1),
            _ptr(res.get("lse")), wp, wn, _stream(dev))
    return res


class _Cache4Struct(ctypes.Structure):
    _fields_ = [("d", _I), ("n_heads", _I), ("n_seqs", _I), ("cu_rows", _PI64), ("k_codes", _VP),
                ("k_scales", _VP), ("v_codes", _VP), ("v_scales", _VP)]


_Cache8Struct = _Cache4Struct  # twinkv_cache8 has the same fields


class Cache4:
    """A cache held in 4 bits (layout in include/twinkv.h): sequence s has the rows
    [cu_rows[s], cu_rows[s + 1]) of every head, a multiple of 32.  Takes the four arrays as they are;
    ``Cache4.empty`` reserves them.  How many rows a problem uses is a separate int32 tensor
    (n_heads, n_seqs), which cache4_compact and cache4_append return."""

    def __init__(self, k_codes, k_scales, v_codes, v_scales, cu_rows):
        u8 = _torch().uint8
        cu = np.array(cu_rows, dtype=np.int64)
        if cu.ndim != 1 or cu.size < 2 or cu[0] != 0 or (cu[1:] < cu[:-1]).any() or (cu & 31).any():
            raise ValueError("cu_rows must start at 0, never decrease, and be multiples of 32")
        if k_codes.dim() != 3:
            raise ValueError("k_codes must be (n_heads, C, d / 2)")
        H, C, d = k_codes.shape[0], int(cu[-1]), 2 * k_codes.shape[2]
        dev = k_codes.device
        for name, x, shape in (("k_codes", k_codes, (H, C, d // 2)), ("k_scales", k_scales, (H, C, d // 32)),
                               ("v_codes", v_codes, (H, C // 8, d, 4)), ("v_scales", v_scales, (H, C // 8, d // 32, 8))):
            if x.shape != shape or x.dtype != u8 or x.device != dev or not x.is_contiguous():
                raise ValueError(f"{name} must be a contiguous uint8 {shape} tensor on {dev}, got {tuple(x.shape)} {x.dtype}")
        if not k_codes.is_cuda:
            raise ValueError("the cache must be on a GPU")
        self.k_codes, self.k_scales, self.v_codes, self.v_scales = k_codes, k_scales, v_codes, v_scales
        self.cu_rows, self.n_heads, self.n_seqs, self.d, self.device = cu, H, cu.size - 1, d, dev
        self._cu = (ctypes.c_int64 * cu.size).from_buffer(cu)
        self._struct = _Cache4Struct(d, H, cu.size - 1, ctypes.cast(self._cu, _PI64), k_codes.data_ptr(),
                                     k_scales.data_ptr(), v_codes.data_ptr(), v_scales.data_ptr())
        self._handle = ctypes.addressof(self._struct)

    @classmethod
    def empty(cls, n_heads: int, capacity, d: int, device="cuda"):
        """Reserves ``capacity[s]`` rows for sequence s of every head, each rounded up to 32."""
        torch = _torch()
        cu = np.concatenate([[0], np.cumsum([(int(c) + 31) // 32 * 32 for c in np.atleast_1d(capacity)])])
        C = int(cu[-1])
        return cls(*(torch.empty(shape, dtype=torch.uint8, device=device) for shape in (
            (n_heads, C, d // 2), (n_heads, C, d // 32), (n_heads, C // 8, d, 4), (n_heads, C // 8, d // 32, 8))), cu)

    def _lens(self, x, name: str):
        return _small(x, (self.n_heads, self.n_seqs), _torch().int32, self.device, name)

    def _offsets(self, cu, T: int, name: str):
        arr, n = _offsets(cu, T, name)
        if n != self.n_seqs:
            raise ValueError(f"{name} must list the cache's {self.n_seqs} sequences")
        return arr


def _cache_rows(keys, values, cache):
    keys, dt = _rows(keys, "keys", None, cache.d, cache.device)
    values, _ = _rows(values, "values", keys.dtype, cache.d, cache.device)
    if keys.shape[0] != cache.n_heads or values.shape != keys.shape:
        raise ValueError(f"keys and values must be ({cache.n_heads}, T, {cache.d})")
    return keys, values, dt


def _cache4_scratch(workspace, cache: Cache4):
    return _scratch(workspace, int(lib().twinkv_cache4_workspace_bytes(cache.n_seqs)), cache.device,
                    "twinkv_cache4_workspace_bytes")


def cache4_compact(keys, values, retained, cache: Cache4, cu_seqlens=None, *, workspace=None) -> dict:
    """``compact`` into a 4-bit cache: the keys and values (n_heads, T, d) at the retained positions of
    every problem become the first rows of its part of ``cache``.  Returns len (n_heads, n_seqs) int32, pos
    (n_heads, C) int32 (-1 on rows not in use) and status (n_heads, n_seqs) int32; a problem that keeps more
    than its rows stores nothing (PROBLEM_BUDGET_MISMATCH, len 0)."""
    torch = _torch()
    keys, values, dt = _cache_rows(keys, values, cache)
    H, T, _ = keys.shape
    dev = cache.device
    cu = cache._offsets(cu_seqlens, T, "cu_seqlens")
    if retained is None:
        raise ValueError("retained is required")
    ret = _mask(retained, H, T, dev, "retained")
    out = {"len": torch.empty((H, cache.n_seqs), dtype=torch.int32, device=dev),
           "pos": torch.empty((H, int(cache.cu_rows[-1])), dtype=torch.int32, device=dev),
           "status": torch.empty((H, cache.n_seqs), dtype=torch.int32, device=dev)}
    ws, wp, wn = _cache4_scratch(workspace, cache)
    _launch(dev, "twinkv_cache4_compact", keys.data_ptr(), values.data_ptr(), dt, cu, keys.stride(0), keys.stride(1),
            values.stride(0), values.stride(1), ret.data_ptr(), cache._handle, out["pos"].data_ptr(),
            out["len"].data_ptr(), out["status"].data_ptr(), wp, wn, _stream(dev))
    return out


def cache4_append(keys, values, cache: Cache4, length, cu_new=None, *, len_out=None, workspace=None) -> dict:
    """The keys and values (n_heads, T, d) of new tokens, [cu_new[s], cu_new[s + 1]) of sequence s, as the
    rows after the ``length`` (n_heads, n_seqs) int32 ones in use.  Returns len (``len_out`` if given, which
    may be ``length`` itself) and status; a problem whose new tokens do not fit stays as it is."""
    torch = _torch()
    keys, values, dt = _cache_rows(keys, values, cache)
    dev = cache.device
    cu = cache._offsets(cu_new, keys.shape[1], "cu_new")
    n_in = cache._lens(length, "length")
    if len_out is None:
        len_out = torch.empty((cache.n_heads, cache.n_seqs), dtype=torch.int32, device=dev)
    elif cache._lens(len_out, "len_out").data_ptr() != len_out.data_ptr():
        raise ValueError("len_out must be contiguous and 16-byte aligned")
    status = torch.empty((cache.n_heads, cache.n_seqs), dtype=torch.int32, device=dev)
    ws, wp, wn = _cache4_scratch(workspace, cache)
    _launch(dev, "twinkv_cache4_append", keys.data_ptr(), values.data_ptr(), dt, cu, keys.stride(0), keys.stride(1),
            values.stride(0), values.stride(1), cache._handle, n_in.data_ptr(), len_out.data_ptr(),
            status.data_ptr(), wp, wn, _stream(dev))
    return {"len": len_out, "status": status}


def cache4_read(cache: Cache4, length, dtype, first=None, cu_out=None, *, want_keys: bool = True,
                want_values: bool = True, workspace=None) -> dict:
    """The values that cached rows stand for, in ``dtype``: keys and values (n_heads, cu_out[-1], d), row
    r of sequence s being cache row first + r (``first`` (n_heads, n_seqs) int32, default 0; ``cu_out``
    defaults to all of the cache's rows).  Rows that are not in use are zeros."""
    torch = _torch()
    if dtype not in (torch.bfloat16, torch.float32):
        raise ValueError(f"unsupported dtype {dtype}")
    dev = cache.device
    cu_out = cache.cu_rows if cu_out is None else cu_out
    cu = cache._offsets(cu_out, int(cu_out[-1]), "cu_out")
    n = cache._lens(length, "length")
    f = cache._lens(first, "first")
    shape = (cache.n_heads, int(cu[-1]), cache.d)
    out = {name: torch.empty(shape, dtype=dtype, device=dev)
           for name, want in (("keys", want_keys), ("values", want_values)) if want}
    ws, wp, wn = _cache4_scratch(workspace, cache)
    _launch(dev, "twinkv_cache4_read", cache._handle, n.data_ptr(), _ptr(f),
            TWINKV_BF16 if dtype == torch.bfloat16 else TWINKV_F32, cu, _ptr(out.get("keys")), _ptr(out.get("values")),
            wp, wn, _stream(dev))
    return out


def cache4_attention(q, cache: Cache4, length, scale: Optional[float] = None, cu_q=None, *,
                     want_lse: bool = False, out=None, workspace=None) -> dict:
    """Attention of q (Hq, Tq, d), the last tokens [cu_q[s], cu_q[s + 1]) of each cached sequence, over the
    ``length`` (n_heads, n_seqs) int32 rows in use: query i of m sees the first length - (m - 1 - i) of
    them.  scale defaults to 1 / sqrt(d).  Returns out, and lse (Hq, Tq) float32 with ``want_lse``.  For bfloat16
    the softmax weights, times the values' scales, are rounded to bfloat16; for float32 they keep 24 bits.  There
    is no gradient: a q that requires one is refused (torch.no_grad() lifts that)."""
    torch = _torch()
    _no_gradient("cache4_attention", q, out)
    dev = cache.device
    q, dt = _rows(q, "q", None, cache.d, dev)
    Hq, Tq, d = q.shape
    group = _group(Hq, cache.n_heads)
    cq = cache._offsets(cu_q, Tq, "cu_q")
    n = cache._lens(length, "length")
    res = {"out": _out_rows(out, (Hq, Tq, d), q, "out")}
    if want_lse:
        res["lse"] = torch.empty((Hq, Tq), dtype=torch.float32, device=dev)
    o = res["out"]
    nb = lib().twinkv_attention_workspace_bytes(dt, d, cache.n_heads, group, cache.n_seqs, cq, cache._cu, 1 << 62, 0)
    ws, wp, wn = _scratch(workspace, int(nb), dev, "twinkv_attention_workspace_bytes")
    _launch(dev, "twinkv_cache4_attention", q.data_ptr(), dt, group, cq, q.stride(0), q.stride(1), cache._handle,
            n.data_ptr(), float(d ** -0.5 if scale is None else scale), o.data_ptr(), o.stride(0), o.stride(1),
            _ptr(res.get("lse")), wp, wn, _stream(dev))
    return res


# ---------------------------------------------------------------- accumulated weights, and the 8-bit cache

def attention_mass(q, k, lse, window: int, n_sink: int = 4, scale: Optional[float] = None, cu_q=None, cu_k=None, *,
                   mass=None, out=None, workspace=None) -> dict:
    """The attention weight that every key has received: for each KV head the sum over its query heads and over the
    queries that see the key of exp(scale q . k - lse), the softmax weights of ``sink_attention`` with the same
    arguments and its ``lse`` (Hq, Tq) float32.  q (Hq, Tq, d) may be a prompt's last tokens only (cu_q), then lse
    is theirs.  Returns mass (H, Tk) float32, the scores that ``select_topk`` takes; ``mass`` (H, Tk) is added to it
    (``out`` may be that tensor).  There is no gradient: inputs that require one are refused (torch.no_grad() lifts
    that)."""
    torch = _torch()
    _no_gradient("attention_mass", q, k, lse, mass, out)
    q, dt = _rows(q, "q")
    Hq, Tq, d = q.shape
    dev = q.device
    k, _ = _rows(k, "k", q.dtype, d, dev)
    H, Tk, _ = k.shape
    group = _group(Hq, H)
    cq, n_seqs = _offsets(cu_q, Tq, "cu_q")
    ck, n_k = _offsets(cu_k, Tk, "cu_k")
    if n_k != n_seqs:
        raise ValueError("cu_q and cu_k must list the same number of sequences")
    if window < 0 or n_sink < 0:
        raise ValueError("window and n_sink must not be negative")
    if lse is None:
        raise ValueError("lse is required")
    f32 = torch.float32
    lse = _small(lse, (Hq, Tq), f32, dev, "lse")
    mass = _small(mass, (H, Tk), f32, dev, "mass")
    out = _own_place(out, (H, Tk), f32, dev, "out")
    window, n_sink = min(int(window), 1 << 62), min(int(n_sink), 1 << 62)
    nb = lib().twinkv_mass_workspace_bytes(dt, d, H, group, n_seqs, cq, ck, window, n_sink)
    ws, wp, wn = _scratch(workspace, int(nb), dev, "twinkv_mass_workspace_bytes")
    _launch(dev, "twinkv_attention_mass", q.data_ptr(), k.data_ptr(), dt, d, H, group, n_seqs, cq, ck, q.stride(0),
            q.stride(1), k.stride(0), k.stride(1), window, n_sink, float(d ** -0.5 if scale is None else scale),
            lse.data_ptr(), _ptr(mass), out.data_ptr(), wp, wn, _stream(dev))
    return {"mass": out}


def _own_place(out, shape, dtype, dev, name: str):
    """The caller's output of an exact shape and type (written in place), or a new one."""
    if out is None:
        return _torch().empty(shape, dtype=dtype, device=dev)
    if _small(out, shape, dtype, dev, name).data_ptr() != out.data_ptr():
        raise ValueError(f"{name} must be contiguous and 16-byte aligned")
    return out


def _rising_by_32(cu) -> bool:
    """Whether offsets never decrease and are multiples of 32 (few of them: without numpy's cost a call)."""
    if cu.size > 16:
        return not ((cu[1:] < cu[:-1]).any() or (cu & 31).any())
    at = cu.tolist()
    return all(x <= y for x, y in zip(at, at[1:])) and not any(x & 31 for x in at)


class Cache8:
    """A cache held in 8 bits, a scale for 32 rows of a head (layout in include/twinkv.h): sequence s has the rows
    [cu_rows[s], cu_rows[s + 1]) of every head, a multiple of 32.  Takes the four arrays as they are;
    ``Cache8.empty`` reserves them.  How many rows a problem uses is a separate int32 tensor (n_heads, n_seqs),
    which cache8_compact, cache8_append and cache8_evict return."""

    def __init__(self, k_codes, k_scales, v_codes, v_scales, cu_rows):
        torch = _torch()
        cu = np.array(cu_rows, dtype=np.int64)
        if cu.ndim != 1 or cu.size < 2 or cu[0] != 0 or not _rising_by_32(cu):
            raise ValueError("cu_rows must start at 0, never decrease, and be multiples of 32")
        if k_codes.dim() != 3:
            raise ValueError("k_codes must be (n_heads, C, d)")
        H, C, d = k_codes.shape[0], int(cu[-1]), k_codes.shape[2]
        dev = k_codes.device
        i8, u8 = torch.int8, torch.uint8
        for name, x, shape, dt in (("k_codes", k_codes, (H, C, d), i8), ("k_scales", k_scales, (H, C // 32), u8),
                                   ("v_codes", v_codes, (H, C // 8, d, 8), i8), ("v_scales", v_scales, (H, C // 32), u8)):
            if x.shape != shape or x.dtype != dt or x.device != dev or not x.is_contiguous():
                raise ValueError(f"{name} must be a contiguous {dt} {shape} tensor on {dev}, got {tuple(x.shape)} {x.dtype}")
        if not k_codes.is_cuda:
            raise ValueError("the cache must be on a GPU")
        self.k_codes, self.k_scales, self.v_codes, self.v_scales = k_codes, k_scales, v_codes, v_scales
        self.cu_rows, self.n_heads, self.n_seqs, self.d, self.device = cu, H, cu.size - 1, d, dev
        self._cu = (ctypes.c_int64 * cu.size).from_buffer(cu)
        self._scales = H * (C // 32)
        self._at = (k_codes.data_ptr(), k_scales.data_ptr(), v_codes.data_ptr(), v_scales.data_ptr())
        self._struct = _Cache8Struct(d, H, cu.size - 1, ctypes.cast(self._cu, _PI64), *self._at)
        self._handle = ctypes.addressof(self._struct)

    @classmethod
    def empty(cls, n_heads: int, capacity, d: int, device="cuda"):
        """Reserves ``capacity[s]`` rows for sequence s of every head, each rounded up to 32."""
        torch = _torch()
        cu = np.concatenate([[0], np.cumsum([(int(c) + 31) // 32 * 32 for c in np.atleast_1d(capacity)])])
        C = int(cu[-1])
        return cls(*(torch.empty(shape, dtype=dt, device=device) for shape, dt in (
            ((n_heads, C, d), torch.int8), ((n_heads, C // 32), torch.uint8),
            ((n_heads, C // 8, d, 8), torch.int8), ((n_heads, C // 32), torch.uint8))), cu)

    _lens = Cache4._lens
    _offsets = Cache4._offsets

    def _spans(self) -> list:
        """The bytes of the four arrays, (first, past the last) each."""
        k, ks, v, vs = self._at
        scales = self._scales
        codes = 32 * scales * self.d
        return [(k, k + codes), (ks, ks + scales), (v, v + codes), (vs, vs + scales)] if scales > 0 else []

    def _weights(self, x, name: str):
        return _small(x, (self.n_heads, int(self.cu_rows[-1])), _torch().float32, self.device, name)


def _cache8_scratch(workspace, cache: Cache8):
    return _scratch(workspace, int(lib().twinkv_cache8_workspace_bytes(cache.n_seqs)), cache.device,
                    "twinkv_cache8_workspace_bytes")


def cache8_compact(keys, values, retained, cache: Cache8, cu_seqlens=None, *, token_mass=None, workspace=None) -> dict:
    """``compact`` into an 8-bit cache: the keys and values (n_heads, T, d) at the retained positions of every problem
    become the first rows of its part of ``cache``.  Returns len (n_heads, n_seqs) int32, pos (n_heads, C) int32 (-1
    on rows not in use) and status (n_heads, n_seqs) int32; a problem that keeps more than its rows stores nothing
    (PROBLEM_BUDGET_MISMATCH, len 0).  With ``token_mass`` (n_heads, T) float32 also mass (n_heads, C), the cached
    rows' weights.  There is no gradient: inputs that require one are refused (torch.no_grad() lifts that)."""
    torch = _torch()
    _no_gradient("cache8_compact", keys, values, token_mass)
    keys, values, dt = _cache_rows(keys, values, cache)
    H, T, _ = keys.shape
    dev, C = cache.device, int(cache.cu_rows[-1])
    cu = cache._offsets(cu_seqlens, T, "cu_seqlens")
    if retained is None:
        raise ValueError("retained is required")
    ret = _mask(retained, H, T, dev, "retained")
    token_mass = _small(token_mass, (H, T), torch.float32, dev, "token_mass")
    out = {"len": torch.empty((H, cache.n_seqs), dtype=torch.int32, device=dev),
           "pos": torch.empty((H, C), dtype=torch.int32, device=dev),
           "status": torch.empty((H, cache.n_seqs), dtype=torch.int32, device=dev)}
    if token_mass is not None:
        out["mass"] = torch.empty((H, C), dtype=torch.float32, device=dev)
    ws, wp, wn = _cache8_scratch(workspace, cache)
    _launch(dev, "twinkv_cache8_compact", keys.data_ptr(), values.data_ptr(), dt, cu, keys.stride(0), keys.stride(1),
            values.stride(0), values.stride(1), ret.data_ptr(), cache._handle, _ptr(token_mass), out["pos"].data_ptr(),
            _ptr(out.get("mass")), out["len"].data_ptr(), out["status"].data_ptr(), wp, wn, _stream(dev))
    return out


def cache8_append(keys, values, cache: Cache8, length, cu_new=None, *, len_out=None, workspace=None) -> dict:
    """The keys and values (n_heads, T, d) of new tokens, [cu_new[s], cu_new[s + 1]) of sequence s, as the rows after
    the ``length`` (n_heads, n_seqs) int32 ones in use.  Returns len (``len_out`` if given, which may be ``length``
    itself) and status; a problem whose new tokens do not fit stays as it is.  Where a row needs a larger scale
    than its block of 32 has, the block's rows are rounded once more.  There is no gradient: inputs that require one
    are refused (torch.no_grad() lifts that)."""
    torch = _torch()
    _no_gradient("cache8_append", keys, values)
    keys, values, dt = _cache_rows(keys, values, cache)
    dev = cache.device
    cu = cache._offsets(cu_new, keys.shape[1], "cu_new")
    n_in = cache._lens(length, "length")
    len_out = torch.empty_like(n_in) if len_out is None else _own_place(len_out, n_in.shape, torch.int32, dev, "len_out")
    status = torch.empty_like(n_in)
    ws, wp, wn = _cache8_scratch(workspace, cache)
    _launch(dev, "twinkv_cache8_append", keys.data_ptr(), values.data_ptr(), dt, cu, keys.stride(0), keys.stride(1),
            values.stride(0), values.stride(1), cache._handle, n_in.data_ptr(), len_out.data_ptr(),
            status.data_ptr(), wp, wn, _stream(dev))
    return {"len": len_out, "status": status}


def cache8_read(cache: Cache8, length, dtype, first=None, cu_out=None, *, want_keys: bool = True,
                want_values: bool = True, workspace=None) -> dict:
    """The values that cached rows stand for, in ``dtype``: keys and values (n_heads, cu_out[-1], d), row r of
    sequence s being cache row first + r (``first`` (n_heads, n_seqs) int32, default 0; ``cu_out`` defaults to all
    of the cache's rows).  Rows that are not in use are zeros."""
    torch = _torch()
    if dtype not in (torch.bfloat16, torch.float32):
        raise ValueError(f"unsupported dtype {dtype}")
    dev = cache.device
    cu_out = cache.cu_rows if cu_out is None else cu_out
    cu = cache._offsets(cu_out, int(cu_out[-1]), "cu_out")
    n = cache._lens(length, "length")
    f = cache._lens(first, "first")
    shape = (cache.n_heads, int(cu[-1]), cache.d)
    out = {name: torch.empty(shape, dtype=dtype, device=dev)
           for name, want in (("keys", want_keys), ("values", want_values)) if want}
    ws, wp, wn = _cache8_scratch(workspace, cache)
    _launch(dev, "twinkv_cache8_read", cache._handle, n.data_ptr(), _ptr(f),
            TWINKV_BF16 if dtype == torch.bfloat16 else TWINKV_F32, cu, _ptr(out.get("keys")), _ptr(out.get("values")),
            wp, wn, _stream(dev))
    return out


def cache8_attention(q, cache: Cache8, length, scale: Optional[float] = None, cu_q=None, *, want_lse: bool = False,
                     want_mass: bool = False, mass=None, mass_out=None, out=None, workspace=None) -> dict:
    """Attention of q (Hq, Tq, d), the last tokens [cu_q[s], cu_q[s + 1]) of each cached sequence, over the
    ``length`` (n_heads, n_seqs) int32 rows in use, as ``cache4_attention`` computes it.  Returns out, with
    ``want_lse`` lse (Hq, Tq) float32, and with ``want_mass``, ``mass`` or ``mass_out`` mass (n_heads, C) float32:
    the rows' weights so far (``mass``; None: 0) and those of this call's queries, 0 on rows not in use.
    ``mass_out`` may be ``mass``; where weights are wanted ``out`` may not be q, which they are computed from.  There is
    no gradient: a q that requires one is refused (torch.no_grad() lifts that)."""
    torch = _torch()
    _no_gradient("cache8_attention", q, mass, mass_out, out)
    dev = cache.device
    q, dt = _rows(q, "q", None, cache.d, dev)
    Hq, Tq, d = q.shape
    group = _group(Hq, cache.n_heads)
    cq = cache._offsets(cu_q, Tq, "cu_q")
    n = cache._lens(length, "length")
    want_mass = want_mass or mass is not None or mass_out is not None
    mass = cache._weights(mass, "mass")
    if want_mass and out is not None and out.data_ptr() == q.data_ptr() and q.numel() > 0:
        raise ValueError("out may not be q where weights are wanted")
    res = {"out": _out_rows(out, (Hq, Tq, d), q, "out")}
    if want_lse:
        res["lse"] = torch.empty((Hq, Tq), dtype=torch.float32, device=dev)
    if want_mass:
        res["mass"] = _own_place(mass_out, (cache.n_heads, int(cache.cu_rows[-1])), torch.float32, dev, "mass_out")
    o = res["out"]
    nb = lib().twinkv_cache8_attention_workspace_bytes(dt, d, cache.n_heads, group, cache.n_seqs, cq, cache._cu,
                                                       1 if want_mass else 0)
    ws, wp, wn = _scratch(workspace, int(nb), dev, "twinkv_cache8_attention_workspace_bytes")
    _launch(dev, "twinkv_cache8_attention", q.data_ptr(), dt, group, cq, q.stride(0), q.stride(1), cache._handle,
            n.data_ptr(), float(d ** -0.5 if scale is None else scale), o.data_ptr(), o.stride(0), o.stride(1),
            _ptr(res.get("lse")), _ptr(mass), _ptr(res.get("mass")), wp, wn, _stream(dev))
    return res


def _ends(n_sink: int, n_recent: int):
    """Numbers of first and last rows as the library takes them, in 32 bits: no problem has more rows."""
    if n_sink < 0 or n_recent < 0:
        raise ValueError("n_sink and n_recent must not be negative")
    return min(int(n_sink), (1 << 31) - 1), min(int(n_recent), (1 << 31) - 1)


def _apart(spans) -> bool:
    """Whether no two of the spans have a byte in common."""
    end = 0
    for x in sorted(spans):
        if x[0] < end:
            return False
        end = x[1]
    return True


def cache8_evict(cache: Cache8, length, mass, budget, to: Cache8, n_sink: int = 4, n_recent: int = 64, *, pos=None,
                 len_out=None, workspace=None) -> dict:
    """Keeps of every problem's ``length`` (n_heads, n_seqs) int32 rows the ``budget`` (an int, or one per sequence)
    that ``select_topk`` would: the first ``n_sink`` and last ``n_recent``, then those of most ``mass`` (n_heads, C)
    float32.  They move, in row order, to the front of another cache ``to``, which shares no memory with this one.
    Returns len, mass and pos of ``to``: pos is what ``pos`` (n_heads, C) int32 held for the rows, or their rows in
    ``cache``; -1, and mass 0, on rows not in use.  ``len_out`` may be ``length``.  There is no gradient: a mass that
    requires one is refused (torch.no_grad() lifts that)."""
    torch = _torch()
    _no_gradient("cache8_evict", mass)
    n_sink, n_recent = _ends(n_sink, n_recent)
    dev = cache.device
    if (to.n_heads, to.n_seqs, to.d, to.device) != (cache.n_heads, cache.n_seqs, cache.d, dev):
        raise ValueError("the caches must have the same heads, sequences, channels and device")
    if not _apart(cache._spans() + to._spans()):
        raise ValueError("the caches must not overlap")
    n = cache._lens(length, "length")
    if mass is None:
        raise ValueError("mass is required")
    mass = cache._weights(mass, "mass")
    pos = _small(pos, (cache.n_heads, int(cache.cu_rows[-1])), torch.int32, dev, "pos")
    keep = _i64_array(_budget(budget, cache.n_seqs))
    C = int(to.cu_rows[-1])
    out = {"len": _own_place(len_out, (cache.n_heads, cache.n_seqs), torch.int32, dev, "len_out"),
           "mass": torch.empty((cache.n_heads, C), dtype=torch.float32, device=dev),
           "pos": torch.empty((cache.n_heads, C), dtype=torch.int32, device=dev)}
    ws, wp, wn = _cache8_scratch(workspace, cache)
    _launch(dev, "twinkv_cache8_evict", cache._handle, n.data_ptr(), mass.data_ptr(), _ptr(pos), keep, n_sink, n_recent,
            to._handle, out["len"].data_ptr(), out["mass"].data_ptr(), out["pos"].data_ptr(), wp, wn, _stream(dev))
    return out
