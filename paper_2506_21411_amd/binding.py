"""ctypes binding of include/dchag.h.  Argument marshalling only.

Tensors are torch tensors on the current ROCm device (torch is used for device memory and
streams, nothing else); they must be contiguous and of dtype float32 (DCHAG_F32) or
bfloat16 (DCHAG_BF16).  Each function has the name and the meaning of the C entry point.
"""
from __future__ import annotations

import ctypes
import functools
import inspect
import os
from dataclasses import dataclass
from typing import List, Optional, Sequence

import torch

DCHAG_F32 = 0
DCHAG_BF16 = 1

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libdchag.so")
_lib = None


class DchagError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"dchag status {status}: {message}")
        self.status = status


class _CLevel(ctypes.Structure):
    _fields_ = [("group_size", ctypes.c_int32), ("kind", ctypes.c_int32),
                ("query", ctypes.c_void_p),
                ("Wq", ctypes.c_void_p), ("Wk", ctypes.c_void_p), ("Wv", ctypes.c_void_p), ("Wo", ctypes.c_void_p),
                ("bq", ctypes.c_void_p), ("bk", ctypes.c_void_p), ("bv", ctypes.c_void_p), ("bo", ctypes.c_void_p)]


class _CLevelGrads(ctypes.Structure):
    _fields_ = [("dquery", ctypes.c_void_p),
                ("dWq", ctypes.c_void_p), ("dWk", ctypes.c_void_p), ("dWv", ctypes.c_void_p), ("dWo", ctypes.c_void_p),
                ("dbq", ctypes.c_void_p), ("dbk", ctypes.c_void_p), ("dbv", ctypes.c_void_p), ("dbo", ctypes.c_void_p)]


class _CAttention(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("heads", "kv_heads", "head_dim", "causal", "sequences", "rows_q", "rows_k")]
                + [("scale", ctypes.c_float)]
                + [(n, ctypes.c_int64) for n in ("ld_q", "ld_k", "ld_v", "ld_out", "ld_dout", "ld_dq", "ld_dk", "ld_dv")]
                + [(n, ctypes.c_void_p) for n in ("q_starts", "k_starts", "k_used", "bias", "borders")]
                + [("n_borders", ctypes.c_int32)])


class _CStageTime(ctypes.Structure):
    _fields_ = [("stage", ctypes.c_int32), ("level", ctypes.c_int32), ("ms", ctypes.c_float)]


STAGE_NAMES = {0: "tokenize", 1: "query", 2: "fold", 3: "scores", 4: "vproj", 5: "softmax_agg", 6: "oproj",
               7: "fused_vagg", 8: "channel_mix", 9: "tokenize_mix", 10: "head_sums", 11: "head_vproj",
               12: "bwd_oproj", 13: "bwd_value", 14: "bwd_softmax", 15: "bwd_tokens", 16: "bwd_key_query",
               17: "bwd_tokenize", 18: "bwd_channel_mix", 19: "fold_value", 20: "tokenize_attend", 21: "key_prep",
               22: "attend", 23: "attend_join", 24: "bwd_attend_query", 25: "bwd_attend_key", 26: "bwd_attend_bias", 27: "pack8",
               28: "unpack8", 29: "weight_grad8", 30: "attend_plan"}

LEVEL_ATTENTION, LEVEL_LINEAR = 0, 1


@dataclass
class LevelWeights:
    """Device tensors of one aggregation level.

    Attention level (kind 0): query [G,D]; Wq..Wo [G,D,D]; biases [G,D] or None.
    Linear level (kind 1, D-CHAG-L): Wv = mixing weights [G,g,D], bv = bias [G,D] or None; the rest None.
    """
    group_size: int
    query: Optional[torch.Tensor]
    Wq: Optional[torch.Tensor]
    Wk: Optional[torch.Tensor]
    Wv: torch.Tensor
    Wo: Optional[torch.Tensor]
    bq: Optional[torch.Tensor] = None
    bk: Optional[torch.Tensor] = None
    bv: Optional[torch.Tensor] = None
    bo: Optional[torch.Tensor] = None
    kind: int = LEVEL_ATTENTION


@dataclass
class LevelGrads:
    """Gradient tensors of one level, shaped like its weights; None = not wanted."""
    dquery: Optional[torch.Tensor] = None
    dWq: Optional[torch.Tensor] = None
    dWk: Optional[torch.Tensor] = None
    dWv: Optional[torch.Tensor] = None
    dWo: Optional[torch.Tensor] = None
    dbq: Optional[torch.Tensor] = None
    dbk: Optional[torch.Tensor] = None
    dbv: Optional[torch.Tensor] = None
    dbo: Optional[torch.Tensor] = None


def library_path() -> str:
    return _LIB_PATH


def use_library(path: str) -> None:
    """Point the binding at another build of the library (the benchmark's timing-probe builds); before the first call."""
    global _LIB_PATH
    if _lib is not None:
        raise RuntimeError("the library is already loaded")
    _LIB_PATH = os.path.abspath(path)


def load_library():
    """Loads libdchag.so (built by `python -m paper_2506_21411_amd.build`); raises if it is not there."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise FileNotFoundError(
            f"{_LIB_PATH} is missing: build it with `python -m paper_2506_21411_amd.build` "
            "(there is no fallback path)")
    lib = ctypes.CDLL(_LIB_PATH)
    i, vp, sz = ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t
    lib.dchag_tokenize.restype = i
    lib.dchag_tokenize.argtypes = [i] * 7 + [vp] * 6
    lib.dchag_aggregate_level.restype = i
    lib.dchag_aggregate_level.argtypes = [i] * 6 + [ctypes.POINTER(_CLevel), vp, vp, vp, sz, vp]
    lib.dchag_yardstick_mfma.restype = i
    lib.dchag_yardstick_mfma.argtypes = [i, vp, sz, ctypes.POINTER(ctypes.c_double), vp]
    lib.dchag_yardstick_copy.restype = i
    lib.dchag_yardstick_copy.argtypes = [vp, vp, sz, vp]
    lib.dchag_yardstick_read.restype = i
    lib.dchag_yardstick_read.argtypes = [vp, sz, vp, vp]
    lib.dchag_debug_reload.restype = None
    lib.dchag_debug_reload.argtypes = []
    lib.dchag_aggregate_level_static.restype = i
    lib.dchag_aggregate_level_static.argtypes = [i] * 6 + [ctypes.POINTER(_CLevel), vp, vp, vp]
    lib.dchag_forward.restype = i
    lib.dchag_forward.argtypes = [i] * 8 + [vp] * 4 + [i, ctypes.POINTER(_CLevel), vp, vp, sz, vp]
    lib.dchag_forward_pos.restype = i
    lib.dchag_forward_pos.argtypes = [i] * 8 + [vp] * 4 + [i, ctypes.POINTER(_CLevel), vp, vp, vp, sz, vp]
    lib.dchag_forward_folded.restype = i
    lib.dchag_forward_folded.argtypes = lib.dchag_forward.argtypes
    lib.dchag_value_fold_bytes.restype = sz
    lib.dchag_value_fold_bytes.argtypes = [i] * 6 + [ctypes.POINTER(_CLevel)]
    lib.dchag_fold_value.restype = i
    lib.dchag_fold_value.argtypes = [i] * 5 + [vp] * 3 + [i, ctypes.POINTER(_CLevel), vp, sz, vp]
    lib.dchag_forward_prefolded.restype = i
    lib.dchag_forward_prefolded.argtypes = [i] * 8 + [vp] * 4 + [i, ctypes.POINTER(_CLevel), vp, vp, vp, sz, vp]
    lib.dchag_backward.restype = i
    lib.dchag_backward.argtypes = ([i] * 8 + [vp] * 4 + [i, ctypes.POINTER(_CLevel), vp, vp, vp, vp,
                                                        ctypes.POINTER(_CLevelGrads), vp, sz, vp])
    lib.dchag_forward_keep.restype = i
    lib.dchag_forward_keep.argtypes = lib.dchag_forward.argtypes
    lib.dchag_backward_kept.restype = i
    lib.dchag_backward_kept.argtypes = lib.dchag_backward.argtypes
    lib.dchag_workspace_bytes.restype = sz
    lib.dchag_workspace_bytes.argtypes = [i] * 9 + [ctypes.POINTER(ctypes.c_int32), i]
    att, i64 = ctypes.POINTER(_CAttention), ctypes.c_int64
    lib.dchag_attend.restype = i
    lib.dchag_attend.argtypes = [i, att] + [vp] * 6 + [sz, vp]
    lib.dchag_attend_backward.restype = i
    lib.dchag_attend_backward.argtypes = [i, att] + [vp] * 11 + [sz, vp]
    lib.dchag_attend_workspace_bytes.restype = sz
    lib.dchag_attend_workspace_bytes.argtypes = [i, att, i]
    lib.dchag_pack8.restype = i
    lib.dchag_pack8.argtypes = [i, i64, i, i64] + [vp] * 4
    lib.dchag_unpack8.restype = i
    lib.dchag_unpack8.argtypes = [i, i64, i, i64] + [vp] * 4
    lib.dchag_weight_grad8.restype = i
    lib.dchag_weight_grad8.argtypes = [i, i, i, i, i64] + [vp] * 6 + [sz, vp]
    lib.dchag_weight_grad8_workspace_bytes.restype = sz
    lib.dchag_weight_grad8_workspace_bytes.argtypes = [i, i, i, i]
    lib.dchag_strerror.restype = ctypes.c_char_p
    lib.dchag_strerror.argtypes = [i]
    lib.dchag_version.restype = ctypes.c_char_p
    lib.dchag_profile_begin.restype = i
    lib.dchag_profile_end.restype = i
    lib.dchag_profile_end.argtypes = [ctypes.POINTER(_CStageTime), i]
    _lib = lib
    return lib


def _check(status: int) -> None:
    if status != 0:
        raise DchagError(status, load_library().dchag_strerror(status).decode())


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return DCHAG_F32
    if t.dtype == torch.bfloat16:
        return DCHAG_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _ptr(t: Optional[torch.Tensor], like: Optional[torch.Tensor] = None):
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("tensors must be contiguous device tensors")
    if like is not None and t.dtype != like.dtype:
        raise TypeError("all tensors of a call must share one dtype")
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream) -> ctypes.c_void_p:
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _clevel(lv: LevelWeights, like: torch.Tensor) -> _CLevel:
    c = _CLevel()
    c.group_size = int(lv.group_size)
    c.kind = int(lv.kind)
    for name in ("query", "Wq", "Wk", "Wv", "Wo", "bq", "bk", "bv", "bo"):
        setattr(c, name, _ptr(getattr(lv, name), like))
    return c


def _workspace(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def dchag_workspace_bytes(dt: int, B: int, C: int, H: int, W: int, p: int, D: int, heads: int,
                          group_sizes: Sequence[int], which: int) -> int:
    arr = (ctypes.c_int32 * len(group_sizes))(*[int(g) for g in group_sizes])
    return int(load_library().dchag_workspace_bytes(dt, B, C, H, W, p, D, heads, len(group_sizes), arr, which))


def dchag_tokenize(x: torch.Tensor, We: torch.Tensor, be: Optional[torch.Tensor], ce: Optional[torch.Tensor],
                   p: int, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """tokens[B,C,N,D] of x[B,C,H,W] with We[C,D,p*p], be/ce [C,D] or None."""
    B, C, H, W = x.shape
    D = We.shape[1]
    if tuple(We.shape) != (C, D, p * p):
        raise ValueError("We must be [C, D, p*p]")
    N = (H // p) * (W // p) if p > 0 else 0
    if out is None:
        out = torch.empty((B, C, N, D), dtype=x.dtype, device=x.device)
    _check(load_library().dchag_tokenize(_dt(x), B, C, H, W, p, D, _ptr(x), _ptr(We, x), _ptr(be, x), _ptr(ce, x),
                                         _ptr(out, x), _stream(stream)))
    return out


def dchag_aggregate_level(tokens_in: torch.Tensor, level: LevelWeights, heads: int,
                          out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                          stream=None) -> torch.Tensor:
    """tokens_out[B,G,N,D] of tokens_in[B,Cin,N,D] for one level."""
    B, Cin, N, D = tokens_in.shape
    g = int(level.group_size)
    G = (Cin + g - 1) // g if g > 0 else 0
    dt = _dt(tokens_in)
    if workspace is None:
        workspace = _workspace(dchag_workspace_bytes(dt, B, Cin, N, 1, 1, D, heads, [g], 0), tokens_in.device)
    if out is None:
        out = torch.empty((B, G, N, D), dtype=tokens_in.dtype, device=tokens_in.device)
    cl = _clevel(level, tokens_in)
    _check(load_library().dchag_aggregate_level(dt, B, Cin, N, D, heads, ctypes.byref(cl), _ptr(tokens_in),
                                                _ptr(out, tokens_in), ctypes.c_void_p(workspace.data_ptr()),
                                                workspace.numel(), _stream(stream)))
    return out


STATIC_SCRATCH_BYTES = 32 << 20


def dchag_aggregate_level_static(tokens_in: torch.Tensor, level: LevelWeights, heads: int, out: torch.Tensor,
                                 stream=None) -> torch.Tensor:
    """dchag_aggregate_level on the library's fixed scratch array: no workspace argument, nothing allocated (the
    caller passes `out`)."""
    B, Cin, N, D = tokens_in.shape
    cl = _clevel(level, tokens_in)
    _check(load_library().dchag_aggregate_level_static(_dt(tokens_in), B, Cin, N, D, heads, ctypes.byref(cl),
                                                       _ptr(tokens_in), _ptr(out, tokens_in), _stream(stream)))
    return out


def dchag_debug_reload() -> None:
    """Re-read the DCHAG_* debugging switches from the environment (the library reads them once, at load)."""
    load_library().dchag_debug_reload()


def dchag_forward(x: torch.Tensor, We: torch.Tensor, be: Optional[torch.Tensor], ce: Optional[torch.Tensor],
                  levels: List[LevelWeights], p: int, heads: int, out: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """out[B,N,D]: tokenize, then every level in turn (the last must leave one group)."""
    B, C, H, W = x.shape
    D = We.shape[1]
    if tuple(We.shape) != (C, D, p * p):
        raise ValueError("We must be [C, D, p*p]")
    N = (H // p) * (W // p) if p > 0 else 0
    dt = _dt(x)
    if workspace is None:
        workspace = _workspace(dchag_workspace_bytes(dt, B, C, H, W, p, D, heads, [lv.group_size for lv in levels], 1),
                               x.device)
    if out is None:
        out = torch.empty((B, N, D), dtype=x.dtype, device=x.device)
    arr = (_CLevel * len(levels))(*[_clevel(lv, x) for lv in levels])
    _check(load_library().dchag_forward(dt, B, C, H, W, p, D, heads, _ptr(x), _ptr(We, x), _ptr(be, x), _ptr(ce, x),
                                        len(levels), arr, _ptr(out, x), ctypes.c_void_p(workspace.data_ptr()),
                                        workspace.numel(), _stream(stream)))
    return out


def dchag_forward_pos(x: torch.Tensor, We: torch.Tensor, be: Optional[torch.Tensor], ce: Optional[torch.Tensor],
                      levels: List[LevelWeights], p: int, heads: int, pos: torch.Tensor,
                      out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                      stream=None) -> torch.Tensor:
    """out[B,N,D] = dchag_forward(...) + pos[N,D], the sum taken in the last projection's epilogue."""
    B, C, H, W = x.shape
    D = We.shape[1]
    if tuple(We.shape) != (C, D, p * p):
        raise ValueError("We must be [C, D, p*p]")
    N = (H // p) * (W // p) if p > 0 else 0
    if tuple(pos.shape) != (N, D):
        raise ValueError("pos must be [N, D]")
    dt = _dt(x)
    if workspace is None:
        workspace = _workspace(dchag_workspace_bytes(dt, B, C, H, W, p, D, heads, [lv.group_size for lv in levels], 1),
                               x.device)
    if out is None:
        out = torch.empty((B, N, D), dtype=x.dtype, device=x.device)
    arr = (_CLevel * len(levels))(*[_clevel(lv, x) for lv in levels])
    _check(load_library().dchag_forward_pos(dt, B, C, H, W, p, D, heads, _ptr(x), _ptr(We, x), _ptr(be, x),
                                            _ptr(ce, x), len(levels), arr, _ptr(pos, x), _ptr(out, x),
                                            ctypes.c_void_p(workspace.data_ptr()), workspace.numel(),
                                            _stream(stream)))
    return out


def dchag_forward_folded(x: torch.Tensor, We: torch.Tensor, be: Optional[torch.Tensor], ce: Optional[torch.Tensor],
                         levels: List[LevelWeights], p: int, heads: int, out: Optional[torch.Tensor] = None,
                         workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """out[B,N,D] as dchag_forward, with the value projection applied after the softmax-weighted sum."""
    B, C, H, W = x.shape
    D = We.shape[1]
    if tuple(We.shape) != (C, D, p * p):
        raise ValueError("We must be [C, D, p*p]")
    N = (H // p) * (W // p) if p > 0 else 0
    dt = _dt(x)
    if workspace is None:
        workspace = _workspace(dchag_workspace_bytes(dt, B, C, H, W, p, D, heads, [lv.group_size for lv in levels], 2),
                               x.device)
    if out is None:
        out = torch.empty((B, N, D), dtype=x.dtype, device=x.device)
    arr = (_CLevel * len(levels))(*[_clevel(lv, x) for lv in levels])
    _check(load_library().dchag_forward_folded(dt, B, C, H, W, p, D, heads, _ptr(x), _ptr(We, x), _ptr(be, x),
                                               _ptr(ce, x), len(levels), arr, _ptr(out, x),
                                               ctypes.c_void_p(workspace.data_ptr()), workspace.numel(),
                                               _stream(stream)))
    return out


def dchag_fold_value(We: torch.Tensor, be: Optional[torch.Tensor], ce: Optional[torch.Tensor],
                     levels: List[LevelWeights], p: int, heads: int, stream=None) -> Optional[torch.Tensor]:
    """Everything of dchag_forward_folded that depends on the weights alone, for dchag_forward_prefolded; None when
    the library does not take that shape's first level from the pixels (dchag_value_fold_bytes == 0)."""
    C, D = We.shape[0], We.shape[1]
    if tuple(We.shape) != (C, D, p * p):
        raise ValueError("We must be [C, D, p*p]")
    dt = _dt(We)
    lib = load_library()
    arr = (_CLevel * len(levels))(*[_clevel(lv, We) for lv in levels])
    need = lib.dchag_value_fold_bytes(dt, C, p, D, heads, len(levels), arr)
    if need == 0:
        return None
    folded = _workspace(need, We.device)
    _check(lib.dchag_fold_value(dt, C, p, D, heads, _ptr(We), _ptr(be, We), _ptr(ce, We), len(levels), arr,
                                ctypes.c_void_p(folded.data_ptr()), folded.numel(), _stream(stream)))
    return folded


def dchag_forward_prefolded(x: torch.Tensor, We: torch.Tensor, be: Optional[torch.Tensor], ce: Optional[torch.Tensor],
                            levels: List[LevelWeights], p: int, heads: int, folded: torch.Tensor,
                            out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                            stream=None) -> torch.Tensor:
    """dchag_forward_folded with the first level's weight-only products taken from `folded` (dchag_fold_value)."""
    B, C, H, W = x.shape
    D = We.shape[1]
    if tuple(We.shape) != (C, D, p * p):
        raise ValueError("We must be [C, D, p*p]")
    N = (H // p) * (W // p) if p > 0 else 0
    dt = _dt(x)
    if workspace is None:
        workspace = _workspace(dchag_workspace_bytes(dt, B, C, H, W, p, D, heads, [lv.group_size for lv in levels], 2),
                               x.device)
    if out is None:
        out = torch.empty((B, N, D), dtype=x.dtype, device=x.device)
    arr = (_CLevel * len(levels))(*[_clevel(lv, x) for lv in levels])
    _check(load_library().dchag_forward_prefolded(dt, B, C, H, W, p, D, heads, _ptr(x), _ptr(We, x), _ptr(be, x),
                                                  _ptr(ce, x), len(levels), arr,
                                                  ctypes.c_void_p(folded.data_ptr()), _ptr(out, x),
                                                  ctypes.c_void_p(workspace.data_ptr()), workspace.numel(),
                                                  _stream(stream)))
    return out


def dchag_forward_keep(x: torch.Tensor, We: torch.Tensor, be: Optional[torch.Tensor], ce: Optional[torch.Tensor],
                       levels: List[LevelWeights], p: int, heads: int, workspace: torch.Tensor,
                       out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """out[B,N,D] as dchag_forward_folded; `workspace` (dchag_workspace_bytes(..., 3) bytes) keeps what
    dchag_backward_kept reads."""
    B, C, H, W = x.shape
    D = We.shape[1]
    if tuple(We.shape) != (C, D, p * p):
        raise ValueError("We must be [C, D, p*p]")
    N = (H // p) * (W // p) if p > 0 else 0
    if out is None:
        out = torch.empty((B, N, D), dtype=x.dtype, device=x.device)
    arr = (_CLevel * len(levels))(*[_clevel(lv, x) for lv in levels])
    _check(load_library().dchag_forward_keep(_dt(x), B, C, H, W, p, D, heads, _ptr(x), _ptr(We, x), _ptr(be, x),
                                             _ptr(ce, x), len(levels), arr, _ptr(out, x),
                                             ctypes.c_void_p(workspace.data_ptr()), workspace.numel(), _stream(stream)))
    return out


def dchag_backward(x: torch.Tensor, We: torch.Tensor, be: Optional[torch.Tensor], ce: Optional[torch.Tensor],
                   levels: List[LevelWeights], p: int, heads: int, dout: torch.Tensor,
                   grads: List[LevelGrads], dx: Optional[torch.Tensor] = None, dWe: Optional[torch.Tensor] = None,
                   dtok_bias: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                   stream=None, kept: bool = False) -> None:
    """Writes the gradients of <dout, dchag_forward(...)> into the given tensors (None = not wanted).
    kept=True calls dchag_backward_kept: `workspace` must be the one a dchag_forward_keep call just filled."""
    B, C, H, W = x.shape
    D = We.shape[1]
    if tuple(We.shape) != (C, D, p * p):
        raise ValueError("We must be [C, D, p*p]")
    if len(grads) != len(levels):
        raise ValueError("one LevelGrads per level")
    dt = _dt(x)
    if workspace is None:
        workspace = _workspace(dchag_workspace_bytes(dt, B, C, H, W, p, D, heads, [lv.group_size for lv in levels], 3),
                               x.device)
    arr = (_CLevel * len(levels))(*[_clevel(lv, x) for lv in levels])
    garr = (_CLevelGrads * len(levels))()
    for j, g in enumerate(grads):
        for name in ("dquery", "dWq", "dWk", "dWv", "dWo", "dbq", "dbk", "dbv", "dbo"):
            setattr(garr[j], name, _ptr(getattr(g, name), x))
    if kept and workspace is None:
        raise ValueError("kept=True needs the workspace of the dchag_forward_keep call")
    fn = load_library().dchag_backward_kept if kept else load_library().dchag_backward
    _check(fn(dt, B, C, H, W, p, D, heads, _ptr(x), _ptr(We, x), _ptr(be, x), _ptr(ce, x),
              len(levels), arr, _ptr(dout, x), _ptr(dx, x), _ptr(dWe, x), _ptr(dtok_bias, x), garr,
              ctypes.c_void_p(workspace.data_ptr()), workspace.numel(), _stream(stream)))


def log_borders(buckets: int, max_distance: int) -> List[int]:
    """Borders for `buckets` buckets a side: the first half of the distances have a bucket each, the other buckets widen by a constant
    factor up to max_distance, from which on all distances share the last.  Border b of the second half is the smallest whole distance r with
    r >= e (max_distance / e)^((b - e) / (buckets - e)), e = buckets // 2, found in whole numbers."""
    e = buckets // 2
    if buckets < 2 or max_distance <= e:
        raise ValueError("need at least two buckets, and a max_distance beyond the first half of them")
    n, out = buckets - e, list(range(1, e + 1))
    for k in range(1, n):
        r, want = out[-1] + 1, e ** (n - k) * max_distance ** k
        while r ** n < want:
            r += 1
        out.append(r)
    return out


def _row_stride(t: torch.Tensor, name: str) -> int:
    """Elements from one row to the next of [rows, heads, d] whose heads lie one behind the other."""
    rows, heads, d = t.shape
    row, head, one = t.stride()
    if ((d > 1 and one != 1) or (heads > 1 and head != d)) and t.numel():
        raise ValueError(f"the heads of a row of {name} must lie one behind the other")
    if rows > 1 and row < heads * d:
        raise ValueError(f"the rows of {name} must not overlap")
    return row if rows > 1 else 0


def _addr(t: torch.Tensor, dtype: torch.dtype, device: int, name: str) -> int:
    """Address of a tensor of that type on the current device; its strides are the caller's business."""
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}")
    if t.get_device() != device:
        raise ValueError(f"{name} must be a tensor on the current device")
    return t.data_ptr()


def _bytes(workspace: torch.Tensor, device: int):
    """Address and size of a workspace; like every tensor of a call it has to be on the current device, and in one piece."""
    if workspace.get_device() != device or not workspace.is_contiguous():
        raise ValueError("the workspace must be a contiguous tensor on the current device")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _vector(t: torch.Tensor, n: int, name: str) -> None:
    if t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous vector of {n}")


def _device(t: torch.Tensor) -> int:
    if not t.is_cuda:
        raise ValueError("tensors must be on the current device")
    return torch.cuda.current_device()


def _raw_stream(device: int) -> int:
    """The current stream's handle, without making a stream object of it, which would take longer than the rest of a call."""
    return torch._C._cuda_getCurrentRawStream(device)


def _on_stream(call):
    """Makes a call on the stream it is given, if it is given one: what the call allocates then is that stream's, too."""
    at = list(inspect.signature(call).parameters).index("stream")  # past every argument that has a place, if it is a keyword

    @functools.wraps(call)
    def on_stream(*args, **kw):
        if len(args) == at + 1 and "stream" not in kw:
            args, kw["stream"] = args[:at], args[at]
        stream = kw.get("stream")
        if stream is None:
            return call(*args, **kw)
        with torch.cuda.stream(stream):
            return call(*args, **kw)
    return on_stream


def _attention(q, k, v, q_starts, k_starts, causal, scale, k_used, bias, borders, device, others=(0, 0, 0, 0, 0)):
    """The C struct of a call, and what it points to on the host; others: row strides of out, dout, dq, dk, dv."""
    if q.dim() != 3 or k.dim() != 3 or v.shape != k.shape:
        raise ValueError("q must be [rows, heads, head_dim], k and v [rows, kv_heads, head_dim]")
    rows_q, heads, d = q.shape
    rows_k, kv_heads, dk = k.shape
    if dk != d:
        raise ValueError("q, k and v must have heads of one size")
    if q_starts.dim() != 1 or q_starts.shape[0] < 1:
        raise ValueError("q_starts must be a vector of one entry more than there are sequences")
    sequences = q_starts.shape[0] - 1
    _vector(q_starts, sequences + 1, "q_starts")
    _vector(k_starts, sequences + 1, "k_starts")
    used = host = bias_at = None
    n = 0
    if k_used is not None:
        _vector(k_used, sequences, "k_used")
        used = _addr(k_used, torch.int32, device, "k_used")
    if (bias is None) != (borders is None):
        raise ValueError("bias and borders come together")
    if bias is not None:
        n = len(borders)
        if tuple(bias.shape) != (heads, (n + 1) * (1 if causal else 2)) or not bias.is_contiguous():
            raise ValueError("bias must be contiguous, [heads, buckets] with one bucket more than borders, twice as many if not causal")
        host = (ctypes.c_int32 * max(1, n))(*borders)
        bias_at = _addr(bias, q.dtype, device, "bias")
    a = _CAttention(heads, kv_heads, d, 1 if causal else 0, sequences, rows_q, rows_k, scale,
                    _row_stride(q, "q"), _row_stride(k, "k"), _row_stride(v, "v"), *others,
                    _addr(q_starts, torch.int32, device, "q_starts"), _addr(k_starts, torch.int32, device, "k_starts"), used, bias_at,
                    None if host is None else ctypes.addressof(host), n)
    return a, host


@_on_stream
def dchag_attend(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q_starts: torch.Tensor, k_starts: torch.Tensor, *,
                 causal: bool = False, scale: float = 0.0, k_used: Optional[torch.Tensor] = None,
                 bias: Optional[torch.Tensor] = None, borders: Optional[Sequence[int]] = None,
                 out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                 workspace: Optional[torch.Tensor] = None, stream=None):
    """(out [rows_q, heads, d], lse [heads, rows_q] float32) of attention over packed sequences: q [rows_q, heads, d], k and v
    [rows_k, kv_heads, d], int32 starts [sequences + 1] on the device.  Rows of a tensor may have gaps between them (columns of a
    joint projection).  Rows of no sequence are not written: give an `out` of your own if they are read later.  Gradients:
    dchag_attend_backward, called with what this returned (autograd does not know the calls)."""
    device = _device(q)
    ld_out = 0
    if out is not None:
        if out.shape != q.shape:
            raise ValueError("out must be shaped like q")
        ld_out = _row_stride(out, "out")
    a, host = _attention(q, k, v, q_starts, k_starts, causal, scale, k_used, bias, borders, device, (ld_out, 0, 0, 0, 0))
    dt, dtype, lib = _dt(q), q.dtype, load_library()
    where = q.device
    if out is None:
        out = torch.empty(q.shape, dtype=dtype, device=where)
    if lse is None:
        lse = torch.empty((a.heads, a.rows_q), dtype=torch.float32, device=where)
    elif tuple(lse.shape) != (a.heads, a.rows_q) or not lse.is_contiguous():
        raise ValueError("lse must be [heads, rows_q] and contiguous")
    if workspace is None:
        workspace = _workspace(lib.dchag_attend_workspace_bytes(dt, a, 0), where)
    _check(lib.dchag_attend(dt, a, _addr(q, dtype, device, "q"), _addr(k, dtype, device, "k"), _addr(v, dtype, device, "v"),
                            _addr(out, dtype, device, "out"), _addr(lse, torch.float32, device, "lse"), *_bytes(workspace, device), _raw_stream(device)))
    return out, lse


@_on_stream
def dchag_attend_backward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, lse: torch.Tensor,
                          dout: torch.Tensor, q_starts: torch.Tensor, k_starts: torch.Tensor, *, causal: bool = False,
                          scale: float = 0.0, k_used: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                          borders: Optional[Sequence[int]] = None, dq: Optional[torch.Tensor] = None,
                          dk: Optional[torch.Tensor] = None, dv: Optional[torch.Tensor] = None,
                          dbias: Optional[torch.Tensor] = None, want_dbias: bool = True,
                          workspace: Optional[torch.Tensor] = None, stream=None):
    """(dq, dk, dv, dbias or None) of <dout, dchag_attend(...)>; out and lse are those of the forward call with the same arguments.
    Rows of no sequence are not written.  Key rows that do not count (k_used) have no gradient: they are zero in the dk and dv that the call
    makes, and left as they were, as rows of no sequence are, in a dk or dv of your own (clear it first if they are read later)."""
    device = _device(q)
    dt, dtype, lib, where = _dt(q), q.dtype, load_library(), q.device
    if dq is None:
        dq = torch.empty(q.shape, dtype=dtype, device=where)
    room = torch.empty if k_used is None else torch.zeros          # the gradient of a key row that does not count
    if dk is None:
        dk = room(k.shape, dtype=dtype, device=where)
    if dv is None:
        dv = room(k.shape, dtype=dtype, device=where)
    if dbias is None and bias is not None and want_dbias:
        dbias = torch.empty(bias.shape, dtype=dtype, device=where)
    if dbias is not None and (bias is None or dbias.shape != bias.shape or not dbias.is_contiguous()):
        raise ValueError("dbias goes with a bias, is shaped like it and contiguous")
    if out.shape != q.shape or dout.shape != q.shape or dq.shape != q.shape or dk.shape != k.shape or dv.shape != k.shape:
        raise ValueError("out, dout and dq must be shaped like q, dk and dv like k")
    a, host = _attention(q, k, v, q_starts, k_starts, causal, scale, k_used, bias, borders, device,
                         (_row_stride(out, "out"), _row_stride(dout, "dout"), _row_stride(dq, "dq"), _row_stride(dk, "dk"), _row_stride(dv, "dv")))
    if tuple(lse.shape) != (a.heads, a.rows_q) or not lse.is_contiguous():
        raise ValueError("lse must be [heads, rows_q] and contiguous")
    if workspace is None:
        workspace = _workspace(lib.dchag_attend_workspace_bytes(dt, a, 1), q.device)
    _check(lib.dchag_attend_backward(
        dt, a, _addr(q, dtype, device, "q"), _addr(k, dtype, device, "k"), _addr(v, dtype, device, "v"), _addr(out, dtype, device, "out"),
        _addr(lse, torch.float32, device, "lse"), _addr(dout, dtype, device, "dout"), _addr(dq, dtype, device, "dq"),
        _addr(dk, dtype, device, "dk"), _addr(dv, dtype, device, "dv"), None if dbias is None else _addr(dbias, dtype, device, "dbias"),
        *_bytes(workspace, device), _raw_stream(device)))
    return dq, dk, dv, dbias


def _matrix(t: torch.Tensor, name: str) -> int:
    """Elements from one row to the next of a matrix whose rows have no gaps inside."""
    if t.dim() != 2 or (t.numel() and t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be a matrix with adjacent columns")
    if t.shape[0] > 1 and t.stride(0) < t.shape[1]:
        raise ValueError(f"the rows of {name} must not overlap")
    return int(t.stride(0)) if t.shape[0] > 1 else 0


def _codes8(codes: torch.Tensor, scales: torch.Tensor, rows: int, D: int) -> None:
    if tuple(codes.shape) != (rows, D) or tuple(scales.shape) != (rows, (D + 31) // 32) or not codes.is_contiguous() or not scales.is_contiguous():
        raise ValueError("codes must be [rows, D] and scales [rows, (D + 31) // 32], contiguous")


@_on_stream
def dchag_pack8(x: torch.Tensor, codes: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None, stream=None):
    """(codes uint8 [rows, D], scales uint8 [rows, (D + 31) // 32]): the rows of x in 8 bits, one exponent for every 32 values."""
    ld, (rows, D), device = _matrix(x, "x"), x.shape, _device(x)
    if codes is None:
        codes = torch.empty((rows, D), dtype=torch.uint8, device=x.device)
    if scales is None:
        scales = torch.empty((rows, (D + 31) // 32), dtype=torch.uint8, device=x.device)
    _codes8(codes, scales, rows, D)
    _check(load_library().dchag_pack8(_dt(x), rows, D, ld, _addr(x, x.dtype, device, "x"), _addr(codes, torch.uint8, device, "codes"),
                                      _addr(scales, torch.uint8, device, "scales"), _raw_stream(device)))
    return codes, scales


@_on_stream
def dchag_unpack8(codes: torch.Tensor, scales: torch.Tensor, dtype: torch.dtype = torch.bfloat16,
                  out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """The rows that codes and scales (dchag_pack8) stand for."""
    (rows, D), device = codes.shape, _device(codes)
    _codes8(codes, scales, rows, D)
    if out is None:
        out = torch.empty((rows, D), dtype=dtype, device=codes.device)
    elif tuple(out.shape) != (rows, D):
        raise ValueError("out must be [rows, D]")
    _check(load_library().dchag_unpack8(_dt(out), rows, D, _matrix(out, "out"), _addr(codes, torch.uint8, device, "codes"),
                                        _addr(scales, torch.uint8, device, "scales"), _addr(out, out.dtype, device, "out"), _raw_stream(device)))
    return out


@_on_stream
def dchag_weight_grad8(dy: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, dW: Optional[torch.Tensor] = None,
                       db: Optional[torch.Tensor] = None, want_db: bool = True, workspace: Optional[torch.Tensor] = None, stream=None):
    """(dW [d_out, d_in], db [d_out] or None) of a linear layer: dy [rows, d_out], its input in 8 bits (dchag_pack8)."""
    ld, (rows, d_out), d_in = _matrix(dy, "dy"), dy.shape, codes.shape[-1]
    _codes8(codes, scales, rows, d_in)
    device, dtype = _device(dy), dy.dtype
    if dW is None:
        dW = torch.empty((d_out, d_in), dtype=dtype, device=dy.device)
    if db is None and want_db:
        db = torch.empty((d_out,), dtype=dtype, device=dy.device)
    if tuple(dW.shape) != (d_out, d_in) or not dW.is_contiguous() or (db is not None and (tuple(db.shape) != (d_out,) or not db.is_contiguous())):
        raise ValueError("dW must be [d_out, d_in], db [d_out], contiguous")
    dt, lib = _dt(dy), load_library()
    if workspace is None:
        workspace = _workspace(lib.dchag_weight_grad8_workspace_bytes(dt, rows, d_out, d_in), dy.device)
    _check(lib.dchag_weight_grad8(dt, rows, d_out, d_in, ld, _addr(dy, dtype, device, "dy"), _addr(codes, torch.uint8, device, "codes"),
                                  _addr(scales, torch.uint8, device, "scales"), _addr(dW, dtype, device, "dW"),
                                  None if db is None else _addr(db, dtype, device, "db"), *_bytes(workspace, device), _raw_stream(device)))
    return dW, db


def dchag_yardstick_mfma(iters: int, sink: torch.Tensor, stream=None) -> float:
    """Launches the MFMA-only yardstick loop; returns the flops it performs.  sink: float32 device scratch."""
    flops = ctypes.c_double(0.0)
    _check(load_library().dchag_yardstick_mfma(int(iters), ctypes.c_void_p(sink.data_ptr()), sink.numel(),
                                               ctypes.byref(flops), _stream(stream)))
    return float(flops.value)


def dchag_yardstick_copy(dst: torch.Tensor, src: torch.Tensor, stream=None) -> int:
    """Launches the stream-copy yardstick dst <- src; returns the bytes read (= the bytes written)."""
    nbytes = src.numel() * src.element_size()
    _check(load_library().dchag_yardstick_copy(ctypes.c_void_p(dst.data_ptr()), ctypes.c_void_p(src.data_ptr()),
                                               nbytes, _stream(stream)))
    return nbytes


def dchag_yardstick_read(src: torch.Tensor, sink: torch.Tensor, stream=None) -> int:
    """Launches the streaming-read yardstick over src; returns the bytes read.  sink: float32 device scratch (>= 256)."""
    nbytes = src.numel() * src.element_size()
    _check(load_library().dchag_yardstick_read(ctypes.c_void_p(src.data_ptr()), nbytes,
                                               ctypes.c_void_p(sink.data_ptr()), _stream(stream)))
    return nbytes


def dchag_profile_begin() -> None:
    """Start bracketing every kernel launch of the library with HIP events (benchmark diagnostic)."""
    _check(load_library().dchag_profile_begin())


def dchag_profile_end(cap: int = 1 << 16):
    """Stop stage timing; returns [(stage name, level, ms)] in launch order."""
    buf = (_CStageTime * cap)()
    n = load_library().dchag_profile_end(buf, cap)
    if n < 0:
        _check(n)
    return [(STAGE_NAMES.get(buf[j].stage, str(buf[j].stage)), int(buf[j].level), float(buf[j].ms))
            for j in range(min(n, cap))]
