"""Thin ctypes binding of the language-model operators (include/cx_lm.h).

Argument marshalling and checks only: every step runs inside libcxlm.so, and there is no fallback.  The functions carry the names of
the C entry points: plain for float32, suffix _bf16 (torch.bfloat16) and _f16 (torch.float16); sizes come from the tensors'
shapes, and a matrix may be a view with longer rows.  Errors are those of cxmix: ValueError for tensors that do not fit a
call, CxError for what the library refuses.

`workspace`: a uint8 tensor of at least the matching *_workspace() bytes; without one the call takes it from torch's
allocator, for the current stream.  A call on another stream by handle brings its own.
"""
from __future__ import annotations

import ctypes
import functools
import os

from . import cxmix
from .cxmix import CX_MAX_ROWS, CxError  # noqa: F401 (part of this module's interface)

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcxlm.so")

CX_MAX_TOKENS, CX_MAX_SEQUENCES, CX_MAX_VOCAB, CX_MAX_WIDTH = 1 << 26, 1 << 22, 1 << 26, 1 << 20
CX_MAX_TOP, CX_MAX_TEACHER, CX_SCAN_CHUNK = 64, 256, 16
CX_MAX_NORM_WIDTH, CX_MAX_TAPS, CX_MAX_STATES = 16384, 4, 16

_TYPED = ["cx_embed_lookup", "cx_embed_grad", "cx_gated_scan", "cx_gated_scan_grad", "cx_token_scores", "cx_distill_loss",
          "cx_distill_grad", "cx_distill_step", "cx_dropout", "cx_add_norm", "cx_add_norm_grad", "cx_short_conv", "cx_short_conv_grad",
          "cx_select_scan", "cx_select_scan_grad"]
EXPORTS = ["cx_lm_abi_version", "cx_embed_workspace", "cx_scan_workspace", "cx_scores_workspace", "cx_distill_workspace",
           "cx_norm_workspace", "cx_conv_workspace", "cx_select_workspace", "cx_select_grad_workspace",
           *(name + suffix for name in _TYPED for suffix in ("", "_bf16", "_f16"))]

_INT32 = 2**31 - 1
_CX_ERR_SHAPE = -2
_lib = None
_torch = None
_dtypes = {}                     # "", "_bf16", "_f16" -> the torch type of the matrices
_calls = {}                      # name -> the library's function
_device_now = None               # the current device's number, without torch's check that it is in use


def lib() -> ctypes.CDLL:
    """The loaded library; raises if it was not built."""
    global _lib, _torch, _device_now
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2012_15198_amd.build` (hipcc, gfx950)")
    import torch                 # first: the library binds to the HIP runtime that owns torch's tensors and streams
    cxmix._know_torch(torch)
    L = ctypes.CDLL(LIB_PATH)
    i32, i64, f32, vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p
    size = ctypes.POINTER(i64)
    L.cx_lm_abi_version.argtypes = []
    L.cx_embed_workspace.argtypes = [i32, i64, i32, i32, size]
    L.cx_scan_workspace.argtypes = [i64, i64, i32, size]
    L.cx_scores_workspace.argtypes = [i64, i32, i32, size]
    L.cx_distill_workspace.argtypes = [i64, i32, size]
    L.cx_norm_workspace.argtypes = [i32, i64, i32, size]
    L.cx_conv_workspace.argtypes = [i32, i64, i64, i32, i32, size]
    L.cx_select_workspace.argtypes = [i64, i64, i32, i32, size]
    L.cx_select_grad_workspace.argtypes = [i64, i64, i32, i32, size]
    row = [vp, i64]
    targets = [i64, i32, i32, vp, vp, vp, f32, f32, f32]
    scratch = [vp, i64, vp]
    typed = {
        "cx_embed_lookup": [*row, i32, i64, i32, i32, vp, i64, f32, *row, vp],
        "cx_embed_grad": [*row, vp, i32, i64, vp, vp, i64, i64, i32, i32, f32, *scratch],
        "cx_gated_scan": [*row, *row, *row, i64, i64, i32, vp, vp, vp, vp, *scratch],
        "cx_gated_scan_grad": [*row, *row, *row, *row, *row, i64, i64, i32, vp, vp, vp, vp, *scratch],
        "cx_token_scores": [*row, i64, i32, vp, f32, vp, vp, i32, vp, vp, *scratch],
        "cx_distill_loss": [*row, *targets, vp, vp, *scratch],
        "cx_distill_grad": [*row, *targets, vp, vp, *row, vp],
        "cx_distill_step": [*row, *targets, vp, vp, *row, *scratch],
        "cx_dropout": [*row, *row, *row, i64, i32, vp, f32, vp],
        "cx_add_norm": [*row, *row, *row, i32, i64, i64, i32, f32, vp, f32, *row, *row, vp, *row, vp, vp],
        "cx_add_norm_grad": [*row, *row, vp, *row, i32, i64, i64, i32, *row, vp, f32, *row, *row, vp, *row, *scratch],
        "cx_short_conv": [*row, *row, i32, i64, *row, i64, i64, i32, i32, i32, vp, vp, vp, vp],
        "cx_short_conv_grad": [*row, *row, *row, i32, i64, *row, vp, *row, i64, i64, i32, i32, i32, vp, vp, *scratch],
        "cx_select_scan": [*row, *row, *row, *row, *row, *row, i32, i64, *row, i64, i64, i32, i32, vp, vp, vp, vp, *scratch],
        "cx_select_scan_grad": [*row, *row, *row, *row, *row, *row, i32, i64, *row, *row, *row, *row, *row, *row, vp, *row, i64, i64, i32, i32, vp, vp,
                                vp, vp, *scratch],
    }
    for name, args in typed.items():
        for suffix in ("", "_bf16", "_f16"):
            getattr(L, name + suffix).argtypes = args
    for name in EXPORTS:
        getattr(L, name).restype = ctypes.c_int
        _calls[name] = getattr(L, name)
    _dtypes.update({"": torch.float32, "_bf16": torch.bfloat16, "_f16": torch.float16})
    _device_now = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    _lib, _torch = L, torch
    return L


def _ok(fn: str, status: int) -> None:
    if status != 0:
        raise CxError(fn, status)


def _call(name, *args) -> None:
    status = _calls[name](*args)
    if status != 0:
        raise CxError(name, status)


# ------------------------------------------------------------------------------------------------------------- checks
# The binding's share of a call is what bounds the smallest ones, so that the checks are plain functions with few queries each:
# cx_embed_lookup_bf16 of 32 tokens, call after call, 7.8 us with an object for every call's checks, 7.1 us with these, of which
# 3.7 us are the library's.
def _matrix(name, arg, t, dtype, rows, columns, device):
    """Row stride of a row-major matrix of the call's type on its device; rows or columns of None: any."""
    shape, stride = t.shape, t.stride()
    if (len(shape) == 2 and t.dtype is dtype and stride[1] == 1 and stride[0] >= shape[1] and (rows is None or shape[0] == rows)
            and (columns is None or shape[1] == columns) and t.get_device() == device):
        return stride[0]
    return _unusual_matrix(name, arg, t, dtype, rows, columns, device)


def _unusual_matrix(name, arg, t, dtype, rows, columns, device):
    """The same for single rows and columns, whose strides mean nothing; raises what does not fit."""
    shape, stride = t.shape, t.stride()
    if t.dtype != dtype:
        raise ValueError(f"{name}: {arg}: expected {dtype}, got {t.dtype}")
    if len(shape) != 2 or (rows is not None and shape[0] != rows) or (columns is not None and shape[1] != columns):
        raise ValueError(f"{name}: {arg}: expected [{'any' if rows is None else rows}][{'any' if columns is None else columns}], got {list(shape)}")
    if t.numel() > 0 and ((shape[1] > 1 and stride[1] != 1) or (shape[0] > 1 and stride[0] < shape[1])):
        raise ValueError(f"{name}: {arg}: expected row-major elements (rows that do not overlap)")
    if t.get_device() != device:
        raise ValueError(f"{name}: {arg}: on another device than the call's first buffer: {t.device}")
    return max(stride[0], shape[1], 1) if shape[0] > 1 else max(shape[1], 1)


def _dense(name, arg, t, dtype, shape, device):
    """Address of a contiguous tensor of exactly this type and shape on the call's device."""
    if t is not None and t.dtype is dtype and t.shape == shape and t.is_contiguous() and t.get_device() == device:
        return t.data_ptr()
    if t is None:
        raise ValueError(f"{name}: {arg} is missing")
    if t.dtype != dtype:
        raise ValueError(f"{name}: {arg}: expected {dtype}, got {t.dtype}")
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name}: {arg}: expected a contiguous tensor {list(shape)}, got {list(t.shape)}, strides {t.stride()}")
    raise ValueError(f"{name}: {arg}: on another device than the call's first buffer: {t.device}")


def _optional(name, arg, t, dtype, shape, device):
    return None if t is None else _dense(name, arg, t, dtype, shape, device)


def _too_wide(name):
    """A size that a 32-bit argument cannot hold, of which ctypes would drop the upper bits: refused as the library refuses what is beyond its limits."""
    raise CxError(name, _CX_ERR_SHAPE)


def _on_device(name, device):
    """Last check before the call."""
    if device < 0:
        raise ValueError(f"{name}: expected device tensors")


def _scratch(name, workspace, size, args, device, stream):
    """The workspace: the caller's, or from torch's allocator what the library's function `size` asks for (None: no call needs one)."""
    _on_device(name, device)
    if size is None and workspace is None:
        return None
    if workspace is not None:
        if workspace.dtype is not _torch.uint8 or not workspace.is_contiguous() or workspace.get_device() != device:
            raise ValueError(f"{name}: workspace: expected a contiguous uint8 tensor on the call's device")
        return workspace
    needed = _size(size, *args)
    if needed == 0:
        return None
    if stream is not None and getattr(stream, "cuda_stream", stream) != cxmix._stream(None):
        raise ValueError(f"{name}: a call on a stream that is not the current one brings its own workspace ({needed} bytes)")
    return _torch.empty(needed, dtype=_torch.uint8, device=device)


def _span(work):
    return (None, 0) if work is None else (work.data_ptr(), work.numel())


_INTS = {int}


def _size(fn, *args) -> int:
    # a training step asks for the same few sizes again: 1 us of a call's 8.  Kept of plain integers alone: a fraction equals one, a tensor may change
    return (_known_size if set(map(type, args)) == _INTS else _asked_size)(fn, *args)


def _asked_size(fn, *args) -> int:
    L = _lib or lib()
    if max(args) > _INT32 or min(args) < -_INT32:        # the 64-bit ones have limits below 2^31 too
        _too_wide(fn)
    n = ctypes.c_int64()
    _ok(fn, getattr(L, fn)(*args, ctypes.byref(n)))
    return n.value


_known_size = functools.lru_cache(maxsize=1024)(_asked_size)


def cx_lm_abi_version() -> int:
    return lib().cx_lm_abi_version()


def cx_embed_workspace(W: int, N: int, V: int, D: int) -> int:
    """Bytes of workspace of cx_embed_grad*."""
    return _size("cx_embed_workspace", W, N, V, D)


def cx_scan_workspace(B: int, T: int, D: int) -> int:
    """Bytes of workspace of cx_gated_scan* and cx_gated_scan_grad*."""
    return _size("cx_scan_workspace", B, T, D)


def cx_scores_workspace(N: int, V: int, K: int) -> int:
    """Bytes of workspace of cx_token_scores*."""
    return _size("cx_scores_workspace", N, V, K)


def cx_distill_workspace(N: int, V: int) -> int:
    """Bytes of workspace of cx_distill_loss* and cx_distill_step*."""
    return _size("cx_distill_workspace", N, V)


def cx_norm_workspace(W: int, N: int, D: int) -> int:
    """Bytes of workspace of cx_add_norm_grad*."""
    return _size("cx_norm_workspace", W, N, D)


def cx_conv_workspace(W: int, B: int, T: int, D: int, K: int) -> int:
    """Bytes of workspace of cx_short_conv_grad*."""
    return _size("cx_conv_workspace", W, B, T, D, K)


def cx_select_workspace(B: int, T: int, D: int, N: int) -> int:
    """Bytes of workspace of cx_select_scan*."""
    return _size("cx_select_workspace", B, T, D, N)


def cx_select_grad_workspace(B: int, T: int, D: int, N: int) -> int:
    """Bytes of workspace of cx_select_scan_grad*."""
    return _size("cx_select_grad_workspace", B, T, D, N)


# ---------------------------------------------------------------------------------------------------------- embeddings
def _lookup(name, suffix, x, tokens, out, offset, V, scale, stream):
    if _lib is None:
        lib()
    dtype, device = _dtypes[suffix], x.get_device()
    if len(tokens.shape) != 2:
        raise ValueError(f"{name}: tokens: expected int32 [W][N]")
    W, N = tokens.shape
    ld = _matrix(name, "x", x, dtype, W, None, device)
    ld_out = _matrix(name, "out", out, dtype, W * N, None, device)
    D = out.shape[1]
    if V > _INT32 or V < -_INT32 or D > _INT32 or W > _INT32:
        _too_wide(name)
    if offset < 0 or offset + V * D > x.shape[1]:
        raise ValueError(f"{name}: a table of {V} x {D} at {offset} does not fit rows of {x.shape[1]}")
    tp = _dense(name, "tokens", tokens, _torch.int32, (W, N), device)
    _on_device(name, device)
    _call(name, x.data_ptr(), ld, W, offset, V, D, tp, N, scale, out.data_ptr(), ld_out, cxmix._stream(stream))


def cx_embed_lookup(x, tokens, out, offset: int, V: int, scale: float = 1.0, stream=None):
    """x: [W][ld] flat rows; tokens: int32 [W][N]; out: [W * N][D].  The table of worker w is x[w, offset : offset + V * D]."""
    _lookup("cx_embed_lookup", "", x, tokens, out, offset, V, scale, stream)


def cx_embed_lookup_bf16(x, tokens, out, offset: int, V: int, scale: float = 1.0, stream=None):
    _lookup("cx_embed_lookup_bf16", "_bf16", x, tokens, out, offset, V, scale, stream)


def cx_embed_lookup_f16(x, tokens, out, offset: int, V: int, scale: float = 1.0, stream=None):
    _lookup("cx_embed_lookup_f16", "_f16", x, tokens, out, offset, V, scale, stream)


def _embed_grad(name, suffix, dout, tokens, g_in, g_out, offset, V, scale, workspace, stream):
    if _lib is None:
        lib()
    dtype, device = _dtypes[suffix], g_out.get_device()
    if len(tokens.shape) != 2:
        raise ValueError(f"{name}: tokens: expected int32 [W][N]")
    W, N = tokens.shape
    ld_dout = _matrix(name, "dout", dout, dtype, W * N, None, device)
    D = dout.shape[1]
    if V > _INT32 or V < -_INT32 or D > _INT32 or W > _INT32:
        _too_wide(name)
    ld = _matrix(name, "g_out", g_out, dtype, W, None, device)
    fits = g_out.shape[1]
    if g_in is not None:
        ld_in = _matrix(name, "g_in", g_in, dtype, W, None, device)
        if W > 1 and ld_in != ld:
            raise ValueError(f"{name}: g_in: row stride {ld_in} differs from g_out's {ld}")
        fits = min(fits, g_in.shape[1])
    if offset < 0 or offset + V * D > fits:
        raise ValueError(f"{name}: a table of {V} x {D} at {offset} does not fit rows of {fits}")
    tp = _dense(name, "tokens", tokens, _torch.int32, (W, N), device)
    work = _scratch(name, workspace, "cx_embed_workspace", (W, N, V, D), device, stream)
    _call(name, dout.data_ptr(), ld_dout, tp, W, N, None if g_in is None else g_in.data_ptr(), g_out.data_ptr(), ld, offset, V, D,
                               scale, *_span(work), cxmix._stream(stream))


def cx_embed_grad(dout, tokens, g_in, g_out, offset: int, V: int, scale: float = 1.0, workspace=None, stream=None):
    """dout: [W * N][D]; tokens: int32 [W][N]; g_out: [W][ld] flat gradient rows.  g_in: None (rows that no token names become
    zeros), g_out itself (added in place) or a second matrix with the same row stride."""
    _embed_grad("cx_embed_grad", "", dout, tokens, g_in, g_out, offset, V, scale, workspace, stream)


def cx_embed_grad_bf16(dout, tokens, g_in, g_out, offset: int, V: int, scale: float = 1.0, workspace=None, stream=None):
    _embed_grad("cx_embed_grad_bf16", "_bf16", dout, tokens, g_in, g_out, offset, V, scale, workspace, stream)


def cx_embed_grad_f16(dout, tokens, g_in, g_out, offset: int, V: int, scale: float = 1.0, workspace=None, stream=None):
    _embed_grad("cx_embed_grad_f16", "_f16", dout, tokens, g_in, g_out, offset, V, scale, workspace, stream)


# ----------------------------------------------------------------------------------------------------- gated recurrence
def scan_states(f, T: int):
    """An empty tensor for the `states` of a scan over f ([B * T][D]) that is to have a gradient."""
    import torch
    B = f.shape[0] // T if T > 0 else 0
    return torch.empty((B, -(-T // CX_SCAN_CHUNK), f.shape[1]), dtype=torch.float32, device=f.device)


def _sequences(name, rows, T, *ends):
    """B of B * T rows; of empty sequences, what the states at their ends say."""
    if T > 0 and rows % T == 0:
        return rows // T
    if T == 0 and rows == 0:
        return next((t.shape[0] for t in ends if t is not None), 0)
    raise ValueError(f"{name}: {rows} rows are no sequences of {T} steps")


def _scan(name, suffix, f, x, y, T, h0, h_last, reset, states, workspace, stream):
    if _lib is None:
        lib()
    dtype, device, f32 = _dtypes[suffix], f.get_device(), _torch.float32
    ldf = _matrix(name, "f", f, dtype, None, None, device)
    rows, D = f.shape
    if D > _INT32:
        _too_wide(name)
    B = _sequences(name, rows, T, h0, h_last)
    ldx = _matrix(name, "x", x, dtype, rows, D, device)
    ldy = _matrix(name, "y", y, dtype, rows, D, device)
    hp = _optional(name, "h0", h0, f32, (B, D), device)
    lp = _optional(name, "h_last", h_last, f32, (B, D), device)
    sp = _optional(name, "states", states, f32, (B, -(-T // CX_SCAN_CHUNK), D), device)
    rp = _optional(name, "reset", reset, _torch.uint8, (B, T), device)
    work = _scratch(name, workspace, None if T <= CX_SCAN_CHUNK else "cx_scan_workspace", (B, T, D), device, stream)
    _call(name, f.data_ptr(), ldf, x.data_ptr(), ldx, y.data_ptr(), ldy, B, T, D, rp, hp, lp, sp, *_span(work),
                               cxmix._stream(stream))


def cx_gated_scan(f, x, y, T: int, h0=None, h_last=None, reset=None, states=None, workspace=None, stream=None):
    """f, x, y: [B * T][D]; h0, h_last: float32 [B][D] (may be one tensor); reset: uint8 [B][T]; states: see scan_states()."""
    _scan("cx_gated_scan", "", f, x, y, T, h0, h_last, reset, states, workspace, stream)


def cx_gated_scan_bf16(f, x, y, T: int, h0=None, h_last=None, reset=None, states=None, workspace=None, stream=None):
    _scan("cx_gated_scan_bf16", "_bf16", f, x, y, T, h0, h_last, reset, states, workspace, stream)


def cx_gated_scan_f16(f, x, y, T: int, h0=None, h_last=None, reset=None, states=None, workspace=None, stream=None):
    _scan("cx_gated_scan_f16", "_f16", f, x, y, T, h0, h_last, reset, states, workspace, stream)


def _scan_grad(name, suffix, f, x, dy, df, dx, T, states, dh_last, dh0, reset, workspace, stream):
    if _lib is None:
        lib()
    dtype, device, f32 = _dtypes[suffix], f.get_device(), _torch.float32
    ldf = _matrix(name, "f", f, dtype, None, None, device)
    rows, D = f.shape
    if D > _INT32:
        _too_wide(name)
    B = _sequences(name, rows, T, dh_last, dh0)
    ldx = _matrix(name, "x", x, dtype, rows, D, device)
    lddy = _matrix(name, "dy", dy, dtype, rows, D, device)
    lddf = _matrix(name, "df", df, dtype, rows, D, device)
    lddx = _matrix(name, "dx", dx, dtype, rows, D, device)
    sp = (_dense if T > 0 else _optional)(name, "states", states, f32, (B, -(-T // CX_SCAN_CHUNK), D), device)
    lp = _optional(name, "dh_last", dh_last, f32, (B, D), device)
    hp = _optional(name, "dh0", dh0, f32, (B, D), device)
    rp = _optional(name, "reset", reset, _torch.uint8, (B, T), device)
    work = _scratch(name, workspace, None if T <= CX_SCAN_CHUNK else "cx_scan_workspace", (B, T, D), device, stream)
    _call(name, f.data_ptr(), ldf, x.data_ptr(), ldx, dy.data_ptr(), lddy, df.data_ptr(), lddf, dx.data_ptr(), lddx, B, T, D, rp, sp,
                               lp, hp, *_span(work), cxmix._stream(stream))


def cx_gated_scan_grad(f, x, dy, df, dx, T: int, states, dh_last=None, dh0=None, reset=None, workspace=None, stream=None):
    """f, x, dy, df, dx: [B * T][D]; states: as cx_gated_scan filled them; dh_last, dh0: float32 [B][D]; reset: uint8 [B][T]."""
    _scan_grad("cx_gated_scan_grad", "", f, x, dy, df, dx, T, states, dh_last, dh0, reset, workspace, stream)


def cx_gated_scan_grad_bf16(f, x, dy, df, dx, T: int, states, dh_last=None, dh0=None, reset=None, workspace=None, stream=None):
    _scan_grad("cx_gated_scan_grad_bf16", "_bf16", f, x, dy, df, dx, T, states, dh_last, dh0, reset, workspace, stream)


def cx_gated_scan_grad_f16(f, x, dy, df, dx, T: int, states, dh_last=None, dh0=None, reset=None, workspace=None, stream=None):
    _scan_grad("cx_gated_scan_grad_f16", "_f16", f, x, dy, df, dx, T, states, dh_last, dh0, reset, workspace, stream)


# ------------------------------------------------------------------------------------------------------------ token scores
def _scores(name, suffix, z, tokens, logp, entropy, top_ids, top_logp, scale, workspace, stream):
    if _lib is None:
        lib()
    device, f32, i32 = z.get_device(), _torch.float32, _torch.int32
    ld = _matrix(name, "z", z, _dtypes[suffix], None, None, device)
    N, V = z.shape
    tp = (_dense if logp is not None else _optional)(name, "tokens", tokens, i32, (N,), device)
    lp = _optional(name, "logp", logp, f32, (N,), device)
    ep = _optional(name, "entropy", entropy, f32, (N,), device)
    K = 0
    ip = pp = None
    if top_ids is not None or top_logp is not None:
        if top_ids is None or len(top_ids.shape) != 2:
            raise ValueError(f"{name}: top_ids: expected int32 [N][K] beside top_logp")
        K = top_ids.shape[1]
        ip = _dense(name, "top_ids", top_ids, i32, (N, K), device)
        pp = _dense(name, "top_logp", top_logp, f32, (N, K), device)
    if V > _INT32 or K > _INT32:
        _too_wide(name)
    work = _scratch(name, workspace, "cx_scores_workspace", (N, V, K), device, stream)
    _call(name, z.data_ptr(), ld, N, V, tp, scale, lp, ep, K, ip, pp, *_span(work), cxmix._stream(stream))


def cx_token_scores(z, tokens, logp, entropy=None, top_ids=None, top_logp=None, scale: float = 1.0, workspace=None, stream=None):
    """z: [N][V] logits; tokens: int32 [N]; logp, entropy: float32 [N]; top_ids: int32 [N][K]; top_logp: float32 [N][K]; what is
    None is not computed.  scale: 1 / temperature."""
    _scores("cx_token_scores", "", z, tokens, logp, entropy, top_ids, top_logp, scale, workspace, stream)


def cx_token_scores_bf16(z, tokens, logp, entropy=None, top_ids=None, top_logp=None, scale: float = 1.0, workspace=None, stream=None):
    _scores("cx_token_scores_bf16", "_bf16", z, tokens, logp, entropy, top_ids, top_logp, scale, workspace, stream)


def cx_token_scores_f16(z, tokens, logp, entropy=None, top_ids=None, top_logp=None, scale: float = 1.0, workspace=None, stream=None):
    _scores("cx_token_scores_f16", "_f16", z, tokens, logp, entropy, top_ids, top_logp, scale, workspace, stream)


# ------------------------------------------------------------------------------------------------------------- distillation
def _targets(name, suffix, z, ids, t, labels, device):
    """The first arguments of the three calls."""
    ld = _matrix(name, "z", z, _dtypes[suffix], None, None, device)
    N, V = z.shape
    if len(ids.shape) != 2:
        raise ValueError(f"{name}: ids: expected int32 [N][K]")
    K = ids.shape[1]
    if V > _INT32 or K > _INT32:
        _too_wide(name)
    ip = _dense(name, "ids", ids, _torch.int32, (N, K), device)
    tp = _dense(name, "t", t, _torch.float32, (N, K), device)
    lp = _optional(name, "labels", labels, _torch.int32, (N,), device)
    return z.data_ptr(), ld, N, V, K, ip, tp, lp


def _distill_loss(name, suffix, z, ids, t, labels, loss, stats, tau, w_kl, w_ce, workspace, stream):
    if _lib is None:
        lib()
    device = z.get_device()
    head = _targets(name, suffix, z, ids, t, labels, device)
    N, V = head[2:4]
    lp = _dense(name, "loss", loss, _torch.float32, (N,), device)
    sp = _optional(name, "stats", stats, _torch.float32, (N, 4), device)
    work = _scratch(name, workspace, "cx_distill_workspace", (N, V), device, stream)
    _call(name, *head, tau, w_kl, w_ce, lp, sp, *_span(work), cxmix._stream(stream))


def cx_distill_loss(z, ids, t, labels, loss, stats, tau: float, w_kl: float, w_ce: float, workspace=None, stream=None):
    """z: [N][V] logits; ids: int32 [N][K] and t: float32 [N][K], the teacher's top tokens and their logits; labels: int32 [N] or
    None; loss: float32 [N]; stats: float32 [N][4] for the gradient, or None."""
    _distill_loss("cx_distill_loss", "", z, ids, t, labels, loss, stats, tau, w_kl, w_ce, workspace, stream)


def cx_distill_loss_bf16(z, ids, t, labels, loss, stats, tau: float, w_kl: float, w_ce: float, workspace=None, stream=None):
    _distill_loss("cx_distill_loss_bf16", "_bf16", z, ids, t, labels, loss, stats, tau, w_kl, w_ce, workspace, stream)


def cx_distill_loss_f16(z, ids, t, labels, loss, stats, tau: float, w_kl: float, w_ce: float, workspace=None, stream=None):
    _distill_loss("cx_distill_loss_f16", "_f16", z, ids, t, labels, loss, stats, tau, w_kl, w_ce, workspace, stream)


def _distill_grad(name, suffix, z, ids, t, labels, stats, gout, dz, tau, w_kl, w_ce, stream):
    if _lib is None:
        lib()
    device = z.get_device()
    head = _targets(name, suffix, z, ids, t, labels, device)
    N, V = head[2:4]
    sp = _dense(name, "stats", stats, _torch.float32, (N, 4), device)
    gp = _dense(name, "gout", gout, _torch.float32, (N,), device)
    ld_dz = _matrix(name, "dz", dz, _dtypes[suffix], N, V, device)
    _on_device(name, device)
    _call(name, *head, tau, w_kl, w_ce, sp, gp, dz.data_ptr(), ld_dz, cxmix._stream(stream))


def cx_distill_grad(z, ids, t, labels, stats, gout, dz, tau: float, w_kl: float, w_ce: float, stream=None):
    """As cx_distill_loss, with its stats; gout: float32 [N]; dz: [N][V], may be z."""
    _distill_grad("cx_distill_grad", "", z, ids, t, labels, stats, gout, dz, tau, w_kl, w_ce, stream)


def cx_distill_grad_bf16(z, ids, t, labels, stats, gout, dz, tau: float, w_kl: float, w_ce: float, stream=None):
    _distill_grad("cx_distill_grad_bf16", "_bf16", z, ids, t, labels, stats, gout, dz, tau, w_kl, w_ce, stream)


def cx_distill_grad_f16(z, ids, t, labels, stats, gout, dz, tau: float, w_kl: float, w_ce: float, stream=None):
    _distill_grad("cx_distill_grad_f16", "_f16", z, ids, t, labels, stats, gout, dz, tau, w_kl, w_ce, stream)


def _distill_step(name, suffix, z, ids, t, labels, gout, loss, dz, tau, w_kl, w_ce, workspace, stream):
    if _lib is None:
        lib()
    device = z.get_device()
    head = _targets(name, suffix, z, ids, t, labels, device)
    N, V = head[2:4]
    gp = _dense(name, "gout", gout, _torch.float32, (N,), device)
    lp = _dense(name, "loss", loss, _torch.float32, (N,), device)
    ld_dz = _matrix(name, "dz", dz, _dtypes[suffix], N, V, device)
    work = _scratch(name, workspace, "cx_distill_workspace", (N, V), device, stream)
    _call(name, *head, tau, w_kl, w_ce, gp, lp, dz.data_ptr(), ld_dz, *_span(work), cxmix._stream(stream))


def cx_distill_step(z, ids, t, labels, gout, loss, dz, tau: float, w_kl: float, w_ce: float, workspace=None, stream=None):
    """cx_distill_loss and cx_distill_grad in one call."""
    _distill_step("cx_distill_step", "", z, ids, t, labels, gout, loss, dz, tau, w_kl, w_ce, workspace, stream)


def cx_distill_step_bf16(z, ids, t, labels, gout, loss, dz, tau: float, w_kl: float, w_ce: float, workspace=None, stream=None):
    _distill_step("cx_distill_step_bf16", "_bf16", z, ids, t, labels, gout, loss, dz, tau, w_kl, w_ce, workspace, stream)


def cx_distill_step_f16(z, ids, t, labels, gout, loss, dz, tau: float, w_kl: float, w_ce: float, workspace=None, stream=None):
    _distill_step("cx_distill_step_f16", "_f16", z, ids, t, labels, gout, loss, dz, tau, w_kl, w_ce, workspace, stream)


# ------------------------------------------------------------------------------------------------- dropout, residual and norm
def _place(name, arg, t, dtype, rows, columns, device):
    """(address, row stride) of a matrix that may be absent."""
    return (None, 0) if t is None else (t.data_ptr(), _matrix(name, arg, t, dtype, rows, columns, device))


def _rng(name, rng, p, device):
    """Address of the generator's two numbers, which a call that drops something needs."""
    return (_dense if p else _optional)(name, "rng", rng, _torch.int64, (2,), device)


def _flat(name, arg, rows, dtype, W, offset, count, device):
    """Row stride of flat rows that hold `count` parameters from `offset` on."""
    ld = _matrix(name, arg, rows, dtype, W, None, device)
    if offset < 0 or offset + count > rows.shape[1]:
        raise ValueError(f"{name}: {arg}: {count} parameters at {offset} do not fit rows of {rows.shape[1]}")
    return ld


def _workers(rows):
    """Workers whose flat rows these are; 0 for what is no matrix, which the checks after it name."""
    shape = rows.shape
    return shape[0] if len(shape) == 2 else 0


def _gradients(name, g_in, g_out, dtype, W, offset, count, device):
    """(address of g_in, address and row stride of g_out) of flat gradient rows."""
    ld = _flat(name, "g_out", g_out, dtype, W, offset, count, device)
    if g_in is not None:
        ld_in = _flat(name, "g_in", g_in, dtype, W, offset, count, device)
        if W > 1 and ld_in != ld:
            raise ValueError(f"{name}: g_in: row stride {ld_in} differs from g_out's {ld}")
    return None if g_in is None else g_in.data_ptr(), g_out.data_ptr(), ld


def _current(name, device):
    """Last check before the call: kernels run on the current device."""
    if device < 0:
        _on_device(name, device)
    if device != _device_now():
        raise ValueError(f"{name}: tensors on cuda:{device}, which is not the current device")


def _narrow(name, *sizes):
    if max(sizes) > _INT32 or min(sizes) < -_INT32:
        _too_wide(name)


def _dropout(name, suffix, x, rng, out, p, residual, stream):
    if _lib is None:
        lib()
    dtype, device = _dtypes[suffix], x.get_device()
    ldx = _matrix(name, "x", x, dtype, None, None, device)
    N, D = x.shape
    if D > _INT32:
        _too_wide(name)
    rp, ldr = _place(name, "residual", residual, dtype, N, D, device)
    ldo = _matrix(name, "out", out, dtype, N, D, device)
    gp = _dense(name, "rng", rng, _torch.int64, (2,), device)
    _current(name, device)
    _call(name, x.data_ptr(), ldx, rp, ldr, out.data_ptr(), ldo, N, D, gp, p, cxmix._stream(stream))


def cx_dropout(x, rng, out, p: float, residual=None, stream=None):
    """x, residual, out: [N][D] (out may be one of the others); rng: int64 [2] on the device, key and draw; p: share that is dropped."""
    _dropout("cx_dropout", "", x, rng, out, p, residual, stream)


def cx_dropout_bf16(x, rng, out, p: float, residual=None, stream=None):
    _dropout("cx_dropout_bf16", "_bf16", x, rng, out, p, residual, stream)


def cx_dropout_f16(x, rng, out, p: float, residual=None, stream=None):
    _dropout("cx_dropout_f16", "_f16", x, rng, out, p, residual, stream)


def _rows_of_workers(name, rows, W, D):
    """Rows of each of W workers."""
    if D > _INT32 or W > _INT32:
        _too_wide(name)
    if W == 0 or rows % W:
        raise ValueError(f"{name}: {rows} rows are not the same number of each of {W} workers")
    return rows // W


def _add_norm(name, suffix, x, residual, weights, offset, s, y, eps, inv, q, scale, p, rng, stream):
    if _lib is None:
        lib()
    dtype, device = _dtypes[suffix], x.get_device()
    ldx = _matrix(name, "x", x, dtype, None, None, device)
    rows, D = x.shape
    W = _workers(weights)
    ldw = _flat(name, "weights", weights, dtype, None, offset, D, device)
    N = _rows_of_workers(name, rows, W, D)
    rp, ldr = _place(name, "residual", residual, dtype, rows, D, device)
    sp, lds = _place(name, "s", s, dtype, rows, D, device)
    yp, ldy = _place(name, "y", y, dtype, rows, D, device)
    ip = None if inv is None else _dense(name, "inv", inv, _torch.float32, (rows,), device)
    qp, ldq, cp = None, 0, None
    if q is not None or scale is not None:
        if q is None or q.dtype not in (_torch.uint8, _torch.float8_e4m3fn):
            raise ValueError(f"{name}: q: expected uint8 or float8_e4m3fn [{rows}][{D}] beside scale")
        qp, ldq = _place(name, "q", q, q.dtype, rows, D, device)
        cp = _dense(name, "scale", scale, _torch.float32, (rows,), device)
    gp = _rng(name, rng, p, device)
    _current(name, device)
    _call(name, x.data_ptr(), ldx, rp, ldr, weights.data_ptr(), ldw, W, offset, N, D, eps, gp, p, sp, lds, yp, ldy, ip, qp, ldq, cp, cxmix._stream(stream))


def cx_add_norm(x, residual, weights, offset: int, s, y, eps: float, inv=None, q=None, scale=None, p: float = 0.0, rng=None, stream=None):
    """x, residual, s, y: [W * N][D], all but x may be None; weights: [W][ld] flat rows, a worker's at weights[w, offset : offset + D]; inv,
    scale: float32 [W * N]; q: uint8 or float8_e4m3fn [W * N][D]; p, rng: as cx_dropout, on x."""
    _add_norm("cx_add_norm", "", x, residual, weights, offset, s, y, eps, inv, q, scale, p, rng, stream)


def cx_add_norm_bf16(x, residual, weights, offset: int, s, y, eps: float, inv=None, q=None, scale=None, p: float = 0.0, rng=None, stream=None):
    _add_norm("cx_add_norm_bf16", "_bf16", x, residual, weights, offset, s, y, eps, inv, q, scale, p, rng, stream)


def cx_add_norm_f16(x, residual, weights, offset: int, s, y, eps: float, inv=None, q=None, scale=None, p: float = 0.0, rng=None, stream=None):
    _add_norm("cx_add_norm_f16", "_f16", x, residual, weights, offset, s, y, eps, inv, q, scale, p, rng, stream)


def _add_norm_grad(name, suffix, dy, s, inv, weights, offset, ds_in, ds, g_in, g_out, dx, p, rng, workspace, stream):
    if _lib is None:
        lib()
    dtype, device = _dtypes[suffix], dy.get_device()
    lddy = _matrix(name, "dy", dy, dtype, None, None, device)
    rows, D = dy.shape
    W = _workers(weights)
    ldw = _flat(name, "weights", weights, dtype, None, offset, D, device)
    N = _rows_of_workers(name, rows, W, D)
    lds = _matrix(name, "s", s, dtype, rows, D, device)
    ip = _dense(name, "inv", inv, _torch.float32, (rows,), device)
    mp, ldm = _place(name, "ds_in", ds_in, dtype, rows, D, device)
    sp, ldds = _place(name, "ds", ds, dtype, rows, D, device)
    xp, lddx = _place(name, "dx", dx, dtype, rows, D, device)
    gip, gop, ldg = _gradients(name, g_in, g_out, dtype, W, offset, D, device)
    gp = _rng(name, rng, p, device)
    _current(name, device)
    work = _scratch(name, workspace, "cx_norm_workspace", (W, N, D), device, stream)
    wp, size = _span(work)
    _call(name, dy.data_ptr(), lddy, s.data_ptr(), lds, ip, weights.data_ptr(), ldw, W, offset, N, D, mp, ldm, gp, p, sp, ldds, xp, lddx, gip, gop, ldg, wp,
          size, cxmix._stream(stream))


def cx_add_norm_grad(dy, s, inv, weights, offset: int, ds_in, ds, g_in, g_out, dx=None, p: float = 0.0, rng=None, workspace=None, stream=None):
    """s, inv: as cx_add_norm left them; ds_in: gradient of s from elsewhere, or None; ds, dx: gradients of residual and x, one of them may be
    None; g_out: [W][ld] flat gradient rows; g_in: None, g_out itself (added in place) or a second matrix with the same row stride."""
    _add_norm_grad("cx_add_norm_grad", "", dy, s, inv, weights, offset, ds_in, ds, g_in, g_out, dx, p, rng, workspace, stream)


def cx_add_norm_grad_bf16(dy, s, inv, weights, offset: int, ds_in, ds, g_in, g_out, dx=None, p: float = 0.0, rng=None, workspace=None,
                          stream=None):
    _add_norm_grad("cx_add_norm_grad_bf16", "_bf16", dy, s, inv, weights, offset, ds_in, ds, g_in, g_out, dx, p, rng, workspace, stream)


def cx_add_norm_grad_f16(dy, s, inv, weights, offset: int, ds_in, ds, g_in, g_out, dx=None, p: float = 0.0, rng=None, workspace=None,
                         stream=None):
    _add_norm_grad("cx_add_norm_grad_f16", "_f16", dy, s, inv, weights, offset, ds_in, ds, g_in, g_out, dx, p, rng, workspace, stream)


# --------------------------------------------------------------------------------------------------------- short convolution
def _by_worker(name, rows, T, W, *ends):
    """B of B * T rows, as many sequences of each of W workers."""
    B = _sequences(name, rows, T, *ends)
    if W == 0 or B % W:
        raise ValueError(f"{name}: {B} sequences are not the same number of each of {W} workers")
    return B


def _short_conv(name, suffix, x, weights, offset, y, T, K, silu, before, after, reset, stream):
    if _lib is None:
        lib()
    dtype, device = _dtypes[suffix], x.get_device()
    ldx = _matrix(name, "x", x, dtype, None, None, device)
    rows, D = x.shape
    W = _workers(weights)
    _narrow(name, D, W, K)
    B = _by_worker(name, rows, T, W, before, after)
    ldw = _flat(name, "weights", weights, dtype, None, offset, D * (K + 1), device)
    ldy = _matrix(name, "y", y, dtype, rows, D, device)
    bp = _optional(name, "before", before, dtype, (B, K - 1, D), device)
    ap = _optional(name, "after", after, dtype, (B, K - 1, D), device)
    rp = _optional(name, "reset", reset, _torch.uint8, (B, T), device)
    _current(name, device)
    _call(name, x.data_ptr(), ldx, weights.data_ptr(), ldw, W, offset, y.data_ptr(), ldy, B, T, D, K, int(bool(silu)), rp, bp, ap, cxmix._stream(stream))


def cx_short_conv(x, weights, offset: int, y, T: int, K: int, silu: bool = True, before=None, after=None, reset=None, stream=None):
    """x, y: [B * T][D]; weights: [W][ld] flat rows with taps [D][K] and biases [D] at offset; before, after: [B][K - 1][D] (may be one tensor);
    reset: uint8 [B][T]."""
    _short_conv("cx_short_conv", "", x, weights, offset, y, T, K, silu, before, after, reset, stream)


def cx_short_conv_bf16(x, weights, offset: int, y, T: int, K: int, silu: bool = True, before=None, after=None, reset=None, stream=None):
    _short_conv("cx_short_conv_bf16", "_bf16", x, weights, offset, y, T, K, silu, before, after, reset, stream)


def cx_short_conv_f16(x, weights, offset: int, y, T: int, K: int, silu: bool = True, before=None, after=None, reset=None, stream=None):
    _short_conv("cx_short_conv_f16", "_f16", x, weights, offset, y, T, K, silu, before, after, reset, stream)


def _short_conv_grad(name, suffix, x, dy, weights, offset, dx, g_in, g_out, T, K, silu, before, reset, workspace, stream):
    if _lib is None:
        lib()
    dtype, device = _dtypes[suffix], x.get_device()
    ldx = _matrix(name, "x", x, dtype, None, None, device)
    rows, D = x.shape
    W = _workers(weights)
    _narrow(name, D, W, K)
    B = _by_worker(name, rows, T, W, before)
    ldw = _flat(name, "weights", weights, dtype, None, offset, D * (K + 1), device)
    lddy = _matrix(name, "dy", dy, dtype, rows, D, device)
    lddx = _matrix(name, "dx", dx, dtype, rows, D, device)
    gip, gop, ldg = _gradients(name, g_in, g_out, dtype, W, offset, D * (K + 1), device)
    bp = _optional(name, "before", before, dtype, (B, K - 1, D), device)
    rp = _optional(name, "reset", reset, _torch.uint8, (B, T), device)
    _current(name, device)
    work = _scratch(name, workspace, "cx_conv_workspace", (W, B, T, D, K), device, stream)
    _call(name, x.data_ptr(), ldx, dy.data_ptr(), lddy, weights.data_ptr(), ldw, W, offset, dx.data_ptr(), lddx, gip, gop, ldg, B, T, D, K, int(bool(silu)),
          rp, bp, *_span(work), cxmix._stream(stream))


def cx_short_conv_grad(x, dy, weights, offset: int, dx, g_in, g_out, T: int, K: int, silu: bool = True, before=None, reset=None,
                       workspace=None, stream=None):
    """x, dy, dx: [B * T][D]; the others as cx_short_conv; g_in, g_out: as cx_add_norm_grad."""
    _short_conv_grad("cx_short_conv_grad", "", x, dy, weights, offset, dx, g_in, g_out, T, K, silu, before, reset, workspace, stream)


def cx_short_conv_grad_bf16(x, dy, weights, offset: int, dx, g_in, g_out, T: int, K: int, silu: bool = True, before=None, reset=None,
                            workspace=None, stream=None):
    _short_conv_grad("cx_short_conv_grad_bf16", "_bf16", x, dy, weights, offset, dx, g_in, g_out, T, K, silu, before, reset, workspace, stream)


def cx_short_conv_grad_f16(x, dy, weights, offset: int, dx, g_in, g_out, T: int, K: int, silu: bool = True, before=None, reset=None,
                           workspace=None, stream=None):
    _short_conv_grad("cx_short_conv_grad_f16", "_f16", x, dy, weights, offset, dx, g_in, g_out, T, K, silu, before, reset, workspace, stream)


# ------------------------------------------------------------------------------------------------------------ selective scan
def select_states(u, T: int, N: int):
    """An empty tensor for the `states` of a selective scan over u ([B * T][D]) with N states that is to have a gradient."""
    import torch
    B = u.shape[0] // T if T > 0 else 0
    return torch.empty((B, -(-T // CX_SCAN_CHUNK), u.shape[1], N), dtype=torch.float32, device=u.device)


def _select_inputs(name, dtype, u, dt, bm, cm, z, params, offset, T, device, *ends):
    """(the first arguments of both calls, B, D, N, W)"""
    ldu = _matrix(name, "u", u, dtype, None, None, device)
    rows, D = u.shape
    lddt = _matrix(name, "dt", dt, dtype, rows, D, device)
    ldb = _matrix(name, "bm", bm, dtype, rows, None, device)
    N = bm.shape[1]
    ldc = _matrix(name, "cm", cm, dtype, rows, N, device)
    zp, ldz = _place(name, "z", z, dtype, rows, D, device)
    W = _workers(params)
    if D > _INT32 or W > _INT32 or N > _INT32:
        _too_wide(name)
    B = _by_worker(name, rows, T, W, *ends)
    ldp = _flat(name, "params", params, dtype, None, offset, D * (N + 2), device)
    return (u.data_ptr(), ldu, dt.data_ptr(), lddt, bm.data_ptr(), ldb, cm.data_ptr(), ldc, zp, ldz, params.data_ptr(), ldp, W, offset), B, D, N, W


def _select_scan(name, suffix, u, dt, bm, cm, params, offset, y, T, z, h0, h_last, reset, states, workspace, stream):
    if _lib is None:
        lib()
    dtype, device, f32 = _dtypes[suffix], u.get_device(), _torch.float32
    head, B, D, N, _ = _select_inputs(name, dtype, u, dt, bm, cm, z, params, offset, T, device, h0, h_last)
    ldy = _matrix(name, "y", y, dtype, u.shape[0], D, device)
    hp = None if h0 is None else _dense(name, "h0", h0, f32, (B, D, N), device)
    lp = None if h_last is None else _dense(name, "h_last", h_last, f32, (B, D, N), device)
    sp = None if states is None else _dense(name, "states", states, f32, (B, -(-T // CX_SCAN_CHUNK), D, N), device)
    rp = None if reset is None else _dense(name, "reset", reset, _torch.uint8, (B, T), device)
    _current(name, device)
    work = _scratch(name, workspace, None if T <= 1 else "cx_select_workspace", (B, T, D, N), device, stream)
    wp, size = _span(work)
    _call(name, *head, y.data_ptr(), ldy, B, T, D, N, rp, hp, lp, sp, wp, size, cxmix._stream(stream))


def cx_select_scan(u, dt, bm, cm, params, offset: int, y, T: int, z=None, h0=None, h_last=None, reset=None, states=None, workspace=None,
                   stream=None):
    """u, dt, z, y: [B * T][D]; bm, cm: [B * T][N]; params: [W][ld] flat rows with A_log [D][N], bias [D] and skip [D] at offset; h0, h_last:
    float32 [B][D][N] (may be one tensor); reset: uint8 [B][T]; states: see select_states()."""
    _select_scan("cx_select_scan", "", u, dt, bm, cm, params, offset, y, T, z, h0, h_last, reset, states, workspace, stream)


def cx_select_scan_bf16(u, dt, bm, cm, params, offset: int, y, T: int, z=None, h0=None, h_last=None, reset=None, states=None, workspace=None,
                        stream=None):
    _select_scan("cx_select_scan_bf16", "_bf16", u, dt, bm, cm, params, offset, y, T, z, h0, h_last, reset, states, workspace, stream)


def cx_select_scan_f16(u, dt, bm, cm, params, offset: int, y, T: int, z=None, h0=None, h_last=None, reset=None, states=None, workspace=None,
                       stream=None):
    _select_scan("cx_select_scan_f16", "_f16", u, dt, bm, cm, params, offset, y, T, z, h0, h_last, reset, states, workspace, stream)


def _select_scan_grad(name, suffix, u, dt, bm, cm, params, offset, dy, du, ddt, dbm, dcm, g_in, g_out, T, states, z, dz, dh_last, dh0, reset, workspace,
                      stream):
    if _lib is None:
        lib()
    dtype, device, f32 = _dtypes[suffix], u.get_device(), _torch.float32
    head, B, D, N, W = _select_inputs(name, dtype, u, dt, bm, cm, z, params, offset, T, device, dh_last, dh0)
    rows = u.shape[0]
    if (z is None) != (dz is None):
        raise ValueError(f"{name}: z and dz go together")
    lddy = _matrix(name, "dy", dy, dtype, rows, D, device)
    lddu = _matrix(name, "du", du, dtype, rows, D, device)
    ldddt = _matrix(name, "ddt", ddt, dtype, rows, D, device)
    lddb = _matrix(name, "dbm", dbm, dtype, rows, N, device)
    lddc = _matrix(name, "dcm", dcm, dtype, rows, N, device)
    zp, lddz = _place(name, "dz", dz, dtype, rows, D, device)
    gip, gop, ldg = _gradients(name, g_in, g_out, dtype, W, offset, D * (N + 2), device)
    sp = (_dense if T > 0 else _optional)(name, "states", states, f32, (B, -(-T // CX_SCAN_CHUNK), D, N), device)
    lp = _optional(name, "dh_last", dh_last, f32, (B, D, N), device)
    hp = _optional(name, "dh0", dh0, f32, (B, D, N), device)
    rp = _optional(name, "reset", reset, _torch.uint8, (B, T), device)
    _current(name, device)
    work = _scratch(name, workspace, "cx_select_grad_workspace", (B, T, D, N), device, stream)
    _call(name, *head, dy.data_ptr(), lddy, du.data_ptr(), lddu, ddt.data_ptr(), ldddt, dbm.data_ptr(), lddb, dcm.data_ptr(), lddc, zp, lddz, gip, gop, ldg,
          B, T, D, N, rp, sp, lp, hp, *_span(work), cxmix._stream(stream))


def cx_select_scan_grad(u, dt, bm, cm, params, offset: int, dy, du, ddt, dbm, dcm, g_in, g_out, T: int, states, z=None, dz=None,
                        dh_last=None, dh0=None, reset=None, workspace=None, stream=None):
    """Gradients beside their inputs: dy, du, ddt, dz: [B * T][D]; dbm, dcm: [B * T][N]; states: as cx_select_scan filled them; dh_last, dh0:
    float32 [B][D][N]; g_in, g_out: as cx_add_norm_grad."""
    _select_scan_grad("cx_select_scan_grad", "", u, dt, bm, cm, params, offset, dy, du, ddt, dbm, dcm, g_in, g_out, T, states, z, dz,
                      dh_last, dh0, reset, workspace, stream)


def cx_select_scan_grad_bf16(u, dt, bm, cm, params, offset: int, dy, du, ddt, dbm, dcm, g_in, g_out, T: int, states, z=None, dz=None,
                             dh_last=None, dh0=None, reset=None, workspace=None, stream=None):
    _select_scan_grad("cx_select_scan_grad_bf16", "_bf16", u, dt, bm, cm, params, offset, dy, du, ddt, dbm, dcm, g_in, g_out, T, states, z,
                      dz, dh_last, dh0, reset, workspace, stream)


def cx_select_scan_grad_f16(u, dt, bm, cm, params, offset: int, dy, du, ddt, dbm, dcm, g_in, g_out, T: int, states, z=None, dz=None,
                            dh_last=None, dh0=None, reset=None, workspace=None, stream=None):
    _select_scan_grad("cx_select_scan_grad_f16", "_f16", u, dt, bm, cm, params, offset, dy, du, ddt, dbm, dcm, g_in, g_out, T, states, z, dz,
                      dh_last, dh0, reset, workspace, stream)

