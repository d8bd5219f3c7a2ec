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
import os

from . import cxmix
from .cxmix import CX_MAX_ROWS, CxError  # noqa: F401 (part of this module's interface)

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcxlm.so")

CX_MAX_TOKENS, CX_MAX_SEQUENCES, CX_MAX_VOCAB, CX_MAX_WIDTH = 1 << 26, 1 << 22, 1 << 26, 1 << 20
CX_MAX_TOP, CX_MAX_TEACHER, CX_SCAN_CHUNK = 64, 256, 16

_TYPED = ["cx_embed_lookup", "cx_embed_grad", "cx_gated_scan", "cx_gated_scan_grad", "cx_token_scores", "cx_distill_loss",
          "cx_distill_grad", "cx_distill_step"]
EXPORTS = ["cx_lm_abi_version", "cx_embed_workspace", "cx_scan_workspace", "cx_scores_workspace", "cx_distill_workspace",
           *(name + suffix for name in _TYPED for suffix in ("", "_bf16", "_f16"))]

_lib = None
_torch = None
_dtypes = {}                     # "", "_bf16", "_f16" -> the torch type of the matrices


def lib() -> ctypes.CDLL:
    """The loaded library; raises if it was not built."""
    global _lib, _torch
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
    }
    for name, args in typed.items():
        for suffix in ("", "_bf16", "_f16"):
            getattr(L, name + suffix).argtypes = args
    for name in EXPORTS:
        getattr(L, name).restype = ctypes.c_int
    _dtypes.update({"": torch.float32, "_bf16": torch.bfloat16, "_f16": torch.float16})
    _lib, _torch = L, torch
    return L


def _ok(fn: str, status: int) -> None:
    if status != 0:
        raise CxError(fn, status)


# ------------------------------------------------------------------------------------------------------------- checks
class _Checks:
    """The tensors of one call: each is checked as it is handed in; done() looks at the devices."""

    def __init__(self, name, suffix):
        lib()
        self.name, self.dtype, self.device, self.host = name, _dtypes[suffix], None, False

    def _seen(self, arg, t):
        if self.device is None:
            self.device, self.host = t.device, not t.is_cuda
        elif t.device != self.device:
            raise ValueError(f"{self.name}: buffers on different devices: {t.device} and {self.device}")
        return t.data_ptr()

    def matrix(self, arg, t, rows=None, columns=None):
        """(address, row stride) of a row-major matrix of the call's type."""
        shape = t.shape
        if t.dtype != self.dtype:
            raise ValueError(f"{self.name}: {arg}: expected {self.dtype}, got {t.dtype}")
        if len(shape) != 2 or (rows is not None and shape[0] != rows) or (columns is not None and shape[1] != columns):
            raise ValueError(f"{self.name}: {arg}: expected [{'any' if rows is None else rows}][{'any' if columns is None else columns}], "
                             f"got {list(shape)}")
        stride = t.stride()
        if (shape[1] > 1 and stride[1] != 1) or (shape[0] > 1 and stride[0] < shape[1]):
            raise ValueError(f"{self.name}: {arg}: expected row-major elements (rows that do not overlap)")
        return self._seen(arg, t), max(stride[0], shape[1]) if shape[0] > 1 else max(shape[1], 1)

    def dense(self, arg, t, dtype, *shape, optional=False):
        """Address of a contiguous tensor of exactly this type and shape."""
        if t is None:
            if optional:
                return None
            raise ValueError(f"{self.name}: {arg} is missing")
        if t.dtype != dtype:
            raise ValueError(f"{self.name}: {arg}: expected {dtype}, got {t.dtype}")
        if t.shape != shape or not t.is_contiguous():
            raise ValueError(f"{self.name}: {arg}: expected a contiguous tensor {list(shape)}, got {list(t.shape)}, strides {t.stride()}")
        return self._seen(arg, t)

    def done(self):
        if self.host:
            raise ValueError(f"{self.name}: expected device tensors")

    def scratch(self, workspace, needed, stream):
        """(tensor to keep alive, address, bytes) of the workspace; all checks are done when this is called."""
        self.done()
        if workspace is None:
            if needed == 0:
                return None, None, 0
            if stream is not None and getattr(stream, "cuda_stream", stream) != cxmix._stream(None):
                raise ValueError(f"{self.name}: a call on a stream that is not the current one brings its own workspace ({needed} bytes)")
            workspace = _torch.empty(needed, dtype=_torch.uint8, device=self.device)
        elif workspace.dtype != _torch.uint8 or not workspace.is_contiguous():
            raise ValueError(f"{self.name}: workspace: expected a contiguous uint8 tensor")
        return workspace, self._seen("workspace", workspace), workspace.numel()


def _size(fn, *args) -> int:
    n = ctypes.c_int64()
    _ok(fn, getattr(lib(), fn)(*args, ctypes.byref(n)))
    return n.value


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


# ---------------------------------------------------------------------------------------------------------- embeddings
def _lookup(suffix, x, tokens, out, offset, V, scale, stream):
    name = "cx_embed_lookup" + suffix
    k = _Checks(name, suffix)
    if tokens.dim() != 2:
        raise ValueError(f"{name}: tokens: expected int32 [W][N]")
    W, N = tokens.shape
    xp, ld = k.matrix("x", x, W)
    op, ld_out = k.matrix("out", out, W * N)
    D = out.shape[1]
    if offset < 0 or offset + V * D > x.shape[1]:
        raise ValueError(f"{name}: a table of {V} x {D} at {offset} does not fit rows of {x.shape[1]}")
    tp = k.dense("tokens", tokens, _torch.int32, W, N)
    k.done()
    _ok(name, getattr(_lib, name)(xp, ld, W, offset, V, D, tp, N, scale, op, ld_out, cxmix._stream(stream)))


def cx_embed_lookup(x, tokens, out, offset: int, V: int, scale: float = 1.0, stream=None):
    """x: [W][ld] flat rows; tokens: int32 [W][N]; out: [W * N][D].  The table of worker w is x[w, offset : offset + V * D]."""
    _lookup("", x, tokens, out, offset, V, scale, stream)


def cx_embed_lookup_bf16(x, tokens, out, offset: int, V: int, scale: float = 1.0, stream=None):
    _lookup("_bf16", x, tokens, out, offset, V, scale, stream)


def cx_embed_lookup_f16(x, tokens, out, offset: int, V: int, scale: float = 1.0, stream=None):
    _lookup("_f16", x, tokens, out, offset, V, scale, stream)


def _embed_grad(suffix, dout, tokens, g_in, g_out, offset, V, scale, workspace, stream):
    name = "cx_embed_grad" + suffix
    k = _Checks(name, suffix)
    if tokens.dim() != 2:
        raise ValueError(f"{name}: tokens: expected int32 [W][N]")
    W, N = tokens.shape
    dp, ld_dout = k.matrix("dout", dout, W * N)
    D = dout.shape[1]
    gp, ld = k.matrix("g_out", g_out, W)
    fits = g_out.shape[1]
    ip = None
    if g_in is not None:
        ip, ld_in = k.matrix("g_in", g_in, W)
        if W > 1 and ld_in != ld:
            raise ValueError(f"{name}: g_in: row stride {ld_in} differs from g_out's {ld}")
        fits = min(fits, g_in.shape[1])
    if offset < 0 or offset + V * D > fits:
        raise ValueError(f"{name}: a table of {V} x {D} at {offset} does not fit rows of {fits}")
    tp = k.dense("tokens", tokens, _torch.int32, W, N)
    keep, wp, wn = k.scratch(workspace, 0 if workspace is not None else cx_embed_workspace(W, N, V, D), stream)
    _ok(name, getattr(_lib, name)(dp, ld_dout, tp, W, N, ip, gp, ld, offset, V, D, scale, wp, wn, cxmix._stream(stream)))


def cx_embed_grad(dout, tokens, g_in, g_out, offset: int, V: int, scale: float = 1.0, workspace=None, stream=None):
    """dout: [W * N][D]; tokens: int32 [W][N]; g_out: [W][ld] flat gradient rows.  g_in: None (rows that no token names become
    zeros), g_out itself (added in place) or a second matrix with the same row stride."""
    _embed_grad("", dout, tokens, g_in, g_out, offset, V, scale, workspace, stream)


def cx_embed_grad_bf16(dout, tokens, g_in, g_out, offset: int, V: int, scale: float = 1.0, workspace=None, stream=None):
    _embed_grad("_bf16", dout, tokens, g_in, g_out, offset, V, scale, workspace, stream)


def cx_embed_grad_f16(dout, tokens, g_in, g_out, offset: int, V: int, scale: float = 1.0, workspace=None, stream=None):
    _embed_grad("_f16", dout, tokens, g_in, g_out, offset, V, scale, workspace, stream)


# ----------------------------------------------------------------------------------------------------- gated recurrence
def scan_states(f, T: int):
    """An empty tensor for the `states` of a scan over f ([B * T][D]) that is to have a gradient."""
    import torch
    B = f.shape[0] // T if T > 0 else 0
    return torch.empty((B, -(-T // CX_SCAN_CHUNK), f.shape[1]), dtype=torch.float32, device=f.device)


def _sequences(name, f, T, *ends):
    """B of a matrix of B * T rows; of empty sequences, what the states at their ends say."""
    if T > 0 and f.shape[0] % T == 0:
        return f.shape[0] // T
    if T == 0 and f.shape[0] == 0:
        return next((t.shape[0] for t in ends if t is not None), 0)
    raise ValueError(f"{name}: {f.shape[0]} rows are no sequences of {T} steps")


def _scan(suffix, f, x, y, T, h0, h_last, reset, states, workspace, stream):
    name = "cx_gated_scan" + suffix
    k = _Checks(name, suffix)
    fp, ldf = k.matrix("f", f)
    rows, D = f.shape
    B = _sequences(name, f, T, h0, h_last)
    xp, ldx = k.matrix("x", x, rows, D)
    yp, ldy = k.matrix("y", y, rows, D)
    f32 = _torch.float32
    hp = k.dense("h0", h0, f32, B, D, optional=True)
    lp = k.dense("h_last", h_last, f32, B, D, optional=True)
    sp = k.dense("states", states, f32, B, -(-T // CX_SCAN_CHUNK), D, optional=True)
    rp = k.dense("reset", reset, _torch.uint8, B, T, optional=True)
    keep, wp, wn = k.scratch(workspace, 0 if workspace is not None else cx_scan_workspace(B, T, D), stream)
    _ok(name, getattr(_lib, name)(fp, ldf, xp, ldx, yp, ldy, B, T, D, rp, hp, lp, sp, wp, wn, cxmix._stream(stream)))


def cx_gated_scan(f, x, y, T: int, h0=None, h_last=None, reset=None, states=None, workspace=None, stream=None):
    """f, x, y: [B * T][D]; h0, h_last: float32 [B][D] (may be one tensor); reset: uint8 [B][T]; states: see scan_states()."""
    _scan("", f, x, y, T, h0, h_last, reset, states, workspace, stream)


def cx_gated_scan_bf16(f, x, y, T: int, h0=None, h_last=None, reset=None, states=None, workspace=None, stream=None):
    _scan("_bf16", f, x, y, T, h0, h_last, reset, states, workspace, stream)


def cx_gated_scan_f16(f, x, y, T: int, h0=None, h_last=None, reset=None, states=None, workspace=None, stream=None):
    _scan("_f16", f, x, y, T, h0, h_last, reset, states, workspace, stream)


def _scan_grad(suffix, f, x, dy, df, dx, T, states, dh_last, dh0, reset, workspace, stream):
    name = "cx_gated_scan_grad" + suffix
    k = _Checks(name, suffix)
    fp, ldf = k.matrix("f", f)
    rows, D = f.shape
    B = _sequences(name, f, T, dh_last, dh0)
    xp, ldx = k.matrix("x", x, rows, D)
    yp, lddy = k.matrix("dy", dy, rows, D)
    dfp, lddf = k.matrix("df", df, rows, D)
    dxp, lddx = k.matrix("dx", dx, rows, D)
    f32 = _torch.float32
    sp = k.dense("states", states, f32, B, -(-T // CX_SCAN_CHUNK), D, optional=T == 0)
    lp = k.dense("dh_last", dh_last, f32, B, D, optional=True)
    hp = k.dense("dh0", dh0, f32, B, D, optional=True)
    rp = k.dense("reset", reset, _torch.uint8, B, T, optional=True)
    keep, wp, wn = k.scratch(workspace, 0 if workspace is not None else cx_scan_workspace(B, T, D), stream)
    _ok(name, getattr(_lib, name)(fp, ldf, xp, ldx, yp, lddy, dfp, lddf, dxp, lddx, B, T, D, rp, sp, lp, hp, wp, wn, cxmix._stream(stream)))


def cx_gated_scan_grad(f, x, dy, df, dx, T: int, states, dh_last=None, dh0=None, reset=None, workspace=None, stream=None):
    """f, x, dy, df, dx: [B * T][D]; states: as cx_gated_scan filled them; dh_last, dh0: float32 [B][D]; reset: uint8 [B][T]."""
    _scan_grad("", f, x, dy, df, dx, T, states, dh_last, dh0, reset, workspace, stream)


def cx_gated_scan_grad_bf16(f, x, dy, df, dx, T: int, states, dh_last=None, dh0=None, reset=None, workspace=None, stream=None):
    _scan_grad("_bf16", f, x, dy, df, dx, T, states, dh_last, dh0, reset, workspace, stream)


def cx_gated_scan_grad_f16(f, x, dy, df, dx, T: int, states, dh_last=None, dh0=None, reset=None, workspace=None, stream=None):
    _scan_grad("_f16", f, x, dy, df, dx, T, states, dh_last, dh0, reset, workspace, stream)


# ------------------------------------------------------------------------------------------------------------ token scores
def _scores(suffix, z, tokens, logp, entropy, top_ids, top_logp, scale, workspace, stream):
    name = "cx_token_scores" + suffix
    k = _Checks(name, suffix)
    zp, ld = k.matrix("z", z)
    N, V = z.shape
    f32, i32 = _torch.float32, _torch.int32
    tp = k.dense("tokens", tokens, i32, N, optional=logp is None)
    lp = k.dense("logp", logp, f32, N, optional=True)
    ep = k.dense("entropy", entropy, f32, N, optional=True)
    K = 0
    ip = pp = None
    if top_ids is not None or top_logp is not None:
        if top_ids is None or top_ids.dim() != 2:
            raise ValueError(f"{name}: top_ids: expected int32 [N][K] beside top_logp")
        K = top_ids.shape[1]
        ip = k.dense("top_ids", top_ids, i32, N, K)
        pp = k.dense("top_logp", top_logp, f32, N, K)
    keep, wp, wn = k.scratch(workspace, 0 if workspace is not None else cx_scores_workspace(N, V, K), stream)
    _ok(name, getattr(_lib, name)(zp, ld, N, V, tp, scale, lp, ep, K, ip, pp, wp, wn, cxmix._stream(stream)))


def cx_token_scores(z, tokens, logp, entropy=None, top_ids=None, top_logp=None, scale: float = 1.0, workspace=None, stream=None):
    """z: [N][V] logits; tokens: int32 [N]; logp, entropy: float32 [N]; top_ids: int32 [N][K]; top_logp: float32 [N][K]; what is
    None is not computed.  scale: 1 / temperature."""
    _scores("", z, tokens, logp, entropy, top_ids, top_logp, scale, workspace, stream)


def cx_token_scores_bf16(z, tokens, logp, entropy=None, top_ids=None, top_logp=None, scale: float = 1.0, workspace=None, stream=None):
    _scores("_bf16", z, tokens, logp, entropy, top_ids, top_logp, scale, workspace, stream)


def cx_token_scores_f16(z, tokens, logp, entropy=None, top_ids=None, top_logp=None, scale: float = 1.0, workspace=None, stream=None):
    _scores("_f16", z, tokens, logp, entropy, top_ids, top_logp, scale, workspace, stream)


# ------------------------------------------------------------------------------------------------------------- distillation
def _targets(k, z, ids, t, labels):
    zp, ld = k.matrix("z", z)
    N, V = z.shape
    if ids.dim() != 2:
        raise ValueError(f"{k.name}: ids: expected int32 [N][K]")
    K = ids.shape[1]
    ip = k.dense("ids", ids, _torch.int32, N, K)
    tp = k.dense("t", t, _torch.float32, N, K)
    lp = k.dense("labels", labels, _torch.int32, N, optional=True)
    return (zp, ld, N, V, K, ip, tp, lp)


def _distill_loss(suffix, z, ids, t, labels, loss, stats, tau, w_kl, w_ce, workspace, stream):
    name = "cx_distill_loss" + suffix
    k = _Checks(name, suffix)
    head = _targets(k, z, ids, t, labels)
    N, V = z.shape
    lp = k.dense("loss", loss, _torch.float32, N)
    sp = k.dense("stats", stats, _torch.float32, N, 4, optional=True)
    keep, wp, wn = k.scratch(workspace, 0 if workspace is not None else cx_distill_workspace(N, V), stream)
    _ok(name, getattr(_lib, name)(*head, tau, w_kl, w_ce, lp, sp, wp, wn, cxmix._stream(stream)))


def cx_distill_loss(z, ids, t, labels, loss, stats, tau: float, w_kl: float, w_ce: float, workspace=None, stream=None):
    """z: [N][V] logits; ids: int32 [N][K] and t: float32 [N][K], the teacher's top tokens and their logits; labels: int32 [N] or
    None; loss: float32 [N]; stats: float32 [N][4] for the gradient, or None."""
    _distill_loss("", z, ids, t, labels, loss, stats, tau, w_kl, w_ce, workspace, stream)


def cx_distill_loss_bf16(z, ids, t, labels, loss, stats, tau: float, w_kl: float, w_ce: float, workspace=None, stream=None):
    _distill_loss("_bf16", z, ids, t, labels, loss, stats, tau, w_kl, w_ce, workspace, stream)


def cx_distill_loss_f16(z, ids, t, labels, loss, stats, tau: float, w_kl: float, w_ce: float, workspace=None, stream=None):
    _distill_loss("_f16", z, ids, t, labels, loss, stats, tau, w_kl, w_ce, workspace, stream)


def _distill_grad(suffix, z, ids, t, labels, stats, gout, dz, tau, w_kl, w_ce, stream):
    name = "cx_distill_grad" + suffix
    k = _Checks(name, suffix)
    head = _targets(k, z, ids, t, labels)
    N, V = z.shape
    sp = k.dense("stats", stats, _torch.float32, N, 4)
    gp = k.dense("gout", gout, _torch.float32, N)
    dp, ld_dz = k.matrix("dz", dz, N, V)
    k.done()
    _ok(name, getattr(_lib, name)(*head, tau, w_kl, w_ce, sp, gp, dp, ld_dz, cxmix._stream(stream)))


def cx_distill_grad(z, ids, t, labels, stats, gout, dz, tau: float, w_kl: float, w_ce: float, stream=None):
    """As cx_distill_loss, with its stats; gout: float32 [N]; dz: [N][V], may be z."""
    _distill_grad("", z, ids, t, labels, stats, gout, dz, tau, w_kl, w_ce, stream)


def cx_distill_grad_bf16(z, ids, t, labels, stats, gout, dz, tau: float, w_kl: float, w_ce: float, stream=None):
    _distill_grad("_bf16", z, ids, t, labels, stats, gout, dz, tau, w_kl, w_ce, stream)


def cx_distill_grad_f16(z, ids, t, labels, stats, gout, dz, tau: float, w_kl: float, w_ce: float, stream=None):
    _distill_grad("_f16", z, ids, t, labels, stats, gout, dz, tau, w_kl, w_ce, stream)


def _distill_step(suffix, z, ids, t, labels, gout, loss, dz, tau, w_kl, w_ce, workspace, stream):
    name = "cx_distill_step" + suffix
    k = _Checks(name, suffix)
    head = _targets(k, z, ids, t, labels)
    N, V = z.shape
    gp = k.dense("gout", gout, _torch.float32, N)
    lp = k.dense("loss", loss, _torch.float32, N)
    dp, ld_dz = k.matrix("dz", dz, N, V)
    keep, wp, wn = k.scratch(workspace, 0 if workspace is not None else cx_distill_workspace(N, V), stream)
    _ok(name, getattr(_lib, name)(*head, tau, w_kl, w_ce, gp, lp, dp, ld_dz, wp, wn, cxmix._stream(stream)))


def cx_distill_step(z, ids, t, labels, gout, loss, dz, tau: float, w_kl: float, w_ce: float, workspace=None, stream=None):
    """cx_distill_loss and cx_distill_grad in one call."""
    _distill_step("", z, ids, t, labels, gout, loss, dz, tau, w_kl, w_ce, workspace, stream)


def cx_distill_step_bf16(z, ids, t, labels, gout, loss, dz, tau: float, w_kl: float, w_ce: float, workspace=None, stream=None):
    _distill_step("_bf16", z, ids, t, labels, gout, loss, dz, tau, w_kl, w_ce, workspace, stream)


def cx_distill_step_f16(z, ids, t, labels, gout, loss, dz, tau: float, w_kl: float, w_ce: float, workspace=None, stream=None):
    _distill_step("_f16", z, ids, t, labels, gout, loss, dz, tau, w_kl, w_ce, workspace, stream)
