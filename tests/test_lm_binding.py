"""CPU-only tests of the language-model operators' interface: the library exports what its header declares, both sides refuse
what does not fit before anything is launched, and the workspaces' sizes are sums that a caller can rely on."""
import ctypes
import os
import re

import pytest
import torch

from paper_2012_15198_amd import cxlm as lm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SUFFIXES = ["", "_bf16", "_f16"]
TYPES = {"": torch.float32, "_bf16": torch.bfloat16, "_f16": torch.float16}


def test_library_exports_every_symbol_the_header_declares():
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "cx_lm.h")).read(), flags=re.S)
    assert set(re.findall(r"\b(cx_[a-z0-9_]+)\s*\(", header)) == set(lm.EXPORTS)
    for name in lm.EXPORTS:
        assert hasattr(lm.lib(), name) and callable(getattr(lm, name)), name
    assert lm.cx_lm_abi_version() == 1
    for name, value in re.findall(r"#define (CX_\w+) (\d+|\(1 << \d+\))", header):
        assert getattr(lm, name) == eval(value), name


def test_header_is_plain_c(tmp_path):
    import subprocess
    src = tmp_path / "use.c"
    src.write_text('#include "cx_lm.h"\nint main(void) { int64_t n; return cx_lm_abi_version() != 1 || cx_embed_workspace(1, 0, 1, 1, &n) != CX_OK; }\n')
    exe, libdir = tmp_path / "use", os.path.join(ROOT, "paper_2012_15198_amd")
    subprocess.check_call(["gcc", "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe),
                           "-L", libdir, "-lcxlm", "-Wl,-rpath," + libdir])
    assert subprocess.run([str(exe)], timeout=120).returncode == 0


# ------------------------------------------------------------------------------------------- the library's own refusals
A, B, C, D, E, F, G, H, S = (k << 28 for k in range(1, 10))          # far apart, aligned; never handed to a kernel


@pytest.mark.parametrize("suffix", SUFFIXES)
def test_embed_refusals(suffix):
    size = 4 if suffix == "" else 2
    fn = getattr(lm.lib(), "cx_embed_lookup" + suffix)
    ok = dict(x=A, ld=1000, W=2, off=10, V=9, D=8, tok=B, N=5, scale=1.0, out=C, ldo=8, st=None)
    call = lambda **kw: fn(*{**ok, **kw}.values())
    assert call(x=None) == -1 and call(tok=None) == -1 and call(out=None) == -1
    for bad in (dict(W=0), dict(W=lm.CX_MAX_ROWS + 1), dict(V=0), dict(V=lm.CX_MAX_VOCAB + 1), dict(D=0), dict(D=lm.CX_MAX_WIDTH + 1), dict(N=-1),
                dict(N=lm.CX_MAX_TOKENS + 1), dict(off=-1), dict(off=929), dict(ld=81), dict(ldo=7), dict(ld=2**62), dict(ldo=2**62)):
        assert call(**bad) == -2, bad
    assert call(x=A + 1) == -5 and call(out=C + 1) == -5 and call(tok=B + 2) == -5
    assert call(out=A + 100 * size) == -6 and call(out=B) == -6
    assert call(N=0, tok=None, out=None) == 0                        # nothing to do, nothing launched

    fn2 = getattr(lm.lib(), "cx_embed_grad" + suffix)
    need = lm.cx_embed_workspace(2, 5, 9, 8)
    ok2 = dict(dout=A, ldd=8, tok=B, W=2, N=5, gi=None, go=C, ld=1000, off=10, V=9, D=8, scale=1.0, ws=D, wn=need, st=None)
    call = lambda **kw: fn2(*{**ok2, **kw}.values())
    assert call(dout=None) == -1 and call(tok=None) == -1 and call(go=None) == -1 and call(ws=None) == -1
    for bad in (dict(W=0), dict(V=0), dict(D=0), dict(N=-1), dict(off=-1), dict(off=929), dict(ldd=7), dict(wn=need - 1), dict(wn=-1)):
        assert call(**bad) == -2, bad
    assert call(go=C + 1) == -5 and call(dout=A + 1) == -5 and call(gi=E + 1) == -5 and call(ws=D + 8) == -5
    assert call(go=A) == -6 and call(gi=C + 8 * size) == -6 and call(ws=C) == -6 and call(ws=A) == -6 and call(go=B) == -6


@pytest.mark.parametrize("suffix", SUFFIXES)
def test_scan_refusals(suffix):
    fn = getattr(lm.lib(), "cx_gated_scan" + suffix)
    ok = dict(f=A, ldf=8, x=B, ldx=8, y=C, ldy=8, B=2, T=40, D=8, reset=None, h0=None, hl=None, states=None, ws=S, wn=1 << 20, st=None)
    call = lambda **kw: fn(*{**ok, **kw}.values())
    assert call(f=None) == -1 and call(x=None) == -1 and call(y=None) == -1
    for bad in (dict(B=-1), dict(T=-1), dict(D=0), dict(ldf=7), dict(ldx=7), dict(ldy=7), dict(T=lm.CX_MAX_TOKENS + 1), dict(D=lm.CX_MAX_WIDTH + 1),
                dict(B=lm.CX_MAX_SEQUENCES + 1)):
        assert call(**bad) == -2, bad
    assert call(T=4000, ws=None) == -1 and call(T=4000, wn=4) == -2       # split: needs its workspace
    assert call(f=A + 1) == -5 and call(h0=D + 2) == -5 and call(states=E + 2) == -5
    assert call(y=A) == -6 and call(y=B) == -6 and call(h0=C) == -6 and call(h0=D, hl=D + 4) == -6 and call(states=C + 64) == -6
    assert call(h0=D, states=D) == -6 and call(reset=C) == -6
    assert call(B=0) == 0

    fn2 = getattr(lm.lib(), "cx_gated_scan_grad" + suffix)
    ok2 = dict(f=A, ldf=8, x=B, ldx=8, dy=C, lddy=8, df=D, lddf=8, dx=E, lddx=8, B=2, T=40, D=8, reset=None, states=F, dl=None, d0=None, ws=S, wn=1 << 20,
               st=None)
    call = lambda **kw: fn2(*{**ok2, **kw}.values())
    for p in ("f", "x", "dy", "df", "dx", "states"):
        assert call(**{p: None}) == -1, p
    assert call(lddf=7) == -2 and call(T=4000, ws=None) == -1 and call(df=D + 1) == -5
    for bad in (dict(df=A), dict(dx=B), dict(df=C), dict(dx=D), dict(df=F), dict(d0=F), dict(dl=D), dict(dl=G, d0=G + 4)):
        assert call(**bad) == -6, bad
    # halves of the rows of one matrix do not share an element; halves that cross do
    size = 4 if suffix == "" else 2
    assert call(B=0, df=D, lddf=16, dx=D + 8 * size, lddx=16) == 0
    assert call(df=D, lddf=16, dx=D + 7 * size, lddx=16) == -6 and call(df=D, lddf=16, dx=D + 9 * size, lddx=16) == -6
    assert call(df=D, lddf=16, dx=D + 8 * size, lddx=17) == -6


@pytest.mark.parametrize("suffix", SUFFIXES)
def test_scores_and_distill_refusals(suffix):
    fn = getattr(lm.lib(), "cx_token_scores" + suffix)
    ok = dict(z=A, ld=50, N=600, V=50, tok=B, scale=1.0, logp=C, ent=D, K=4, ids=E, top=F, ws=None, wn=0, st=None)
    call = lambda **kw: fn(*{**ok, **kw}.values())
    assert call(z=None) == -1 and call(tok=None) == -1 and call(ids=None) == -1 and call(top=None) == -1
    for bad in (dict(N=-1), dict(V=0), dict(K=-1), dict(K=lm.CX_MAX_TOP + 1), dict(K=51, V=50), dict(ld=49), dict(scale=0.0), dict(scale=-1.0),
                dict(scale=float("nan")), dict(scale=float("inf"))):
        assert call(**bad) == -2, bad
    long = dict(N=1, V=4_000_000, ld=4_000_000)                           # split, so that a workspace is needed
    assert lm.cx_scores_workspace(1, 4_000_000, 4) > 0 and lm.cx_distill_workspace(1, 4_000_000) > 0
    assert call(**long) == -1 and call(**long, ws=S, wn=8) == -2
    assert call(z=A + 1) == -5 and call(logp=C + 2) == -5
    assert call(logp=A) == -6 and call(ent=C) == -6 and call(top=E) == -6 and call(ids=B) == -6
    assert call(N=0, z=None) == 0

    names = ("z", "ld", "N", "V", "K", "ids", "t", "lab", "tau", "kl", "ce")
    head = dict(zip(names, (A, 50, 600, 50, 4, B, C, D, 2.0, 0.5, 0.5)))
    loss = lambda **kw: getattr(lm.lib(), "cx_distill_loss" + suffix)(*{**head, "loss": E, "stats": F, "ws": None, "wn": 0, "st": None, **kw}.values())
    grad = lambda **kw: getattr(lm.lib(), "cx_distill_grad" + suffix)(*{**head, "stats": F, "gout": E, "dz": G, "lddz": 50, "st": None, **kw}.values())
    step = lambda **kw: getattr(lm.lib(), "cx_distill_step" + suffix)(*{**head, "gout": E, "loss": F, "dz": G, "lddz": 50, "ws": None, "wn": 0, "st": None,
                                                                        **kw}.values())
    for call in (loss, grad, step):
        assert call(z=None) == -1 and call(ids=None) == -1 and call(t=None) == -1
        for bad in (dict(N=-1), dict(V=0), dict(K=-1), dict(K=lm.CX_MAX_TEACHER + 1), dict(ld=49), dict(tau=0.0), dict(tau=float("nan")), dict(kl=-1.0),
                    dict(ce=float("inf")), dict(ce=float("nan"))):
            assert call(**bad) == -2, bad
        assert call(z=A + 1) == -5 and call(t=C + 2) == -5
        assert call(N=0, z=None) == 0
    assert loss(loss=None) == -1 and grad(stats=None) == -1 and grad(dz=None) == -1 and grad(gout=None) == -1 and step(loss=None) == -1
    assert loss(loss=A) == -6 and loss(stats=E) == -6 and grad(dz=B) == -6 and step(dz=F) == -6 and step(loss=E) == -6
    assert grad(dz=A + 100) == -6 and step(dz=A, lddz=51) == -6           # in place means exactly there
    assert step(lddz=49) == -2 and step(**long, lddz=4_000_000) == -1 and loss(**long) == -1
    assert step(**long, lddz=4_000_000, ws=S, wn=8) == -2 and loss(**long, ws=S, wn=8) == -2


def test_workspace_sizes():
    n = ctypes.c_int64(5)
    assert lm.lib().cx_embed_workspace(0, 1, 1, 1, ctypes.byref(n)) == -2 and n.value == 0
    assert lm.lib().cx_embed_workspace(1, 1, 1, 1, None) == -1 and lm.lib().cx_scan_workspace(1, 1, 1, None) == -1
    assert lm.lib().cx_scores_workspace(1, 1, 1, None) == -1 and lm.lib().cx_distill_workspace(1, 1, None) == -1
    assert lm.cx_embed_workspace(2, 100, 10, 8) >= 2 * 11 * 4 + 2 * 100 * 4 + 2 * 2 * 2 * 8 * 4
    assert lm.cx_scan_workspace(4, 1, 64) == 0 and lm.cx_scan_workspace(1, 100_000, 64) > 0 and lm.cx_scan_workspace(0, 5, 1) == 0
    assert lm.cx_scores_workspace(10_000, 50_000, 4) == 0 and lm.cx_distill_workspace(10_000, 50_000) == 0
    assert lm.cx_scores_workspace(1, 4_000_000, 4) > 0 and lm.cx_distill_workspace(1, 4_000_000) > 0
    with pytest.raises(lm.CxError, match="CX_ERR_SHAPE"):
        lm.cx_scores_workspace(1, 10, 11)


# -------------------------------------------------------------------------------------------------- the binding's checks
def t(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype)


def ints(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def refuses(fn, *args, match, **kw):
    with pytest.raises(ValueError, match=match):
        fn(*args, **kw)


@pytest.mark.parametrize("suffix", SUFFIXES)
def test_binding_refuses_what_does_not_fit(suffix):
    """Host tensors: the device check comes last, so the all-correct call raises that one and every mismatch is reachable."""
    ty = TYPES[suffix]
    other = torch.float64
    m = lambda *s: t(*s, dtype=ty)
    fn = getattr(lm, "cx_embed_lookup" + suffix)
    refuses(fn, m(2, 100), ints(2, 3), m(6, 8), 4, 12, match="device tensors")
    refuses(fn, m(2, 99), ints(2, 3), m(6, 8), 4, 12, match="does not fit")
    refuses(fn, m(2, 100), ints(2, 3), m(6, 8), -1, 12, match="does not fit")
    refuses(fn, m(3, 100), ints(2, 3), m(6, 8), 4, 12, match="x: expected")
    refuses(fn, m(2, 100), ints(2, 3), m(5, 8), 4, 12, match="out: expected")
    refuses(fn, t(2, 100, dtype=other), ints(2, 3), m(6, 8), 4, 12, match="x: expected torch")
    refuses(fn, m(2, 100), ints(2, 3).long(), m(6, 8), 4, 12, match="tokens: expected")
    refuses(fn, m(2, 100), ints(2, 6)[:, ::2], m(6, 8), 4, 12, match="tokens: expected")
    refuses(fn, m(2, 200)[:, ::2], ints(2, 3), m(6, 8), 4, 12, match="row-major")
    refuses(fn, m(1, 100).expand(2, 100), ints(2, 3), m(6, 8), 4, 12, match="do not overlap")

    fn = getattr(lm, "cx_embed_grad" + suffix)
    refuses(fn, m(6, 8), ints(2, 3), None, m(2, 100), 4, 12, match="device tensors")
    refuses(fn, m(6, 8), ints(2, 3), m(2, 120), m(2, 100), 4, 12, match="row stride")
    refuses(fn, m(6, 8), ints(2, 3), m(2, 100)[:, :50], m(2, 100), 4, 12, match="does not fit")
    refuses(fn, m(7, 8), ints(2, 3), None, m(2, 100), 4, 12, match="dout: expected")

    fn = getattr(lm, "cx_gated_scan" + suffix)
    refuses(fn, m(6, 8), m(6, 8), m(6, 8), 3, match="device tensors")
    refuses(fn, m(6, 8), m(6, 8), m(6, 8), 4, match="no sequences")
    refuses(fn, m(6, 8), m(6, 8), m(6, 8), 0, match="no sequences")
    refuses(fn, m(6, 8), m(6, 9), m(6, 8), 3, match="x: expected")
    refuses(fn, m(6, 8), m(6, 8), m(6, 8), 3, h0=t(2, 9), match="h0: expected")
    refuses(fn, m(6, 8), m(6, 8), m(6, 8), 3, h0=t(2, 8, dtype=other), match="h0: expected")
    refuses(fn, m(6, 8), m(6, 8), m(6, 8), 3, reset=torch.zeros((2, 3), dtype=torch.bool), match="reset: expected")
    refuses(fn, m(6, 8), m(6, 8), m(6, 8), 3, states=t(2, 2, 8), match="states: expected")
    fn = getattr(lm, "cx_gated_scan_grad" + suffix)
    ok = (m(6, 8), m(6, 8), m(6, 8), m(6, 8), m(6, 8), 3)
    refuses(fn, *ok, t(2, 1, 8), match="device tensors")
    refuses(fn, *ok, None, match="states is missing")
    refuses(fn, *ok, t(2, 1, 7), match="states: expected")

    fn = getattr(lm, "cx_token_scores" + suffix)
    refuses(fn, m(4, 9), ints(4), t(4), t(4), ints(4, 2), t(4, 2), match="device tensors")
    refuses(fn, m(4, 9), None, t(4), match="tokens is missing")
    refuses(fn, m(4, 9), ints(4), t(4), t(4), None, t(4, 2), match="top_ids")
    refuses(fn, m(4, 9), ints(4), t(4), t(4), ints(4, 2), None, match="top_logp is missing")
    refuses(fn, m(4, 9), ints(4), t(4), t(4), ints(4, 2), t(4, 3), match="top_logp: expected")
    refuses(fn, m(4, 9), ints(5), t(4), match="tokens: expected")

    loss = getattr(lm, "cx_distill_loss" + suffix)
    refuses(loss, m(4, 9), ints(4, 2), t(4, 2), ints(4), t(4), t(4, 4), 1.0, 1.0, 1.0, match="device tensors")
    refuses(loss, m(4, 9), ints(4, 2), t(4, 3), ints(4), t(4), t(4, 4), 1.0, 1.0, 1.0, match="t: expected")
    refuses(loss, m(4, 9), ints(8), t(4, 2), ints(4), t(4), t(4, 4), 1.0, 1.0, 1.0, match="ids: expected")
    refuses(loss, m(4, 9), ints(4, 2), t(4, 2), ints(4), t(4), t(4, 3), 1.0, 1.0, 1.0, match="stats: expected")
    grad = getattr(lm, "cx_distill_grad" + suffix)
    refuses(grad, m(4, 9), ints(4, 2), t(4, 2), ints(4), t(4, 4), t(4), m(4, 9), 1.0, 1.0, 1.0, match="device tensors")
    refuses(grad, m(4, 9), ints(4, 2), t(4, 2), ints(4), t(4, 4), t(4), m(4, 8), 1.0, 1.0, 1.0, match="dz: expected")
    step = getattr(lm, "cx_distill_step" + suffix)
    refuses(step, m(4, 9), ints(4, 2), t(4, 2), None, t(4), t(4), m(4, 9), 1.0, 1.0, 1.0, match="device tensors")
    refuses(step, m(4, 9), ints(4, 2), t(4, 2), None, None, t(4), m(4, 9), 1.0, 1.0, 1.0, match="gout is missing")
