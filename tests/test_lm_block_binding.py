"""CPU-only tests of the residual block's operators' interface: both sides refuse what does not fit before anything is launched, every overlap that
the header excludes among it, and the workspaces' sizes are sums that a caller can rely on."""
import ctypes
import math

import pytest
import torch

from paper_2012_15198_amd import cxlm as lm

SUFFIXES = ["", "_bf16", "_f16"]
TYPES = {"": torch.float32, "_bf16": torch.bfloat16, "_f16": torch.float16}
SIZE = {"": 4, "_bf16": 2, "_f16": 2}
PLACES = [k << 28 for k in range(1, 32)]                             # far apart, aligned; never handed to a kernel
ROOM = 1 << 26


def caller(name, suffix, **ok):
    fn = getattr(lm.lib(), name + suffix)
    return lambda **kw: fn(*{**ok, **kw}.values())


def dropout(suffix):
    x, r, o, g = PLACES[:4]
    return caller("cx_dropout", suffix, x=x, ldx=8, r=r, ldr=8, out=o, ldo=8, N=6, D=8, rng=g, p=0.5, st=None)


def add_norm(suffix):
    x, r, w, g, s, y, inv, q, sc = PLACES[:9]
    return caller("cx_add_norm", suffix, x=x, ldx=8, r=r, ldr=8, w=w, ldw=20, W=2, off=3, N=5, D=8, eps=1e-6, rng=g, p=0.5, s=s, lds=8, y=y, ldy=8, inv=inv, q=q,
                  ldq=8, scale=sc, st=None)


def add_norm_grad(suffix):
    dy, s, inv, w, di, g, ds, dx, gi, go, ws = PLACES[:11]
    return caller("cx_add_norm_grad", suffix, dy=dy, lddy=8, s=s, lds=8, inv=inv, w=w, ldw=20, W=2, off=3, N=5, D=8, di=di, ldi=8, rng=g, p=0.5, ds=ds, ldds=8,
                  dx=dx, lddx=8, gi=gi, go=go, ldg=20, ws=ws, wn=ROOM, st=None)


def conv(suffix):
    x, w, y, reset, before, after = PLACES[:6]
    return caller("cx_short_conv", suffix, x=x, ldx=8, w=w, ldw=50, W=2, off=3, y=y, ldy=8, B=4, T=40, D=8, K=4, silu=1, reset=reset, before=before, after=after,
                  st=None)


def conv_grad(suffix):
    x, dy, w, dx, gi, go, reset, before, ws = PLACES[:9]
    return caller("cx_short_conv_grad", suffix, x=x, ldx=8, dy=dy, lddy=8, w=w, ldw=50, W=2, off=3, dx=dx, lddx=8, gi=gi, go=go, ldg=50, B=4, T=40, D=8, K=4,
                  silu=1, reset=reset, before=before, ws=ws, wn=ROOM, st=None)


def select(suffix, T=400):
    u, dt, bm, cm, z, w, y, reset, h0, hl, st, ws = PLACES[:12]
    return caller("cx_select_scan", suffix, u=u, ldu=8, dt=dt, lddt=8, bm=bm, ldb=5, cm=cm, ldc=5, z=z, ldz=8, w=w, ldw=60, W=2, off=3, y=y, ldy=8, B=4, T=T, D=8, N=5,
                  reset=reset, h0=h0, hl=hl, states=st, ws=ws, wn=ROOM, st=None)


def select_grad(suffix):
    u, dt, bm, cm, z, w, dy, du, ddt, db, dc, dz, gi, go, reset, st, dl, d0, ws = PLACES[:19]
    return caller("cx_select_scan_grad", suffix, u=u, ldu=8, dt=dt, lddt=8, bm=bm, ldb=5, cm=cm, ldc=5, z=z, ldz=8, w=w, ldw=60, W=2, off=3, dy=dy, lddy=8, du=du,
                  lddu=8, ddt=ddt, ldddt=8, db=db, lddb=5, dc=dc, lddc=5, dz=dz, lddz=8, gi=gi, go=go, ldg=60, B=4, T=400, D=8, N=5, reset=reset, states=st, dl=dl,
                  d0=d0, ws=ws, wn=ROOM, st=None)


def refuses_overlaps(call, ok, ins, outs, allowed):
    """ok: the places of the buffers by name."""
    for out in outs:
        for other in (*ins, *outs):
            if other != out and (out, other) not in allowed and (other, out) not in allowed:
                assert call(**{out: ok[other]}) == -6, (out, other)


def places(call):
    """The default places of a caller's buffers, by name."""
    cells = dict(zip(call.__code__.co_freevars, (c.cell_contents for c in call.__closure__)))
    return {k: v for k, v in cells["ok"].items() if isinstance(v, int) and v in PLACES}


@pytest.mark.parametrize("suffix", SUFFIXES)
def test_dropout_refusals(suffix):
    call, size = dropout(suffix), SIZE[suffix]
    for p in ("x", "out", "rng"):
        assert call(**{p: None}) == -1, p
    for bad in (dict(N=-1), dict(N=(1 << 31) + 1), dict(D=0), dict(D=lm.CX_MAX_WIDTH + 1), dict(ldx=7), dict(ldr=7), dict(ldo=7), dict(p=-0.1), dict(p=1.0),
                dict(p=float("nan")), dict(p=0.999999), dict(N=1 << 30, D=64, ldx=64, ldr=64, ldo=64)):
        assert call(**bad) == -2, bad
    assert call(x=PLACES[0] + 1) == -5 and call(rng=PLACES[3] + 4) == -5
    refuses_overlaps(call, places(call), ["rng"], ["out"], [])
    assert call(out=PLACES[0] + 8 * size) == -6 and call(out=PLACES[1] + size) == -6 and call(out=PLACES[0], ldo=9) == -6
    assert call(N=0, x=None) == 0


@pytest.mark.parametrize("suffix", SUFFIXES)
def test_norm_refusals(suffix):
    call, size = add_norm(suffix), SIZE[suffix]
    assert call(x=None) == -1 and call(w=None) == -1 and call(rng=None) == -1 and call(scale=None) == -1 and call(s=None, y=None, q=None) == -1
    for bad in (dict(W=0), dict(W=lm.CX_MAX_ROWS + 1), dict(N=-1), dict(N=lm.CX_MAX_TOKENS + 1), dict(D=0), dict(D=lm.CX_MAX_NORM_WIDTH + 1, ldx=1 << 20), dict(off=-1),
                dict(off=13), dict(ldx=7), dict(ldr=7), dict(lds=7), dict(ldy=7), dict(ldq=7), dict(eps=-1e-9), dict(eps=math.inf), dict(eps=math.nan), dict(p=1.0)):
        assert call(**bad) == -2, bad
    for p in ("x", "r", "w", "s", "y", "inv", "scale"):
        assert call(**{p: places(call)[p] + 1}) == -5, p
    refuses_overlaps(call, places(call), ["x", "r", "w", "rng"], ["s", "y", "inv", "q", "scale"], [("s", "x"), ("s", "r"), ("y", "x")])
    assert call(s=PLACES[0] + size) == -6 and call(y=PLACES[0], ldy=9) == -6 and call(s=PLACES[0], y=PLACES[0]) == -6
    assert call(N=0, x=None) == 0

    call = add_norm_grad(suffix)
    for p in ("dy", "s", "inv", "w", "rng", "go", "ws"):
        assert call(**{p: None}) == -1, p
    assert call(ds=None, dx=None) == -1
    for bad in (dict(W=0), dict(D=0), dict(off=13), dict(ldg=10), dict(lddy=7), dict(ldi=7), dict(ldds=7), dict(lddx=7), dict(lds=7), dict(p=-1.0),
                dict(wn=lm.cx_norm_workspace(2, 5, 8) - 1)):
        assert call(**bad) == -2, bad
    for p in ("dy", "s", "inv", "w", "di", "ds", "dx", "gi", "go", "ws"):
        assert call(**{p: places(call)[p] + 1}) == -5, p
    refuses_overlaps(call, places(call), ["dy", "s", "inv", "w", "di", "rng", "gi"], ["ds", "dx", "go", "ws"],
                     [("ds", "dy"), ("ds", "di"), ("dx", "dy"), ("dx", "di"), ("go", "gi")])
    assert call(N=0, dy=None, gi=PLACES[9]) == 0


@pytest.mark.parametrize("suffix", SUFFIXES)
def test_conv_refusals(suffix):
    call = conv(suffix)
    for p in ("x", "w", "y"):
        assert call(**{p: None}) == -1, p
    common = (dict(W=0), dict(W=3), dict(B=-2), dict(T=-1), dict(T=lm.CX_MAX_TOKENS + 1), dict(D=0), dict(D=lm.CX_MAX_WIDTH + 1), dict(K=0), dict(K=lm.CX_MAX_TAPS + 1),
              dict(off=-1), dict(off=11), dict(ldx=7), dict(B=2 * lm.CX_MAX_SEQUENCES))
    for bad in (*common, dict(ldy=7)):
        assert call(**bad) == -2, bad
    for p in ("x", "w", "y", "before", "after"):
        assert call(**{p: places(call)[p] + 1}) == -5, p
    refuses_overlaps(call, places(call), ["x", "w", "reset", "before"], ["y", "after"], [("after", "before")])
    assert call(after=PLACES[4] + SIZE[suffix]) == -6 and call(B=0, x=None) == 0
    call = conv_grad(suffix)
    for p in ("x", "dy", "w", "dx", "go", "ws"):
        assert call(**{p: None}) == -1, p
    for bad in (*common, dict(lddy=7), dict(lddx=7), dict(ldg=40), dict(wn=lm.cx_conv_workspace(2, 4, 40, 8, 4) - 1)):
        assert call(**bad) == -2, bad
    for p in ("x", "dy", "w", "dx", "before", "gi", "go", "ws"):
        assert call(**{p: places(call)[p] + 1}) == -5, p
    refuses_overlaps(call, places(call), ["x", "dy", "w", "reset", "before", "gi"], ["dx", "go", "ws"], [("go", "gi")])
    assert call(B=0, x=None, gi=PLACES[5]) == 0 and call(T=0, x=None, gi=PLACES[5]) == 0


@pytest.mark.parametrize("suffix", SUFFIXES)
def test_select_refusals(suffix):
    assert lm.cx_select_workspace(4, 400, 8, 5) > 0
    call = select(suffix)
    for p in ("u", "dt", "bm", "cm", "w", "y", "ws"):
        assert call(**{p: None}) == -1, p
    common = (dict(W=0), dict(W=3), dict(B=-2), dict(T=-1), dict(T=lm.CX_MAX_TOKENS + 1), dict(D=0), dict(N=0), dict(N=lm.CX_MAX_STATES + 1, ldb=99, ldc=99), dict(off=-1),
              dict(off=5), dict(ldu=7), dict(lddt=7), dict(ldb=4), dict(ldc=4), dict(ldz=7), dict(ldu=(1 << 24) + 1), dict(B=2 * lm.CX_MAX_SEQUENCES),
              dict(B=(1 << 20) + 2, D=512))
    for bad in (*common, dict(ldy=7), dict(wn=lm.cx_select_workspace(4, 400, 8, 5) - 1)):
        assert call(**bad) == -2, bad
    for p in ("u", "dt", "bm", "cm", "z", "w", "y", "h0", "hl", "states", "ws"):
        assert call(**{p: places(call)[p] + 1}) == -5, p
    ins, outs = ["u", "dt", "bm", "cm", "z", "w", "reset", "h0"], ["y", "hl", "states"]
    refuses_overlaps(call, places(call), ins, outs + ["ws"], [("hl", "h0")])
    for T in (1, 40):
        refuses_overlaps(select(suffix, T), places(call), ins, outs, [("hl", "h0")])
    assert call(hl=PLACES[8] + 4) == -6 and call(B=0, u=None) == 0
    call = select_grad(suffix)
    for p in ("u", "dt", "bm", "cm", "w", "dy", "du", "ddt", "db", "dc", "go", "states", "ws"):
        assert call(**{p: None}) == -1, p
    assert call(z=None) == -1 and call(dz=None) == -1
    for bad in (*common, dict(lddy=7), dict(lddu=7), dict(ldddt=7), dict(lddb=4), dict(lddc=4), dict(lddz=7), dict(ldg=40), dict(lddy=(1 << 24) + 1),
                dict(wn=lm.cx_select_grad_workspace(4, 400, 8, 5) - 1)):
        assert call(**bad) == -2, bad
    for p in ("u", "dt", "bm", "cm", "z", "w", "dy", "du", "ddt", "db", "dc", "dz", "gi", "go", "states", "dl", "d0", "ws"):
        assert call(**{p: places(call)[p] + 1}) == -5, p
    refuses_overlaps(call, places(call), ["u", "dt", "bm", "cm", "z", "w", "dy", "reset", "states", "dl", "gi"], ["du", "ddt", "db", "dc", "dz", "go", "d0", "ws"],
                     [("d0", "dl"), ("go", "gi")])
    assert call(d0=PLACES[16] + 4) == -6 and call(B=0, u=None, gi=PLACES[13]) == 0


def test_parts_of_one_wide_matrix_do_not_overlap():
    """Rows of [x | gate | its gradients] and of [dt | B | C]: neighbours are taken (no sequence is left to work on), crossing by one element is not."""
    u, size = PLACES[20], 4
    call = select_grad("")
    apart = dict(u=u, ldu=42, du=u + 8 * size, lddu=42, dt=u + 16 * size, lddt=42, ddt=u + 24 * size, ldddt=42, db=u + 32 * size, lddb=42, dc=u + 37 * size, lddc=42)
    assert call(**apart, ws=PLACES[18] + 1) == -5                    # the last check before the overlaps
    for name in ("du", "ddt", "db", "dc"):
        for off in (-1, 1):
            assert call(**{**apart, name: apart[name] + off * size}) == -6, (name, off)


def test_workspace_sizes():
    n = ctypes.c_int64(5)
    for name, args in (("cx_norm_workspace", (1, 1, 1)), ("cx_conv_workspace", (1, 1, 1, 1, 1)), ("cx_select_workspace", (1, 1, 1, 1)), ("cx_select_grad_workspace", (1, 1, 1, 1))):
        fn = getattr(lm.lib(), name)
        assert fn(*args, None) == -1 and fn(*args[:-1], -1, ctypes.byref(n)) == -2 and n.value == 0
        for k in range(len(args)):
            for wide in (2**32 + 9, 9 - 2**32, 2**64 + 9):
                with pytest.raises(lm.CxError, match="CX_ERR_SHAPE"):
                    getattr(lm, name)(*args[:k], wide, *args[k + 1:])
    assert lm.cx_norm_workspace(2, 0, 8) == 0 and lm.cx_norm_workspace(2, 5, 8) >= 2 * 8 * 4
    assert lm.cx_conv_workspace(2, 0, 9, 8, 4) == 0 and lm.cx_conv_workspace(2, 4, 40, 8, 4) >= 4 * 8 * 5 * 4
    assert lm.cx_select_workspace(4, 1, 64, 16) == 0 and lm.cx_select_workspace(1, 100_000, 64, 16) > 0 and lm.cx_select_workspace(2000, 64, 64, 16) == 0
    assert lm.cx_select_grad_workspace(4, 1, 64, 16) >= 4 * (2 * 16 + 64 * 18) * 4 and lm.cx_select_grad_workspace(0, 7, 1, 1) == 0


# -------------------------------------------------------------------------------------------------- the binding's checks
def t(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype)


def refuses(fn, *args, match, **kw):
    with pytest.raises(ValueError, match=match):
        fn(*args, **kw)


@pytest.mark.parametrize("suffix", SUFFIXES)
def test_binding_refuses_what_does_not_fit(suffix):
    """Host tensors: the device check comes last, so the all-correct call raises that one and every mismatch is reachable."""
    ty, other = TYPES[suffix], torch.float64
    m = lambda *s: t(*s, dtype=ty)
    rng, bytes_ = t(2, dtype=torch.int64), lambda *s: t(*s, dtype=torch.uint8)
    fn = getattr(lm, "cx_dropout" + suffix)
    refuses(fn, m(4, 9), rng, m(4, 9), 0.5, residual=m(4, 9), match="device tensors")
    refuses(fn, m(4, 9), None, m(4, 9), 0.5, match="rng is missing")
    refuses(fn, m(4, 9), rng.int(), m(4, 9), 0.5, match="rng: expected")
    refuses(fn, m(4, 9), rng, m(4, 8), 0.5, match="out: expected")
    refuses(fn, m(4, 9), rng, m(4, 9), 0.5, residual=m(5, 9), match="residual: expected")
    refuses(fn, m(4, 18)[:, ::2], rng, m(4, 9), 0.5, match="row-major")

    fn = getattr(lm, "cx_add_norm" + suffix)
    ok = (m(6, 9), m(6, 9), m(2, 20), 5, m(6, 9), m(6, 9), 1e-6)
    refuses(fn, *ok, inv=t(6), q=bytes_(6, 9), scale=t(6), match="device tensors")
    refuses(fn, m(5, 9), None, m(2, 20), 5, None, m(5, 9), 1e-6, match="same number")
    refuses(fn, *ok[:3], 12, *ok[4:], match="do not fit")
    refuses(fn, *ok[:3], -1, *ok[4:], match="do not fit")
    refuses(fn, *ok[:2], t(2, 20, dtype=other), *ok[3:], match="weights: expected")
    refuses(fn, *ok[:4], m(6, 8), *ok[5:], match="s: expected")
    refuses(fn, *ok, inv=t(5), match="inv: expected")
    refuses(fn, *ok, q=bytes_(6, 9), match="scale is missing")
    refuses(fn, *ok, scale=t(6), match="q: expected")
    refuses(fn, *ok, q=t(6, 9, dtype=torch.int8), scale=t(6), match="q: expected")
    refuses(fn, *ok, p=0.5, match="rng is missing")
    fn = getattr(lm, "cx_add_norm_grad" + suffix)
    ok = (m(6, 9), m(6, 9), t(6), m(2, 20), 5, m(6, 9), m(6, 9), None, m(2, 30))
    refuses(fn, *ok, dx=m(6, 9), match="device tensors")
    refuses(fn, *ok[:2], None, *ok[3:], match="inv is missing")
    refuses(fn, *ok[:8], m(3, 30), match="g_out: expected")
    refuses(fn, *ok[:8], m(2, 13), match="do not fit")
    refuses(fn, *ok[:7], m(2, 31), m(2, 30), match="row stride")
    refuses(fn, *ok, dx=m(6, 8), match="dx: expected")
    refuses(fn, *ok, p=0.5, match="rng is missing")

    fn = getattr(lm, "cx_short_conv" + suffix)
    ok = (m(12, 9), m(2, 60), 5, m(12, 9), 3, 4)
    refuses(fn, *ok, before=m(4, 3, 9), after=m(4, 3, 9), reset=bytes_(4, 3), match="device tensors")
    refuses(fn, *ok[:4], 5, 4, match="no sequences")
    refuses(fn, m(9, 9), *ok[1:3], m(9, 9), 3, 4, match="same number")
    refuses(fn, *ok[:2], 16, *ok[3:], match="do not fit")
    refuses(fn, *ok, before=m(4, 4, 9), match="before: expected")
    refuses(fn, *ok, after=t(4, 3, 9, dtype=other), match="after: expected")
    refuses(fn, *ok, reset=t(4, 3, dtype=torch.bool), match="reset: expected")
    fn = getattr(lm, "cx_short_conv_grad" + suffix)
    ok = (m(12, 9), m(12, 9), m(2, 60), 5, m(12, 9), None, m(2, 60), 3, 4)
    refuses(fn, *ok, match="device tensors")
    refuses(fn, m(12, 9), m(12, 8), *ok[2:], match="dy: expected")
    refuses(fn, *ok[:6], m(2, 40), 3, 4, match="do not fit")

    fn = getattr(lm, "cx_select_scan" + suffix)
    ok = (m(12, 9), m(12, 9), m(12, 5), m(12, 5), m(2, 70), 5, m(12, 9), 3)
    refuses(fn, *ok, z=m(12, 9), h0=t(4, 9, 5), h_last=t(4, 9, 5), reset=bytes_(4, 3), states=t(4, 1, 9, 5), match="device tensors")
    refuses(fn, *ok[:3], m(12, 4), *ok[4:], match="cm: expected")
    refuses(fn, *ok[:4], m(2, 60), *ok[5:], match="do not fit")
    refuses(fn, *ok[:4], m(3, 70), *ok[5:], match="same number")
    refuses(fn, *ok, z=m(12, 8), match="z: expected")
    refuses(fn, *ok, h0=t(4, 5, 9), match="h0: expected")
    refuses(fn, *ok, states=t(4, 2, 9, 5), match="states: expected")
    fn = getattr(lm, "cx_select_scan_grad" + suffix)
    ok = (*ok[:6], m(12, 9), m(12, 9), m(12, 9), m(12, 5), m(12, 5), None, m(2, 70), 3, t(4, 1, 9, 5))
    refuses(fn, *ok, z=m(12, 9), dz=m(12, 9), match="device tensors")
    refuses(fn, *ok, z=m(12, 9), match="go together")
    refuses(fn, *ok[:14], None, match="states is missing")
    refuses(fn, *ok[:9], m(12, 4), *ok[10:], match="dbm: expected")
    refuses(fn, *ok, dh0=t(4, 9, 4), match="dh0: expected")


@pytest.mark.parametrize("suffix", SUFFIXES)
def test_sizes_beyond_32_bits_are_refused(suffix):
    shape = lambda *s, dtype=torch.float32: torch.empty(s, dtype=dtype, device="meta")
    m, wide = lambda *s: shape(*s, dtype=TYPES[suffix]), 2**32 + 9
    rng = shape(2, dtype=torch.int64)
    for name, args in (("cx_dropout", (m(2, wide), rng, m(2, wide), 0.5)), ("cx_add_norm", (m(2, wide), None, m(1, wide), 0, None, m(2, wide), 1e-6)),
                       ("cx_add_norm_grad", (m(2, wide), m(2, wide), shape(2), m(1, wide), 0, None, m(2, wide), None, m(1, wide))),
                       ("cx_short_conv", (m(2, wide), m(1, 5 * wide), 0, m(2, wide), 2, 4)), ("cx_short_conv", (m(2, 9), m(1, 99), 0, m(2, 9), 2, 2**32 + 4)),
                       ("cx_short_conv", (m(2, 9), m(1, 99), 0, m(2, 9), 2, 4 - 2**32)),
                       ("cx_select_scan", (m(2, wide), m(2, wide), m(2, 5), m(2, 5), m(1, 7 * wide), 0, m(2, wide), 2)),
                       ("cx_select_scan", (m(2, 9), m(2, 9), m(2, wide), m(2, wide), m(1, 10 * wide), 0, m(2, 9), 2))):
        with pytest.raises(lm.CxError, match="CX_ERR_SHAPE"):
            getattr(lm, name + suffix)(*args)


@pytest.mark.parametrize("argv", [["--blocks", "-1"], ["--dropout", "0.1"]])
def test_training_command_refuses(argv):
    from paper_2012_15198_amd import codistill
    with pytest.raises(SystemExit):
        codistill.main(argv)
