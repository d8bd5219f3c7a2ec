"""CPU-only: the recurrence refuses every overlap that its header excludes, before anything is launched."""
import pytest

from paper_2012_15198_amd import cxlm as lm

SUFFIXES = ["", "_bf16", "_f16"]
A, B, C, D, E, F, G, H, R, S = (k << 28 for k in range(1, 11))       # far apart, aligned; never handed to a kernel
LONG = 4000                                                          # steps that are split, so that the workspace is written
ROOM = 1 << 20


@pytest.mark.parametrize("suffix", SUFFIXES)
@pytest.mark.parametrize("T", [1, 40, LONG])
def test_the_forward_call_refuses_overlaps(suffix, T):
    ok = dict(f=A, ldf=8, x=B, ldx=8, y=C, ldy=8, B=2, T=T, D=8, reset=R, h0=D, hl=E, states=F, ws=S, wn=ROOM, st=None)
    call = lambda **kw: getattr(lm.lib(), "cx_gated_scan" + suffix)(*{**ok, **kw}.values())
    for out in ("y", "hl", "states", *(["ws"] if T == LONG else [])):
        for other in ("f", "x", "reset", "h0", "y", "hl", "states"):
            if other == out or (out, other) == ("hl", "h0"):         # the state in place
                continue
            assert call(**{out: ok[other]}) == -6, (out, other)
    assert call(hl=D + 4) == -6 and call(hl=A + 4) == -6 and call(states=B + 8 * 2 - 4) == -6


@pytest.mark.parametrize("suffix", SUFFIXES)
@pytest.mark.parametrize("T", [1, 40, LONG])
def test_the_gradient_refuses_overlaps(suffix, T):
    ok = dict(f=A, ldf=8, x=B, ldx=8, dy=C, lddy=8, df=D, lddf=8, dx=E, lddx=8, B=2, T=T, D=8, reset=R, states=F, dl=G, d0=H, ws=S, wn=ROOM, st=None)
    call = lambda **kw: getattr(lm.lib(), "cx_gated_scan_grad" + suffix)(*{**ok, **kw}.values())
    for out in ("df", "dx", "d0", *(["ws"] if T == LONG else [])):
        for other in ("f", "x", "dy", "reset", "states", "dl", "df", "dx", "d0"):
            if other == out or (out, other) == ("d0", "dl"):
                continue
            assert call(**{out: ok[other]}) == -6, (out, other)
    assert call(d0=G + 4) == -6 and call(d0=C + 4) == -6
