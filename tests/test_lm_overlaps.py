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


@pytest.mark.parametrize("suffix", SUFFIXES)
def test_matrices_that_cross_by_one_element(suffix):
    """Halves of the rows of one wide matrix share nothing; one element more to either side, or another pitch, does."""
    size = 4 if suffix == "" else 2
    head = (A, 100, 600, 50, 4, B, C, D, 2.0, 0.5, 0.5)
    step = lambda dz, ld=100: getattr(lm.lib(), "cx_distill_step" + suffix)(*head, E, F, dz, ld, None, 0, None)
    grad = lambda dz, ld=100: getattr(lm.lib(), "cx_distill_grad" + suffix)(*head, F, E, dz, ld, None)
    for call in (step, grad):
        for off in (1, 49, 51, 99, 149, 151, -1, -49, -51):
            assert call(A + off * size) == -6, off
        assert call(A + 50 * size, 101) == -6 and call(A, 101) == -6
    need = lm.cx_embed_workspace(2, 5, 9, 8)
    rows = lambda g_in, g_out: getattr(lm.lib(), "cx_embed_grad" + suffix)(B, 8, C, 2, 5, g_in, g_out, 164, 10, 9, 8, 1.0, S, need, None)
    for off in (1, 81, 83, 163):
        assert rows(A, A + off * size) == -6 and rows(A + off * size, A) == -6, off
    scores = lambda logp: getattr(lm.lib(), "cx_token_scores" + suffix)(A, 100, 600, 50, B, 1.0, logp, None, 0, None, None, None, 0, None)
    assert scores(A + 48 * size) == -6 and scores(A + 52 * size) == -6      # 600 results reach into the next row
