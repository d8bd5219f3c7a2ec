"""cx_dropout, cx_add_norm and cx_add_norm_grad against their formulas in 64 bits."""
import pytest
import torch

import lm_block_reference as B
import lm_reference as R
from lm_block_util import DEV, edges, flat_rows, gradient_rows, place, untouched
from paper_2012_15198_amd import cxlm as lm

pytestmark = pytest.mark.gpu
RNG = (0x1234567_89ABCDEF, -5_000_000_001)


def rng_of(pair=RNG):
    return torch.tensor(pair, dtype=torch.int64, device=DEV)


# ------------------------------------------------------------------------------------------------------------------ dropout
@pytest.mark.parametrize("suffix", R.SUFFIXES)
@pytest.mark.parametrize("strided", [False, True])
@pytest.mark.parametrize("N,D,p,added", [(1, 1, 0.5, False), (3, 7, 0.25, True), (1, 8, 0.1, True), (37, 65, 0.9, False), (129, 515, 0.1, True),
                                         (2, 5001, 0.3, True), (300, 1024, 0.0, False), (70, 16, 1e-6, True)])
def test_dropout(suffix, strided, N, D, p, added):
    gen, dtype = torch.Generator().manual_seed(N + D), R.TYPES[suffix]
    x, r = (torch.randn((N, D), generator=gen).to(dtype) for _ in range(2))
    out = place(torch.full_like(x, 9.0), strided)
    getattr(lm, "cx_dropout" + suffix)(place(x, strided), rng_of(), out, p, residual=place(r, strided) if added else None)
    keep = B.factor(RNG, N, D, p)
    ref, slack = B.dropout(x, r if added else None, keep)
    R.check(out, ref, slack)
    if not added:
        assert torch.equal(out.cpu() == 0, (keep == 0) | (x == 0))
    if strided:
        assert untouched(out)


@pytest.mark.parametrize("suffix", R.SUFFIXES)
def test_dropout_in_place_drops_nan_and_infinity(suffix):
    N, D, dtype = 40, 33, R.TYPES[suffix]
    x = torch.randn((N, D), generator=torch.Generator().manual_seed(1)).to(dtype)
    keep = B.factor(RNG, N, D, 0.4)
    dirty = torch.where(keep == 0, torch.tensor([torch.nan, torch.inf]).to(dtype)[torch.arange(D) % 2], x)
    r = torch.randn((N, D), generator=torch.Generator().manual_seed(2)).to(dtype)
    outs = []
    for values in (x, dirty):
        alone, on_x, on_r = values.to(DEV), values.to(DEV), r.to(DEV)
        getattr(lm, "cx_dropout" + suffix)(alone, rng_of(), alone, 0.4)
        getattr(lm, "cx_dropout" + suffix)(on_x, rng_of(), on_x, 0.4, residual=on_r)
        getattr(lm, "cx_dropout" + suffix)(values.to(DEV), rng_of(), on_r, 0.4, residual=on_r)
        assert torch.equal(on_x, on_r)
        outs.append((alone, on_x))
    for a, b in zip(*outs):
        assert a.isfinite().all() and torch.equal(a, b)


def test_masks_of_keys_and_draws():
    """Another key or draw is another mask; every mask drops its share; the counter's upper halves count."""
    x, share = torch.ones((400, 500), device=DEV), 0.3
    masks = []
    for pair in ((0, 0), (1, 0), (0, 1), (2**32, 0), (0, 2**32), (-1, -1)):
        out = torch.empty_like(x)
        lm.cx_dropout(x, rng_of(pair), out, share)
        assert torch.equal(out.cpu() != 0, B.factor(pair, 400, 500, share) != 0)
        masks.append(out != 0)
        assert abs(float(masks[-1].double().mean()) - 0.7) < 6 * (0.21 / x.numel())**0.5
    for i, a in enumerate(masks):
        for b in masks[:i]:
            assert abs(float((a == b).double().mean()) - 0.58) < 0.02


# --------------------------------------------------------------------------------------------------------------------- norm
SHAPES = [  # W, N, D
    (1, 1, 1), (2, 3, 2), (1, 5, 8), (3, 7, 9), (1, 33, 64), (2, 50, 129), (5, 11, 515), (1, 20, 768), (2, 9, 1024), (1, 6, 1537), (2, 3, 4097), (1, 3, 8200),
    (1, 2, 16384), (16, 1, 40), (1, 700, 24)]


def make(suffix, W, N, D, p, strided, residual):
    gen, dtype = torch.Generator().manual_seed(W * N + D), R.TYPES[suffix]
    x, r, dy, more = (torch.randn((W * N, D), generator=gen).to(dtype) for _ in range(4))
    rows = flat_rows([torch.randn((W, D), generator=gen) * 0.3 + 1], 5, dtype, gen)
    w = rows[:, 5:5 + D].repeat_interleave(N, 0)
    return gen, dtype, x, r if residual else None, dy, more, rows, w, B.factor(RNG, W * N, D, p)


@pytest.mark.parametrize("suffix", R.SUFFIXES)
@pytest.mark.parametrize("p,strided,residual", [(0.0, False, True), (0.3, True, True), (0.1, False, False), (0.0, True, False)])
@pytest.mark.parametrize("W,N,D", SHAPES)
def test_forward(suffix, p, strided, residual, W, N, D):
    _, dtype, x, r, _, _, rows, w, keep = make(suffix, W, N, D, p, strided, residual)
    s, y = (place(torch.full_like(x, 9.0), strided) for _ in range(2))
    inv, scale = (torch.full((W * N,), 9.0, device=DEV) for _ in range(2))
    q = torch.full((W * N, D + 3), 5, dtype=torch.uint8, device=DEV)[:, 1:1 + D] if strided else torch.full((W * N, D), 5, dtype=torch.uint8, device=DEV)
    getattr(lm, "cx_add_norm" + suffix)(place(x, strided), None if r is None else place(r, strided), rows.to(DEV), 5, s, y, 1e-6, inv=inv, q=q, scale=scale,
                                        p=p, rng=rng_of())
    ref = B.add_norm(x, r, w, keep, float(torch.tensor(1e-6)))
    R.check(s, ref["t"], ref["t_err"], "s")
    R.check(y, ref["y"], ref["y_err"], "y")
    R.check(inv, ref["inv"], ref["inv_err"], "inv")
    most = (ref["y"].abs() + ref["y_err"]).amax(1)
    R.check(scale, (ref["y"].abs().amax(1) / 448).clamp_min(2.0**-126), (most - ref["y"].abs().amax(1)) / 448 + 2 * R.U * most / 448, "scale")
    held, by = q.cpu().view(torch.float8_e4m3fn).double() if not strided else q.contiguous().cpu().view(torch.float8_e4m3fn).double(), scale.cpu().double()[:, None]
    want, slack = ref["y"] / by, ref["y_err"] / by + 3 * R.U * (ref["y"] / by).abs()
    assert ((held - want).abs() <= B.half_step8(want.abs() + slack) + slack).all() and held.abs().amax() <= 448
    if strided:
        assert untouched(s) and untouched(y) and (q._base[:, 0] == 5).all() and (q._base[:, 1 + D:] == 5).all()


@pytest.mark.parametrize("suffix", R.SUFFIXES)
@pytest.mark.parametrize("p,strided,mode", [(0.0, False, "alone"), (0.3, True, "added"), (0.1, False, "in place")])
@pytest.mark.parametrize("W,N,D", SHAPES + [(2, 3000, 40), (1, 1100, 200)])
def test_gradient(suffix, p, strided, mode, W, N, D):
    gen, dtype, x, r, dy, more, rows, w, keep = make(suffix, W, N, D, p, strided, True)
    s, inv = place(torch.empty_like(x), strided), torch.empty(W * N, device=DEV)
    getattr(lm, "cx_add_norm" + suffix)(x.to(DEV), r.to(DEV), rows.to(DEV), 5, s, None, 1e-5, inv=inv, p=p, rng=rng_of())
    ds, dx = (place(torch.full_like(x, 9.0), strided) for _ in range(2))
    g_in, g_out, base = gradient_rows(mode, rows, dtype, gen)
    before = edges(g_out, 5, D)
    getattr(lm, "cx_add_norm_grad" + suffix)(place(dy, strided), s, inv, rows.to(DEV), 5, place(more, strided) if mode == "added" else None, ds, g_in, g_out,
                                             dx=dx, p=p, rng=rng_of())
    ref = B.add_norm_grad(dy, s.cpu(), inv.cpu(), w, more if mode == "added" else None, keep)
    R.check(ds, ref["ds"], ref["ds_err"], "ds")
    R.check(dx, ref["dx"], ref["dx_err"], "dx")
    unit = s.cpu().double() * inv.cpu().double()[:, None]
    terms = dy.double() * unit
    want, slack = B.summed(terms, 3 * R.U * terms.abs(), terms.abs(), W, 1, None if base is None else base[:, 5:5 + D])
    R.check(g_out[:, 5:5 + D], want, slack, "dw")
    assert torch.equal(edges(g_out, 5, D), before)
    if strided:
        assert untouched(ds) and untouched(dx)


@pytest.mark.parametrize("suffix", R.SUFFIXES)
def test_buffers_in_place(suffix):
    """s in x's or the residual's place, y in x's; ds and dx in the places of dy and ds_in."""
    W, N, D, p = 2, 30, 200, 0.2
    _, dtype, x, r, dy, more, rows, _, _ = make(suffix, W, N, D, p, False, True)
    forward, backward = getattr(lm, "cx_add_norm" + suffix), getattr(lm, "cx_add_norm_grad" + suffix)
    on, w = lambda t: t.to(DEV), rows.to(DEV)
    s, y, inv, g = torch.empty_like(on(x)), torch.empty_like(on(x)), torch.empty(W * N, device=DEV), torch.empty_like(w)
    forward(on(x), on(r), w, 5, s, y, 1e-6, inv=inv, p=p, rng=rng_of())
    a, b, inv2 = on(x), on(r), torch.empty_like(inv)
    forward(a, b, w, 5, b, a, 1e-6, inv=inv2, p=p, rng=rng_of())
    assert torch.equal(a, y) and torch.equal(b, s) and torch.equal(inv, inv2)
    a = on(x)
    forward(a, on(r), w, 5, a, None, 1e-6, p=p, rng=rng_of())
    assert torch.equal(a, s)
    ds, dx = torch.empty_like(s), torch.empty_like(s)
    backward(on(dy), s, inv, w, 5, on(more), ds, None, g, dx=dx, p=p, rng=rng_of())
    for swap in (False, True):
        a, b, g2 = on(dy), on(more), torch.empty_like(g)
        backward(a, s, inv, w, 5, b, a if swap else b, None, g2, dx=b if swap else a, p=p, rng=rng_of())
        assert torch.equal(a, ds if swap else dx) and torch.equal(b, dx if swap else ds) and torch.equal(g[:, 5:5 + D], g2[:, 5:5 + D])
    alone = torch.empty_like(s)
    backward(on(dy), s, inv, w, 5, on(more), None, None, g, dx=alone, p=p, rng=rng_of())
    assert torch.equal(alone, dx)


def test_the_norm_drops_what_dropout_drops():
    """One mask of a matrix, whichever operator reads it: s of the norm is what cx_dropout gives, and ds = dx where nothing is dropped."""
    x, r = torch.randn((60, 77), device=DEV), torch.randn((60, 77), device=DEV)
    w, out, s = torch.ones((3, 77), device=DEV), torch.empty_like(x), torch.empty_like(x)
    lm.cx_dropout(x, rng_of(), out, 0.35, residual=r)
    lm.cx_add_norm(x, r, w, 0, s, None, 1e-6, p=0.35, rng=rng_of())
    assert torch.equal(out, s)


@pytest.mark.parametrize("suffix", R.SUFFIXES)
def test_rows_at_their_ends(suffix):
    """Rows of zeros, one large value, the least and largest normal values, NaN and infinity; each row by itself."""
    dtype, D = R.TYPES[suffix], 70
    tiny, huge = torch.finfo(dtype).tiny, 1e18 if suffix != "_f16" else 60000.0
    x = torch.zeros((7, D))
    x[1, 3], x[2], x[3], x[4, 5], x[5, 6] = huge, tiny, huge / 16, torch.nan, torch.inf
    x[6] = torch.linspace(-2, 2, D)
    x = x.to(dtype)
    y, scale, q = torch.empty((7, D), dtype=dtype, device=DEV), torch.empty(7, device=DEV), torch.empty((7, D), dtype=torch.float8_e4m3fn, device=DEV)
    getattr(lm, "cx_add_norm" + suffix)(x.to(DEV), None, torch.ones((1, D), dtype=dtype, device=DEV), 0, None, y, 1e-6, q=q, scale=scale)
    fine = [0, 1, 2, 3, 6]
    ref = B.add_norm(x[fine], None, torch.ones((5, D), dtype=dtype), torch.ones((5, D), dtype=torch.float64), float(torch.tensor(1e-6)))
    R.check(y[fine], ref["y"], ref["y_err"] + 2.0**-126)
    assert y[4].isnan().all() and y[5, 6].isnan() and (y[5, :6] == 0).all() and scale[4:6].isnan().all()
    held = q.cpu().double() * scale.cpu().double()[:, None]
    assert held[4].isnan().all() and scale[0] == 2.0**-126 and (held[0] == 0).all() and (scale > 0)[fine].all()
    assert ((held[fine] - ref["y"]).abs() <= ref["y"].abs() * 2.0**-4 + scale.cpu().double()[fine, None] * 2.0**-10 + 1e-6 * ref["y"].abs()).all()


def test_no_rows():
    w, empty, g = torch.ones((2, 9), device=DEV), torch.empty((0, 9), device=DEV), torch.full((2, 9), 4.0, device=DEV)
    lm.cx_add_norm(empty, None, w, 0, empty, empty, 1e-6)
    lm.cx_dropout(empty, rng_of(), empty, 0.5)
    lm.cx_add_norm_grad(empty, empty, torch.empty(0, device=DEV), w, 0, None, empty, g, g)
    assert (g == 4).all()
    lm.cx_add_norm_grad(empty, empty, torch.empty(0, device=DEV), w, 0, None, empty, None, g)
    assert (g == 0).all()


def test_gradient_against_differences():
    """Central differences of sum(y c) + sum(s k) in 64 bits, at drawn places of x, residual and w."""
    W, N, D, p, gen = 2, 5, 19, 0.3, torch.Generator().manual_seed(3)
    _, _, x, r, dy, more, rows, w, keep = make("", W, N, D, p, False, True)
    s, inv, ds, dx, g = torch.empty((W * N, D), device=DEV), torch.empty(W * N, device=DEV), *(torch.empty((W * N, D), device=DEV) for _ in range(2)), torch.empty_like(rows.to(DEV))
    lm.cx_add_norm(x.to(DEV), r.to(DEV), rows.to(DEV), 5, s, None, 1e-3, inv=inv, p=p, rng=rng_of())
    lm.cx_add_norm_grad(dy.to(DEV), s, inv, rows.to(DEV), 5, more.to(DEV), ds, None, g, dx=dx, p=p, rng=rng_of())

    def value(x, r, w):
        f = B.add_norm(x, r, w.repeat_interleave(N, 0), keep, 1e-3)
        return float((f["y"] * dy.double()).sum() + (f["t"] * more.double()).sum())

    args = [x.double(), r.double(), rows[:, 5:5 + D].double()]
    for which, grad in ((0, dx), (1, ds), (2, g[:, 5:5 + D])):
        for at in torch.randint(0, args[which].numel(), (12,), generator=gen).tolist():
            ends = []
            for sign in (1, -1):
                moved = [a.clone() for a in args]
                moved[which].view(-1)[at] += sign * 1e-5
                ends.append(value(*moved))
            slope = (ends[0] - ends[1]) / 2e-5
            assert abs(slope - float(grad.reshape(-1)[at])) < 2e-5 * (1 + abs(slope)), (which, at)
