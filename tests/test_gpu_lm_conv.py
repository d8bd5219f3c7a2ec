"""cx_short_conv and cx_short_conv_grad against the convolution in 64 bits, step by step."""
import pytest
import torch

import lm_block_reference as BR
import lm_reference as R
from lm_block_util import DEV, edges, flat_rows, gradient_rows, place, untouched
from paper_2012_15198_amd import cxlm as lm

pytestmark = pytest.mark.gpu
OFFSET = 3


def make(suffix, W, B, T, D, K, packed, seed=0):
    gen, dtype = torch.Generator().manual_seed(seed + B * T + D * K), R.TYPES[suffix]
    x, dy = (torch.randn((B * T, D), generator=gen).to(dtype) for _ in range(2))
    rows = flat_rows([torch.randn((W, D * K), generator=gen) * 0.6, torch.randn((W, D), generator=gen) * 0.3], OFFSET, dtype, gen)
    before = torch.randn((B, K - 1, D), generator=gen).to(dtype)
    reset = None
    if packed:
        reset = (torch.rand((B, T), generator=gen) < 0.2).to(torch.uint8) * 5
        reset[0, 0] = 1
        if B > 1:
            reset[1] = 1
        reset[B - 1, T - 1] = 1
    of = lambda begin, *shape: rows[:, OFFSET + begin:OFFSET + begin + D * (shape[-1] if len(shape) > 1 else 1)].repeat_interleave(B // W, 0).view(B, *shape)
    return gen, dtype, x, dy, rows, of(0, D, K), of(D * K, D), before, reset


SHAPES = [  # W, B, T, D, K
    (1, 1, 1, 1, 1), (1, 1, 1, 3, 4), (2, 4, 2, 9, 4), (1, 2, 3, 64, 3), (3, 3, 7, 65, 2), (1, 2, 8, 8, 4), (1, 3, 9, 515, 4), (2, 2, 31, 16, 1),
    (2, 4, 33, 24, 4), (1, 1, 300, 40, 3), (1, 2, 1111, 7, 4), (1, 1, 67, 1030, 2), (5, 40, 5, 12, 4)]


@pytest.mark.parametrize("suffix", R.SUFFIXES)
@pytest.mark.parametrize("packed,strided,silu,mode", [(False, False, True, "alone"), (True, True, True, "in place"), (True, False, False, "added"),
                                                      (False, True, False, "alone")])
@pytest.mark.parametrize("W,B,T,D,K", SHAPES)
def test_both_directions(suffix, packed, strided, silu, mode, W, B, T, D, K):
    gen, dtype, x, dy, rows, w, bias, before, reset = make(suffix, W, B, T, D, K, packed)
    on = lambda t: None if t is None else t.to(DEV)
    carried = None if mode == "added" else before
    xd, y, dx = place(x, strided), place(torch.full_like(x, 9.0), strided), place(torch.full_like(x, 9.0), strided)
    after = torch.full_like(before, 9.0).to(DEV)
    getattr(lm, "cx_short_conv" + suffix)(xd, rows.to(DEV), OFFSET, y, T, K, silu=silu, before=on(carried), after=after, reset=on(reset))
    ref = BR.conv(x, w, bias, T, K, silu, carried, reset)
    R.check(y.reshape(B, T, D), ref["y"], ref["y_err"], "y")
    assert torch.equal(after.cpu().double(), ref["after"])
    count = D * (K + 1)
    g_in, g_out, base = gradient_rows(mode, rows, dtype, gen)
    around = edges(g_out, OFFSET, count)
    getattr(lm, "cx_short_conv_grad" + suffix)(xd, place(dy, strided), rows.to(DEV), OFFSET, dx, g_in, g_out, T, K, silu=silu, before=on(carried), reset=on(reset))
    ref = BR.conv_grad(x, dy, w, bias, T, K, silu, carried, reset)
    R.check(dx.reshape(B, T, D), ref["dx"], ref["dx_err"], "dx")
    part = lambda begin, n: None if base is None else base[:, OFFSET + begin:OFFSET + begin + n]
    R.check(g_out[:, OFFSET:OFFSET + D * K], *BR.summed(ref["dw"], ref["dw_err"], ref["dw_size"], W, T, part(0, D * K)), "dw")
    R.check(g_out[:, OFFSET + D * K:OFFSET + count], *BR.summed(ref["dbias"], ref["dbias_err"], ref["dbias_size"], W, T, part(D * K, D)), "dbias")
    assert torch.equal(edges(g_out, OFFSET, count), around)
    if strided:
        assert untouched(y) and untouched(dx)


@pytest.mark.parametrize("suffix", R.SUFFIXES)
@pytest.mark.parametrize("K", [1, 2, 3, 4])
def test_steps_one_by_one_with_the_state_in_place_equal_the_sequence(suffix, K):
    W, B, T, D = 1, 3, 23, 130
    _, dtype, x, _, rows, w, bias, before, reset = make(suffix, W, B, T, D, K, True)
    whole, state, out = torch.empty((B * T, D), dtype=dtype, device=DEV), before.to(DEV), torch.empty((B, D), dtype=dtype, device=DEV)
    rd, wd, xd = reset.to(DEV), rows.to(DEV), x.to(DEV).view(B, T, D)
    getattr(lm, "cx_short_conv" + suffix)(x.to(DEV), wd, OFFSET, whole, T, K, before=before.to(DEV), reset=rd)
    for t in range(T):
        getattr(lm, "cx_short_conv" + suffix)(xd[:, t], wd, OFFSET, out, 1, K, before=state, after=state, reset=rd[:, t:t + 1].contiguous())
        assert torch.equal(out, whole.view(B, T, D)[:, t])
    assert torch.equal(state.cpu().double(), BR.taps(x, T, K, before, reset)[1])


@pytest.mark.parametrize("suffix", R.SUFFIXES)
@pytest.mark.parametrize("cuts", [(2,), (1, 2, 3), (40,), (33, 34)])
def test_a_sequence_in_chunks_with_the_state_in_place(suffix, cuts):
    W, B, T, D, K = 1, 2, 70, 33, 4
    _, dtype, x, _, rows, _, _, before, reset = make(suffix, W, B, T, D, K, True)
    whole, state, wd = torch.empty((B * T, D), dtype=dtype, device=DEV), before.to(DEV), rows.to(DEV)
    getattr(lm, "cx_short_conv" + suffix)(x.to(DEV), wd, OFFSET, whole, T, K, before=before.to(DEV), reset=reset.to(DEV))
    for begin, end in zip((0, *cuts), (*cuts, T)):
        n = end - begin
        piece = x.view(B, T, D)[:, begin:end].reshape(B * n, D).to(DEV)
        out = torch.empty_like(piece)
        getattr(lm, "cx_short_conv" + suffix)(piece, wd, OFFSET, out, n, K, before=state, after=state, reset=reset[:, begin:end].contiguous().to(DEV))
        assert torch.equal(out.view(B, n, D), whole.view(B, T, D)[:, begin:end])


@pytest.mark.parametrize("suffix", R.SUFFIXES)
def test_nothing_crosses_a_reset(suffix):
    """NaN and infinities in one document leave the others as they are, forward and backward, where no parameter joins them."""
    W, B, T, D, K, cut = 1, 1, 90, 20, 4, 61
    _, dtype, x, dy, rows, _, _, before, _ = make(suffix, W, B, T, D, K, False)
    reset = torch.zeros((B, T), dtype=torch.uint8)
    reset[0, cut] = 1
    dirty, late = x.clone(), dy.clone()
    dirty[cut - 1], dirty[cut - 2, ::2] = torch.nan, torch.inf
    late[cut], late[cut + 1, ::2] = torch.nan, torch.inf
    outs = []
    for xs, gs in ((x, dy), (dirty, dy), (x, late)):
        y, dx, after, g = (torch.empty_like(t.to(DEV)) for t in (x, x, before, rows))
        getattr(lm, "cx_short_conv" + suffix)(xs.to(DEV), rows.to(DEV), OFFSET, y, T, K, before=before.to(DEV), after=after, reset=reset.to(DEV))
        getattr(lm, "cx_short_conv_grad" + suffix)(xs.to(DEV), gs.to(DEV), rows.to(DEV), OFFSET, dx, None, g, T, K, before=before.to(DEV), reset=reset.to(DEV))
        outs.append((y, dx, after))
    assert outs[0][0].isfinite().all() and torch.equal(outs[0][0][cut:], outs[1][0][cut:]) and torch.equal(outs[0][1][cut:], outs[1][1][cut:])
    assert torch.equal(outs[0][1][:cut], outs[2][1][:cut]) and torch.equal(outs[0][2], outs[1][2])
    last = torch.zeros((B, T), dtype=torch.uint8)
    last[0, T - 1] = 1                                    # what lies before the last reset does not leave either
    dirty = x.clone()
    dirty[T - 2] = torch.nan
    after = torch.full_like(before, 9.0).to(DEV)
    getattr(lm, "cx_short_conv" + suffix)(dirty.to(DEV), rows.to(DEV), OFFSET, torch.empty_like(x.to(DEV)), T, K, after=after, reset=last.to(DEV))
    assert (after[:, :K - 2] == 0).all() and torch.equal(after[0, K - 2].cpu(), x[T - 1])


def test_no_steps():
    before = torch.randn((2, 3, 5), device=DEV)
    after, rows, empty = torch.empty_like(before), torch.randn((1, 25), device=DEV), torch.empty((0, 5), device=DEV)
    lm.cx_short_conv(empty, rows, 0, empty, 0, 4, before=before, after=after)
    assert torch.equal(after, before)
    lm.cx_short_conv(empty, rows, 0, empty, 0, 4, after=after)
    assert (after == 0).all()
    g = torch.full_like(rows, 3.0)
    lm.cx_short_conv_grad(empty, empty, rows, 0, empty, g, g, 0, 4)
    assert (g == 3).all()
    lm.cx_short_conv_grad(empty, empty, rows, 0, empty, None, g, 0, 4)
    assert (g == 0).all()


def test_gradient_against_differences():
    W, B, T, D, K = 2, 2, 20, 3, 4
    gen, _, x, dy, rows, w, bias, before, reset = make("", W, B, T, D, K, True)
    reset[1] = 0
    dx, g = torch.empty((B * T, D), device=DEV), torch.empty_like(rows.to(DEV))
    lm.cx_short_conv_grad(x.to(DEV), dy.to(DEV), rows.to(DEV), OFFSET, dx, None, g, T, K, before=before.to(DEV), reset=reset.to(DEV))
    value = lambda x, w, b: float((BR.conv(x, w, b, T, K, True, before, reset)["y"].reshape(B * T, D) * dy.double()).sum())
    args = [x.double(), w.double().clone(), bias.double().clone()]
    for which, grad in ((0, dx), (1, g[:, OFFSET:OFFSET + D * K]), (2, g[:, OFFSET + D * K:OFFSET + D * (K + 1)])):
        for at in torch.randint(0, args[which].numel(), (12,), generator=gen).tolist():
            ends = []
            for sign in (1, -1):
                moved = [a.clone() for a in args]
                moved[which].view(-1)[at] += sign * 1e-5
                ends.append(value(*moved))
            slope = (ends[0] - ends[1]) / 2e-5
            assert abs(slope - float(grad.reshape(-1)[at])) < 2e-5 * (1 + abs(slope)), (which, at)
