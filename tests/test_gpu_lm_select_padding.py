"""Steps of padding in cx_select_scan and cx_select_scan_grad: rows whose dt are all -inf leave the states as they are and, where their dy are 0, no
gradient, whatever their other operands hold."""
import pytest
import torch

import lm_reference as R
from lm_block_util import DEV
from paper_2012_15198_amd import cxlm as lm
from test_gpu_lm_select import Case

pytestmark = pytest.mark.gpu
SIZES = [(1, 30, 5), (1, 130, 16), (9, 70, 1), (50, 30, 5), (50, 129, 16), (300, 70, 12), (900, 33, 7)]


def dirty(c, pad, k):
    """Everything but dt and dy of the padded rows holds NaN or an infinity."""
    for j, t in enumerate((c.u, c.bm, c.cm, c.z)):
        t[pad] = (torch.nan, torch.inf, -torch.inf)[(j + k) % 3]


@pytest.mark.parametrize("suffix", R.SUFFIXES)
@pytest.mark.parametrize("T,D,N", SIZES)
@pytest.mark.parametrize("k", [None, 0, 1, 2])
def test_rows_of_padding_hold_anything(suffix, T, D, N, k):
    """Padding rows in runs inside tiles, over whole tiles and at the end: what the other rows, the states and the parameters get is what it is with
    finite ones, to the bit."""
    outs, B = [], 2
    pad = ((torch.arange(B * T) % 11 >= 7) | ((torch.arange(B * T) // 16) % 5 == 3) | (torch.arange(B * T) % T == T - 1)) & (T > 1)
    if T == 1:
        pad[1] = True
    for which in (None, k):
        c = Case(suffix, 1, B, T, D, N)
        c.dt[pad], c.dy[pad] = -torch.inf, 0
        if which is not None:
            dirty(c, pad, which)
        d, on = c.on(), lambda t: t.to(DEV)
        y, h_last, dh0, g = torch.empty_like(d["u"]), torch.empty((B, D, N), device=DEV), torch.empty((B, D, N), device=DEV), torch.zeros_like(on(c.rows))
        states = lm.select_states(y, T, N)
        c.forward(d, y, states, on(c.h0), h_last)
        grads = c.backward(d, states, None, g, on(c.dh), dh0)
        assert all((v[pad.to(DEV)] == 0).all() for v in grads.values())
        outs.append([y[~pad.to(DEV)], h_last, states, dh0, g, *grads.values()])
    if T == 1:
        assert torch.equal(outs[1][1][1].cpu(), c.h0[1])
    for j, (clean, other) in enumerate(zip(*outs)):
        assert clean.isfinite().all() and torch.equal(clean, other), j


@pytest.mark.parametrize("suffix", R.SUFFIXES)
@pytest.mark.parametrize("T", [1, 40, 300])
def test_a_column_of_padding_takes_nothing_of_u(suffix, T):
    """dt of -inf in single columns, whose u are not finite, beside open ones; reduced gradients take nothing of them."""
    outs, B, D, N, shut = [], 1, 70, 6, torch.tensor([0, 5, 66, 69])
    for value in (0.5, torch.nan, torch.inf):
        c = Case(suffix, 1, B, T, D, N)
        c.dt[:, shut], c.dy[:, shut], c.u[:, shut] = -torch.inf, 0, value
        d, on = c.on(), lambda t: t.to(DEV)
        y, h_last, dh0, g = torch.empty_like(d["u"]), torch.empty((B, D, N), device=DEV), torch.empty((B, D, N), device=DEV), torch.zeros_like(on(c.rows))
        states = lm.select_states(y, T, N)
        c.forward(d, y, states, on(c.h0), h_last)
        grads = c.backward(d, states, None, g, on(c.dh), dh0)
        assert torch.equal(h_last[:, shut].cpu(), c.h0[:, shut])
        rest = torch.ones(D, dtype=torch.bool)
        rest[shut] = False
        outs.append([y[:, rest.to(DEV)], h_last, states, dh0, g, *grads.values()])
    for other in outs[1:]:
        for j, (clean, got) in enumerate(zip(outs[0], other)):
            assert clean.isfinite().all() and torch.equal(clean, got), j
