"""The bounds that the recurrence is tested with: they hold for a plain fp32 evaluation and agree with the step-by-step reference, and they are
narrow enough that a state held in bfloat16 or an error of one part in 10,000 is found, at the longest lengths too."""
import pytest
import torch

import lm_bounds as bounds
import lm_reference as R

SHAPES = [(1, 1, 1), (3, 40, 7), (1, 1111, 33), (2, 2050, 5), (1, 8189, 3)]


def inputs(B, T, D, packed, seed=1):
    gen = torch.Generator().manual_seed(seed)
    normal = lambda m, s, *shape: torch.randn(shape, generator=gen) * s + m
    f, x, dy = normal(2.0, 1.5, B * T, D), normal(0.0, 1.0, B * T, D), normal(0.0, 1.0, B * T, D)
    reset = (torch.rand((B, T), generator=gen) < 0.05).to(torch.uint8) if packed else None
    return f, x, dy, normal(0.0, 1.0, B, D), normal(0.0, 1.0, B, D), reset


def found(got, ref, slack):
    try:
        R.check(got, ref, slack)
    except AssertionError:
        return True
    return False


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("B,T,D", SHAPES)
def test_bounds(B, T, D, packed):
    f, x, dy, h0, dh, reset = inputs(B, T, D, packed)
    s, g = bounds.scan(f, x, T, h0, reset), bounds.scan_grad(f, x, dy, T, h0, reset, dh)
    ry, rh, _ = R.scan(f, x, T, h0, reset)
    rf, rx, r0, _ = R.scan_grad(f, x, dy, T, h0, reset, dh)
    for mine, other in ((s["y"], ry), (s["h_last"], rh), (g["df"], rf), (g["dx"], rx), (g["dh0"], r0)):
        assert (mine - other.reshape(mine.shape)).abs().max() < 1e-12
    # step by step in fp32
    a, b = torch.sigmoid(f).view(B, T, D), torch.sigmoid(-f).view(B, T, D)
    keep = torch.ones((B, T, 1)) if reset is None else (reset == 0).float()[..., None]
    h, ys, before = h0, torch.empty((B, T, D)), torch.empty((B, T, D))
    for t in range(T):
        before[:, t] = keep[:, t] * h
        h = a[:, t] * before[:, t] + b[:, t] * x.view(B, T, D)[:, t]
        ys[:, t] = h
    r, dfs, dxs = dh, torch.empty_like(ys), torch.empty_like(ys)
    for t in range(T - 1, -1, -1):
        r = dy.view(B, T, D)[:, t] + r
        dxs[:, t] = b[:, t] * r
        dfs[:, t] = dxs[:, t] * a[:, t] * (before[:, t] - x.view(B, T, D)[:, t])
        r = keep[:, t] * a[:, t] * r
    fine = ((ys, s["y"], s["y_err"]), (h, s["h_last"], s["h_last_err"]), (dxs, g["dx"], g["dx_err"]), (dfs, g["df"], g["df_err"]), (r, g["dh0"], g["dh0_err"]))
    for got, ref, slack in fine:
        R.check(got, ref, slack)
    if T < 40:
        return
    for got, ref, slack in fine:
        assert found(got.bfloat16().float(), ref, slack) and found(got * 1.01, ref, slack) and found(got * 1.0001, ref, slack)
    # a state that is held in bfloat16 from step to step
    h, low = h0, torch.empty_like(ys)
    for t in range(T):
        h = (a[:, t] * keep[:, t] * h + b[:, t] * x.view(B, T, D)[:, t]).bfloat16().float()
        low[:, t] = h
    assert found(low, s["y"], s["y_err"])
