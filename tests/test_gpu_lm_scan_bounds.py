"""cx_gated_scan and cx_gated_scan_grad within the fp32 error bound of every element: short, long and split sequences, kept states included."""
import pytest
import torch

import lm_bounds as bounds
import lm_reference as R
from paper_2012_15198_amd import cxlm as lm

DEV = "cuda:0"
pytestmark = pytest.mark.gpu

SHAPES = [  # B, T, D
    (1, 1, 1), (3, 1, 65), (2, 2, 3), (1, 16, 64), (2, 17, 129), (3, 127, 65), (1, 128, 257), (2, 129, 7), (1, 1111, 33), (2, 2050, 5), (130, 40, 20),
    (300, 33, 65), (66, 131, 200),                              # two 16-bit columns to a lane
    (2, 700, 65), (2, 700, 129), (1, 1500, 131), (5, 390, 193), (20, 300, 323),      # 16-bit gradients of odd widths, split
    (1, 8189, 3), (1, 8192, 2), (1, 16_300, 65), (2, 4_000, 70)]                     # 18 to 64 spans


def one(suffix, B, T, D, packed, strided, seed):
    dtype, gen = R.TYPES[suffix], torch.Generator().manual_seed(seed)
    normal = lambda m, s, *shape: torch.randn(shape, generator=gen) * s + m
    f, x, dy = (normal(m, s, B * T, D).to(dtype) for m, s in ((2.0, 1.5), (0.0, 1.0), (0.0, 1.0)))
    h0, dh = normal(0.0, 1.0, B, D), normal(0.0, 1.0, B, D)
    reset = None
    if packed:
        reset = (torch.rand((B, T), generator=gen) < 0.03).to(torch.uint8) * 3
        reset[B - 1, 0] = 1
        reset[:, T // 128 * 128 if T % 128 else T - 1] = 1      # at the beginning of a tile

    def place(t):
        if not strided:
            return t.to(DEV)
        wide = torch.full((t.shape[0], t.shape[1] + 3), 3.0, dtype=t.dtype, device=DEV)
        wide[:, 1:1 + t.shape[1]] = t.to(DEV)
        return wide[:, 1:1 + t.shape[1]]

    on = lambda t: None if t is None else t.to(DEV)
    fd, xd, dyd = place(f), place(x), place(dy)
    y, df, dx = (place(torch.full_like(f, torch.nan)) for _ in range(3))
    h_last, dh0 = (torch.full((B, D), torch.nan, device=DEV) for _ in range(2))
    states = lm.scan_states(fd, T).fill_(torch.nan)
    getattr(lm, "cx_gated_scan" + suffix)(fd, xd, y, T, h0=on(h0), h_last=h_last, reset=on(reset), states=states)
    getattr(lm, "cx_gated_scan_grad" + suffix)(fd, xd, dyd, df, dx, T, states, dh_last=on(dh), dh0=dh0, reset=on(reset))
    s, g = bounds.scan(f, x, T, h0, reset), bounds.scan_grad(f, x, dy, T, h0, reset, dh)
    each = slice(None, None, lm.CX_SCAN_CHUNK)
    R.check(y.view(B, T, D), s["y"], s["y_err"], "y")
    R.check(h_last, s["h_last"], s["h_last_err"], "h_last")
    R.check(states, s["before"][:, each], s["before_err"][:, each], "states")
    R.check(dx.view(B, T, D), g["dx"], g["dx_err"], "dx")
    R.check(df.view(B, T, D), g["df"], g["df_err"], "df")
    R.check(dh0, g["dh0"], g["dh0_err"], "dh0")
    if strided:
        for t in (y, df, dx):
            assert (t._base[:, 0] == 3).all() and (t._base[:, 1 + D:] == 3).all()


@pytest.mark.parametrize("suffix", R.SUFFIXES)
@pytest.mark.parametrize("packed,strided", [(False, False), (True, True)])
@pytest.mark.parametrize("B,T,D", SHAPES)
def test_every_element(suffix, packed, strided, B, T, D):
    one(suffix, B, T, D, packed, strided, B * T + D)
