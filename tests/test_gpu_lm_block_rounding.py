"""What the residual block's operators round, and where."""
import pytest
import torch

import lm_block_reference as B
import lm_reference as R
from lm_block_util import DEV
from paper_2012_15198_amd import cxlm as lm

pytestmark = pytest.mark.gpu


def rows_at_midpoints(dtype, gen):
    """[W][D] weights whose quotients by their scale lie at or next to the midpoints of e4m3; a row's largest first."""
    W = 128
    most = 1 + torch.arange(W) / 128 if dtype == torch.bfloat16 else 1 + torch.rand(W, generator=gen)
    most = most.to(dtype)
    middle = torch.cat([torch.arange(17, 32, 2) * 2.0**k for k in range(-4, 4)])
    at = (middle * most.float()[:, None] / 448).to(dtype)
    whole = torch.int32 if dtype == torch.float32 else torch.int16
    return torch.cat([most[:, None], *((at.view(whole) + k).view(dtype) for k in range(-2, 3))], 1)


@pytest.mark.parametrize("suffix,power", [("", 0), ("", -100), ("", 122), ("_bf16", 0), ("_bf16", -100), ("_bf16", 122), ("_f16", 0)])
def test_the_8_bit_output_is_the_quotient_by_the_scale(suffix, power):
    """Rows of ones and eps = 0: inv is 1 and y the weights.  A product with the scale's reciprocal would be off by a step of e4m3 in some places."""
    dtype = R.TYPES[suffix]
    rows = rows_at_midpoints(dtype, torch.Generator().manual_seed(1))
    rows = rows.clamp(max=rows[:, :1]) * 2.0**power
    W, D = rows.shape
    y = rows.float()
    scale = y.amax(1) / 448
    want, product = (y / scale[:, None]).to(torch.float8_e4m3fn).float(), (y * (1 / scale)[:, None]).to(torch.float8_e4m3fn).float()
    assert (want != product).sum() >= 32
    q, by = torch.empty((W, D), dtype=torch.float8_e4m3fn, device=DEV), torch.empty(W, device=DEV)
    getattr(lm, "cx_add_norm" + suffix)(torch.ones((W, D), dtype=dtype, device=DEV), None, rows.to(DEV), 0, None, None, 0.0, q=q, scale=by)
    assert torch.equal(by.cpu(), scale)
    assert torch.equal(q.cpu().float(), want)


@pytest.mark.parametrize("suffix", R.SUFFIXES)
@pytest.mark.parametrize("D", [9, 700])
def test_an_infinite_result_has_an_infinite_scale(suffix, D):
    rows = torch.ones((2, D), dtype=R.TYPES[suffix])
    rows[0, 3], rows[0, 5] = torch.inf, -torch.inf
    q, scale = torch.empty((2, D), dtype=torch.float8_e4m3fn, device=DEV), torch.empty(2, device=DEV)
    getattr(lm, "cx_add_norm" + suffix)(torch.ones_like(rows).to(DEV), None, rows.to(DEV), 0, None, None, 0.0, q=q, scale=scale)
    held = q.cpu().float()
    assert scale[0] == torch.inf and held[0, 3].isnan() and held[0, 5].isnan() and held[0].isnan().sum() == 2 and (held[0].nan_to_num(0.0) == 0).all()
    assert (held[1] == 448).all()


@pytest.mark.parametrize("suffix", R.SUFFIXES)
@pytest.mark.parametrize("W,N,D", [(2, 3_000, 40), (1, 500, 515)])
def test_gradient_of_the_parameters_against_the_sum_that_was_not_rounded(suffix, W, N, D):
    """s is the sum t rounded to the rows' type: each term of dw is off by no more than dy inv times that rounding, beside the error in 32 bits."""
    gen, dtype = torch.Generator().manual_seed(N + D), R.TYPES[suffix]
    x, r, dy = ((torch.randn((W * N, D), generator=gen) * a).to(dtype) for a in (1.0, 3.0, 1.0))
    rows = (1 + 0.2 * torch.randn((W, D), generator=gen)).to(dtype)
    s, ds, inv, g = torch.empty_like(x.to(DEV)), torch.empty_like(x.to(DEV)), torch.empty(W * N, device=DEV), torch.empty_like(rows.to(DEV))
    getattr(lm, "cx_add_norm" + suffix)(x.to(DEV), r.to(DEV), rows.to(DEV), 0, s, None, 1e-6, inv=inv)
    getattr(lm, "cx_add_norm_grad" + suffix)(dy.to(DEV), s, inv, rows.to(DEV), 0, None, ds, None, g)
    ref = B.add_norm(x, r, rows.repeat_interleave(N, 0), torch.ones((W * N, D), dtype=torch.float64), float(torch.tensor(1e-6)))
    t, by = ref["t"], ref["inv"][:, None]
    terms = dy.double() * t * by
    err = dy.double().abs() * (by * (R.half_ulp(t, dtype) + ref["t_err"]) + t.abs() * ref["inv_err"][:, None]) + 3 * R.U * terms.abs()
    R.check(g, *B.summed(terms, err, terms.abs(), W, 1), "dw")


@pytest.mark.parametrize("suffix", R.SUFFIXES)
def test_slopes_of_the_gate_far_out(suffix):
    """silu' is 1 at +inf and 0 at -inf: the gradients of the convolution's input and of the scan's gate stay finite there."""
    dtype = R.TYPES[suffix]
    D, T, w = 5, 6, 0.5
    x = torch.ones((T, D), dtype=dtype)
    x[1], x[3], x[4, 2] = torch.inf, -torch.inf, torch.nan
    dy = torch.randn((T, D), generator=torch.Generator().manual_seed(1)).to(dtype)
    rows, dx = torch.cat([torch.full((1, D), w), torch.zeros((1, D))], 1).to(dtype).to(DEV), torch.empty((T, D), dtype=dtype, device=DEV)
    getattr(lm, "cx_short_conv_grad" + suffix)(x.to(DEV), dy.to(DEV), rows, 0, dx, None, torch.empty_like(rows), T, 1)
    assert torch.equal(dx[1].cpu(), (dy[1].float() * w).to(dtype)) and (dx[3] == 0).all() and dx[4, 2].isnan()
    assert dx.isnan().sum() == 1

    u, steps, bm = (torch.full((T, n), 0.5, dtype=dtype, device=DEV) for n in (D, D, 2))
    params = torch.full((1, D * 4), 0.25, dtype=dtype, device=DEV)
    read, y = (torch.empty((T, D), dtype=dtype, device=DEV) for _ in range(2))
    states = lm.select_states(u, T, 2)
    getattr(lm, "cx_select_scan" + suffix)(u, steps, bm, bm, params, 0, read, T)
    getattr(lm, "cx_select_scan" + suffix)(u, steps, bm, bm, params, 0, y, T, z=x.to(DEV), states=states)
    assert (y[1] == torch.inf).all() and (y[3] == 0).all()
    out = {k: torch.empty_like(u) for k in ("du", "ddt", "dz")}
    getattr(lm, "cx_select_scan_grad" + suffix)(u, steps, bm, bm, params, 0, dy.to(DEV), out["du"], out["ddt"], torch.empty_like(bm), torch.empty_like(bm), None,
                                                torch.empty_like(params), T, states, z=x.to(DEV), dz=out["dz"])
    want = dy[1].double() * read[1].cpu().double()
    assert ((out["dz"][1].cpu().double() - want).abs() <= 3 * torch.finfo(dtype).eps * want.abs()).all()          # read and dz are rounded once each
    assert (out["dz"][3] == 0).all() and out["dz"].isnan().sum() == 1
