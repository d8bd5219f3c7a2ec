"""cx_gated_scan and cx_gated_scan_grad against the recurrence in 64 bits, step by step."""
import pytest
import torch

import lm_reference as R
from paper_2012_15198_amd import cxlm as lm

DEV = "cuda:0"
pytestmark = pytest.mark.gpu


def inputs(B, T, D, dtype, seed, packed, strided):
    gen = torch.Generator().manual_seed(seed)
    wide = (lambda s: (torch.randn((B * T, 3 * D + 1), generator=gen) * s).to(dtype)) if strided else None
    normal = lambda m, s: (torch.randn((B * T, D), generator=gen) * s + m).to(dtype)
    f, x, dy = normal(2.0, 1.5), normal(0.0, 1.0), normal(0.0, 1.0)
    h0, dh = torch.randn((B, D), generator=gen), torch.randn((B, D), generator=gen)
    reset = None
    if packed:
        reset = (torch.rand((B, T), generator=gen) < 0.15).to(torch.uint8) * 7
        reset[0, 0] = 1                                        # at the first step: h0 is not used
        if B > 1:
            reset[1] = 1                                       # every step a document of its own
        if T > 1:
            reset[:, T - 1] = 1
    return f, x, dy, h0, dh, reset, wide


def place(t, strided):
    """On the device; strided: inside longer rows that begin at an odd element."""
    if not strided:
        return t.to(DEV)
    wide = torch.full((t.shape[0], t.shape[1] + 5), 3.0, dtype=t.dtype, device=DEV)
    wide[:, 1:1 + t.shape[1]] = t.to(DEV)
    return wide[:, 1:1 + t.shape[1]]


SHAPES = [  # B, T, D
    (1, 1, 1), (3, 1, 2), (2, 1, 300), (1, 2, 1), (2, 15, 3), (1, 16, 64), (2, 17, 129), (3, 127, 65), (1, 128, 257), (2, 129, 7),
    (1, 300, 128), (1, 1111, 33), (2, 2050, 5), (130, 40, 20)]


@pytest.mark.parametrize("suffix", R.SUFFIXES)
@pytest.mark.parametrize("packed,strided", [(False, False), (True, True), (True, False), (False, True)])
@pytest.mark.parametrize("B,T,D", SHAPES)
def test_both_directions(suffix, packed, strided, B, T, D):
    dtype = R.TYPES[suffix]
    f, x, dy, h0, dh, reset, _ = inputs(B, T, D, dtype, B * T + D, packed, strided)
    on = lambda t: None if t is None else t.to(DEV)
    fd, xd, dyd = (place(t, strided) for t in (f, x, dy))
    y, df, dx = (place(torch.full_like(f, torch.nan), strided) for _ in range(3))
    h_last, dh0 = (torch.full((B, D), torch.nan, device=DEV) for _ in range(2))
    states = lm.scan_states(fd, T)
    getattr(lm, "cx_gated_scan" + suffix)(fd, xd, y, T, h0=on(h0), h_last=h_last, reset=on(reset), states=states)
    getattr(lm, "cx_gated_scan_grad" + suffix)(fd, xd, dyd, df, dx, T, states, dh_last=on(dh), dh0=dh0, reset=on(reset))
    ry, rh, before = R.scan(f, x, T, h0, reset)
    rf, rx, r0, high = R.scan_grad(f, x, dy, T, h0, reset, dh)
    M = float(torch.maximum(x.double().abs().max(), h0.double().abs().max()))
    L, reach = R.memory(f, T), float(f.double().abs().max())
    err_h = R.U * M * (16 + reach) * (1 + L)
    R.check(y, ry, err_h, "y")
    R.check(h_last, rh, err_h, "h_last")
    R.check(states.reshape(B, -1, D), before[:, ::lm.CX_SCAN_CHUNK], err_h, "states") if reset is None else None
    err_r = R.U * high * (16 + reach) * (1 + L)
    R.check(dx, rx, err_r, "dx")
    R.check(df, rf, 2 * M * err_r + high * err_h, "df")
    R.check(dh0, r0, err_r, "dh0")
    if strided:
        for t in (y, df, dx):
            assert (t._base[:, 0] == 3).all() and (t._base[:, 1 + D:] == 3).all()


@pytest.mark.parametrize("suffix", R.SUFFIXES)
@pytest.mark.parametrize("packed,strided", [(False, False), (True, True)])
@pytest.mark.parametrize("B,T,D", [(300, 1, 65), (140, 37, 129), (66, 131, 200), (50, 259, 258), (260, 20, 2), (70, 300, 3)])
def test_columns_of_a_lane_at_many_and_few_sequences(suffix, packed, strided, B, T, D):
    test_both_directions(suffix, packed, strided, B, T, D)


@pytest.mark.parametrize("suffix", R.SUFFIXES)
def test_defaults_and_halves_of_one_projection(suffix):
    """No states at the ends; gates and inputs (and their gradients) as the two halves of the rows of one matrix."""
    dtype, B, T, D = R.TYPES[suffix], 2, 70, 33
    f, x, dy, _, _, _, _ = inputs(B, T, D, dtype, 3, False, False)
    both = torch.cat([f, x], 1).to(DEV)
    grads = torch.empty_like(both)
    y = torch.empty((B * T, D), dtype=dtype, device=DEV)
    states = lm.scan_states(y, T)
    getattr(lm, "cx_gated_scan" + suffix)(both[:, :D], both[:, D:], y, T, states=states)
    getattr(lm, "cx_gated_scan_grad" + suffix)(both[:, :D], both[:, D:], dy.to(DEV), grads[:, :D], grads[:, D:], T, states)
    ry, _, _ = R.scan(f, x, T, None, None)
    rf, rx, _, high = R.scan_grad(f, x, dy, T, None, None, None)
    M, L, reach = float(x.double().abs().max()), R.memory(f, T), float(f.double().abs().max())
    err = R.U * (16 + reach) * (1 + L)
    R.check(y, ry, M * err)
    R.check(grads[:, D:], rx, high * err)
    R.check(grads[:, :D], rf, 3 * M * high * err)


@pytest.mark.parametrize("suffix", R.SUFFIXES)
@pytest.mark.parametrize("D", [1, 129, 256])
def test_steps_one_by_one_with_the_state_in_place_equal_the_sequence(suffix, D):
    dtype, B, T = R.TYPES[suffix], 3, 37
    f, x, _, h0, _, reset, _ = inputs(B, T, D, dtype, 8, True, False)
    state = h0.to(DEV)
    fd, xd, rd = f.to(DEV).view(B, T, D), x.to(DEV).view(B, T, D), reset.to(DEV)
    y = torch.empty((B, D), dtype=dtype, device=DEV)
    ry, rh, _ = R.scan(f, x, T, h0, reset)
    M, L, reach = float(max(x.double().abs().max(), h0.abs().max())), R.memory(f, T), float(f.double().abs().max())
    err = R.U * M * (16 + reach) * (1 + L)
    for t in range(T):
        getattr(lm, "cx_gated_scan" + suffix)(fd[:, t], xd[:, t], y, 1, h0=state, h_last=state, reset=rd[:, t:t + 1].contiguous())
        R.check(y, ry.view(B, T, D)[:, t], err)
    R.check(state, rh, err)


@pytest.mark.parametrize("T,h_alias", [(2000, True), (64, True), (2000, False)])
def test_state_in_place_over_long_and_split_sequences(T, h_alias):
    B, D = 1, 129
    f, x, _, h0, _, _, _ = inputs(B, T, D, torch.bfloat16, 5, False, False)
    state = h0.to(DEV)
    last = state if h_alias else torch.empty_like(state)
    y = torch.empty((T, D), dtype=torch.bfloat16, device=DEV)
    lm.cx_gated_scan_bf16(f.to(DEV), x.to(DEV), y, T, h0=state, h_last=last)
    ry, rh, _ = R.scan(f, x, T, h0, None)
    err = R.U * float(max(x.double().abs().max(), h0.abs().max())) * (16 + float(f.double().abs().max())) * (1 + R.memory(f, T))
    R.check(y, ry, err)
    R.check(last, rh, err)


@pytest.mark.parametrize("suffix", R.SUFFIXES)
@pytest.mark.parametrize("T", [9, 200, 1500])
def test_nothing_crosses_a_reset(suffix, T):
    """NaN and infinities in one document leave the others as they are, forward and backward."""
    dtype, B, D, cut = R.TYPES[suffix], 1, 40, T * 2 // 3
    f, x, dy, h0, dh, _, _ = inputs(B, T, D, dtype, 2, False, False)
    reset = torch.zeros((B, T), dtype=torch.uint8)
    reset[0, cut] = 1
    dirty = [t.clone() for t in (f, x, dy)]
    dirty[1][cut - 1, ::2] = torch.inf
    dirty[0][cut - 1, 1::3] = torch.nan
    dirty[1][0, 3] = torch.nan
    outs = []
    for ff, xx, gg in ((f, x, dy), dirty):
        y, df, dx = (torch.empty((T, D), dtype=dtype, device=DEV) for _ in range(3))
        h_last, dh0 = (torch.empty((B, D), device=DEV) for _ in range(2))
        states = lm.scan_states(y, T)
        ff, xx, gg = ff.to(DEV), xx.to(DEV), gg.to(DEV)
        getattr(lm, "cx_gated_scan" + suffix)(ff, xx, y, T, h0=h0.to(DEV), h_last=h_last, reset=reset.to(DEV), states=states)
        getattr(lm, "cx_gated_scan_grad" + suffix)(ff, xx, gg, df, dx, T, states, dh_last=dh.to(DEV), dh0=dh0, reset=reset.to(DEV))
        outs.append((y[cut:], h_last, df[cut:], dx[cut:]))
    for clean, got in zip(*outs):
        assert clean.isfinite().all() and torch.equal(clean, got)
    # and a NaN in the later document's gradient does not reach the earlier one's
    late = dy.clone()
    late[cut, 5] = torch.nan
    grads = []
    for gg, last in ((dy, dh), (late, torch.full_like(dh, torch.inf))):
        y, df, dx = (torch.empty((T, D), dtype=dtype, device=DEV) for _ in range(3))
        states = lm.scan_states(y, T)
        getattr(lm, "cx_gated_scan" + suffix)(f.to(DEV), x.to(DEV), y, T, reset=reset.to(DEV), states=states)
        getattr(lm, "cx_gated_scan_grad" + suffix)(f.to(DEV), x.to(DEV), gg.to(DEV), df, dx, T, states, dh_last=last.to(DEV), reset=reset.to(DEV))
        grads.append((df[:cut], dx[:cut]))
    for clean, got in zip(*grads):
        assert clean.isfinite().all() and torch.equal(clean, got)


def test_gates_at_their_ends():
    """Gates of 0 and 1 to the last bit, infinite ones included: the state is replaced or kept, and nothing becomes NaN."""
    f = torch.tensor([[torch.inf], [200.0], [88.0], [-torch.inf], [-200.0], [-88.0], [0.0]])
    x = torch.arange(1.0, 8.0)[:, None]
    y = torch.empty((7, 1), device=DEV)
    lm.cx_gated_scan(f.to(DEV), x.to(DEV), y, 7, h0=torch.full((1, 1), 9.0, device=DEV))
    ref = R.scan(f, x, 7, torch.full((1, 1), 9.0), None)[0]
    R.check(y, ref, 1e-6 * ref.abs())


def test_no_steps():
    h0 = torch.randn((4, 6), device=DEV)
    out = torch.empty_like(h0)
    empty = torch.empty((0, 6), device=DEV)
    lm.cx_gated_scan(empty, empty, empty, 0, h0=h0, h_last=out)
    assert torch.equal(out, h0)
    lm.cx_gated_scan(empty, empty, empty, 0, h_last=out)
    assert (out == 0).all()
    lm.cx_gated_scan_grad(empty, empty, empty, empty, empty, 0, None, dh_last=h0, dh0=out)
    assert torch.equal(out, h0)


def test_gradient_against_differences():
    """Central differences of sum(y * c) + sum(h_last * k) in 64 bits through the reference forward, at drawn places."""
    B, T, D, gen = 2, 50, 4, torch.Generator().manual_seed(6)
    f, x, dy, h0, dh, reset, _ = inputs(B, T, D, torch.float32, 6, True, False)
    reset[1] = 0
    df, dx = torch.empty((B * T, D), device=DEV), torch.empty((B * T, D), device=DEV)
    dh0, y = torch.empty((B, D), device=DEV), torch.empty((B * T, D), device=DEV)
    states = lm.scan_states(y, T)
    lm.cx_gated_scan(f.to(DEV), x.to(DEV), y, T, h0=h0.to(DEV), reset=reset.to(DEV), states=states)
    lm.cx_gated_scan_grad(f.to(DEV), x.to(DEV), dy.to(DEV), df, dx, T, states, dh_last=dh.to(DEV), dh0=dh0, reset=reset.to(DEV))

    def value(f, x, h0):
        ys, last, _ = R.scan(f, x, T, h0, reset)
        return float((ys * dy.double()).sum() + (last * dh.double()).sum())

    args = [f.double(), x.double(), h0.double()]
    for which, grad in ((0, df), (1, dx), (2, dh0)):
        for place in torch.randint(0, args[which].numel(), (12,), generator=gen).tolist():
            step = 1e-5
            ends = []
            for sign in (1, -1):
                moved = [a.clone() for a in args]
                moved[which].view(-1)[place] += sign * step
                ends.append(value(*moved))
            slope = (ends[0] - ends[1]) / (2 * step)
            assert abs(slope - float(grad.reshape(-1)[place])) < 2e-5 * (1 + abs(slope)), (which, place)
