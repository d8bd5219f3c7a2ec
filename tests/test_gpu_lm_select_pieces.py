"""cx_select_scan and cx_select_scan_grad where a span of steps is composed of several pieces, against the scan in 64 bits: a few columns of
many, with nothing pulling on the others."""
import pytest
import torch

import lm_block_reference as BR
import lm_reference as R
from lm_block_util import DEV
from lm_split import FORWARD_AT_ONCE, GRADIENT_AT_ONCE, empty_pieces, split, workspaces
from paper_2012_15198_amd import cxlm as lm
from test_gpu_lm_select import OFFSET, Case

pytestmark = pytest.mark.gpu

CASES = [  # suffix, W, B, T, D, N, packed: what is composed, forward and backward
    ("_bf16", 2, 8, 390, 2_048, 16, True),       # 4 spans of 2 pieces, the last piece of all empty; 2 of 5, likewise
    ("", 1, 8, 390, 2_048, 10, False),           # the same with three states a lane
    ("_f16", 2, 6, 1_111, 515, 7, True),         # backward 9 spans of 3 pieces, the last one empty
    ("_f16", 1, 3, 2_099, 505, 3, True),         # forward 33 of 2: enter in eight stretches
    ("_bf16", 3, 3, 2_067, 250, 6, True),        # backward 33 of 2: enter in eight stretches
    ("", 1, 3, 2_067, 250, 16, False),
]


@pytest.mark.parametrize("suffix,W,B,T,D,N,packed", CASES)
def test_spans_of_several_pieces(suffix, W, B, T, D, N, packed):
    forward, backward = split(B, T, D, FORWARD_AT_ONCE), split(B, T, D, GRADIENT_AT_ONCE)
    assert forward[0] > 1 and max(forward[1], backward[1]) > 1
    assert (lm.cx_select_workspace(B, T, D, N), lm.cx_select_grad_workspace(B, T, D, N)) == workspaces(B, T, D, N)
    if T < 2_000:
        assert empty_pieces(T, *backward) > 0
    else:
        assert max((s[0] - 1) * s[1] for s in (forward, backward)) >= 64
    c = Case(suffix, W, B, T, D, N)
    if packed:
        c.reset = (torch.rand((B, T), generator=c.gen) < 0.004).to(torch.uint8) * 7          # some pieces forget, some do not
        c.reset[B - 1] = 0
    at = torch.tensor([0, 17, 63, 64 % D, D // 2, D - 2, D - 1])
    others = torch.ones(D, dtype=torch.bool)
    others[at] = False
    c.dy[:, others], c.dh[:, others] = 0, 0
    d, on = c.on(), lambda t: None if t is None else t.to(DEV)
    y, h_last, dh0, g = torch.empty_like(d["u"]), torch.empty((B, D, N), device=DEV), torch.empty((B, D, N), device=DEV), torch.empty_like(on(c.rows))
    states = lm.select_states(y, T, N)
    c.forward(d, y, states, on(c.h0), h_last, on(c.reset))
    grads = c.backward(d, states, None, g, on(c.dh), dh0, on(c.reset))

    some = [t[:, at].contiguous() for t in (c.u, c.dt)], [t[:, at].contiguous() for t in (c.A_log, c.bias, c.skip)]
    args = (*some[0], c.bm, c.cm, c.z[:, at].contiguous(), T, *some[1], c.h0[:, at], c.reset)
    columns = lambda t: t.cpu()[:, at]
    ref = BR.select(*args)
    R.check(columns(y).reshape(B, T, -1), ref["y"], ref["y_err"], "y")
    R.check(columns(h_last), ref["h_last"], ref["h_last_err"], "h_last")
    if not packed:
        R.check(states.cpu()[:, :, at], ref["before"][:, ::16], ref["before_err"][:, ::16], "states")
    ref = BR.select_grad(*args, c.dy[:, at], c.dh[:, at])
    for key, name in (("u", "du"), ("dt", "ddt"), ("z", "dz")):
        R.check(columns(grads[key]).reshape(B, T, -1), ref[name], ref[name + "_err"], name)
        assert (grads[key].cpu()[:, others] == 0).all(), name
    for key, name in (("bm", "db"), ("cm", "dc")):
        R.check(grads[key].reshape(B, T, N), ref[name], ref[name + "_err"], name)
    R.check(columns(dh0), ref["dh0"], ref["dh0_err"], "dh0")
    g = g.cpu()[:, OFFSET:]
    for name, got in (("dA", g[:, :D * N].reshape(W, D, N)[:, at].reshape(W, -1)), ("dbias", g[:, D * N:D * (N + 1)][:, at]),
                      ("dskip", g[:, D * (N + 1):D * (N + 2)][:, at])):
        R.check(got, *BR.summed(ref[name], ref[name + "_err"], ref[name + "_size"], W, T), name)
