"""Buffers that lie between the rows of another one share nothing with it: such calls are taken, and what lies beside stays as it was."""
import pytest
import torch

import lm_reference as R
from paper_2012_15198_amd import cxlm as lm

DEV = "cuda:0"
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("suffix", R.SUFFIXES)
def test_gradient_rows_in_two_halves_of_one_matrix(suffix):
    W, N, V, D = 3, 200, 40, 13
    gen = torch.Generator().manual_seed(5)
    P, dtype = V * D + 2, R.TYPES[suffix]
    both = torch.randn((W, 2 * P), generator=gen).to(dtype)
    tokens = torch.randint(-1, V, (W, N), generator=gen).int()
    dout = torch.randn((W * N, D), generator=gen).to(dtype)
    on = both.to(DEV)
    getattr(lm, "cx_embed_grad" + suffix)(dout.to(DEV), tokens.to(DEV), on[:, P:], on[:, :P], 1, V)
    ref, size = R.embed_grad(dout, tokens, both[:, P:], 1, V, D, 1.0)
    longest = max(int(torch.bincount(t[t >= 0].long()).max()) for t in tokens)
    R.check(on[:, 1:1 + V * D], ref, (longest + 3) * R.U * size)
    assert torch.equal(on[:, P:].cpu(), both[:, P:]) and torch.equal(on[:, 0].cpu(), both[:, 0]) and torch.equal(on[:, P - 1].cpu(), both[:, P - 1])


@pytest.mark.parametrize("suffix", R.SUFFIXES)
@pytest.mark.parametrize("N", [3, 520])
def test_logits_and_their_gradient_in_two_halves_of_one_matrix(suffix, N):
    V, K, dtype = 1_003, 5, R.TYPES[suffix]
    gen = torch.Generator().manual_seed(N)
    both = torch.full((N, 2 * V), 7.0, dtype=dtype)
    both[:, V:] = (torch.randn((N, V), generator=gen) * 2).to(dtype)
    ids, labels = torch.randint(0, V, (N, K), generator=gen).int(), torch.randint(0, V, (N,), generator=gen).int()
    t, gout = torch.randn((N, K), generator=gen), torch.rand(N, generator=gen) + 0.5
    ref, grad, slack, grad_slack = R.distill(both[:, V:], ids, t, labels, gout, 2.0, 0.7, 0.3)
    for step in (True, False):
        on, loss, stats = both.to(DEV), torch.empty(N, device=DEV), torch.empty((N, 4), device=DEV)
        head = (on[:, V:], ids.to(DEV), t.to(DEV), labels.to(DEV))
        if step:
            getattr(lm, "cx_distill_step" + suffix)(*head, gout.to(DEV), loss, on[:, :V], 2.0, 0.7, 0.3)
        else:
            getattr(lm, "cx_distill_loss" + suffix)(*head, loss, stats, 2.0, 0.7, 0.3)
            getattr(lm, "cx_distill_grad" + suffix)(*head, stats, gout.to(DEV), on[:, :V], 2.0, 0.7, 0.3)
        R.check(loss, ref, slack)
        R.check(on[:, :V], grad, grad_slack)
        assert torch.equal(on[:, V:].cpu(), both[:, V:])


def test_scores_beside_their_logits():
    """float32 results of two rows in the columns behind the first one's logits."""
    V = 900
    wide = torch.randn((2, V + 8), generator=torch.Generator().manual_seed(3))
    on = wide.to(DEV)
    tokens = torch.tensor([17, 899], dtype=torch.int32)
    lm.cx_token_scores(on[:, :V], tokens.to(DEV), on[0, V:V + 2], on[0, V + 2:V + 4])
    logp, entropy, _, _ = R.scores(wide[:, :V], tokens, 0, 1.0)
    R.check(on[0, V:V + 2], logp, R.lse_slack(wide[:, :V], 1.0) + 8 * R.U)
    R.check(on[0, V + 2:V + 4], entropy, R.U * (64 + V / 256) * 20)
    assert torch.equal(on[:, :V].cpu(), wide[:, :V]) and torch.equal(on[0, V + 4:].cpu(), wide[0, V + 4:]) and torch.equal(on[1].cpu(), wide[1])


def test_states_between_the_rows_of_a_projection():
    """One sequence: the state that enters and the one that leaves lie beside the gates of two steps."""
    T, D = 300, 33
    wide = torch.randn((T, 3 * D), generator=torch.Generator().manual_seed(9))
    on, y = wide.to(DEV), torch.empty((T, D), device=DEV)
    lm.cx_gated_scan(on[:, :D], on[:, D:2 * D], y, T, h0=on[0:1, 2 * D:], h_last=on[1:2, 2 * D:])
    want, last = torch.empty_like(y), torch.empty((1, D), device=DEV)
    f, x, h0 = (wide[:, k * D:(k + 1) * D].contiguous().to(DEV) for k in range(3))
    lm.cx_gated_scan(f, x, want, T, h0=h0[:1].clone(), h_last=last)
    assert torch.equal(y, want) and torch.equal(on[1:2, 2 * D:], last)
    assert torch.equal(on[:, :2 * D].cpu(), wide[:, :2 * D]) and torch.equal(on[0, 2 * D:].cpu(), wide[0, 2 * D:]) and torch.equal(on[2:].cpu(), wide[2:])
