"""Calls of more tokens or rows than one launch or one piece length takes: gradients of more than 16,384 tokens a worker, logits of more than
65,535 rows."""
import pytest
import torch

import lm_reference as R
from paper_2012_15198_amd import cxlm as lm

DEV = "cuda:0"
pytestmark = pytest.mark.gpu


def tokens_of(kind, W, N, V, gen):
    if kind == "one":
        t = torch.full((W, N), V // 2)
    elif kind == "two":                                        # long lists whose ends share a piece
        t = torch.where(torch.arange(N) % 3 == 0, V - 1, V // 3).expand(W, N).clone()
    else:
        t = (V ** torch.rand((W, N), generator=gen, dtype=torch.float64)).long().clamp(0, V - 1)
        t[torch.rand((W, N), generator=gen) < 0.05] = -1
    return t.int()


@pytest.mark.parametrize("suffix", R.SUFFIXES)
@pytest.mark.parametrize("mode", ["alone", "added", "in place"])
@pytest.mark.parametrize("W,N,V,D,kind", [(2, 20_011, 700, 3, "zipf"), (1, 20_011, 90, 3, "one"), (1, 16_385, 50, 129, "two"), (2, 20_011, 2_500, 129, "zipf"),
                                          (1, 20_011, 300, 140, "one"), (1, 32_768, 4_000, 768, "zipf"), (1, 16_384, 600, 33, "zipf"),
                                          (1, 16_389, 300_000, 3, "zipf")])
def test_gradients_of_many_tokens(suffix, mode, W, N, V, D, kind):
    gen = torch.Generator().manual_seed(N + V + D)
    dtype, scale, offset = R.TYPES[suffix], 1.5, 3
    tokens = tokens_of(kind, W, N, V, gen)
    dout = torch.randn((W * N, D), generator=gen).to(dtype)
    base = torch.randn((W, offset + V * D + 1), generator=gen).to(dtype)
    g_in = None if mode == "alone" else base.to(DEV)
    g_out = g_in if mode == "in place" else torch.full_like(base, torch.nan).to(DEV)
    getattr(lm, "cx_embed_grad" + suffix)(dout.to(DEV), tokens.to(DEV), g_in, g_out, offset, V, scale)
    ref, size = R.embed_grad(dout, tokens, None if mode == "alone" else base, offset, V, D, scale)
    # additions on the way of a term: within its piece of at most 64 tokens, then the pieces of its list; the scale and g_in
    longest = max(int(torch.bincount(t[t >= 0].long()).max()) for t in tokens)
    R.check(g_out[:, offset:offset + V * D], ref, (min(longest, 64) + -(-longest // 16) + 5) * R.U * size)
    edges = torch.cat([g_out[:, :offset], g_out[:, offset + V * D:]], 1).cpu()
    want = torch.cat([base[:, :offset], base[:, offset + V * D:]], 1) if mode == "in place" else torch.full_like(edges, torch.nan)
    assert torch.equal(edges.nan_to_num(9.0), want.nan_to_num(9.0))


ROWS = 65_535 + 70


@pytest.mark.parametrize("suffix", R.SUFFIXES)
@pytest.mark.parametrize("V,K,labels", [(37, 5, True), (21, 0, True), (50, 50, False)])
def test_scores_of_many_rows(suffix, V, K, labels):
    gen = torch.Generator().manual_seed(V)
    z = (torch.randn((ROWS, V), generator=gen) * 3).to(R.TYPES[suffix])
    tokens = torch.randint(-1, V + 1, (ROWS,), generator=gen).int()
    on = torch.full((ROWS, V + 3), torch.nan, dtype=z.dtype, device=DEV)[:, 1:1 + V]
    on.copy_(z)
    logp, entropy = (torch.full((ROWS,), 5.0, device=DEV) for _ in range(2))
    ids, top = torch.full((ROWS, K), -7, dtype=torch.int32, device=DEV), torch.full((ROWS, K), 5.0, device=DEV)
    getattr(lm, "cx_token_scores" + suffix)(on, tokens.to(DEV) if labels else None, logp if labels else None, entropy, ids if K else None, top if K else None)
    want = R.scores(z, tokens, K, 1.0)
    slack = R.lse_slack(z, 1.0) + R.U * z.double().abs().amax(1) * 2
    if labels:
        R.check(logp, want[0], slack)
    R.check(entropy, want[1], R.U * 64 * 30)
    assert torch.equal(ids.cpu(), want[2])
    R.check(top, want[3], slack[:, None])


@pytest.mark.parametrize("suffix", R.SUFFIXES)
@pytest.mark.parametrize("V,K,labels", [(37, 5, True), (21, 0, True), (50, 50, False)])
def test_distillation_of_many_rows(suffix, V, K, labels):
    gen = torch.Generator().manual_seed(V)
    z = (torch.randn((ROWS, V), generator=gen) * 2).to(R.TYPES[suffix])
    ids = torch.randint(-1, V, (ROWS, K), generator=gen).int()
    t, gout = torch.randn((ROWS, K), generator=gen) * 2, torch.rand(ROWS, generator=gen) + 0.5
    label = torch.randint(-1, V, (ROWS,), generator=gen).int() if labels else None
    loss, grad, slack, grad_slack = R.distill(z, ids, t, label, gout, 2.0, 0.7, 0.3)
    for step in (True, False):
        on = torch.full((ROWS, V + 3), 3.0, dtype=z.dtype, device=DEV)
        on[:, 1:1 + V] = z.to(DEV)
        dz = torch.full((ROWS, V + 5), 3.0, dtype=z.dtype, device=DEV)
        got, stats = torch.full((ROWS,), 5.0, device=DEV), torch.empty((ROWS, 4), device=DEV)
        head = (on[:, 1:1 + V], ids.to(DEV), t.to(DEV), None if label is None else label.to(DEV))
        if step:
            getattr(lm, "cx_distill_step" + suffix)(*head, gout.to(DEV), got, dz[:, 2:2 + V], 2.0, 0.7, 0.3)
        else:
            getattr(lm, "cx_distill_loss" + suffix)(*head, got, stats, 2.0, 0.7, 0.3)
            getattr(lm, "cx_distill_grad" + suffix)(*head, stats, gout.to(DEV), dz[:, 2:2 + V], 2.0, 0.7, 0.3)
        R.check(got, loss, slack, "loss")
        R.check(dz[:, 2:2 + V], grad, grad_slack, "dz")
        assert (dz[:, :2] == 3).all() and (dz[:, 2 + V:] == 3).all() and (on[:, 0] == 3).all() and (on[:, 1 + V:] == 3).all()


def test_long_rows_of_a_second_launch_equal_the_same_rows_alone():
    """65,605 float32 rows of 16,401: the gradient reads them again, past what one workgroup's registers hold of it.  Rows around the launches' seam."""
    V, K = 16_401, 3
    gen = torch.Generator(DEV).manual_seed(1)
    z = torch.empty((ROWS, V), device=DEV).normal_(0.0, 2.0, generator=gen)
    ids, labels = (torch.randint(0, V, s, device=DEV, generator=gen).int() for s in ((ROWS, K), (ROWS,)))
    t, gout = (torch.randn(s, device=DEV, generator=gen) for s in ((ROWS, K), (ROWS,)))
    loss, stats, dz = torch.empty(ROWS, device=DEV), torch.empty((ROWS, 4), device=DEV), torch.empty_like(z)
    lm.cx_distill_loss(z, ids, t, labels, loss, stats, 2.0, 0.7, 0.3)
    lm.cx_distill_grad(z, ids, t, labels, stats, gout, dz, 2.0, 0.7, 0.3)
    for rows in (slice(0, 600), slice(65_000, ROWS)):
        part = [v[rows] for v in (z, ids, t, labels)]
        n = part[0].shape[0]
        loss2, stats2, dz2 = torch.empty(n, device=DEV), torch.empty((n, 4), device=DEV), torch.empty((n, V), device=DEV)
        lm.cx_distill_loss(*part, loss2, stats2, 2.0, 0.7, 0.3)
        lm.cx_distill_grad(*part, stats2, gout[rows], dz2, 2.0, 0.7, 0.3)
        assert torch.equal(loss[rows], loss2) and torch.equal(stats[rows], stats2) and torch.equal(dz[rows], dz2)
