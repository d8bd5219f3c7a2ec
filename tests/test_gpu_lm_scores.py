"""cx_token_scores against log-softmax, entropy and a stable sort in 64 bits."""
import pytest
import torch

import lm_reference as R
from paper_2012_15198_amd import cxlm as lm

DEV = "cuda:0"
pytestmark = pytest.mark.gpu


def run(suffix, z, tokens, K, scale=1.0, offset=0):
    """offset: the rows begin that many elements into longer ones."""
    N, V = z.shape
    zd = torch.full((N, V + offset + (3 if offset else 0)), torch.nan, dtype=z.dtype, device=DEV)[:, offset:offset + V]
    zd.copy_(z)
    logp, entropy = (torch.full((N,), 5.0, device=DEV) for _ in range(2))
    ids, top = torch.full((N, K), -7, dtype=torch.int32, device=DEV), torch.full((N, K), 5.0, device=DEV)
    getattr(lm, "cx_token_scores" + suffix)(zd, tokens.to(DEV), logp, entropy, ids if K else None, top if K else None, scale)
    return logp, entropy, ids, top


def compare(suffix, z, tokens, K, scale=1.0, offset=0):
    got = run(suffix, z, tokens, K, scale, offset)
    logp, entropy, ids, top = R.scores(z, tokens, K, scale)
    slack = R.lse_slack(z, scale) + R.U * torch.where(z.isfinite(), z.double().abs(), 0.0).amax(1) * scale * 2
    R.check(got[0], logp, slack, "logp")
    spread = 4 + min(40.0, float(z[z.isfinite()].double().abs().max()) * 2 * scale if z.isfinite().any() else 0.0)
    R.check(got[1], entropy, R.U * (64 + z.shape[1] / 256) * spread, "entropy")
    assert torch.equal(got[2].cpu(), ids), "ids"
    R.check(got[3], top, slack[:, None], "top")


@pytest.mark.parametrize("suffix", R.SUFFIXES)
@pytest.mark.parametrize("N,V,K", [(1, 1, 1), (1, 2, 2), (3, 7, 7), (2, 9, 0), (5, 64, 64), (4, 300, 60), (2, 1000, 5), (3, 4097, 64),
                                   (700, 515, 3), (2, 8192, 20), (1, 33_333, 64), (600, 17_001, 9), (1, 131_073, 20), (513, 40, 40),
                                   (130, 219, 28), (5, 3557, 63), (40, 900, 32), (40, 900, 33), (30, 318, 54), (3, 512, 64)])
def test_rows(suffix, N, V, K):
    gen = torch.Generator().manual_seed(N + V)
    z = (torch.randn((N, V), generator=gen) * 3).to(R.TYPES[suffix])
    tokens = torch.randint(0, V, (N,), generator=gen).int()
    if N > 2:
        tokens[0], tokens[1] = -1, V
    compare(suffix, z, tokens, K, scale=0.7, offset=N % 3)


@pytest.mark.parametrize("suffix", R.SUFFIXES)
@pytest.mark.parametrize("N,V", [(2, 30_000), (600, 5_000), (1, 300)])
def test_ties_go_to_the_lower_id(suffix, N, V):
    """All logits equal (an output layer of zeros), few values, and two zeros of different sign."""
    gen = torch.Generator().manual_seed(V)
    few = torch.randint(-2, 3, (N, V), generator=gen).float()
    few[few == 0] = torch.where(torch.rand(int((few == 0).sum()), generator=gen) < 0.5, 0.0, -0.0)
    for z in (torch.zeros((N, V)), few, torch.where(torch.rand((N, V), generator=gen) < 0.5, 0.0, -0.0)):
        compare(suffix, z.to(R.TYPES[suffix]), torch.zeros(N, dtype=torch.int32), 64)


@pytest.mark.parametrize("suffix", R.SUFFIXES)
@pytest.mark.parametrize("V,K", [(70_000, 64), (20_000, 33), (3_000, 64)])
def test_orders_that_crowd_the_threshold(suffix, V, K):
    """Rising and falling rows, and rows whose large values all lie in few threads' vectors, at any stride."""
    up = torch.linspace(-4, 4, V).repeat(2, 1)
    crowded = torch.linspace(-1, 0, V).repeat(4, 1)
    at = torch.arange(V)
    for row, (width, period) in enumerate(((8, 4096), (4, 2048), (512, 16384), (1600, V))):
        inside = at % period < width
        crowded[row, inside] += 5 + torch.rand(int(inside.sum()), generator=torch.Generator().manual_seed(row))
    for z in (up, up.flip(1), crowded):
        compare(suffix, z.to(R.TYPES[suffix]), torch.zeros(z.shape[0], dtype=torch.int32), K)
        many = z.repeat(300, 1)[:513].to(R.TYPES[suffix])               # a workgroup a row
        compare(suffix, many, torch.zeros(513, dtype=torch.int32), K)


@pytest.mark.parametrize("suffix", R.SUFFIXES)
@pytest.mark.parametrize("N,V", [(9, 12_345), (9, 21), (640, 2_049)])
def test_masks_infinities_and_nan(suffix, N, V):
    gen = torch.Generator().manual_seed(N * V)
    dtype = R.TYPES[suffix]
    z = (torch.randn((N, V), generator=gen) * 2).to(dtype)
    z[0, torch.rand(V, generator=gen) < 0.9] = -torch.inf
    z[1] = -torch.inf                                                   # nothing left
    z[2] = -torch.inf
    z[2, V - 1] = 1.0                                                   # one left
    z[3] = torch.finfo(dtype).min                                       # the lowest value everywhere: uniform
    z[4, : V // 2] = torch.finfo(dtype).min
    z[5, V // 3] = torch.nan
    z[6, V // 3] = torch.inf
    z[7] = torch.nan
    z[8, ::2], z[8, 1::2] = torch.finfo(dtype).max, torch.finfo(dtype).min
    tokens = torch.randint(0, V, (N,), generator=gen).int()
    tokens[2] = V - 1
    got = run(suffix, z, tokens, 16, 1.0)
    logp, entropy, ids, top = R.scores(z, tokens, 16, 1.0)
    ordinary = torch.ones(N, dtype=torch.bool)
    ordinary[[3, 4, 8]] = False
    slack = R.lse_slack(z[ordinary], 1.0)
    R.check(got[0].cpu()[ordinary], logp[ordinary], slack)
    R.check(got[1].cpu()[ordinary], entropy[ordinary], R.U * (64 + V / 256) * 44)
    R.check(got[3].cpu()[ordinary], top[ordinary], slack[:, None])
    # rows with extreme values: log sum exp is not representable beside them, differences are
    equal = torch.log(torch.tensor(float(V)))
    assert abs(float(got[1][3]) - equal) < 1e-4 and abs(float(got[0][3]) + equal) < 1e-4 and abs(float(got[3][3, 0]) + equal) < 1e-4
    assert abs(float(got[1][8]) - torch.log(torch.tensor((V + 1) // 2.0))) < 1e-4
    R.check(got[1].cpu()[4:5], entropy[4:5], R.U * (64 + V / 256) * 44)
    assert torch.equal(got[2].cpu(), ids)


def test_outputs_that_are_not_wanted_and_no_rows():
    z = torch.randn((3, 50), device=DEV)
    entropy = torch.empty(3, device=DEV)
    lm.cx_token_scores(z, None, None, entropy)
    R.check(entropy, R.scores(z.cpu(), torch.zeros(3, dtype=torch.int32), 0, 1.0)[1], R.U * 64 * 20)
    ids, top = torch.empty((3, 4), dtype=torch.int32, device=DEV), torch.empty((3, 4), device=DEV)
    lm.cx_token_scores(z, None, None, None, ids, top)
    assert torch.equal(ids.cpu(), R.order(z.cpu())[:, :4].int())
    lm.cx_token_scores(torch.empty((0, 50), device=DEV), torch.empty(0, dtype=torch.int32, device=DEV), torch.empty(0, device=DEV))


@pytest.mark.parametrize("suffix", R.SUFFIXES)
@pytest.mark.parametrize("V", [700, 70_000])
def test_scales_at_the_ends_of_their_range(suffix, V):
    """The largest scale leaves the maximum alone, shared by the logits that equal it; the smallest makes every row uniform."""
    z = torch.randn((3, V), generator=torch.Generator().manual_seed(V)).to(R.TYPES[suffix])
    z[1, 100], z[1, 650] = 20.0, 20.0
    best = z.double().amax(1, keepdim=True)
    at = (z.double() == best).double()
    tokens = at.argmax(1).int()
    tokens[2] = int(z[2].double().argmin())
    for scale, count in ((2.3e38, at.sum(1)), (1e-38, torch.full((3,), float(V), dtype=torch.float64))):
        logp, entropy, ids, _ = run(suffix, z, tokens, 2, scale)
        want = -count.log()
        if scale > 1:
            want[2] = -torch.inf
        R.check(logp, want, R.U * (64 + V / 256) * 20)
        R.check(entropy, count.log(), R.U * (64 + V / 256) * 20)
        assert torch.equal(ids.cpu(), R.order(z)[:, :2].int())
