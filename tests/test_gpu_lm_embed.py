"""cx_embed_lookup and cx_embed_grad against their definitions in 64 bits."""
import pytest
import torch

import lm_reference as R
from paper_2012_15198_amd import cxlm as lm

DEV = "cuda:0"
pytestmark = pytest.mark.gpu


def tokens_of(kind, W, N, V, gen):
    if kind == "zipf":
        t = ((torch.rand((W, N), generator=gen, dtype=torch.float64) * (V + 1.0)).log().clamp_min(0).exp() - 1).long().clamp(0, V - 1)
        t = (V ** torch.rand((W, N), generator=gen, dtype=torch.float64)).long().clamp(0, V - 1) if V > 1 else t * 0
        t[torch.rand((W, N), generator=gen) < 0.1] = -1
    elif kind == "one":                       # a single token again and again: one list, cut into pieces
        t = torch.full((W, N), V // 2)
    elif kind == "two":                       # two long lists that share a piece
        t = torch.where(torch.arange(N) % 3 == 0, V - 1, V // 3).expand(W, N).clone()
    elif kind == "none":                      # padding alone, on both sides of the vocabulary
        t = torch.where(torch.arange(N) % 2 == 0, -1, V).expand(W, N).clone()
        if N:
            t[0, 0] = 2**31 - 1
            t[0, -1] = -2**31
    else:
        t = torch.randint(0, V, (W, N), generator=gen)
    return t.int()


SHAPES = [  # W, N, V, D, offset, extra row length, tokens
    (1, 1, 1, 1, 0, 0, "any"), (1, 1, 5, 8, 0, 0, "any"), (2, 7, 11, 3, 5, 3, "any"), (3, 64, 40, 33, 1, 0, "zipf"),
    (2, 65, 513, 16, 7, 1, "zipf"), (1, 300, 512, 129, 0, 5, "one"), (2, 1000, 1025, 65, 3, 0, "two"), (1, 200, 3, 520, 9, 2, "any"),
    (4, 129, 700, 7, 0, 0, "none"), (1, 5000, 2000, 31, 0, 0, "zipf"), (2, 33, 90, 1030, 11, 0, "any"), (1, 513, 1, 64, 0, 0, "any"),
    (2, 70, 50, 13, 2, 0, "any"), (1, 90, 30, 26, 0, 1, "zipf"), (2, 300, 60, 527, 4, 0, "zipf"), (1, 40, 20, 9, 1, 0, "two"),
    (2, 40, 700, 33, 3, 2, "zipf"), (1, 5, 90, 7, 1, 0, "any"), (3, 300, 5000, 65, 5, 3, "two"), (2, 33, 1500, 130, 1, 1, "none")]


def rows(gen, W, ld, dtype):
    return torch.randn((W, ld), generator=gen).to(dtype)


@pytest.mark.parametrize("suffix", R.SUFFIXES)
@pytest.mark.parametrize("W,N,V,D,offset,extra,kind", SHAPES)
def test_lookup(suffix, W, N, V, D, offset, extra, kind):
    gen = torch.Generator().manual_seed(N + D)
    dtype, scale = R.TYPES[suffix], D ** 0.5
    x = rows(gen, W, offset + V * D + extra, dtype)
    tokens = tokens_of(kind, W, N, V, gen)
    out = torch.full((W * N, D + 3), 7.0, dtype=dtype, device=DEV)
    getattr(lm, "cx_embed_lookup" + suffix)(x.to(DEV), tokens.to(DEV), out[:, 2:2 + D], offset, V, scale)
    ref = R.lookup(x, tokens, offset, V, D, scale)
    R.check(out[:, 2:2 + D], ref, 2 * R.U * ref.abs())                # scale as fp32, the product's rounding
    assert (out[:, :2] == 7).all() and (out[:, 2 + D:] == 7).all()


@pytest.mark.parametrize("suffix", R.SUFFIXES)
@pytest.mark.parametrize("W,N,D", [(1, 262_150, 13), (2, 70_001, 131), (1, 40_003, 1001)])
def test_lookup_of_many_tokens(suffix, W, N, D):
    test_lookup(suffix, W, N, 300, D, 3, 0, "any")


@pytest.mark.parametrize("suffix", R.SUFFIXES)
@pytest.mark.parametrize("mode", ["alone", "added", "in place"])
@pytest.mark.parametrize("W,N,V,D,offset,extra,kind", SHAPES)
def test_grad(suffix, mode, W, N, V, D, offset, extra, kind):
    gen = torch.Generator().manual_seed(N * 3 + D)
    dtype, scale = R.TYPES[suffix], D ** 0.5
    tokens = tokens_of(kind, W, N, V, gen)
    dout = torch.randn((W * N, D + 2), generator=gen).to(dtype)[:, 1:1 + D]
    dout[((tokens < 0) | (tokens >= V)).flatten()] = torch.nan        # rows of padding are not looked at
    base = rows(gen, W, offset + V * D + extra, dtype)
    g_in = None if mode == "alone" else base.to(DEV)
    g_out = g_in if mode == "in place" else torch.full_like(base, torch.nan).to(DEV)
    wide = torch.empty((W * N, D + 2), dtype=dtype, device=DEV)[:, 1:1 + D]
    wide.copy_(dout)
    getattr(lm, "cx_embed_grad" + suffix)(wide, tokens.to(DEV), g_in, g_out, offset, V, scale)
    ref, size = R.embed_grad(dout, tokens, None if mode == "alone" else base, offset, V, D, scale)
    longest = max((int(torch.bincount(t[(t >= 0) & (t < V)].long(), minlength=1).max()) for t in tokens), default=0)
    R.check(g_out[:, offset:offset + V * D], ref, (longest + 3) * R.U * size)
    around = g_out.cpu().clone()
    around[:, offset:offset + V * D] = 0
    want = base.clone() if mode == "in place" else torch.full_like(base, torch.nan)
    want[:, offset:offset + V * D] = 0
    assert torch.equal(around.nan_to_num(9.0), want.nan_to_num(9.0))


def test_grad_of_no_tokens_is_zero_and_twice_the_same():
    g = torch.full((2, 100), torch.nan, device=DEV)
    empty = torch.empty((0, 5), device=DEV)
    lm.cx_embed_grad(empty, torch.empty((2, 0), dtype=torch.int32, device=DEV), None, g, 10, 12)
    assert (g[:, 10:70] == 0).all() and g[:, :10].isnan().all() and g[:, 70:].isnan().all()
    lm.cx_embed_lookup(torch.zeros((2, 100), device=DEV), torch.empty((2, 0), dtype=torch.int32, device=DEV), empty, 10, 12)
    # the order of the sums is fixed: bit for bit the same, whatever the workspace held before
    gen = torch.Generator().manual_seed(4)
    tokens = tokens_of("zipf", 3, 3000, 700, gen).to(DEV)
    dout = torch.randn((9000, 40), generator=gen).to(DEV)
    got = []
    for fill in (0, 255):
        g = torch.empty((3, 28000), device=DEV)
        work = torch.full((lm.cx_embed_workspace(3, 3000, 700, 40),), fill, dtype=torch.uint8, device=DEV)
        lm.cx_embed_grad(dout, tokens, None, g, 0, 700, workspace=work)
        got.append(g)
    assert torch.equal(*got)


def test_grad_against_differences():
    """d/d table of sum(lookup * c) by central differences of the lookup in fp32; linear in the table, so rounding alone counts."""
    gen = torch.Generator().manual_seed(1)
    W, N, V, D, scale = 2, 90, 13, 6, 1.5
    tokens = tokens_of("zipf", W, N, V, gen)
    x, c = rows(gen, W, V * D, torch.float32), torch.randn((W * N, D), generator=gen)
    g = torch.empty((W, V * D), device=DEV)
    lm.cx_embed_grad(c.to(DEV), tokens.to(DEV), None, g, 0, V, scale)

    def value(x):
        out = torch.empty((W * N, D), device=DEV)
        lm.cx_embed_lookup(x.to(DEV), tokens.to(DEV), out, 0, V, scale)
        return float((out.cpu().double() * c.double()).sum())

    for w, i in ((0, 0), (0, 40), (1, 5), (1, V * D - 1)):
        up, down = x.clone(), x.clone()
        up[w, i] += 1.0
        down[w, i] -= 1.0
        slope = (value(up) - value(down)) / float(up[w, i].double() - down[w, i].double())
        assert abs(slope - float(g[w, i])) < 1e-3 * (1 + abs(slope))


@pytest.mark.parametrize("suffix", ["", "_bf16"])
def test_tables_beyond_32_bits_of_elements(suffix):
    """A table whose rows lie beyond 2^31 elements of the flat row: lookup and gradient in place touch the right ones."""
    dtype, V, D, offset = R.TYPES[suffix], 9, 64, 2**31 + 5
    x = torch.zeros((1, offset + V * D + 1), dtype=dtype, device=DEV)
    x[0, offset:offset + V * D] = torch.arange(V * D, device=DEV).remainder(200).to(dtype)
    tokens = torch.tensor([[8, 0, 3]], dtype=torch.int32, device=DEV)
    out = torch.empty((3, D), dtype=dtype, device=DEV)
    getattr(lm, "cx_embed_lookup" + suffix)(x, tokens, out, offset, V)
    assert torch.equal(out, x[0, offset:offset + V * D].view(V, D)[tokens[0].long()])
    before = x[0, offset:offset + V * D].clone().view(V, D)
    getattr(lm, "cx_embed_grad" + suffix)(out, tokens, x, x, offset, V)
    after = before.clone()
    after[tokens[0].long()] = (before[tokens[0].long()].float() * 2).to(dtype)
    assert torch.equal(x[0, offset:offset + V * D].view(V, D), after)
    assert (x[0, :offset].view(-1)[:1 << 20] == 0).all() and float(x[0, offset + V * D]) == 0
