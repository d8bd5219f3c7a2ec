"""The language-model operators in 64 bits, from their definitions, on the CPU, with the bounds that their tests use.

Bounds.  u = 2^-24 is fp32's rounding unit; half_ulp() is the error of one rounding to an output type.  Each operator's bound adds to
that the errors of its fp32 arithmetic: every operation's rounding times the magnitude that it can carry, with the one-ulp
exponential and reciprocal counted as four roundings, and arguments of exponentials contributing their own size."""
import numpy as np
import torch

U = 2.0 ** -24
TYPES = {"": torch.float32, "_bf16": torch.bfloat16, "_f16": torch.float16}
SUFFIXES = list(TYPES)


def half_ulp(ref, dtype):
    """Half the spacing of `dtype` at |ref|, the subnormals' spacing included."""
    bits, lowest = {torch.float32: (24, -126), torch.bfloat16: (8, -126), torch.float16: (11, -14)}[dtype]
    exponent = torch.frexp(ref.abs().clamp_min(2.0 ** lowest))[1] - 1
    return torch.ldexp(torch.full_like(ref, 0.5), exponent - (bits - 1))


def check(got, ref, slack, what=""):
    """|got - ref| <= one rounding to got's type at |ref| + slack, and slack; NaN and infinities in the same places."""
    got64, ref = got.detach().cpu().double(), ref.double()
    assert got64.shape == ref.shape, what
    assert torch.equal(got64.isnan(), ref.isnan()), what
    slack = torch.as_tensor(slack, dtype=torch.float64).expand_as(ref)
    fine = ref.isfinite()
    assert torch.equal(got64[~fine & ~ref.isnan()], ref[~fine & ~ref.isnan()]), what
    ref, slack, got64 = ref[fine], slack[fine], got64[fine]
    allowed = half_ulp(ref.abs() + slack, got.dtype) + slack
    off = (got64 - ref).abs()
    bad = off > allowed
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()}, worst {float((off / allowed).max()):.3g} times the bound"


# ---------------------------------------------------------------------------------------------------------- embeddings
def lookup(x, tokens, offset, V, D, scale):
    W, N = tokens.shape
    out = torch.zeros((W * N, D), dtype=torch.float64)
    for w in range(W):
        for n in range(N):
            v = int(tokens[w, n])
            if 0 <= v < V:
                out[w * N + n] = x[w, offset + v * D:offset + (v + 1) * D].double() * scale
    return out


def embed_grad(dout, tokens, g_in, offset, V, D, scale):
    """(gradient [W][V * D], sum of |terms|)"""
    W, N = tokens.shape
    out, size = (torch.zeros((W, V, D), dtype=torch.float64) for _ in range(2))
    for w in range(W):
        known = ((tokens[w] >= 0) & (tokens[w] < V)).nonzero()[:, 0]
        rows = dout.reshape(W, N, D)[w, known].double() * scale
        out[w].index_add_(0, tokens[w, known].long(), rows)
        size[w].index_add_(0, tokens[w, known].long(), rows.abs())
    out, size = out.reshape(W, V * D), size.reshape(W, V * D)
    if g_in is not None:
        base = g_in[:, offset:offset + V * D].double()
        out, size = out + base, size + base.abs()
    return out, size


# ----------------------------------------------------------------------------------------------------- gated recurrence
def scan(f, x, T, h0, reset):
    """(y [B * T][D], h_last, what enters every step) in 64 bits."""
    D = f.shape[1]
    B = f.shape[0] // T
    f, x = f.double().reshape(B, T, D), x.double().reshape(B, T, D)
    a, b = torch.special.expit(f), torch.special.expit(-f)
    h = torch.zeros((B, D), dtype=torch.float64) if h0 is None else h0.double()
    ys, before = torch.empty_like(x), torch.empty_like(x)
    for t in range(T):
        if reset is not None:
            h = torch.where(reset[:, t, None] != 0, 0.0, h)
        before[:, t] = h
        h = a[:, t] * h + b[:, t] * x[:, t]
        ys[:, t] = h
    return ys.reshape(B * T, D), h, before


def scan_grad(f, x, dy, T, h0, reset, dh_last):
    """(df, dx, dh0, largest |r|) in 64 bits."""
    D = f.shape[1]
    B = f.shape[0] // T
    _, _, before = scan(f, x, T, h0, reset)
    f, x, dy = (t.double().reshape(B, T, D) for t in (f, x, dy))
    a, b = torch.special.expit(f), torch.special.expit(-f)
    r = torch.zeros((B, D), dtype=torch.float64) if dh_last is None else dh_last.double()
    df, dx, high = torch.empty_like(x), torch.empty_like(x), 0.0
    for t in range(T - 1, -1, -1):
        r = dy[:, t] + r
        high = max(high, float(r.abs().max()))
        dx[:, t] = b[:, t] * r
        df[:, t] = r * (before[:, t] - x[:, t]) * a[:, t] * b[:, t]
        r = a[:, t] * r
        if reset is not None:
            r = torch.where(reset[:, t, None] != 0, 0.0, r)
    return df.reshape(B * T, D), dx.reshape(B * T, D), r, high


def memory(f, T):
    """Steps over which errors of a scan add up: min(T, 1 / (1 - the largest gate))."""
    return min(T, 1.0 / float(torch.special.expit(-f.double()).min()))


# ------------------------------------------------------------------------------------------------------------ token scores
def order(z):
    """Ids of each row by logit, largest first, the lower id first among equal ones; NaN last."""
    z = z.double() + 0.0
    z = torch.where(z.isnan(), -torch.inf, z)
    return torch.sort(-z, dim=1, stable=True).indices


def scores(z, tokens, K, scale):
    """(logp, entropy, top ids, top logp): rows as the header defines them."""
    raw, N = z, z.shape[0]
    z = z.double() * scale
    broken = (z.isnan() | (z == torch.inf)).any(1)
    empty = (z == -torch.inf).all(1)
    lse = torch.logsumexp(z, 1)
    lp = z - lse[:, None]
    p = lp.exp()
    entropy = -torch.where(p > 0, p * lp, 0.0).sum(1)
    entropy[empty] = 0.0
    entropy[broken] = torch.nan
    lp[empty] = -torch.inf
    lp[broken] = torch.nan
    known = (tokens >= 0) & (tokens < z.shape[1])
    logp = torch.where(known, lp.gather(1, torch.where(known, tokens, 0).long()[:, None])[:, 0], 0.0)
    ids = order(raw)[:, :K]
    top = lp.gather(1, ids)
    gone = raw.gather(1, ids).isnan()
    return logp, entropy, torch.where(gone, -1, ids).int(), top


def lse_slack(z, scale, parts=1.0):
    """Bound of the error of log sum exp of rows of z at `scale`."""
    z = z.double()
    high = torch.where(z.isfinite(), z.abs(), 0.0).amax(1) * scale
    return U * (32 + z.shape[1] / 512 + 4 * high)


# ------------------------------------------------------------------------------------------------------------- distillation
def distill(z, ids, t, labels, gout, tau, w_kl, w_ce):
    """(loss, dz, slack of the loss, slack of dz)"""
    N, V = z.shape
    z = z.double()
    empty = (z == -torch.inf).all(1)
    z = torch.where(empty[:, None], 0.0, z)
    soft, hard = z / tau - torch.logsumexp(z / tau, 1, keepdim=True), z - torch.logsumexp(z, 1, keepdim=True)
    known = (ids >= 0) & (ids < V) & (t != -torch.inf)
    lt = torch.where(known, t.double() / tau, -torch.inf)
    has = known.any(1) & ~empty & (w_kl != 0)
    log_q = lt - torch.where(known.any(1), torch.logsumexp(lt, 1), 0.0)[:, None]
    q = torch.where(known & has[:, None], log_q.exp(), 0.0)
    at = torch.where(known, ids, 0).long()
    lp = soft.gather(1, at)
    terms = torch.where(q > 0, q * (torch.where(known, log_q, 0.0) - lp), 0.0)
    sizes = torch.where(q > 0, q * (torch.where(known, log_q, 0.0).abs() + lp.abs()), 0.0)
    loss, size = w_kl * tau**2 * terms.sum(1), w_kl * tau**2 * sizes.sum(1)
    label = torch.full((N,), -1) if labels is None else labels
    lab = (label >= 0) & (label < V) & ~empty & (w_ce != 0)
    one = torch.where(lab, label, 0).long()[:, None]
    loss = loss - torch.where(lab, w_ce * hard.gather(1, one)[:, 0], 0.0)
    size = size + torch.where(lab, w_ce * hard.gather(1, one)[:, 0].abs(), 0.0)
    kl, ce = has.double()[:, None] * w_kl * tau, lab.double()[:, None] * w_ce
    targets = (w_kl * tau * q).double()
    grad = torch.where(kl > 0, kl * soft.exp(), 0.0) + torch.where(ce > 0, ce * hard.exp(), 0.0)
    grad_size = grad.clone()
    grad = grad.scatter_add(1, at, -targets).scatter_add(1, one, -ce)
    grad_size = grad_size.scatter_add(1, at, targets).scatter_add(1, one, ce)
    g = gout.double()[:, None]
    low = torch.where(z.isfinite(), z, torch.inf).amin(1)
    spread = torch.where(z.isfinite(), z, -torch.inf).amax(1) - low
    rel = U * (64 + V / 512 + 8 * spread.clamp(max=200.0) * max(1.0, 1.0 / tau))
    return loss, torch.where((kl + ce) > 0, g * grad, 0.0), rel * (size + w_kl * tau**2 + w_ce), rel[:, None] * g.abs() * grad_size
