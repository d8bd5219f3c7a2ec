"""Dropout, norm, short convolution and selective scan in 64 bits, from their definitions, on the CPU, each with a bound of the fp32 error of every
element of its results.

U = 2^-24.  An operation adds U of its result; the one-ulp exponential and reciprocal count as four.  sigmoid(v) is off by at most
(2 |v| + 10) U of itself: the exponent's constant and product 2 |v|, exponential and reciprocal 4 each, the sum and the product."""
import numpy as np
import torch

U = 2.0 ** -24


# ------------------------------------------------------------------------------------------------------------------ dropout
def border(p):
    return round(float(np.float32(p)) * 65536)


def factor(rng, n, D, p):
    """0 or 1 / (1 - p) of each element of [n][D]: Philox4x32 of ten rounds, eight 16-bit halves a block."""
    k = border(p)
    if k == 0:
        return torch.ones((n, D), dtype=torch.float64)
    key, draw = (int(v) % 2**64 for v in rng)
    blocks = -(-D // 8)
    at = np.arange(n * blocks, dtype=np.uint64)
    low, up = np.uint64(2**32 - 1), np.uint64(32)
    c = [at & low, at >> up, np.full_like(at, draw % 2**32), np.full_like(at, draw >> 32)]
    keys = [key % 2**32, key >> 32]
    for _ in range(10):
        first, second = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(second >> up) ^ c[1] ^ np.uint64(keys[0]), second & low, (first >> up) ^ c[3] ^ np.uint64(keys[1]), first & low]
        keys = [(keys[0] + 0x9E3779B9) % 2**32, (keys[1] + 0xBB67AE85) % 2**32]
    halves = np.stack(c, 1).astype("<u4").view("<u2").reshape(n, -1)[:, :D]
    return torch.from_numpy((halves >= k) * (65536.0 / (65536 - k)))


def dropped(v, keep):
    return torch.where(keep == 0, 0.0, v * keep)


def dropout(x, residual, keep):
    """(result, bound): the scale's rounding, the product, the sum."""
    v = dropped(x.double(), keep)
    r = torch.zeros_like(v) if residual is None else residual.double()
    return r + v, U * (3 * v.abs() + r.abs())


# --------------------------------------------------------------------------------------------------------------------- norm
ADDS = 50                      # additions on a term's way through a row's sum: 32 columns of a lane, 6 across lanes, 8 wavefronts


def add_norm(x, residual, w, keep, eps):
    """x, w [n][D]; {t, y, inv} with bounds."""
    t, et = dropout(x, residual, keep)
    w = w.double()
    D = t.shape[1]
    inv = 1 / (t.square().mean(1, keepdim=True) + eps).sqrt()
    size = t.square().sum(1, keepdim=True) + eps * D
    rel = (et * t.abs() + et * et).sum(1, keepdim=True) / size + U * (ADDS / 2 + 5)
    y = t * inv * w
    return {"t": t, "t_err": et, "inv": inv[:, 0], "inv_err": (inv * rel)[:, 0], "y": y, "y_err": y.abs() * (rel + 3 * U) + (et * inv * w).abs()}


def half_step8(v):
    """Half the spacing of e4m3 at v."""
    exponent = torch.frexp(v.abs().clamp_min(2.0**-6))[1] - 1
    return torch.ldexp(torch.full_like(v, 0.5), exponent - 3)


def add_norm_grad(dy, s, inv, w, ds_in, keep):
    """From the s and inv that the forward call left.  dw of all rows together."""
    dy, s, w, inv = dy.double(), s.double(), w.double(), inv.double()[:, None]
    D, n = s.shape[1], s.shape[0]
    unit, g = s * inv, dy * w
    m = (g * unit).mean(1, keepdim=True)
    em = U * (ADDS + 6) * (g * unit).abs().mean(1, keepdim=True)
    own = g - unit * m
    ds = inv * own + (0 if ds_in is None else ds_in.double())
    err = inv * (unit.abs() * em + U * (4 * (unit * m).abs() + 3 * g.abs())) + U * (2 * (inv * own).abs() + ds.abs())
    dw, size = (dy * unit).sum(0), (dy * unit).abs().sum(0)
    return {"ds": ds, "ds_err": err, "dx": dropped(ds, keep), "dx_err": keep * err + 2 * U * (keep * ds).abs(), "dw": dw, "dw_size": size, "dw_err": U * (n + 40) * size}


# -------------------------------------------------------------------------------------------------------- short convolution
def taps(x, T, K, before, reset):
    """[B][T][K][D] of what each tap sees, and what the step after the last sees, [B][K - 1][D]."""
    D = x.shape[1]
    x = x.double().reshape(-1, T, D)
    B = x.shape[0]
    window = torch.zeros((B, K - 1, D), dtype=torch.float64) if before is None else before.double().clone()
    out = torch.zeros((B, T, K, D), dtype=torch.float64)
    for t in range(T):
        if reset is not None:
            window = torch.where(reset[:, t, None, None] != 0, 0.0, window)
        out[:, t, :K - 1], out[:, t, K - 1] = window, x[:, t]
        window = out[:, t, 1:].clone()
    return out, window


def conv(x, w, bias, T, K, silu, before, reset):
    """w [B][D][K], bias [B][D]."""
    seen, after = taps(x, T, K, before, reset)
    w, bias = w.double().transpose(1, 2)[:, None], bias.double()[:, None]
    v = bias + (w * seen).sum(2)
    ev = U * (K + 1) * (bias.abs() + (w * seen).abs().sum(2))
    e = torch.special.expit(v)
    y = v * e if silu else v
    err = 1.1 * ev + y.abs() * (2 * v.abs() + 12) * U + 2.0**-110 * v.abs() if silu else ev
    return {"y": y, "y_err": err, "after": after, "v": v, "ev": ev, "seen": seen, "e": e}


def conv_grad(x, dy, w, bias, T, K, silu, before, reset):
    """dx [B][T][D]; dw [B][D][K] and dbias [B][D] of each sequence with the sizes of their terms."""
    f = conv(x, w, bias, T, K, silu, before, reset)
    v, e, seen = f["v"], f["e"], f["seen"]
    B, _, D = v.shape
    dy = dy.double().reshape(v.shape)
    d, ed = dy, torch.zeros_like(dy)
    if silu:
        d = dy * e * (1 + v * (1 - e))
        ed = dy.abs() * (0.5 * f["ev"] + e * (1 + v.abs()) * (2 * (2 * v.abs() + 10) + 4) * U)
    w = w.double()
    dx, err = torch.zeros_like(v), torch.zeros_like(v)
    since = torch.full((B,), K, dtype=torch.long)              # steps that a step's taps may look back
    for t in range(T):
        since = since + 1
        if reset is not None:
            since = torch.where(reset[:, t] != 0, 0, since)
        for j in range(min(K, t + 1)):
            sees = (since >= j).double()[:, None]
            dx[:, t - j] += torch.where(sees > 0, w[:, :, K - 1 - j] * d[:, t], 0.0)
            err[:, t - j] += sees * (w[:, :, K - 1 - j].abs() * ed[:, t] + U * (K + 1) * (w[:, :, K - 1 - j] * d[:, t]).abs())
    over = lambda a, b: torch.einsum("btd,btkd->bdk", a, b)
    dw, dw_err, dw_size = over(d, seen), over(ed, seen.abs()), over(d.abs(), seen.abs())
    return {"dx": dx, "dx_err": err, "dw": dw, "dw_err": dw_err, "dw_size": dw_size, "dbias": d.sum(1), "dbias_err": ed.sum(1), "dbias_size": d.abs().sum(1)}


# ------------------------------------------------------------------------------------------------------------ selective scan
def _steps(u, dt, bm, T, A_log, bias):
    """Gates and their bounds: delta, x = delta R of [B][T][D][N] and the relative errors cd of delta, cr of R, ca of a."""
    D, N = u.shape[1], bm.shape[1]
    B = u.shape[0] // T
    u, v = u.double().reshape(B, T, D), dt.double().reshape(B, T, D) + bias.double()[:, None]
    R = A_log.double().exp()
    delta = torch.where(v < -700, 0.0, torch.nn.functional.softplus(v, threshold=700.0))
    av = torch.where(v.isinf(), 0.0, v.abs())
    cd, cr = (3 * av + 24) * U, (2 * A_log.double().abs() + 8) * U
    return u, v, av, R, delta, cd, cr


def select(u, dt, bm, cm, z, T, A_log, bias, skip, h0, reset):
    """A_log [B][D][N], bias and skip [B][D].  A step's error of a state: the gate's ca of what it keeps and 5 more for the joining of spans
    (whose sum of steps adds U a step, weighed by x exp(-x) < 0.37), cd + 3 U of what is new, 3 U of the state."""
    D, N = u.shape[1], bm.shape[1]
    u, v, av, R, delta, cd, cr = _steps(u, dt, bm, T, A_log, bias)
    B = u.shape[0]
    bm, cm = bm.double().reshape(B, T, N), cm.double().reshape(B, T, N)
    h = torch.zeros((B, D, N), dtype=torch.float64) if h0 is None else h0.double()
    H, err = h.abs(), torch.zeros_like(h)
    shape = (B, T, D, N)
    before, before_err, before_H, after, after_err, after_H, a_all, ca_all = (torch.empty(shape, dtype=torch.float64) for _ in range(8))
    keep = torch.ones((B, T)) if reset is None else (reset == 0).double()
    for t in range(T):
        x = delta[:, t, :, None] * R
        a, ca = (-x).exp(), x * (cd[:, t, :, None] + cr + 4 * U) + 4 * U
        k = keep[:, t, None, None]
        fresh = (delta[:, t] * u[:, t])[..., None] * bm[:, t, None]
        before[:, t], before_err[:, t], before_H[:, t] = torch.where(k == 0, 0.0, h), torch.where(k == 0, 0.0, err), torch.where(k == 0, 0.0, H)
        h = a * before[:, t] + fresh
        newH = a * before_H[:, t] + fresh.abs()
        err = a * before_err[:, t] + (ca + 5 * U) * a * before_H[:, t] + (cd[:, t, :, None] + 3 * U) * fresh.abs() + 3 * U * newH
        H = newH
        after[:, t], after_err[:, t], after_H[:, t], a_all[:, t], ca_all[:, t] = h, err, H, a, ca
    skip = skip.double()[:, None]
    read = (after * cm[:, :, None]).sum(3) + skip * u
    size = (after_H * cm[:, :, None].abs()).sum(3) + (skip * u).abs()
    read_err = (after_err * cm[:, :, None].abs()).sum(3) + (N + 6) * U * size
    y, y_err = read, read_err
    if z is not None:
        z = z.double().reshape(B, T, D)
        e = torch.special.expit(z)
        y, y_err = read * z * e, read_err * (z * e).abs() + (read * z * e).abs() * (2 * z.abs() + 14) * U
    return {"y": y, "y_err": y_err, "h_last": h, "h_last_err": err, "before": before, "before_err": before_err, "before_H": before_H, "after": after,
            "after_err": after_err, "after_H": after_H, "a": a_all, "ca": ca_all, "read": read, "read_err": read_err, "keep": keep, "delta": delta, "cd": cd,
            "cr": cr, "R": R, "v": v, "av": av, "u": u, "z": z, "bm": bm, "cm": cm, "skip": skip}


def select_grad(u, dt, bm, cm, z, T, A_log, bias, skip, h0, reset, dy, dh_last):
    """Gradients with bounds; those of A_log, bias and skip of each sequence, with the sizes of their terms for the sums over steps and parts."""
    f = select(u, dt, bm, cm, z, T, A_log, bias, skip, h0, reset)
    u, v, av, delta, cd, cr, R, z, bm, cm, skip = (f[k] for k in ("u", "v", "av", "delta", "cd", "cr", "R", "z", "bm", "cm", "skip"))
    B, _, D = u.shape
    N = bm.shape[2]
    dy = dy.double().reshape(B, T, D)
    out = {}
    if z is None:
        g, cg = dy, torch.full_like(dy, U)
    else:
        e = torch.special.expit(z)
        g, cg = dy * z * e, (2 * z.abs() + 13) * U
        slope = e * (1 + z * (1 - e))
        out["dz"] = dy * slope * f["read"]
        out["dz_err"] = dy.abs() * (e * (1 + z.abs()) * (2 * (2 * z.abs() + 10) + 8) * U * f["read"].abs() + slope.abs() * f["read_err"]) + 2 * U * out["dz"].abs()
    r = torch.zeros((B, D, N), dtype=torch.float64) if dh_last is None else dh_last.double()
    G, err = r.abs(), torch.zeros_like(r)
    names = ("du", "ddt", "db", "dc")
    for k in names:
        out[k], out[k + "_err"] = (torch.empty((B, T, D if k[1] not in "bc" else N), dtype=torch.float64) for _ in range(2))
    dA, dA_err, dA_size = (torch.zeros((B, D, N), dtype=torch.float64) for _ in range(3))
    slabs = -(-D // 64)
    for t in range(T - 1, -1, -1):
        gt, cgt, d, cdt = g[:, t], cg[:, t], delta[:, t], cd[:, t]
        pull = gt[..., None] * cm[:, t, None]
        r, G = r + pull, G + pull.abs()
        err = err + (cgt[..., None] + 2 * U) * pull.abs() + U * G
        a, ca, k = f["a"][:, t], f["ca"][:, t], f["keep"][:, t, None, None]
        b = bm[:, t, None]
        into, into_size = (r * b).sum(2), (G * b.abs()).sum(2)
        into_err = (err * b.abs()).sum(2) + (N + 4) * U * into_size
        moved, M = r * a * f["before"][:, t], G * a * f["before_H"][:, t]
        moved_err = err * a * f["before_H"][:, t] + G * a * f["before_err"][:, t] + err * a * f["before_err"][:, t] + (ca + 3 * U) * M
        across = -(moved * R).sum(2)
        across_err = (R * moved_err + (cr + (N + 4) * U) * R * M).sum(2)
        sg = skip[:, 0] * gt
        out["du"][:, t] = d * into + sg
        out["du_err"][:, t] = d * (into_err + (cdt + 2 * U) * into_size) + (cgt + 3 * U) * sg.abs()
        both, s = across + u[:, t] * into, torch.special.expit(v[:, t])
        size = (R * M).sum(2) + u[:, t].abs() * into_size
        out["ddt"][:, t] = both * s
        out["ddt_err"][:, t] = s * (across_err + u[:, t].abs() * into_err + (3 * av[:, t] + 16) * U * size)
        du_ = d * u[:, t]
        out["db"][:, t] = (r * du_[..., None]).sum(1)
        out["db_err"][:, t] = ((err + (cdt[..., None] + (14 + slabs) * U) * G) * du_.abs()[..., None]).sum(1)
        out["dc"][:, t] = (f["after"][:, t] * gt[..., None]).sum(1)
        out["dc_err"][:, t] = ((f["after_err"][:, t] + (cgt[..., None] + (14 + slabs) * U) * f["after_H"][:, t]) * gt.abs()[..., None]).sum(1)
        dA -= R * d[..., None] * moved
        dA_err += R * d[..., None] * (moved_err + (cr + cdt[..., None] + 4 * U) * M)
        dA_size += R * d[..., None] * M
        r, G, err = (torch.where(k == 0, 0.0, w) for w in (a * r, a * G, a * err + (ca + 5 * U) * a * G))
    out.update(dh0=r, dh0_err=err, dA=dA, dA_err=dA_err, dA_size=dA_size, dbias=out["ddt"].sum(1), dbias_err=out["ddt_err"].sum(1),
               dbias_size=(out["ddt"].abs() + out["ddt_err"]).sum(1), dskip=(g * u).sum(1), dskip_err=(cg * (g * u).abs()).sum(1), dskip_size=(g * u).abs().sum(1))
    return out


# -------------------------------------------------------------------------------------------------------- sums over a worker
def summed(each, err, size, W, steps, g_in=None):
    """Sums of [B][...] over each worker's sequences, flattened, with the bound of `steps` additions of every sequence's terms and those of the parts."""
    over = lambda t: t.reshape(W, -1, *t.shape[1:]).sum(1).reshape(W, -1)
    value, bound = over(each), over(err) + U * (steps * (each.shape[0] // W) + 40) * over(size)
    if g_in is not None:
        value, bound = value + g_in.double(), bound + U * (g_in.double().abs() + value.abs())
    return value, bound
