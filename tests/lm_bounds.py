"""The gated recurrence in 64 bits with a bound of the fp32 error of every element, forward and backward, on the CPU.

U = 2^-24.  A step's gates a = sigmoid(f) and b = sigmoid(-f) are off by at most (2 |f| + 10) U of themselves: the exponent's constant and
product 2 |f|, the one-ulp exponential and reciprocal 4 each, the sum and e * a one each.  The products and sums of a step add 2, the
joining of pieces and spans, which is rarer than once a step, 4 more: c = 16 + 2 |f|.  Errors are carried through the steps like values:

    H_t = a_t H_{t-1} + b_t |x_t|      what |h_t| cannot exceed         err_t = a_t err_{t-1} + c_t U H_t
    G_t = |dy_t| + a_{t+1} G_{t+1}     the same of r_t                  errg_t = a_{t+1} errg_{t+1} + c_{t+1} U a_{t+1} G_{t+1} + U G_t

which bounds any order of composing the steps, since a composed map's terms are terms of H and G.  A reset drops what came before it."""
import torch

U = 2.0 ** -24


def _split(f, x, T, reset):
    D = f.shape[1]
    f, x = f.double().reshape(-1, T, D), x.double().reshape(-1, T, D)
    keep = torch.ones_like(f) if reset is None else (reset == 0).double()[..., None].expand_as(f)
    return f, x, torch.special.expit(f), torch.special.expit(-f), keep, 16 + 2 * f.abs()


def scan(f, x, T, h0, reset):
    """y, what enters each step (before its reset), h_last, and the bounds of the three, [B][T][D] and [B][D]."""
    f, x, a, b, keep, c = _split(f, x, T, reset)
    h = torch.zeros_like(f[:, 0]) if h0 is None else h0.double()
    H, err = h.abs(), torch.zeros_like(h)
    out = [torch.empty_like(f) for _ in range(6)]
    for t in range(T):
        for to, v in zip(out[:3], (h, err, H)):
            to[:, t] = v
        k = keep[:, t]
        h = torch.where(k == 0, 0.0, a[:, t] * h) + b[:, t] * x[:, t]
        H = k * a[:, t] * H + b[:, t] * x[:, t].abs()
        err = k * a[:, t] * err + c[:, t] * U * H
        for to, v in zip(out[3:], (h, err, H)):
            to[:, t] = v
    before, before_err, before_H, y, y_err, _ = out
    return {"y": y, "y_err": y_err, "before": before, "before_err": before_err, "before_H": before_H, "h_last": h, "h_last_err": err}


def scan_grad(f, x, dy, T, h0, reset, dh_last):
    """df, dx, dh0 and their bounds."""
    s = scan(f, x, T, h0, reset)
    f, x, a, b, keep, c = _split(f, x, T, reset)
    dy = dy.double().reshape(f.shape)
    r = torch.zeros_like(f[:, 0]) if dh_last is None else dh_last.double()
    R, err = r.abs(), torch.zeros_like(r)
    df, df_err, dx, dx_err = (torch.empty_like(f) for _ in range(4))
    for t in range(T - 1, -1, -1):
        at, bt, k, cu = a[:, t], b[:, t], keep[:, t], c[:, t] * U
        g, G = dy[:, t] + r, dy[:, t].abs() + R
        errg = err + U * G
        dx[:, t], dx_err[:, t] = bt * g, bt * (errg + cu * G)
        off = torch.where(k == 0, 0.0, s["before"][:, t]) - x[:, t]
        off_err = k * s["before_err"][:, t] + U * (k * s["before_H"][:, t] + x[:, t].abs())
        df[:, t] = at * bt * g * off
        df_err[:, t] = at * bt * (G * off_err + off.abs() * errg + off_err * errg + (2 * cu + 2 * U) * G * (off.abs() + off_err))
        r, R, err = k * at * g, k * at * G, k * (at * errg + cu * at * G)
    return {"df": df, "df_err": df_err, "dx": dx, "dx_err": dx_err, "dh0": r, "dh0_err": err}
