"""Inputs of the tests of the residual block's operators: matrices inside longer rows, flat parameter rows."""
import torch

DEV = "cuda:0"


def place(t, strided, fill=3.0):
    """On the device; strided: inside longer rows that begin at an odd element."""
    if not strided:
        return t.to(DEV)
    wide = torch.full((t.shape[0], t.shape[1] + 5), fill, dtype=t.dtype, device=DEV)
    wide[:, 1:1 + t.shape[1]] = t.to(DEV)
    return wide[:, 1:1 + t.shape[1]]


def untouched(t, fill=3.0):
    """Whether what lies beside a strided matrix still holds its fill."""
    base, width = t._base, t.shape[1]
    return bool((base[:, 0] == fill).all() and (base[:, 1 + width:] == fill).all())


def flat_rows(parts, offset, dtype, gen):
    """[W][ld] rows with the parts ([W][any]) from `offset` on, something else around them."""
    W = parts[0].shape[0]
    edge = lambda n: torch.randn((W, n), generator=gen)
    return torch.cat([edge(offset), *parts, edge(3)], 1).to(dtype)


def gradient_rows(mode, rows, dtype, gen):
    """(g_in on the device or None, g_out, host copy of g_in) for the three ways of adding."""
    base = torch.randn(rows.shape, generator=gen).to(dtype)
    if mode == "alone":
        return None, torch.full_like(base, 7.0).to(DEV), None
    g_in = base.to(DEV)
    return g_in, g_in if mode == "in place" else torch.full_like(base, 7.0).to(DEV), base


def edges(rows, offset, count):
    return torch.cat([rows[:, :offset], rows[:, offset + count:]], 1).cpu()
