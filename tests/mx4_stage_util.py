"""The 4-bit FFN's two products checked one by one: the second from the hidden rows as they were stored, so that its bound holds one
float sum and one rounding and no rounding of the first is counted again in every term.

The hidden rows lie at the start of the workspace until the next call uses it."""
from __future__ import annotations

import torch

import mx4_util as M


def sums(rows, W, bias):
    """(rows W^T + bias, bound of its float sum): rows [R, K], W [N, K] and bias [N] or None, all double."""
    out = rows @ W.T
    size = rows.abs() @ W.abs().T
    if bias is not None:
        out, size = out + bias, size + bias.abs()
    return out, (W.shape[1] + 2) * 2.0 ** -23 * size


def rounded(value, off, dtype):
    """Bound of a value that is off by ``off`` and rounded once."""
    return off + M.HALF[dtype] * (value.abs() + off) + 1e-38


def hidden(u, off_u, dtype):
    """(gelu(u), bound of what is stored): gelu' is at most 1.13, the form is off by 1e-6 and a few float roundings at most."""
    g = M.gelu(u)
    return g, rounded(g, 1.13 * off_u + 1e-6 + 2.0 ** -22 * g.abs(), dtype)


def stored_hidden(workspace, rows, F, dtype):
    """The hidden rows [rows, F] that the forward call left in its workspace."""
    size = torch.empty((), dtype=dtype).element_size()
    return workspace[:rows * F * size].view(dtype).reshape(rows, F).clone()


def excess(got, want, tol):
    """The largest error in units of its bound."""
    return float(((got - want).abs() / tol).max())
