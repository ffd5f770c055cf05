"""Plain double-precision forms of the 4-bit expert calls and of the layer's gradients, on the CPU, and their error bounds.

Bounds count roundings: half a step of bf16 is 2^-8 relative, of float 2^-24; a float sum of n products is off by at most
n 2^-23 times the sum of their magnitudes (2^-23 rather than 2^-24: the matrix cores may cut instead of rounding)."""
from __future__ import annotations

import math

import numpy as np
import torch

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
MAGNITUDE = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])
CODE_VALUE = np.concatenate([MAGNITUDE, -MAGNITUDE])


def decode(codes, scales):
    """float64 values [..., cols] of codes [..., cols / 2] and scales [..., cols / 32] (uint8 tensors)."""
    c = codes.cpu().numpy()
    v = np.empty(c.shape[:-1] + (c.shape[-1] * 2,))
    v[..., 0::2], v[..., 1::2] = CODE_VALUE[c & 15], CODE_VALUE[c >> 4]
    s = scales.cpu().numpy().astype(np.float64)
    s = np.where(s == 255, np.nan, np.exp2(s - 127.0))
    return torch.from_numpy(v * np.repeat(s, 32, axis=-1))


def random_codes(gen, experts, rows, cols, std=0.05):
    """All codes with equal probability and scales of four powers of two around ``std`` (uint8 CPU tensors)."""
    codes = torch.randint(0, 256, (experts, rows, cols // 2), generator=gen, dtype=torch.uint8)
    e = int(round(math.log2(std / 3.0)))
    scales = torch.randint(127 + e - 1, 127 + e + 3, (experts, rows, cols // 32), generator=gen, dtype=torch.int32).to(torch.uint8)
    return codes, scales


def gelu(u):
    return 0.5 * u * torch.erfc(-u / math.sqrt(2.0))


def gelu_slope(u):
    return 0.5 * torch.erfc(-u / math.sqrt(2.0)) + u * torch.exp(-0.5 * u * u) / math.sqrt(2.0 * math.pi)


def ffn(x, offsets, experts, W1, b1, W2, b2, dtype):
    """(u, h, bound of u, bound of h) of packed rows x (float64); W1, W2: float64 values."""
    R, d = x.shape
    F = W1.shape[1]
    u, h = torch.zeros((R, F), dtype=torch.float64), torch.zeros((R, d), dtype=torch.float64)
    tu, th = torch.zeros_like(u), torch.zeros_like(h)
    for s, e in enumerate(experts):
        lo, hi = offsets[s], offsets[s + 1]
        a, b = W1[e], W2[e]
        u[lo:hi] = x[lo:hi] @ a.T + (0.0 if b1 is None else b1[e])
        sum_u = (d + 2) * 2.0 ** -23 * (x[lo:hi].abs() @ a.abs().T + (0.0 if b1 is None else b1[e].abs()))
        g = gelu(u[lo:hi])
        # gelu' is at most 1.13; the value of gelu itself is off by 1e-6 at most
        off_g = 1.13 * sum_u + 1e-6 + HALF[dtype] * (g.abs() + 1e-6 + 1.13 * sum_u)
        h[lo:hi] = g @ b.T + (0.0 if b2 is None else b2[e])
        sum_h = off_g @ b.abs().T + (F + 2) * 2.0 ** -23 * ((g.abs() + off_g) @ b.abs().T + (0.0 if b2 is None else b2[e].abs()))
        tu[lo:hi] = sum_u + HALF[dtype] * (u[lo:hi].abs() + sum_u)
        th[lo:hi] = sum_h + HALF[dtype] * (h[lo:hi].abs() + sum_h)
    return u, h, tu + 1e-38, th + 1e-38


def times_weights(y, offsets, experts, W, dtype):
    """(y W_e, bound) of packed rows y: one grouped product, one rounding."""
    out = torch.zeros((y.shape[0], W.shape[2]), dtype=torch.float64)
    tol = torch.zeros_like(out)
    for s, e in enumerate(experts):
        lo, hi = offsets[s], offsets[s + 1]
        out[lo:hi] = y[lo:hi] @ W[e]
        off = (W.shape[1] + 2) * 2.0 ** -23 * (y[lo:hi].abs() @ W[e].abs())
        tol[lo:hi] = off + HALF[dtype] * (out[lo:hi].abs() + off)
    return out, tol + 1e-38


def within(got, want, tol, what=""):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = ((got - want).abs() > tol)
    assert not over.any(), f"{what}: {int(over.sum())} of {got.numel()} beyond the bound, worst {float(((got - want).abs() / tol).max()):.3g} of it"


def route(gen, T, E, k, drop=0.0, used=None):
    """Distinct experts per pair, dropped pairs, and the order by (expert, pair): idx, live, offsets, perm, inv, rows."""
    pool = torch.arange(E) if used is None else torch.tensor(used)
    idx = pool[torch.rand((T, len(pool)), generator=gen).argsort(1)[:, :k]].reshape(T, k)
    live = torch.rand((T, k), generator=gen) >= drop
    key = torch.where(live, idx, E).flatten()
    order = torch.argsort(key, stable=True)
    rows = int(live.sum())
    perm = torch.full((T * k,), -1, dtype=torch.int32)
    perm[:rows] = order[:rows].to(torch.int32)
    inv = torch.full((T * k,), -1, dtype=torch.int32)
    inv[order[:rows]] = torch.arange(rows, dtype=torch.int32)
    counts = torch.bincount(key, minlength=E + 1)[:E]
    offsets = [0] + counts.cumsum(0).tolist()
    return idx.to(torch.int32), live, offsets, perm, inv, rows
