"""The backward pass of a layer with as many rows as a context takes: byte offsets up to 2^32 and beyond, sampled tokens and rows."""
import pytest
import torch

import mx4_stage_util as S
import mx4_util as M
from paper_2411_16786_amd import binding as B

pytestmark = pytest.mark.gpu


def test_as_many_rows_as_a_context_takes():
    T, d, F, E, k = (1 << 24) - 32, 64, 64, 4, 2                    # T * k * d = 2^31 - 4096
    with pytest.raises(B.MoeError):
        B.Context(T + 32, d, F, E, k, "bf16")
    ctx, N, bf = B.Context(T, d, F, E, k, "bf16"), T * k, torch.bfloat16
    gen = torch.Generator(device="cuda").manual_seed(1)
    normal = lambda *s: torch.empty(s, dtype=bf, device="cuda").normal_(generator=gen)
    new = lambda *s, dt=bf: torch.full(s, 3.0, dtype=dt, device="cuda")
    probs = torch.softmax(torch.randn((T, E), generator=gen, device="cuda"), 1)
    scores, idx = torch.topk(probs, k, 1)
    order = torch.argsort(idx.flatten().to(torch.uint8), stable=True)
    perm, inv = order.to(torch.int32), torch.empty(N, dtype=torch.int32, device="cuda")
    inv[order] = torch.arange(N, dtype=torch.int32, device="cuda")
    offsets = [0] + torch.bincount(idx.flatten(), minlength=E).cumsum(0).tolist()
    seg, experts, idx = torch.tensor(offsets, dtype=torch.int32, device="cuda"), torch.arange(E, dtype=torch.int32, device="cuda"), idx.to(torch.int32)
    bits = lambda *s: torch.randint(0, 256, s, generator=gen, device="cuda", dtype=torch.uint8)
    level = lambda *s: torch.randint(120, 124, s, generator=gen, device="cuda", dtype=torch.int32).to(torch.uint8)
    W1, W2 = (bits(E, F, d // 2), level(E, F, d // 32)), (bits(E, d, F // 2), level(E, d, F // 32))
    x, dy, Wg = normal(T, d), normal(T, d), normal(E, d)
    ws = torch.empty(ctx.workspace_bytes(), dtype=torch.uint8, device="cuda")
    u, h, dh, dxp, dx = new(N, F), new(N, d), new(N, d), new(N, d), new(T, d)
    ds, dz, dWg, dbg = (new(*s, dt=torch.float32) for s in ((T, k), (T, E), (E, d), (E,)))
    print("forward", flush=True)
    ctx.moe_expert_ffn_mx4(x, perm, None, seg, experts, N, W1, None, W2, None, u, h, ws)
    ctx.moe_expert_ffn_status(ws)
    kept = ws[:N * F * 2].view(bf).reshape(N, F)
    pick = torch.cat([torch.tensor([0, 1, N - 2, N - 1, N // 2], device="cuda"), torch.randint(0, N, (500,), generator=gen, device="cuda")])
    pick = torch.cat([pick, *(torch.tensor([lo, hi - 1], device="cuda") for lo, hi in zip(offsets, offsets[1:]))])
    kept = kept[pick].clone()
    print("backward", flush=True)
    ctx.moe_combine_backward(dy, h, inv, scores.contiguous(), dh, ds)
    ctx.moe_expert_ffn_mx4_backward(dh, u, seg, experts, N, W1, W2, None, dxp, ws)
    ctx.moe_route_backward(x, Wg, idx, probs, ds, None, None, dxp, inv, dx, dz, dWg, dbg, ws)
    torch.cuda.synchronize()

    half = M.HALF["bf16"]
    for e in range(E):
        at = (pick >= offsets[e]) & (pick < offsets[e + 1])
        rows, pair = pick[at], order[pick[at]]
        v1, v2 = (M.decode(W[0][e], W[1][e]) for W in (W1, W2))
        f64 = lambda t: t.cpu().double()
        want, off = S.sums(f64(x[pair // k]), v1, None)
        M.within(u[rows], want, S.rounded(want, off, "bf16"), "u")
        M.within(kept[at], *S.hidden(want, off, "bf16"), "hidden")
        want, off = S.sums(f64(kept[at]), v2, None)
        M.within(h[rows], want, S.rounded(want, off, "bf16"), "h")
        want = f64(scores.flatten()[pair])[:, None] * f64(dy[pair // k])
        M.within(dh[rows], want, half * want.abs() * (1 + 1e-6) + 2.0 ** -24 * want.abs() + 1e-38, "dh")
        prod = f64(h[rows]) * f64(dy[pair // k])
        M.within(ds.flatten()[pair], prod.sum(1), (d + 2) * 2.0 ** -24 * prod.abs().sum(1) + 1e-38, "dscores")
        # dx_packed through du, which is not kept: its rounding and its sum's bound go through the second product's magnitudes
        raw, off = S.sums(f64(dh[rows]), v2.T.contiguous(), None)
        du = raw * M.gelu_slope(f64(u[rows]))
        off = S.rounded(du, 1.13 * off + 4e-6 * (raw.abs() + off), "bf16")
        want, more = S.sums(du, v1.T.contiguous(), None)
        off = off @ v1.abs() + 2 * more
        M.within(dxp[rows], want, off + half * (want.abs() + off), "dx_packed")
    tok = torch.cat([torch.tensor([0, 1, T - 1], device="cuda"), torch.randint(0, T, (300,), generator=gen, device="cuda")])
    P, g = probs[tok].cpu().double(), torch.zeros((len(tok), E), dtype=torch.float64)
    g.scatter_add_(1, idx[tok].cpu().long(), ds[tok].cpu().double())
    want = P * (g - (P * g).sum(1, keepdim=True))
    off = (E + 3 * k + 8) * 2.0 ** -24 * (P * (g.abs() + (P * g.abs()).sum(1, keepdim=True))) + 1e-38
    M.within(dz[tok], want, off, "dz")
    rows = dxp[inv.view(T, k)[tok].long()].cpu().double()
    W = Wg.cpu().double()
    off, mag = off @ W.abs(), want.abs() @ W.abs() + rows.abs().sum(1)
    want = rows.sum(1) + want @ W
    off = off + (E + k + 2) * 2.0 ** -23 * mag
    M.within(dx[tok], want, off + half * (want.abs() + off) + 1e-38, "dx")
    assert torch.isfinite(dWg).all() and torch.isfinite(dbg).all()
    for t in (u, h, dxp, dx):                                       # every row was written
        assert not any(bool((part == 3.0).all(1).any()) for part in t.split(1 << 22))
