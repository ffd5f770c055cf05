"""The 4-bit FFN product by product: the hidden rows against gelu of the first, the second from the hidden rows as stored."""
import numpy as np
import pytest
import torch

import mx4_plan_util as P
import mx4_stage_util as S
import mx4_util as M
import test_gpu_mx4
import test_gpu_mx4_tiles
from paper_2411_16786_amd import binding as B

pytestmark = pytest.mark.gpu

ROWS_CHECKED = 32


def check(shape):
    """One forward and one backward call of a shape, sampled rows of every expert."""
    R, d, F, E, kernels = shape
    plans = P.plans(R, E, d, F)
    for place, name in kernels:
        assert plans[place] == name, (place, plans)
    print("shape", shape, plans, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(R + 3 * d + F)
    rng = np.random.default_rng(R + d + F)
    counts = rng.multinomial(R, rng.dirichlet(np.full(E, 2.0)))
    offsets = np.concatenate([[0], np.cumsum(counts)])
    ctx = B.Context(R, d, F, E, 1, "bf16")
    bits = lambda *s: torch.randint(0, 256, s, generator=gen, device="cuda", dtype=torch.uint8)
    level = lambda *s: torch.randint(120, 124, s, generator=gen, device="cuda", dtype=torch.int32).to(torch.uint8)
    W1, W2 = (bits(E, F, d // 2), level(E, F, d // 32)), (bits(E, d, F // 2), level(E, d, F // 32))
    b1, b2 = (torch.randn(s, generator=gen, device="cuda") * 0.1 for s in ((E, F), (E, d)))
    x = (torch.randn((R, d), generator=gen, device="cuda") * 8.0 / d ** 0.5).bfloat16()
    dh = torch.randn((R, d), generator=gen, device="cuda").bfloat16()
    seg, experts = torch.tensor(offsets, dtype=torch.int32, device="cuda"), torch.arange(E, dtype=torch.int32, device="cuda")
    ws = torch.empty(ctx.workspace_bytes(), dtype=torch.uint8, device="cuda")
    # 64 rows of guard behind the outputs: columns past the end of a row would land in the next one, those of the last row here
    u, h, du, dx = (torch.full((R + 64, n), 3.0, dtype=torch.bfloat16, device="cuda") for n in (F, d, F, d))
    ctx.moe_expert_ffn_mx4(x, None, None, seg, experts, R, W1, b1, W2, b2, u, h, ws)
    kept = S.stored_hidden(ws, R, F, torch.bfloat16)
    ctx.moe_expert_ffn_mx4_backward(dh, u, seg, experts, R, W1, W2, du, dx, ws)
    torch.cuda.synchronize()
    for t in (u, h, du, dx):
        assert (t[R:] == 3.0).all() and not (t[:R] == 3.0).all(1).any()
    for e in range(E):
        lo, hi = int(offsets[e]), int(offsets[e + 1])
        if lo == hi:
            continue
        rows = torch.from_numpy(np.unique(np.concatenate([[lo, hi - 1], rng.integers(lo, hi, ROWS_CHECKED)]))).cuda()
        v1, v2 = (test_gpu_mx4_tiles._decode(W[0][e], W[1][e]) for W in (W1, W2))

        def near(got, want, tol, what):
            M.within(got, want.cpu(), tol.cpu(), f"{what} of expert {e}")

        want, off = S.sums(x[rows].double(), v1, b1[e].double())
        near(u[rows], want, S.rounded(want, off, "bf16"), "u")
        near(kept[rows], *S.hidden(want, off, "bf16"), "hidden")
        want, off = S.sums(kept[rows].double(), v2, b2[e].double())
        near(h[rows], want, S.rounded(want, off, "bf16"), "h")
        raw, off = S.sums(dh[rows].double(), v2.T.contiguous(), None)
        slope = M.gelu_slope(u[rows].double())
        off = 1.13 * off + 4e-6 * (raw.abs() + off)
        near(du[rows], raw * slope, S.rounded(raw * slope, off, "bf16"), "du")
        want, off = S.sums(du[rows].double(), v1.T.contiguous(), None)
        near(dx[rows], want, S.rounded(want, off, "bf16"), "dx")


@pytest.mark.parametrize("shape", test_gpu_mx4_tiles.SHAPES, ids=lambda s: "-".join(map(str, s[:4])))
def test_products(shape):
    check(shape)


@pytest.mark.parametrize("case", test_gpu_mx4.CASES, ids=lambda c: "-".join(map(str, c[:6])))
def test_products_of_small_shapes(case):
    T, d, F, E, k, dtype, bias, drop, used = case
    print("products", case, flush=True)
    c = test_gpu_mx4.Case(T, d, F, E, k, dtype, bias, drop, used)
    _, h = c.forward()
    kept = S.stored_hidden(c.ws, c.rows, F, c.dt).cpu()
    for e in range(E):
        lo, hi = c.offsets[e], c.offsets[e + 1]
        b1, b2 = (None if b is None else b[e].double() for b in (c.b1, c.b2))
        want, off = S.sums(c.xp[lo:hi], c.v1[e], b1)
        M.within(kept[lo:hi], *S.hidden(want, off, dtype), f"hidden of expert {e}")
        want, off = S.sums(kept[lo:hi].double(), c.v2[e], b2)
        M.within(h[lo:hi], want, S.rounded(want, off, dtype), f"h of expert {e}")
