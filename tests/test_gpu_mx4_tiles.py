"""Every kernel and tile of the 4-bit FFN at shapes that take it, ragged segments, sampled rows against double precision."""
import numpy as np
import pytest
import torch

import mx4_plan_util as P
import mx4_util as M
from paper_2411_16786_amd import binding as B

pytestmark = pytest.mark.gpu

# rows, d, F, experts, and the kernels that the shape is here for: (place of the product: first and second of the forward, first and second of
# the gradient; its kernel)
SHAPES = [
    (1, 64, 256, 4, [(0, "rows16"), (1, "rows16"), (2, "rows"), (3, "rows")]),
    (2, 64, 16384, 4, [(0, "rows32")]),
    (16, 1792, 7168, 16, [(1, "rows32")]),
    (26, 64, 256, 4, [(0, "32x64/4"), (1, "32x64/4"), (2, "32x128/4"), (3, "32x128/4")]),
    (26, 512, 2048, 4, [(0, "32x64/4+"), (1, "32x64/4+")]),
    (26, 64, 16384, 4, [(0, "32x128/2"), (2, "32x128/2")]),
    (40, 2048, 8192, 16, [(0, "32x128/2+")]),
    (100, 64, 16384, 4, [(0, "64x128")]),
    (128, 64, 7680, 2, [(0, "64x128/2")]),
    (600, 512, 2048, 4, [(0, "64x128/2+")]),
    (600, 64, 16384, 4, [(0, "128x128")]),
    (1000, 64, 7680, 2, [(0, "128x256"), (2, "64x256")]),
    (1000, 1792, 7168, 16, [(1, "64x128+")]),
    (3000, 1024, 4096, 8, [(0, "128x256+")]),
    (3000, 384, 1536, 16, [(1, "64x128/2+")]),
    (3000, 2048, 8192, 16, [(1, "128x256+")]),
    (600, 2048, 8192, 16, [(1, "32x128/2+")]),
    (8192, 64, 256, 4, [(1, "64x128/2")]),
    (8192, 320, 1280, 4, [(1, "64x128")]),
    (8192, 512, 2048, 4, [(3, "64x256")]),
    (16384, 64, 256, 4, [(3, "32x128/2")]),
    (16384, 320, 1280, 4, [(1, "128x128")]),
    (16384, 384, 1536, 16, [(1, "128x128+")]),
    (2000, 1152, 4608, 8, [(0, "64x128"), (3, "32x128/2")]),
]
ROWS_CHECKED = 48                                                   # per expert, its first and last rows among them


def _decode(codes, scales):
    table = torch.tensor(M.CODE_VALUE, device="cuda")
    v = torch.stack([table[(codes & 15).int()], table[(codes >> 4).int()]], -1).reshape(codes.shape[0], -1)
    return v * torch.exp2(scales.double() - 127.0).repeat_interleave(32, dim=1)


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s[:4])))
def test_shape(shape):
    R, d, F, E, kernels = shape
    plans = P.plans(R, E, d, F)
    for place, name in kernels:
        assert plans[place] == name, (place, plans)
    print("shape", shape, plans, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(R + d + F)
    rng = np.random.default_rng(R + d)
    share = rng.dirichlet(np.full(E, 2.0))
    if E > 2 and R > 4:
        share[1] = 0.0                                              # an expert without rows
    counts = rng.multinomial(R, share / share.sum())
    offsets = np.concatenate([[0], np.cumsum(counts)])
    ctx = B.Context(R, d, F, E, 1, "bf16")
    bits = lambda *s: torch.randint(0, 256, s, generator=gen, device="cuda", dtype=torch.uint8)
    level = lambda *s: torch.randint(120, 124, s, generator=gen, device="cuda", dtype=torch.int32).to(torch.uint8)
    W1, W2 = (bits(E, F, d // 2), level(E, F, d // 32)), (bits(E, d, F // 2), level(E, d, F // 32))
    b1, b2 = (torch.randn(s, generator=gen, device="cuda") * 0.1 for s in ((E, F), (E, d)))
    scale = 8.0 / d ** 0.5                                          # pre-activations of order one
    x = (torch.randn((R, d), generator=gen, device="cuda") * scale).bfloat16()
    seg, experts = torch.tensor(offsets, dtype=torch.int32, device="cuda"), torch.arange(E, dtype=torch.int32, device="cuda")
    ws = torch.empty(ctx.workspace_bytes(), dtype=torch.uint8, device="cuda")
    u, h = torch.full((R, F), 3.0, dtype=torch.bfloat16, device="cuda"), torch.full((R, d), 3.0, dtype=torch.bfloat16, device="cuda")
    perm = torch.randperm(R, generator=gen, device="cuda").to(torch.int32)
    ctx.moe_expert_ffn_mx4(x, perm, None, seg, experts, R, W1, b1, W2, b2, u, h, ws)
    dh = torch.randn((R, d), generator=gen, device="cuda").bfloat16()
    du, dx = torch.empty_like(u), torch.empty_like(h)
    ctx.moe_expert_ffn_mx4_backward(dh, u, seg, experts, R, W1, W2, du, dx, ws)
    torch.cuda.synchronize()
    ctx.moe_expert_ffn_status(ws)

    for e in range(E):
        lo, hi = int(offsets[e]), int(offsets[e + 1])
        if lo == hi:
            continue
        pick = np.unique(np.concatenate([[lo, hi - 1], rng.integers(lo, hi, ROWS_CHECKED)]))
        rows = torch.from_numpy(pick).cuda()
        v1, v2 = _decode(W1[0][e], W1[1][e])[None], _decode(W2[0][e], W2[1][e])[None]
        ends = [0, len(pick)]
        with torch.device("cuda"):
            ref = M.ffn(x[perm[rows].long()].double(), ends, [0], v1, b1[e:e + 1].double(), v2, b2[e:e + 1].double(), "bf16")
            ref = [t.cpu() for t in ref]
            raw, tol = M.times_weights(dh[rows].double(), ends, [0], v2, "f32")
            back, back_tol = M.times_weights(du[rows].double(), ends, [0], v1, "bf16")
        M.within(u[rows], ref[0], ref[2], f"u of expert {e}")
        M.within(h[rows], ref[1], ref[3], f"h of expert {e}")
        slope = M.gelu_slope(u[rows].double())
        want = raw * slope
        off = 1.13 * tol + 4e-6 * (raw.abs() + tol)
        M.within(du[rows], want.cpu(), (off + M.HALF["bf16"] * (want.abs() + off)).cpu(), f"du of expert {e}")
        M.within(dx[rows], back.cpu(), back_tol.cpu(), f"dx of expert {e}")
    assert not (u == 3.0).all(1).any() and not (h == 3.0).all(1).any()          # every row was written
