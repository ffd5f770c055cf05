"""What the bounds of the 4-bit FFN's tests let through, on the CPU: a right result stays well within them, a lost stage of a reduction,
a wrong scale and a GELU of another form do not, at the widths the GPU tests use."""
import pytest
import torch

import mx4_stage_util as S
import mx4_util as M
import test_gpu_mx4
import test_gpu_mx4_partial_columns
import test_gpu_mx4_tiles

WIDTHS = sorted({("bf16", s[1], s[2]) for s in test_gpu_mx4_tiles.SHAPES + test_gpu_mx4_partial_columns.PARTIAL} | {(c[5], c[1], c[2]) for c in test_gpu_mx4.CASES})
ROWS = 8


@pytest.mark.parametrize("dtype,d,F", WIDTHS)
def test_planted_mistakes_exceed_the_bounds(dtype, d, F):
    gen = torch.Generator().manual_seed(d + F)
    bits = lambda *s: torch.randint(0, 256, s, generator=gen, dtype=torch.uint8)
    level = lambda *s: torch.randint(120, 124, s, generator=gen, dtype=torch.int32).to(torch.uint8)
    W1, W2 = (M.decode(bits(n, K // 2), level(n, K // 32)) for n, K in ((F, d), (d, F)))
    b1, b2 = (torch.randn(n, generator=gen, dtype=torch.float64) * 0.1 for n in (F, d))
    x = (torch.randn((ROWS, d), generator=gen) * 8.0 / d ** 0.5).to(M.DT[dtype]).double()
    store = lambda t: t.to(M.DT[dtype]).double()

    u, off_u = S.sums(x, W1, b1)
    g, tol_g = S.hidden(u, off_u, dtype)
    kept = store(g)
    h, off_h = S.sums(kept, W2, b2)
    tol_u, tol_h = S.rounded(u, off_u, dtype), S.rounded(h, off_h, dtype)
    single = lambda a, W, b: (a.float() @ W.float().T + b.float()).double()
    assert S.excess(store(single(x, W1, b1)), u, tol_u) <= 1 and S.excess(store(single(kept, W2, b2)), h, tol_h) <= 1
    assert S.excess(kept, g, tol_g) <= 1

    def mistakes(rows, W, b, want, tol):
        last = min(64, W.shape[1] // 2)                             # a stage of the tiles, or what stands for it in a short reduction
        cut = rows.clone()
        cut[:, -last:] = 0.0
        doubled = W.clone()
        doubled[:, :32] *= 2.0
        assert S.excess(store(S.sums(cut, W, b)[0]), want, tol) > 2, "a lost stage"
        assert S.excess(store(S.sums(rows, doubled, b)[0]), want, tol) > 2, "a doubled scale"

    mistakes(x, W1, b1, u, tol_u)
    mistakes(kept, W2, b2, h, tol_h)
    assert S.excess(store(u * torch.sigmoid(1.702 * u)), g, tol_g) > 2, "a sigmoid for the normal distribution"
