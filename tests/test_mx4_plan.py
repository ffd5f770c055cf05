"""Rules by which the 4-bit FFN picks kernels and tiles, on the CPU."""
import pytest

import mx4_plan_util as P


def test_every_tile_fits_the_lds_and_every_size_has_a_kernel():
    L = P.lib()
    for K in [64 * i for i in (1, 2, 3, 7, 8, 16, 18, 28, 32, 72, 112, 128, 200, 256, 300, 512, 1024, 2048, 4096, 16384)]:
        for N in (64, 192, 1152, 4608, 8192, 1 << 20):
            for n_seg in (1, 4, 16, 1024):
                for rows in (0, 1, 15, 16, 17, 64, 100, 1000, 8192):
                    t = L.tile(rows, n_seg, N, K)
                    assert -1 <= t < len(P.TILES)
                    if t >= 0:
                        assert L.lds(t, K) <= 160 * 1024, (t, K)
                    assert -1 <= L.tile_t(rows, n_seg, N) < len(P.TILES_T)


@pytest.mark.parametrize("rows,n_seg,BM,tiles", [(0, 4, 16, 1), (1, 4, 16, 1), (3, 4, 16, 3), (16, 1, 16, 2), (17, 2, 16, 3), (1000, 8, 128, 15), (5, 1024, 32, 5)])
def test_tile_bound(rows, n_seg, BM, tiles):
    """No table of n segments with that many rows has more tiles: checked against the worst table, one-row segments first."""
    assert P.lib().bound(rows, n_seg, BM) == tiles
    counts = [1] * min(rows, n_seg - 1)
    counts.append(rows - len(counts))
    assert sum((c + BM - 1) // BM for c in counts) <= tiles


@pytest.mark.parametrize("rows,n_seg,d,F,names", [
    (2, 8, 1152, 4608, ("rows16", "rows16", "rows", "rows")),                      # one token
    (16, 8, 1152, 4608, ("rows32", "rows16", "rows", "rows")),
    (200, 8, 1152, 4608, ("32x128/2", "32x64/4+", "32x128/2", "32x128/4")),
    (2000, 8, 1152, 4608, ("64x128", "64x128/2+", "64x256", "32x128/2")),
    (8192, 8, 1152, 4608, ("128x256", "64x128", "64x256", "64x256")),              # the headline batch
    (8192, 16, 2048, 8192, ("128x256+", "128x128+", "64x256", "64x256")),
])
def test_choices(rows, n_seg, d, F, names):
    assert P.plans(rows, n_seg, d, F) == names


@pytest.mark.parametrize("rows,n_seg,d,F,names", [
    (2, 8, 1152, 4608, ("rows16", "rows16")),
    (120, 16, 384, 1536, ("rows32", "rows16")),
    (1000, 16, 384, 1536, ("rows64", "rows32")),
    (2000, 8, 1152, 4608, ("rows64", "rows64")),
])
def test_choices_in_float(rows, n_seg, d, F, names):
    assert (P.plan_float(rows, n_seg, F), P.plan_float(rows, n_seg, d)) == names
