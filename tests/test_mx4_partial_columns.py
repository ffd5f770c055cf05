"""Every tile of the 4-bit FFN that can have a last block of columns with less than all of them is tested with one.  Needs no GPU."""
import mx4_plan_util as P
import test_gpu_mx4_partial_columns
import test_gpu_mx4_tiles


def _runs(partial):
    """(transposed, kernel) of all products of the tile tests' shapes, those with columns left over only if ``partial``."""
    found = set()
    for R, d, F, E, _ in test_gpu_mx4_tiles.SHAPES + test_gpu_mx4_partial_columns.PARTIAL:
        for place, name in enumerate(P.plans(R, E, d, F)):
            if not partial or P.columns_left(name, (F, d, F, d)[place]):
                found.add((place >= 2, name))
    return found


def test_every_tile_runs_and_runs_with_columns_left_over():
    tiles = {(False, t + c) for t in P.TILES for c in ("", "+")} | {(True, t) for t in P.TILES_T}
    assert tiles <= _runs(False)
    whole = {(False, "32x64/4"), (False, "32x64/4+")}               # N is a multiple of 64: their blocks are always whole
    assert tiles - whole <= _runs(True)
    assert (True, "rows") in _runs(True)
