"""Every tile of the 4-bit FFN where its last block of columns is not whole."""
import pytest

import mx4_plan_util as P
from test_gpu_mx4_stages import check

pytestmark = pytest.mark.gpu

# As test_gpu_mx4_tiles.SHAPES: the place's product has columns left over behind the last whole block of the kernel named (256 columns:
# 64, 128 and 192 of them, i.e. two, four or six wavefronts with work in the last block of the forward product, one to three of the gradient's)
PARTIAL = [
    (400, 64, 1600, 16, [(0, "64x128/2")]),
    (200, 64, 7232, 8, [(0, "64x128")]),
    (2000, 1088, 7168, 16, [(1, "64x128+")]),
    (8192, 64, 512, 2, [(1, "64x128/2+")]),
    (16384, 64, 320, 2, [(0, "128x128")]),
    (16384, 320, 1536, 2, [(1, "128x128+")]),
    (600, 64, 7744, 8, [(0, "128x256")]),
    (3000, 64, 4224, 2, [(0, "128x256")]),
    (3000, 64, 2240, 2, [(0, "128x256")]),
    (600, 512, 7744, 8, [(0, "128x256+")]),
    (3000, 512, 4224, 2, [(0, "128x256+")]),
    (3000, 512, 2240, 2, [(0, "128x256+")]),
    (26, 64, 6208, 16, [(0, "32x128/2")]),
    (26, 512, 6208, 16, [(0, "32x128/2+")]),
    (40, 64, 6208, 8, [(2, "32x128/2")]),
    (26, 64, 192, 2, [(2, "32x128/4")]),
    (400, 64, 6208, 8, [(2, "64x256")]),
    (1000, 64, 4224, 2, [(2, "64x256")]),
    (16384, 64, 192, 2, [(2, "64x256")]),
    (26, 64, 192, 8, [(2, "rows")]),
    (8192, 1152, 4608, 8, [(3, "64x256")]),                         # the headline batch
]


@pytest.mark.parametrize("shape", PARTIAL, ids=lambda s: "-".join(map(str, s[:4])))
def test_last_block_of_columns(shape):
    R, d, F, E, kernels = shape
    for place, name in kernels:
        assert P.columns_left(name, (F, d, F, d)[place]) > 0
    check(shape)
