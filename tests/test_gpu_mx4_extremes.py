"""4-bit experts at the ends of the number range: the largest weights."""

import numpy as np
import pytest
import torch

import mx4_util as M
from paper_2411_16786_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_largest_weights_stand_for_numbers(dtype):
    """Scales end at 2^125, whose largest code value, 1.5 2^127, is a number; what lies above it becomes that."""
    end = torch.finfo(M.DT[dtype]).max
    tops = [1.5 * 2.0 ** 127, 1.75 * 2.0 ** 127, 1.875 * 2.0 ** 127, end, -end, 2.0 ** 127, 7.0 * 2.0 ** 124, 7.5 * 2.0 ** 124]
    rest = np.array([0, .25, .75, 1, 1.25, 2.5, 3, 3.5, 3.75, 4, 5, 5.5, 6, 7]) * 2.0 ** 125
    w = torch.zeros((len(tops), 32), dtype=torch.float64)
    for i, top in enumerate(tops):
        fits = rest[rest <= abs(top)]
        w[i, 0], w[i, 1:1 + len(fits)] = top, torch.from_numpy(fits * (-1.0) ** np.arange(len(fits)))
    ctx = B.Context(1, 64, 64, 1, 1, dtype)
    codes, scales, values = (torch.empty(s, dtype=t, device="cuda") for s, t in (((len(tops), 16), torch.uint8), ((len(tops), 1), torch.uint8), ((len(tops), 32), M.DT[dtype])))
    ctx.moe_quantize_mx4(w.to(M.DT[dtype]).cuda(), codes, scales, values)
    byte = np.array([127 + 125 if abs(t) > 7.0 * 2.0 ** 124 else 127 + 124 for t in tops])
    assert np.array_equal(scales.cpu().numpy()[:, 0], byte)
    got = values.cpu().double().numpy()
    assert np.isfinite(got).all()
    assert np.array_equal(got, M.decode(codes, scales).numpy())
    step = np.exp2(byte - 127.0)[:, None]
    v = w.abs().numpy() / step
    even = np.array([0, 2, 4, 6, 1, 3, 5, 7])                       # the even code of a tie comes first
    code = even[np.argmin(np.abs(v[..., None] - M.MAGNITUDE[even]), axis=-1)]
    assert np.array_equal(np.abs(got), M.MAGNITUDE[code] * step)
    assert np.array_equal(np.signbit(got), np.signbit(w.numpy()))
