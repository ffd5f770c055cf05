"""4-bit experts at the ends of the number range: the largest weights, infinite pre-activations, the tails of GELU and of its slope."""
import math

import numpy as np
import pytest
import torch

import mx4_stage_util as S
import mx4_util as M
from paper_2411_16786_amd import binding as B

pytestmark = pytest.mark.gpu

INF = float("inf")


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


class Ends:
    """Rows through designed weights of one expert, d = 64, F = 128, all scales 1."""

    def __init__(self, T, dtype):
        self.T, self.dtype, self.dt = T, dtype, M.DT[dtype]
        self.ctx = B.Context(T, 64, 128, 1, 1, dtype)
        self.seg, self.one = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([0, T], [0]))
        self.ws = torch.empty(self.ctx.workspace_bytes(), dtype=torch.uint8, device="cuda")

    @staticmethod
    def weights(code):
        """codes [rows, cols] 0 .. 15 as the calls take them."""
        code = code.to(torch.uint8)
        return (code[:, 0::2] | (code[:, 1::2] << 4)).contiguous()[None].cuda(), torch.full((1, code.shape[0], code.shape[1] // 32), 127, dtype=torch.uint8).cuda()

    def forward(self, x, W1, W2):
        u, h = (torch.full((self.T, n), 3.0, dtype=self.dt, device="cuda") for n in (128, 64))
        self.ctx.moe_expert_ffn_mx4(x.to(self.dt).cuda(), None, None, self.seg, self.one, self.T, W1, None, W2, None, u, h, self.ws)
        kept = S.stored_hidden(self.ws, self.T, 128, self.dt).cpu().double()
        return u.cpu().double(), kept, h.cpu().double()

    def slopes(self, u):
        """gelu'(u) [T, 128] through a gradient whose product is exactly 1 everywhere."""
        code = torch.zeros((64, 128))
        code[0] = 2                                                 # the first row of W2 holds ones, and dh selects it
        dh = torch.zeros((self.T, 64))
        dh[:, 0] = 1.0
        du, dx = (torch.empty((self.T, n), dtype=self.dt, device="cuda") for n in (128, 64))
        self.ctx.moe_expert_ffn_mx4_backward(dh.to(self.dt).cuda(), u.to(self.dt).cuda(), self.seg, self.one, self.T, self.weights(torch.zeros((128, 64))),
                                             self.weights(code), du, dx, self.ws)
        return du.cpu().double()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [4, 300])
def test_infinite_pre_activations(dtype, T):
    """Sums that overflow are infinite, gelu of -infinity is (near) zero, and the second product gives what arithmetic with infinities gives."""
    c = Ends(T, dtype)
    gen = torch.Generator().manual_seed(T)
    n = torch.arange(128)
    code1 = torch.randint(0, 8, (128, 64), generator=gen)           # column 0: 0, 4, -4, 2 in turn; column 1: -4
    code1[:, 0], code1[:, 1] = torch.tensor([0, 6, 14, 4])[n % 4], 14
    x = torch.zeros((T, 64))
    kind = torch.arange(T) % 4
    x[kind == 0, 0], x[kind == 1, 0], x[kind == 2, 1], x[kind == 3, 0] = 3e38, -3e38, 3e38, 0.5
    code2 = torch.randint(0, 16, (64, 128), generator=gen)
    code2[0], code2[1], code2[2] = 4, 12, 0                         # 2, -2 and 0 everywhere
    code2[3] = torch.tensor([4, 4, 4, 12])[n % 4]                   # 2, 2, 2, -2
    code2[4] = torch.where(n % 4 == 2, 0, 4)
    u, kept, h = c.forward(x, c.weights(code1), c.weights(code2))
    ends = torch.tensor([0.0, INF, -INF, INF])[n % 4].double()
    assert torch.isinf(u).any()
    assert torch.equal(u[kind == 0], ends.expand(int((kind == 0).sum()), 128)) and torch.equal(u[kind == 1], -ends.expand(int((kind == 1).sum()), 128))
    assert (u[kind == 2] == -INF).all()
    assert not torch.isnan(kept).any()
    assert torch.equal(torch.isinf(kept), u == INF) and (kept[u == -INF].abs() < 1e-8).all()
    up = h[kind == 0]                                               # infinite where n % 4 is 1 or 3
    assert (up[:, 0] == INF).all() and (up[:, 1] == -INF).all() and torch.isnan(up[:, 2:4]).all() and (up[:, 4] == INF).all()
    down = h[kind == 1]                                             # ... where it is 2
    assert (down[:, 0] == INF).all() and (down[:, 1] == -INF).all() and torch.isnan(down[:, 2]).all() and (down[:, 3] == INF).all() and torch.isnan(down[:, 4]).all()
    assert (h[kind == 2].abs() < 1e-5).all()                        # 128 terms of 6e-9 times 6 at most
    small = h[kind == 3]
    g, v2 = M.gelu(torch.tensor([0.0, 2.0, -2.0, 1.0]).double())[n % 4], torch.from_numpy(M.CODE_VALUE[code2.numpy()])
    want, size = v2 @ g, v2.abs() @ g.abs()
    off = (M.HALF[dtype] + 130 * 2.0 ** -23) * size + 1e-6 * v2.abs().sum(1)        # one rounding of the hidden value, the sum, the form of GELU
    assert ((small - want).abs() <= off + M.HALF[dtype] * (want.abs() + off)).all()


@pytest.mark.parametrize("T", [7, 300])
def test_float_gelu_keeps_its_digits_in_the_tail(T):
    """Relative to gelu(u) = u Phi(u), u from -12 to 0: erfc(x), x = -u / sqrt 2, amplifies the two roundings of x by at most 2 x^2 + 1 = u^2 + 1
    each; 16 half steps for erfc itself and the products."""
    c = Ends(T, "f32")
    u = -12.0 * torch.rand(T, generator=torch.Generator().manual_seed(T))
    u[0], u[1], u[2] = -5.0, -5.5, -12.0
    code1 = torch.zeros((128, 64))
    code1[:, 0] = 2
    x = torch.zeros((T, 64))
    x[:, 0] = u
    got_u, kept, _ = c.forward(x, c.weights(code1), c.weights(torch.zeros((64, 128))))
    v = u.double()[:, None].expand(T, 128)
    assert torch.equal(got_u, v)
    want = M.gelu(v)
    assert ((kept - want).abs() <= (2 * (v * v + 1) + 16) * 2.0 ** -24 * want.abs()).all(), S.excess(kept, want, 2.0 ** -24 * want.abs())


@pytest.mark.parametrize("T", [7, 300])
def test_float_slope_keeps_its_digits_in_the_tail(T):
    """Relative to Phi(u) + |u| phi(u), u from -12 to 12: as above for Phi; the exponent u^2 / 2 of phi has two roundings, so u^2 half steps,
    and 16 more for exp and the products."""
    c = Ends(T, "f32")
    u = torch.linspace(-12.0, 12.0, T * 128).reshape(T, 128)
    u[0, :4] = torch.tensor([-5.0, -5.5, -6.0, -0.75])
    got, v = c.slopes(u), u.double()
    phi = torch.exp(-0.5 * v * v) / math.sqrt(2.0 * math.pi)
    Phi = 0.5 * torch.erfc(-v / math.sqrt(2.0))
    tol = ((2 * (v * v + 1) + 16) * Phi + (v * v + 16) * v.abs() * phi) * 2.0 ** -24
    want = Phi + v * phi
    assert ((got - want).abs() <= tol).all(), S.excess(got, want, tol)


@pytest.mark.parametrize("T", [7, 300])
def test_bf16_slope_beyond_its_polynomial(T):
    """gelu' is below 1e-13 in magnitude from -8 on and as near to 1 from 8 on: 0 and 1 in bf16."""
    c = Ends(T, "bf16")
    u = torch.tensor([-8.0, -9.5, -60.0, -1e30, -INF, 8.0, 9.5, 60.0, 1e30, INF])[torch.arange(T * 128) % 10].reshape(T, 128)
    assert torch.equal(c.slopes(u).abs(), (u > 0).double())
