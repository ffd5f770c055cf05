"""4-bit experts on the GPU against double precision: quantisation, the FFN and the gradient of its rows."""
import numpy as np
import pytest
import torch

import mx4_util as M
from paper_2411_16786_amd import binding as B

pytestmark = pytest.mark.gpu

F64 = torch.float64


def say(*a):
    print(*a, flush=True)


def dev(t, dtype=None):
    return t.to(dtype).cuda() if dtype is not None else t.cuda()


# ---- quantisation

def _expected(w):
    """Scale bytes and signed code values / scale, by search: w float64 [groups, 32]."""
    top = w.abs().amax(1).numpy()
    byte = np.ones(len(top), dtype=np.int64)
    for b in range(2, 255):
        byte = np.where(top > 7.0 * 2.0 ** (byte - 127.0), b, byte)
    v = (w.abs().numpy() / np.exp2(byte - 127.0)[:, None])
    dist = np.abs(v[..., None] - M.MAGNITUDE)
    best = dist.min(-1, keepdims=True)
    tied = dist == best
    even = np.array([0, 2, 4, 6, 1, 3, 5, 7])                 # the even code of a tie comes first
    code = even[np.argmax(tied[..., even], axis=-1)]
    code = code + 8 * np.signbit(w.numpy())
    return byte, code


def _check_quantize(w, dtype):
    """w: float64 [rows, cols], exact in dtype."""
    rows, cols = w.shape
    ctx = B.Context(1, 64, 64, 1, 1, dtype)
    W = dev(w, M.DT[dtype])
    codes = torch.full((rows * cols // 2 + 64,), 171, dtype=torch.uint8, device="cuda")
    scales = torch.full((rows * cols // 32 + 64,), 171, dtype=torch.uint8, device="cuda")
    values = torch.full((rows * cols + 64,), 5.0, dtype=M.DT[dtype], device="cuda")
    ctx.moe_quantize_mx4(W, codes[:rows * cols // 2], scales[:rows * cols // 32], values[:rows * cols])
    torch.cuda.synchronize()
    assert (codes[rows * cols // 2:] == 171).all() and (scales[rows * cols // 32:] == 171).all() and (values[rows * cols:] == 5.0).all()
    c = codes[:rows * cols // 2].cpu().numpy()
    got = np.stack([c & 15, c >> 4], -1).reshape(-1, 32)
    byte, code = _expected(w.reshape(-1, 32))
    assert np.array_equal(scales[:rows * cols // 32].cpu().numpy(), byte)
    assert np.array_equal(got, code), (got != code).sum()
    want = M.CODE_VALUE[code] * np.exp2(byte - 127.0)[:, None]
    assert np.array_equal(values[:rows * cols].cpu().double().numpy().reshape(-1, 32), want)
    only = torch.empty_like(codes[:rows * cols // 2])         # without the values
    ctx.moe_quantize_mx4(W, only, torch.empty_like(scales[:rows * cols // 32]))
    assert torch.equal(only, codes[:rows * cols // 2])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(1, 32), (3, 96), (257, 64), (64, 1152)])
def test_quantize_random(dtype, rows, cols):
    gen = torch.Generator().manual_seed(rows * cols)
    w = torch.randn((rows, cols), generator=gen) * torch.exp2(torch.randint(-40, 40, (rows, 1), generator=gen).float())
    _check_quantize(w.to(M.DT[dtype]).double(), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_ties_borders_and_extremes(dtype):
    ties = np.array([0, .25, .5, .75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7])
    step = 2.0 ** (-7 if dtype == "bf16" else -20)
    rows = []
    for scale in (1.0, 2.0 ** 60, 2.0 ** -100, 2.0 ** -126, 2.0 ** -127, 2.0 ** 124):
        for top in (4.0, 6.0, 7.0):                           # the group's largest magnitude, at scale 1
            small = ties[ties <= top]
            group = np.concatenate([small, -small])[:31]
            rows.append(np.concatenate([group, np.zeros(31 - len(group)), [top]]) * scale)
            near = np.concatenate([small[1:] * (1 + step), -small[1:] * (1 - step)])[:31]      # to either side of every border
            near = np.clip(near, -top, top)
            rows.append(np.concatenate([near, np.zeros(31 - len(near)), [top]]) * scale)
        rows.append(np.concatenate([[7.0 + 8 * step], np.zeros(31)]) * scale)                # just beyond 7: the next scale
    rows.append(np.zeros(32))
    rows.append(np.full(32, -0.0))
    w = torch.from_numpy(np.stack(rows)).to(M.DT[dtype])
    w = torch.where(torch.isfinite(w), w, torch.zeros_like(w)).double()
    _check_quantize(w, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_marks_groups_that_are_not_finite(dtype):
    w = torch.randn((4, 96), generator=torch.Generator().manual_seed(5)).to(M.DT[dtype])
    w[0, 3], w[1, 40], w[2, 95], w[3, 64] = float("nan"), float("inf"), -float("inf"), -float("nan")
    ctx = B.Context(1, 64, 64, 1, 1, dtype)
    codes, scales, values = (torch.empty(s, dtype=t, device="cuda") for s, t in (((4, 48), torch.uint8), ((4, 3), torch.uint8), ((4, 96), M.DT[dtype])))
    ctx.moe_quantize_mx4(dev(w), codes, scales, values)
    bad = torch.zeros((4, 3), dtype=torch.bool)
    bad[0, 0] = bad[1, 1] = bad[2, 2] = bad[3, 2] = True
    assert torch.equal(scales.cpu() == 255, bad)
    assert torch.equal(torch.isnan(values.cpu().float()).reshape(4, 3, 32).all(-1), bad)
    assert torch.equal(torch.isnan(values.cpu().float()).reshape(4, 3, 32).any(-1), bad)
    assert (codes.cpu().reshape(4, 3, 16)[bad] == 0).all()


def test_quantize_beyond_32_bit_offsets():
    """2^33 weights and some: more than one launch, offsets beyond 32 bits; every piece as the call on it alone gives it."""
    ctx = B.Context(1, 64, 64, 1, 1, "bf16")
    rows, cols = (1 << 20) + 3, 8192
    gen = torch.Generator(device="cuda").manual_seed(5)
    W = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    places = [0, 1, (1 << 18) - 1, 1 << 18, (1 << 19) + 5, (1 << 20) - 1, 1 << 20, rows - 1]        # 2^32 bytes and 2^33 elements among them
    W[places] = torch.randn((len(places), cols), generator=gen, device="cuda").bfloat16()
    codes = torch.full((rows, cols // 2), 171, dtype=torch.uint8, device="cuda")
    scales = torch.full((rows, cols // 32), 171, dtype=torch.uint8, device="cuda")
    ctx.moe_quantize_mx4(W, codes, scales)
    few = W[places].contiguous()
    few_codes, few_scales = torch.empty_like(codes[:len(places)]), torch.empty_like(scales[:len(places)])
    ctx.moe_quantize_mx4(few, few_codes, few_scales)
    torch.cuda.synchronize()
    assert torch.equal(codes[places], few_codes) and torch.equal(scales[places], few_scales)
    codes[places], scales[places] = 0, 1
    assert int(codes.amax()) == 0 and int(scales.amax()) == 1 and int(scales.amin()) == 1


# ---- the FFN and its gradient

class Case:
    def __init__(self, T, d, F, E, k, dtype, bias=False, drop=0.0, used=None, n_shared=0, seed=0):
        gen = torch.Generator().manual_seed(1000 * T + 7 * d + F + seed)
        self.dtype, self.dt, self.d, self.F, self.k = dtype, M.DT[dtype], d, F, k
        self.ctx = B.Context(max(T, 1), d, F, E, k, dtype, n_shared=n_shared)
        n = E + n_shared
        self.idx, self.live, self.offsets, self.perm, self.inv, self.rows = M.route(gen, T, n, k + n_shared, drop, used)
        self.N = T * (k + n_shared)
        self.W1, self.W2 = M.random_codes(gen, n, F, d), M.random_codes(gen, n, d, F)
        self.v1, self.v2 = M.decode(*self.W1), M.decode(*self.W2)
        self.b1 = torch.randn((n, F), generator=gen) * 0.1 if bias else None
        self.b2 = torch.randn((n, d), generator=gen) * 0.1 if bias else None
        self.x = torch.randn((T, d), generator=gen).to(self.dt)
        self.g1 = tuple(t.cuda() for t in self.W1)
        self.g2 = tuple(t.cuda() for t in self.W2)
        self.gb1, self.gb2 = (None if b is None else b.cuda() for b in (self.b1, self.b2))
        self.seg = torch.tensor(self.offsets, dtype=torch.int32).cuda()
        self.seg_expert = torch.arange(n, dtype=torch.int32).cuda()
        self.ws = torch.empty(self.ctx.workspace_bytes(), dtype=torch.uint8, device="cuda")
        self.gen = gen
        tok = (self.perm[:self.rows] // (k + n_shared)).long()
        self.xp = self.x[tok].double()
        self.ref = M.ffn(self.xp, self.offsets, range(n), self.v1, self._64(self.b1), self.v2, self._64(self.b2), dtype)

    @staticmethod
    def _64(b):
        return None if b is None else b.double()

    def forward(self, x=None, row_pairs="perm", out_pairs=None, keep=True, max_rows=None, h_rows=None):
        h = torch.full((self.N if h_rows is None else h_rows, self.d), 3.0, dtype=self.dt, device="cuda")
        u = torch.full((self.N, self.F), 3.0, dtype=self.dt, device="cuda") if keep else None
        self.ctx.moe_expert_ffn_mx4(self.x.cuda() if x is None else x, self.perm.cuda() if isinstance(row_pairs, str) else row_pairs, out_pairs,
                                    self.seg, self.seg_expert, self.N if max_rows is None else max_rows, self.g1, self.gb1, self.g2, self.gb2,
                                    u, h, self.ws)
        torch.cuda.synchronize()
        return u, h

    def check_forward(self, u, h):
        R = self.rows
        M.within(h[:R], self.ref[1], self.ref[3], "h")
        assert (h[R:] == 3.0).all()
        if u is not None:
            M.within(u[:R], self.ref[0], self.ref[2], "u")
            assert (u[R:] == 3.0).all()

    def backward(self, dh, u, keep=True, max_rows=None):
        du = torch.full((self.N, self.F), 3.0, dtype=self.dt, device="cuda") if keep else None
        dx = torch.full((self.N, self.d), 3.0, dtype=self.dt, device="cuda")
        self.ctx.moe_expert_ffn_mx4_backward(dh, u, self.seg, self.seg_expert, self.N if max_rows is None else max_rows, self.g1, self.g2, du, dx, self.ws)
        torch.cuda.synchronize()
        return du, dx

    def check_backward(self):
        R, n = self.rows, len(self.offsets) - 1
        dh = torch.randn((self.N, self.d), generator=self.gen).to(self.dt)
        u = (2.0 * torch.randn((self.N, self.F), generator=self.gen)).to(self.dt)
        du, dx = self.backward(dh.cuda(), u.cuda())
        raw, tol = M.times_weights(dh[:R].double(), self.offsets, range(n), self.v2, "f32")
        slope = M.gelu_slope(u[:R].double())
        want = raw * slope
        # the slope itself is off by 4e-6 at most (bf16; 4e-7 in float), and at most 1.13
        off = 1.13 * tol + (4e-6 if self.dtype == "bf16" else 4e-7) * (raw.abs() + tol)
        M.within(du[:R], want, off + M.HALF[self.dtype] * (want.abs() + off), "du")
        # dx is formed from du as it was stored: one product, one rounding
        back, tol = M.times_weights(du[:R].cpu().double(), self.offsets, range(n), self.v1, self.dtype)
        M.within(dx[:R], back, tol, "dx")
        assert (du[R:] == 3.0).all() and (dx[R:] == 3.0).all()
        alone = self.backward(dh.cuda(), u.cuda(), keep=False)[1]
        assert torch.equal(alone, dx)


# T, d, F, E, k, dtype, bias, drop, experts in use
CASES = [
    (1, 64, 256, 4, 2, "bf16", False, 0.0, None),                    # one token, one step of the reduction
    (1, 64, 64, 1, 1, "bf16", True, 0.0, None),
    (1, 1152, 4608, 8, 2, "bf16", True, 0.0, None),                  # one token at the DiT-MoE-XL widths
    (3, 192, 320, 4, 1, "bf16", True, 0.0, None),                    # reductions that end inside a step of 128
    (15, 64, 448, 3, 2, "bf16", True, 0.3, None),
    (17, 128, 256, 64, 3, "bf16", False, 0.0, None),                 # more experts than rows of some
    (33, 384, 1536, 16, 2, "bf16", True, 0.0, None),
    (64, 64, 256, 4, 2, "bf16", True, 1.0, None),                    # no pair left
    (100, 128, 192, 5, 2, "bf16", True, 0.2, [1, 3]),                # experts without a row
    (129, 320, 576, 4, 1, "bf16", True, 0.0, [2]),                   # all rows at one expert, one beyond a tile
    (300, 256, 512, 4, 2, "bf16", False, 0.1, None),
    (1000, 192, 384, 8, 4, "bf16", True, 0.0, None),
    (777, 384, 1536, 2, 2, "bf16", True, 0.0, None),
    (1, 32, 32, 1, 1, "f32", True, 0.0, None),
    (1, 64, 256, 4, 2, "f32", False, 0.0, None),
    (19, 96, 160, 4, 2, "f32", True, 0.2, None),
    (64, 64, 256, 4, 2, "f32", True, 0.0, None),
    (200, 384, 1536, 16, 2, "f32", True, 0.0, None),
    (333, 224, 288, 3, 3, "f32", True, 0.1, [0, 1, 2]),
    (500, 384, 1536, 16, 2, "f32", True, 0.1, None),                 # 64 columns a workgroup in the first product
    (1300, 1056, 288, 2, 1, "f32", True, 0.0, None),                 # ... in the second, whose last 64 are half there
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[:6])))
def test_forward(case):
    T, d, F, E, k, dtype, bias, drop, used = case
    say("forward", case)
    c = Case(T, d, F, E, k, dtype, bias, drop, used)
    u, h = c.forward()
    c.check_forward(u, h)
    assert torch.equal(c.forward(keep=False)[1], h)                  # without the pre-activations: the same rows
    xp = torch.zeros((c.N, d), dtype=c.dt)
    xp[:c.rows] = c.xp.to(c.dt)
    u2, h2 = c.forward(x=xp.cuda(), row_pairs=None)                  # packed rows instead of the gather
    assert torch.equal(u2, u) and torch.equal(h2, h)
    out = torch.arange(c.N, dtype=torch.int32).flip(0).cuda()        # rows scattered
    assert torch.equal(c.forward(out_pairs=out)[1].flip(0), h)
    c.ctx.moe_expert_ffn_status(c.ws)


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[:6])))
def test_backward(case):
    T, d, F, E, k, dtype, bias, drop, used = case
    say("backward", case)
    Case(T, d, F, E, k, dtype, bias, drop, used).check_backward()


def test_no_row():
    c = Case(0, 64, 256, 4, 2, "bf16")
    c.forward()
    c.ctx.moe_expert_ffn_status(c.ws)
    e = torch.empty((0, 64), dtype=c.dt, device="cuda")
    c.ctx.moe_expert_ffn_mx4_backward(e, torch.empty((0, 256), dtype=c.dt, device="cuda"), c.seg, c.seg_expert, 0, c.g1, c.g2, None, e, c.ws)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype,T", [("bf16", 40), ("bf16", 700), ("f32", 40)])
def test_rows_from_the_bound_on_are_left_alone(dtype, T):
    c = Case(T, 128, 256, 4, 2, dtype, bias=True)
    whole_u, whole_h = c.forward()
    bound = c.N // 2 + 3                                             # inside a tile of some segment
    u, h = c.forward(max_rows=bound)
    assert torch.equal(u[:bound], whole_u[:bound]) and torch.equal(h[:bound], whole_h[:bound])
    assert (u[bound:] == 3.0).all() and (h[bound:] == 3.0).all()
    with pytest.raises(B.MoeError) as e:
        c.ctx.moe_expert_ffn_status(c.ws)
    assert e.value.status == B.MOE_ERR_SHAPE
    dh, u = torch.ones_like(h), torch.ones_like(u)
    du, dx = c.backward(dh, u, max_rows=bound)
    assert (du[bound:] == 3.0).all() and (dx[bound:] == 3.0).all()
    full_du, full_dx = c.backward(dh, u)
    assert torch.equal(du[:bound], full_du[:bound]) and torch.equal(dx[:bound], full_dx[:bound])
    c.ctx.moe_expert_ffn_status(c.ws)


@pytest.mark.parametrize("W,E_loc", [(4, 4), (64, 16), (9, 8)])
def test_segments_of_a_receive_buffer(W, E_loc):
    """[source rank][local expert] segments, many of them empty, up to 1024."""
    say("segments", W, E_loc)
    T, d, F = 160, 128, 192
    gen = torch.Generator().manual_seed(W)
    counts = torch.zeros(W * E_loc, dtype=torch.int32)
    for i in torch.randint(0, W * E_loc, (T,), generator=gen).tolist():
        counts[i] += 1
    if W == 9:                                                       # the last segment, behind the first 64, holds most rows
        counts[:] = 0
        counts[3], counts[W * E_loc - 1] = 31, T - 31
    offsets = [0] + counts.cumsum(0).tolist()
    experts = [s % E_loc for s in range(W * E_loc)]
    c = Case(T, d, F, E_loc, 1, "bf16", bias=True, seed=W)
    c.seg, c.seg_expert = torch.tensor(offsets, dtype=torch.int32).cuda(), torch.tensor(experts, dtype=torch.int32).cuda()
    x = torch.randn((T, d), generator=gen).to(c.dt)
    ref = M.ffn(x.double(), offsets, experts, c.v1, c.b1.double(), c.v2, c.b2.double(), "bf16")
    u, h = c.forward(x=x.cuda(), row_pairs=None)
    M.within(u, ref[0], ref[2], "u")
    M.within(h, ref[1], ref[3], "h")
    dh = torch.randn((T, d), generator=gen).to(c.dt)
    du, dx = c.backward(dh.cuda(), u)
    back, tol = M.times_weights(du.cpu().double(), offsets, experts, c.v1, "bf16")
    M.within(dx, back, tol, "dx")


def test_segments_of_unknown_experts_have_no_rows():
    c = Case(40, 64, 128, 4, 1, "bf16")
    u, h = c.forward()
    c.seg_expert = torch.tensor([0, 4, -1, 3], dtype=torch.int32).cuda()
    u2, h2 = c.forward()
    o = c.offsets
    assert torch.equal(h2[:o[1]], h[:o[1]]) and torch.equal(h2[o[3]:o[4]], h[o[3]:o[4]])
    assert (h2[o[1]:o[3]] == 3.0).all() and (u2[o[1]:o[3]] == 3.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [5, 300])
def test_values_that_are_not_finite_stay_in_their_rows(dtype, T):
    c = Case(T, 128, 256, 2, 1, dtype, bias=True)
    u, h = c.forward()
    x = c.x.clone()
    x[2, 5], x[T - 1, 127] = float("nan"), float("inf")
    u2, h2 = c.forward(x=x.cuda())
    bad = torch.zeros(T, dtype=torch.bool)
    bad[[2, T - 1]] = True
    bad = bad[(c.perm // 1).long()]
    assert torch.equal(h2[~bad], h[~bad]) and torch.equal(u2[~bad], u[~bad])
    assert not torch.isfinite(u2[bad].float()).any(1).all() or torch.isnan(h2[bad].float()).any(1).all()
    assert torch.isnan(h2[bad].float()).all()                        # a NaN or infinite pre-activation reaches every column
    dh = torch.randn((T, 128), generator=c.gen).to(c.dt)
    ones = torch.ones((T, 256), dtype=c.dt)
    clean = c.backward(dh.cuda(), ones.cuda())
    dirty = ones.clone()
    dirty[3, 7] = float("nan")
    du, dx = c.backward(dh.cuda(), dirty.cuda())
    other = torch.arange(T) != 3
    assert torch.equal(dx[other], clean[1][other]) and torch.equal(du[other], clean[0][other])
    assert torch.isnan(du[3, 7]) and torch.isnan(dx[3].float()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [5, 300])
def test_slope_of_infinite_and_large_pre_activations(dtype, T):
    """gelu' is 1 at +infinity and 0 at -infinity; far out it is within the forms' 4e-6 of that."""
    c = Case(T, 128, 256, 1, 1, dtype)
    ends = torch.tensor([float("inf"), -float("inf"), 1e30, -1e30, 60.0, -60.0, 7.0, -7.0])
    u = ends[torch.randint(0, 8, (T, 256), generator=c.gen)].to(c.dt)
    dh = torch.randn((T, 128), generator=c.gen).to(c.dt)
    du, dx = c.backward(dh.cuda(), u.cuda())
    raw, tol = M.times_weights(dh.double(), c.offsets, range(1), c.v2, "f32")
    want = raw * (u > 0)
    off = tol + 4e-6 * (raw.abs() + tol)
    M.within(du, want, off + M.HALF[dtype] * (want.abs() + off), "du")
    assert torch.isfinite(dx.float()).all()


def test_scale_byte_255_is_nan_and_its_column_alone():
    c = Case(6, 128, 256, 2, 1, "bf16")
    u, _ = c.forward()
    c.g1[1][0, 9, 1] = 255                                           # expert 0, hidden column 9
    u2, h2 = c.forward()
    mine = slice(0, c.offsets[1])
    assert torch.isnan(u2[mine, 9].float()).all() and torch.isnan(h2[mine].float()).all()
    keep = torch.arange(256) != 9
    assert torch.equal(u2[:, keep], u[:, keep]) and torch.equal(u2[c.offsets[1]:], u[c.offsets[1]:])


def test_large_activations_reach_infinity_without_nan():
    """Magnitudes near the end of bf16: sums overflow to infinity or stay, GELU of a large negative number is zero."""
    c = Case(4, 64, 128, 1, 1, "bf16")
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    x[:, 0] = torch.tensor([1e30, -1e30, 3e38, -3e38])
    u, h = c.forward(x=x.cuda())
    want = x[(c.perm // 1).long()].double() @ c.v1[0].T
    got = u.cpu().double()
    fits = want.abs() < 3.3e38
    assert ((got - want).abs() <= 2.0 ** -7 * want.abs())[fits].all()
    assert not torch.isnan(h.float()).any() or torch.isinf(u.float()).any()


@pytest.mark.parametrize("dtype,T", [("bf16", 1), ("bf16", 50), ("bf16", 600), ("f32", 50)])
def test_graph_replays_and_streams(dtype, T):
    say("graph", dtype, T)
    c = Case(T, 192, 448, 4, 2, dtype, bias=True)
    x, perm = c.x.cuda(), c.perm.cuda()
    h, u = torch.zeros((c.N, c.d), dtype=c.dt, device="cuda"), torch.zeros((c.N, c.F), dtype=c.dt, device="cuda")
    dx = torch.zeros_like(h)

    def both():
        c.ctx.moe_expert_ffn_mx4(x, perm, None, c.seg, c.seg_expert, c.N, c.g1, c.gb1, c.g2, c.gb2, u, h, c.ws)
        c.ctx.moe_expert_ffn_mx4_backward(h, u, c.seg, c.seg_expert, c.N, c.g1, c.g2, None, dx, c.ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for turn in range(3):
        x.copy_(torch.randn((T, c.d), generator=c.gen).to(c.dt))
        both()
        torch.cuda.synchronize()
        want = [t.clone() for t in (u, h, dx)]
        for t in (u, h, dx):
            t.fill_(9.0)
        c.ws.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((u, h, dx), want)), turn


def test_two_workspaces_on_two_streams():
    """Two calls at once, each with its own workspace, give what they give alone."""
    a, b = Case(200, 256, 512, 4, 2, "bf16", bias=True), Case(210, 256, 512, 4, 2, "bf16", bias=True, seed=1)
    alone = [c.forward()[1] for c in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.zeros_like(h) for h in alone]
    xs, perms = [c.x.cuda() for c in (a, b)], [c.perm.cuda() for c in (a, b)]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, s, o, x, p in zip((a, b), streams, outs, xs, perms):
            with torch.cuda.stream(s):
                c.ctx.moe_expert_ffn_mx4(x, p, None, c.seg, c.seg_expert, c.N, c.g1, c.gb1, c.g2, c.gb2, None, o, c.ws)
    torch.cuda.synchronize()
    for c, o, h in zip((a, b), outs, alone):
        assert torch.equal(o[:c.rows], h[:c.rows])


def test_cached_layer_takes_the_rows():
    """moe_route, the 4-bit FFN scattering into the cache, and moe_combine reading it: the synchronous layer of Conditional
    Communication, two steps, against the same layer with packed rows."""
    T, d, F, E, k = 130, 128, 256, 4, 2
    c = Case(T, d, F, E, k, "bf16", bias=True)
    gen = c.gen
    Wg = (torch.randn((E, d), generator=gen) / d ** 0.5).to(c.dt).cuda()
    ys = []
    for scatter in (True, False):
        buf = B.LayerBuffers(c.ctx, "cuda", with_cache=True)
        y = []
        for step, policy in enumerate((B.Policy(B.REFRESH_ALL), B.Policy(B.REFRESH_ALG4, step_t=1, stride_n=2))):
            x = (c.x.float() + 0.1 * step * torch.randn((T, d), generator=torch.Generator().manual_seed(step))).to(c.dt).cuda()
            c.ctx.moe_route(x, Wg, None, policy, buf.scores, buf.expert_idx, buf.mask, buf.n_refresh, None, buf.counts, buf.offsets, buf.perm,
                            buf.inv, buf.workspace)
            rows, _ = c.ctx.moe_policy_refreshed_pairs(policy, T)
            h = buf.H_cache.view(T * k, d) if scatter else buf.h_packed
            c.ctx.moe_expert_ffn_mx4(x, buf.perm, buf.perm if scatter else None, buf.offsets, buf.seg_expert, rows, c.g1, c.gb1, c.g2, c.gb2,
                                     None, h, buf.workspace)
            c.ctx.moe_expert_ffn_status(buf.workspace)
            c.ctx.moe_combine(None if scatter else h, buf.inv, buf.scores, buf.mask, buf.H_cache, buf.S_cache, False, buf.y)
            y.append(buf.y.clone())
        ys.append(y)
    assert all(torch.equal(a, b) for a, b in zip(*ys))
    assert torch.isfinite(ys[0][1].float()).all() and not torch.equal(ys[0][0], ys[0][1])
