"""Gradients of combine, router and dispatch on the GPU against double precision, and the whole backward pass of a layer with 4-bit
experts against differentiation of a plain layer and against differences."""
import pytest
import torch

import mx4_util as M
from paper_2411_16786_amd import binding as B

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, flush=True)


SHAPES = [
    # T, d, E, k, n_shared, dtype, drop
    (1, 64, 1, 1, 0, "bf16", 0.0),
    (1, 16, 1, 1, 0, "f32", 0.0),
    (1, 1152, 8, 2, 0, "bf16", 0.0),
    (15, 64, 4, 2, 0, "bf16", 0.3),
    (16, 192, 16, 3, 0, "bf16", 0.0),
    (17, 320, 17, 4, 1, "bf16", 0.2),
    (63, 48, 5, 2, 0, "f32", 0.1),
    (65, 80, 33, 6, 2, "f32", 0.2),
    (64, 64, 4, 2, 0, "bf16", 1.0),
    (130, 576, 64, 5, 0, "bf16", 0.0),
    (257, 384, 16, 2, 0, "bf16", 0.1),
    (1000, 128, 8, 2, 2, "bf16", 0.1),
    (3001, 64, 60, 2, 0, "bf16", 0.0),
    (2500, 32, 40, 1, 0, "f32", 0.1),
    (9000, 64, 4, 2, 0, "bf16", 0.0),
    (4200, 2048, 16, 2, 0, "bf16", 0.1),                             # several tiles of tokens per wavefront
    (4133, 2048, 40, 1, 0, "bf16", 0.0),
    (2100, 1024, 8, 6, 1, "f32", 0.1),
    (513, 1152, 8, 2, 0, "bf16", 0.0),
]
IDS = ["-".join(map(str, s)) for s in SHAPES]


@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
def test_combine_backward(shape):
    T, d, E, k, ns, dtype, drop = shape
    say("combine_backward", shape)
    gen = torch.Generator().manual_seed(T + d)
    slots, dt = k + ns, M.DT[dtype]
    _, live, _, perm, inv, R = M.route(gen, T, E + ns, slots, drop)
    dy, h = torch.randn((T, d), generator=gen).to(dt), torch.randn((T * slots, d), generator=gen).to(dt)
    s = torch.rand((T, slots), generator=gen)
    ctx = B.Context(T, d, 64, E, k, dtype, n_shared=ns)
    h[R:] = float("nan")                                             # rows that no pair has are not read
    dh = torch.full((T * slots, d), 3.0, dtype=dt, device="cuda")
    ds = torch.full((T, slots), 3.0, device="cuda")
    ctx.moe_combine_backward(dy.cuda(), h.cuda(), inv.cuda(), s.cuda(), dh, ds)
    pair = perm[:R].long()
    want = s.flatten()[pair].double()[:, None] * dy[pair // slots].double()
    M.within(dh[:R], want, M.HALF[dtype] * want.abs() * (1 + 1e-6) + 2.0 ** -24 * want.abs() + 1e-38, "dh")
    assert (dh[R:] == 3.0).all()
    prod = h[:R].double() * dy[pair // slots].double()
    dots, tol = torch.zeros(T * slots, dtype=torch.float64), torch.zeros(T * slots, dtype=torch.float64)
    dots[pair], tol[pair] = prod.sum(1), (d + 2) * 2.0 ** -24 * prod.abs().sum(1)
    M.within(ds.flatten(), dots, tol + 1e-38, "dscores")
    assert (ds.flatten()[inv.cuda() < 0] == 0).all()


class Route:
    def __init__(self, shape, renorm, aux, seed=0):
        T, d, E, k, ns, dtype, drop = shape
        gen = self.gen = torch.Generator().manual_seed(T + d + seed)
        self.shape, self.renorm, self.dt, slots = shape, renorm, M.DT[dtype], k + ns
        z = torch.randn((T, E), generator=gen)
        self.probs = torch.softmax(z, 1)
        top = torch.topk(z, k, 1).indices
        shared = torch.arange(E, E + ns).expand(T, ns)
        self.idx = torch.cat([top, shared], 1).to(torch.int32).contiguous()
        _, _, _, self.perm, self.inv, self.R = M.route(gen, T, E + ns, slots, drop)
        self.x, self.Wg = (torch.randn(s, generator=gen).to(self.dt) for s in ((T, d), (E, d)))
        self.dxp = torch.randn((T * slots, d), generator=gen).to(self.dt)
        self.dxp[self.R:] = float("nan")
        self.ds = torch.randn((T, slots), generator=gen)
        self.ds[:, k:] = float("nan")                                # the shared slots' scores are constants
        self.dP = torch.randn((T, E), generator=gen) if aux else None
        self.dL = torch.randn((T, E), generator=gen) if aux else None
        self.ctx = B.Context(T, d, 64, E, k, dtype, renorm_topk=renorm, n_shared=ns)
        self.ws = torch.empty(self.ctx.workspace_bytes(), dtype=torch.uint8, device="cuda")

    def run(self, rows=True, want=("dz", "dWg", "dbg")):
        T, d, E = self.shape[:3]
        new = lambda name, *s: torch.full(s, 3.0, device="cuda") if name in want else None
        self.dx = torch.full((T, d), 3.0, dtype=self.dt, device="cuda")
        self.dz, self.dWg, self.dbg = new("dz", T, E), new("dWg", E, d), new("dbg", E)
        c = lambda t: None if t is None else t.cuda()
        self.ctx.moe_route_backward(c(self.x), c(self.Wg), c(self.idx), c(self.probs), c(self.ds), c(self.dP), c(self.dL),
                                    c(self.dxp) if rows else None, c(self.inv) if rows else None, self.dx, self.dz, self.dWg, self.dbg, self.ws)
        torch.cuda.synchronize()

    def expected_dz(self):
        """By the formula, in double, and a bound: magnitudes summed, 2^-24 for each of the few operations."""
        T, d, E, k = self.shape[:4]
        P, idx, ds = self.probs.double(), self.idx[:, :k].long(), self.ds[:, :k].double()
        g = torch.zeros_like(P) if self.dP is None else self.dP.double()
        size = g.abs()
        if self.renorm:
            p = torch.gather(P, 1, idx)
            total = p.sum(1, keepdim=True)
            mean = (ds * p).sum(1, keepdim=True) / total
            add, mag = (ds - mean) / total, (ds.abs() + (ds.abs() * p).sum(1, keepdim=True) / total) / total
        else:
            add, mag = ds, ds.abs()
        g, size = g.scatter_add(1, idx, add), size.scatter_add(1, idx, mag)
        dz = P * (g - (P * g).sum(1, keepdim=True))
        mag = P * (size + (P * size).sum(1, keepdim=True))
        if self.dL is not None:
            dz, mag = dz + self.dL.double(), mag + self.dL.double().abs()
        return dz, (E + 3 * k + 8) * 2.0 ** -24 * mag + 1e-38

    def expected_rows(self, rows):
        """(sum of the dispatch's rows, sum of magnitudes)."""
        T, d, E, k, ns = self.shape[:5]
        out, mag = torch.zeros((T, d), dtype=torch.float64), torch.zeros((T, d), dtype=torch.float64)
        if rows:
            inv = self.inv.reshape(T, k + ns).long()
            for j in range(k + ns):
                t = (inv[:, j] >= 0).nonzero().flatten()
                v = self.dxp[inv[t, j]].double()
                out[t] += v
                mag[t] += v.abs()
        return out, mag

    def check(self, rows=True):
        T, d, E, k, ns, dtype = self.shape[:6]
        dz, tol = self.expected_dz()
        if self.dz is not None:
            M.within(self.dz, dz, tol, "dz")
        W, x = self.Wg.double(), self.x.double()
        want, mag = self.expected_rows(rows)
        want, mag = want + dz @ W, mag + dz.abs() @ W.abs()
        off = (E + k + ns + 2) * 2.0 ** -23 * mag + tol @ W.abs()
        M.within(self.dx, want, off + M.HALF[dtype] * (want.abs() + off) + 1e-38, "dx")
        if self.dWg is not None:
            off = (T + 8) * 2.0 ** -23 * (dz.abs().T @ x.abs()) + tol.T @ x.abs()
            M.within(self.dWg, dz.T @ x, off + 1e-38, "dWg")
        if self.dbg is not None:
            M.within(self.dbg, dz.sum(0), (T + 8) * 2.0 ** -24 * dz.abs().sum(0) + tol.sum(0), "dbg")


@pytest.mark.parametrize("renorm,aux", [(False, False), (True, True), (False, True)])
@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
def test_route_backward(shape, renorm, aux):
    say("route_backward", shape, renorm, aux)
    r = Route(shape, renorm, aux)
    r.run()
    r.check()


@pytest.mark.parametrize("shape", [SHAPES[5], SHAPES[7], SHAPES[10], SHAPES[14]], ids=lambda s: "-".join(map(str, s)))
def test_route_backward_in_parts(shape):
    """Without the dispatch's rows, and without outputs that nobody wants."""
    r = Route(shape, True, False)
    r.run(rows=False)
    r.check(rows=False)
    whole = (r.dx.clone(), r.dz.clone(), r.dWg.clone(), r.dbg.clone())
    r.run(rows=False, want=())
    assert torch.equal(r.dx, whole[0])
    r.run(rows=False, want=("dbg",))
    assert torch.equal(r.dbg, whole[3]) and torch.equal(r.dx, whole[0])
    r.run(rows=False, want=("dWg",))
    assert torch.equal(r.dWg, whole[2])


@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
def test_dispatch_backward_alone(shape):
    T, d, E, k, ns, dtype, _ = shape
    r = Route(shape, False, False)
    dx = torch.full((T, d), 3.0, dtype=r.dt, device="cuda")
    r.ctx.moe_route_backward(None, None, None, None, None, None, None, r.dxp.cuda(), r.inv.cuda(), dx, None, None, None, None)
    want, mag = r.expected_rows(True)
    off = (k + ns) * 2.0 ** -24 * mag
    M.within(dx, want, off + M.HALF[dtype] * (want.abs() + off) + 1e-38, "dx")


def test_no_token():
    ctx = B.Context(4, 64, 64, 4, 2, "bf16")
    ws = torch.empty(ctx.workspace_bytes(), dtype=torch.uint8, device="cuda")
    e = lambda *s, dt=torch.float32: torch.empty(s, dtype=dt, device="cuda")
    bf, i32 = torch.bfloat16, torch.int32
    Wg, dWg, dbg = torch.ones((4, 64), dtype=bf, device="cuda"), torch.full((4, 64), 3.0, device="cuda"), torch.full((4,), 3.0, device="cuda")
    ctx.moe_route_backward(e(0, 64, dt=bf), Wg, e(0, 2, dt=i32), e(0, 4), e(0, 2), None, None, e(0, 64, dt=bf), e(0, dt=i32), e(0, 64, dt=bf), e(0, 4),
                           dWg, dbg, ws)
    assert (dWg == 0).all() and (dbg == 0).all()
    ctx.moe_combine_backward(e(0, 64, dt=bf), e(0, 64, dt=bf), e(0, dt=i32), e(0, 2), e(0, 64, dt=bf), e(0, 2))
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_not_a_number_stays_with_its_token(dtype):
    shape = (70, 64, 6, 2, 0, dtype, 0.0)
    r = Route(shape, False, False)
    r.run()
    clean = (r.dx.clone(), r.dz.clone())
    r.ds[5, 1] = float("nan")
    r.run()
    other = torch.arange(70) != 5
    assert torch.equal(r.dx[other], clean[0][other]) and torch.equal(r.dz[other], clean[1][other])
    assert torch.isnan(r.dz[5]).all() and torch.isnan(r.dx[5].float()).all() and torch.isnan(r.dWg).all() and torch.isnan(r.dbg).all()


# ---- the pass as a whole

def _plain_layer(x, Wg, bg, v1, b1, v2, b2, idx, renorm):
    """y of a layer with the selection given, double, differentiable."""
    T, k = idx.shape
    P = torch.softmax(x @ Wg.T + bg, 1)
    s = torch.gather(P, 1, idx)
    if renorm:
        s = s / s.sum(1, keepdim=True)
    y = torch.zeros_like(x)
    for e in range(Wg.shape[0]):
        t, j = (idx == e).nonzero(as_tuple=True)
        h = M.gelu(x[t] @ v1[e].T + b1[e]) @ v2[e].T + b2[e]
        y = y.index_add(0, t, s[t, j][:, None] * h)
    return y


class Layer:
    """Forward and backward pass of a layer with 4-bit experts through the public calls."""

    def __init__(self, T, d, F, E, k, dtype, renorm, seed=0):
        gen = self.gen = torch.Generator().manual_seed(seed)
        self.dt, self.renorm = M.DT[dtype], renorm
        self.T, self.d, self.F, self.E, self.k = T, d, F, E, k
        self.ctx = B.Context(T, d, F, E, k, dtype, renorm_topk=renorm)
        self.buf = B.LayerBuffers(self.ctx, "cuda", with_debug=True)
        w1, w2 = (torch.randn(s, generator=gen) * 0.1 for s in ((E, F, d), (E, d, F)))
        self.W1 = self.quantized(w1)
        self.W2 = self.quantized(w2)
        self.b1, self.b2 = torch.randn((E, F), generator=gen) * 0.1, torch.randn((E, d), generator=gen) * 0.1
        self.Wg = (torch.randn((E, d), generator=gen) / d ** 0.5).to(self.dt)
        self.bg = torch.randn(E, generator=gen) * 0.3
        self.x = torch.randn((T, d), generator=gen).to(self.dt)
        self.dy = torch.randn((T, d), generator=gen).to(self.dt)
        g = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt, device="cuda")
        N = T * k
        self.u, self.dh, self.dxp = g(N, F, dt=self.dt), g(N, d, dt=self.dt), g(N, d, dt=self.dt)
        self.ds, self.dx, self.dz, self.dWg, self.dbg = g(T, k), g(T, d, dt=self.dt), g(T, E), g(E, d), g(E)
        self.on = {n: getattr(self, n).cuda() for n in ("b1", "b2", "Wg", "bg", "x", "dy")}

    def quantized(self, w):
        codes = torch.empty(w.shape[:-1] + (w.shape[-1] // 2,), dtype=torch.uint8, device="cuda")
        scales = torch.empty(w.shape[:-1] + (w.shape[-1] // 32,), dtype=torch.uint8, device="cuda")
        self.ctx.moe_quantize_mx4(w.to(self.dt).cuda(), codes, scales)
        return codes, scales

    def step(self):
        o, b, c = self.on, self.buf, self.ctx
        c.moe_route(o["x"], o["Wg"], o["bg"], None, b.scores, b.expert_idx, None, None, None, b.counts, b.offsets, b.perm, b.inv, b.workspace,
                    probs_all=b.probs)
        N = self.T * self.k
        c.moe_expert_ffn_mx4(o["x"], b.perm, None, b.offsets, b.seg_expert, N, self.W1, o["b1"], self.W2, o["b2"], self.u, b.h_packed, b.workspace)
        c.moe_combine(b.h_packed, b.inv, b.scores, None, None, None, False, b.y)
        c.moe_combine_backward(o["dy"], b.h_packed, b.inv, b.scores, self.dh, self.ds)
        c.moe_expert_ffn_mx4_backward(self.dh, self.u, b.offsets, b.seg_expert, N, self.W1, self.W2, None, self.dxp, b.workspace)
        c.moe_route_backward(o["x"], o["Wg"], b.expert_idx, b.probs, self.ds, None, None, self.dxp, b.inv, self.dx, self.dz, self.dWg, self.dbg, b.workspace)
        return b.y, self.dx, self.dz, self.dWg, self.dbg

    def plain(self):
        return [t.double() for t in (self.x, self.Wg, self.bg)], [M.decode(*self.W1), self.b1.double(), M.decode(*self.W2), self.b2.double(),
                                                                   self.buf.expert_idx.cpu().long(), self.renorm]


@pytest.mark.parametrize("dtype,renorm,T", [("f32", False, 37), ("f32", True, 37), ("bf16", False, 300), ("bf16", True, 5)])
def test_whole_pass_against_the_plain_layer(dtype, renorm, T):
    say("whole pass", dtype, renorm, T)
    L = Layer(T, 64, 128, 5, 2, dtype, renorm)
    y, dx, dz, dWg, dbg = L.step()
    leaves, rest = L.plain()
    leaves = [t.requires_grad_() for t in leaves]
    want = _plain_layer(*leaves, *rest)
    grads = torch.autograd.grad(want, leaves, L.dy.double())
    want = want.detach()
    # Every stored intermediate (u, gelu(u), h, dh, du, dx_packed) is rounded once: 8 roundings in a row, each 2^-8 relative in bf16
    # of its own row's size, and float sums of up to 128 terms: 8 + 128 2^-16 halves of a step, of the norm of the result in float64.
    tol = 8 * M.HALF["bf16"] if dtype == "bf16" else 128 * 2.0 ** -23
    for name, got, ref in (("y", y, want), ("dx", dx, grads[0]), ("dWg", dWg, grads[1]), ("dbg", dbg, grads[2])):
        err = float((got.cpu().double() - ref).norm() / ref.norm())
        say(name, f"{err:.2e} of {tol:.2e}")
        assert err <= tol, (name, err, tol)


def test_whole_pass_against_differences():
    """Directional differences of the double-precision layer: h^2 error of the central difference, h = 1e-5."""
    L = Layer(29, 64, 128, 5, 2, "f32", True, seed=3)
    _, dx, _, dWg, dbg = L.step()
    leaves, rest = L.plain()
    dy = L.dy.double()
    for i, got in enumerate((dx, dWg, dbg)):
        for seed in range(3):
            way = torch.randn(leaves[i].shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)
            ends = []
            for sign in (1, -1):
                moved = list(leaves)
                moved[i] = leaves[i] + sign * 1e-5 * way
                ends.append((_plain_layer(*moved, *rest) * dy).sum())
            slope = float((ends[0] - ends[1]) / 2e-5)
            mine = float((got.cpu().double() * way).sum())
            size = float(got.cpu().double().norm() * way.norm())
            assert abs(slope - mine) <= 1e-5 * size, (i, slope, mine, size)


@pytest.mark.parametrize("T", [7, 500])
def test_whole_pass_captured(T):
    """The pass in one graph, replayed with other inputs and the program's own work in between."""
    L = Layer(T, 128, 256, 6, 2, "bf16", False)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        L.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = L.step()
    for turn in range(4):
        L.on["x"].copy_(torch.randn((T, 128), generator=L.gen).to(L.dt))
        L.on["dy"].copy_(torch.randn((T, 128), generator=L.gen).to(L.dt))
        L.step()
        torch.cuda.synchronize()
        want = [t.clone() for t in outs]
        for t in outs:
            t.fill_(9.0)
        L.buf.workspace.fill_(turn)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), turn


def test_side_stream():
    """A call goes to the current stream: on a side stream it waits for that stream's work alone."""
    L = Layer(64, 128, 256, 4, 2, "bf16", False)
    want = [t.clone() for t in L.step()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for t in (L.dx, L.dWg, L.buf.y):
            t.zero_()
        got = L.step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
