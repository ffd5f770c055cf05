"""Cases of the operators around a MoE layer with 4-bit experts and of the layer's gradients.

Five operators, each through its public entry point (``binding.Context``):

* ``quantize``     weights to 4-bit codes with a power-of-two scale per 32 columns (MXFP4), and the values they stand for
* ``ffn``          the grouped expert FFN on such weights, W1 -> GELU -> W2, rows read by token through the dispatch's order
* ``ffn_bwd``      its gradient with respect to the rows, through the frozen weights
* ``combine_bwd``  gradient of the weighted sum over a token's experts: rows and scores
* ``route_bwd``    gradient of router and dispatch: tokens, router weight and bias

``own`` False computes them with elementary torch operations, True calls the framework.  Inputs are the same either way.
Widths are those of ``workloads.CONFIGS``; activations are N(0, 1), expert weights N(0, 0.02), router rows N(0, 1/sqrt(d)), the
expert load is uniform or Zipf.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
GROUP = 32                                    # columns that share a scale

# (d, F, E): tiny, DiT-MoE-S, DiT-MoE-XL, DiT-MoE-G, expert-parallel widths
TINY, SMALL, XL, G, EP = (64, 256, 4), (384, 1536, 16), (1152, 4608, 8), (1792, 7168, 16), (2048, 8192, 16)

MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)       # what codes 0..7 stand for; bit 3 is the sign


def _case(kind, widths, T=0, name=None, dtype="bf16", k=2, bias=False, zipf=False, renorm=False, keep=False, drop=0.0, aux=False):
    d, F, E = widths
    case = dict(kind=kind, T=T, d=d, F=F, E=E, k=k, dtype=dtype, bias=bias, zipf=zipf, renorm=renorm, keep=keep, drop=drop, aux=aux)
    if name is not None:
        case["name"] = name
    return case


def listed():
    return [
        # loading a DiT-MoE-XL layer in 4 bits: one of its two weight arrays
        _case("quantize", XL, name="quantize-xl"),
        # a DiT-MoE-S layer from float weights
        _case("quantize", SMALL, name="quantize-s-f32", dtype="f32"),
        # serving one token: launches and the weights of two experts
        _case("ffn", XL, 1, "ffn-xl-1"),
        # a few tokens under an uneven load at the expert-parallel widths: the weights of most experts are the traffic
        _case("ffn", EP, 13, "ffn-ep-13-zipf", zipf=True),
        # a small ragged batch in training: biases, the pre-activations kept for the backward pass
        _case("ffn", XL, 1000, "ffn-xl-1000-bias-keep", bias=True, keep=True),
        # the headline layer's batch: 16 x 256 tokens
        _case("ffn", XL, 4096, "ffn-xl-4096"),
        # gradient in float at the DiT-MoE-S widths: validating a model
        _case("ffn_bwd", SMALL, 500, "ffn-bwd-s-f32-500", dtype="f32", bias=True, keep=True),
        # gradient of the headline batch through frozen experts
        _case("ffn_bwd", XL, 4096, "ffn-bwd-xl-4096"),
        # the smallest gradient: one 8x8 latent in float
        _case("combine_bwd", TINY, 64, "combine-bwd-tiny-f32-64", dtype="f32"),
        # a 512px batch at the expert-parallel widths, Zipf load
        _case("combine_bwd", EP, 8192, "combine-bwd-ep-8192", zipf=True),
        # router of DiT-MoE-S over an odd batch, scores renormalised, a tenth of the pairs dropped, a loss on the probabilities
        _case("route_bwd", SMALL, 1019, "route-bwd-s-1019-renorm-drop", renorm=True, drop=0.1, aux=True),
        # the 512px batch
        _case("route_bwd", EP, 8192, "route-bwd-ep-8192", zipf=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MAX_FLOPS = 4.0 * 8192 * 1152 * 4608          # the largest listed case


def draw(rng):
    while True:
        kind = rng.choice(["quantize", "ffn", "ffn", "ffn", "ffn_bwd", "ffn_bwd", "combine_bwd", "route_bwd"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        widths = rng.choice([TINY, SMALL, XL, XL, G, EP] if dtype == "bf16" else [TINY, SMALL, XL])
        k = rng.choice([1, 2, 2, 2, 3, 4])
        zipf, bias, keep = rng.random() < 0.4, rng.random() < 0.3, rng.random() < 0.3
        if kind == "quantize":
            case = _case("quantize", widths, dtype=dtype)
        elif kind in ("ffn", "ffn_bwd"):
            T = _log_int(rng, 1, 4096 if dtype == "bf16" else 512)
            case = _case(kind, widths, T, dtype=dtype, k=k, bias=bias, zipf=zipf, keep=keep)
        elif kind == "combine_bwd":
            case = _case(kind, widths, _log_int(rng, 1, 8192), dtype=dtype, k=k, zipf=zipf, drop=rng.choice([0.0, 0.0, 0.1, 0.5]))
        else:
            case = _case(kind, widths, _log_int(rng, 1, 8192), dtype=dtype, k=k, zipf=zipf, renorm=rng.random() < 0.5,
                         drop=rng.choice([0.0, 0.0, 0.1, 0.5]), aux=rng.random() < 0.5, bias=bias)
        w = work(case)
        if w["flops"] <= MAX_FLOPS and w["bytes"] <= 6e8:
            return case


def _touched(case):
    """Experts that a uniform choice of T * k pairs is expected to reach."""
    return case["E"] * (1.0 - (1.0 - case["k"] / case["E"]) ** case["T"])


def work(case):
    """Each input read once and each output written once (the hidden activations of the FFN are neither)."""
    T, d, F, E, k, kind = (case[n] for n in ("T", "d", "F", "E", "k", "kind"))
    b = 2 if case["dtype"] == "bf16" else 4
    R = T * k
    if kind == "quantize":
        n = E * F * d
        return {"bytes": 2 * n * b + n / 2 + n / GROUP, "flops": 4.0 * n}
    weights = 2 * _touched(case) * d * F * (0.5 + 1.0 / GROUP)
    if kind == "ffn":
        return {"bytes": weights + min(T, R) * d * b + R * d * b + (R * F * b if case["keep"] else 0), "flops": 4.0 * R * d * F}
    if kind == "ffn_bwd":
        return {"bytes": weights + 2 * R * d * b + R * F * b * (2 if case["keep"] else 1), "flops": 4.0 * R * d * F}
    live = int(round(R * (1.0 - case["drop"])))
    if kind == "combine_bwd":
        return {"bytes": T * d * b + 2 * live * d * b + 12 * R, "flops": 3.0 * live * d}
    return {"bytes": live * d * b + 2 * T * d * b + E * d * (b + 4) + T * E * 4 * (3 if case["aux"] else 2) + 12 * R,
            "flops": 4.0 * T * E * d + live * d}


# ---- inputs

def _normal(gen, shape, std, dtype):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).mul_(std).to(dtype)


def _quantized(w):
    """Codes [rows, cols / 2] (column 2c in the low half of byte c) and scale bytes [rows, cols / 32] of float w: a group's scale
    is the smallest power of two, 2^-126 or more, of which its largest magnitude is at most 7 (what rounds to the code of 6 with the error
    of half a step); byte 127 + exponent.  Codes are nearest, ties to the even code."""
    rows, cols = w.shape
    g = w.float().reshape(rows, cols // GROUP, GROUP)
    mantissa, exponent = torch.frexp(g.abs().amax(-1))
    scale = torch.clamp(exponent - torch.where(mantissa <= 0.875, 3, 2) + 127, min=1)
    v = torch.ldexp(g.abs(), (127 - scale)[..., None])
    code = ((v > 0.25).to(torch.uint8) + (v >= 0.75) + (v > 1.25) + (v >= 1.75) + (v > 2.5) + (v >= 3.5) + (v > 5.0)).to(torch.uint8)
    code = (code | (torch.signbit(g).to(torch.uint8) << 3)).reshape(rows, cols // 2, 2)
    return (code[..., 0] | (code[..., 1] << 4)).contiguous(), scale.to(torch.uint8).contiguous()


def _expert_codes(gen, E, rows, cols):
    codes = torch.empty((E, rows, cols // 2), dtype=torch.uint8, device=DEV)
    scales = torch.empty((E, rows, cols // GROUP), dtype=torch.uint8, device=DEV)
    for e in range(E):
        codes[e], scales[e] = _quantized(_normal(gen, (rows, cols), 0.02, torch.float32))
    return codes, scales


def _routing(case, gen):
    """What router and dispatch leave: probabilities, selected experts, scores, and the order of the pairs by expert."""
    T, E, k = case["T"], case["E"], case["k"]
    z = torch.randn((T, E), generator=gen, device=DEV)
    if case["zipf"]:
        z = z - 1.2 * torch.log(torch.arange(1, E + 1, device=DEV, dtype=torch.float32))
    probs = torch.softmax(z, 1)
    top = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :k]
    scores = torch.gather(probs, 1, top)
    if case["renorm"]:
        scores = scores / scores.sum(1, keepdim=True)
    live = torch.rand((T, k), generator=gen, device=DEV) >= case["drop"]
    expert = torch.where(live, top, E).flatten()              # dropped pairs sort behind the last expert
    order = torch.sort(expert, stable=True).indices
    rows = int(live.sum())
    perm = torch.where(torch.arange(T * k, device=DEV) < rows, order, -1)
    inv = torch.full((T * k,), -1, dtype=torch.int64, device=DEV)
    inv[order[:rows]] = torch.arange(rows, device=DEV)
    counts = torch.bincount(expert, minlength=E + 1)[:E]
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), counts.cumsum(0)])
    i32 = lambda t: t.to(torch.int32).contiguous()
    return dict(probs=probs.contiguous(), idx=i32(top), scores=scores.contiguous(), perm=i32(perm), inv=i32(inv),
                offsets=i32(offsets), rows=rows, ends=offsets.tolist())


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    T, d, F, E, k, kind = (case[n] for n in ("T", "d", "F", "E", "k", "kind"))
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    s = {"case": case, "dt": dt}
    if kind == "quantize":
        s["W"] = torch.cat([_normal(gen, (1, F, d), 0.02, dt) for _ in range(E)])
    else:
        s.update(_routing(case, gen))
        N = T * k
        if kind in ("ffn", "ffn_bwd"):
            s["W1"], s["W2"] = _expert_codes(gen, E, F, d), _expert_codes(gen, E, d, F)
            if kind == "ffn":
                s["x"] = _normal(gen, (T, d), 1.0, dt)
                s["b1"] = _normal(gen, (E, F), 0.1, torch.float32) if case["bias"] else None
                s["b2"] = _normal(gen, (E, d), 0.1, torch.float32) if case["bias"] else None
            else:
                s["dh"] = _normal(gen, (N, d), 1e-2, dt)
                s["u"] = _normal(gen, (N, F), 0.7, dt)        # pre-activations as N(0, 1) rows through N(0, 0.02) weights give them
        elif kind == "combine_bwd":
            s["dy"] = _normal(gen, (T, d), 1e-2, dt)
            s["h"] = _normal(gen, (N, d), 0.5, dt)
        else:
            s["x"] = _normal(gen, (T, d), 1.0, dt)
            s["Wg"] = _normal(gen, (E, d), 1.0 / math.sqrt(d), dt)
            s["dxp"] = _normal(gen, (N, d), 1e-2, dt)
            s["dscores"] = _normal(gen, (T, k), 0.3, torch.float32)
            s["dprobs"] = _normal(gen, (T, E), 0.01, torch.float32) if case["aux"] else None
            s["dlogits"] = _normal(gen, (T, E), 0.01, torch.float32) if case["aux"] else None
    if own:
        _own_state(s)
    return s


def _own_state(s):
    """The context, the buffers and the workspace that a program keeps."""
    from paper_2411_16786_amd import binding as B
    case, dt = s["case"], s["dt"]
    T, d, F, E, k, kind = (case[n] for n in ("T", "d", "F", "E", "k", "kind"))
    ctx = s["ctx"] = B.Context(max(T, 1), d, F, E, k, case["dtype"], renorm_topk=case["renorm"])
    new = lambda shape, dtype=dt: torch.empty(shape, dtype=dtype, device=DEV)
    N = T * k
    if kind == "quantize":
        s["codes"], s["scales"] = new((E, F, d // 2), torch.uint8), new((E, F, d // GROUP), torch.uint8)
        s["values"] = new((E, F, d))
        return
    s["workspace"] = new((ctx.workspace_bytes(),), torch.uint8)
    s["seg_expert"] = torch.arange(E, dtype=torch.int32, device=DEV)
    if kind == "ffn":
        s["u_out"], s["h_out"] = (new((N, F)) if case["keep"] else None), new((N, d))
    elif kind == "ffn_bwd":
        s["du_out"], s["dxp_out"] = (new((N, F)) if case["keep"] else None), new((N, d))
    elif kind == "combine_bwd":
        s["dh_out"], s["ds_out"] = new((N, d)), new((T, k), torch.float32)
    else:
        s["dx_out"], s["dz_out"] = new((T, d)), new((T, E), torch.float32)
        s["dWg_out"], s["dbg_out"] = new((E, d), torch.float32), new((E,), torch.float32)


# ---- one pass

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    case, ctx = s["case"], s["ctx"]
    N, kind = case["T"] * case["k"], case["kind"]
    if kind == "quantize":
        ctx.moe_quantize_mx4(s["W"], s["codes"], s["scales"], s["values"])
        return {"codes": s["codes"], "scales": s["scales"], "values": s["values"]}
    if kind == "ffn":
        ctx.moe_expert_ffn_mx4(s["x"], s["perm"], None, s["offsets"], s["seg_expert"], N, s["W1"], s["b1"], s["W2"], s["b2"],
                               s["u_out"], s["h_out"], s["workspace"])
        return {"h": s["h_out"], "u": s["u_out"]} if case["keep"] else {"h": s["h_out"]}
    if kind == "ffn_bwd":
        ctx.moe_expert_ffn_mx4_backward(s["dh"], s["u"], s["offsets"], s["seg_expert"], N, s["W1"], s["W2"], s["du_out"],
                                        s["dxp_out"], s["workspace"])
        return {"dx": s["dxp_out"], "du": s["du_out"]} if case["keep"] else {"dx": s["dxp_out"]}
    if kind == "combine_bwd":
        ctx.moe_combine_backward(s["dy"], s["h"], s["inv"], s["scores"], s["dh_out"], s["ds_out"])
        return {"dh": s["dh_out"][:s["rows"]], "dscores": s["ds_out"]}
    ctx.moe_route_backward(s["x"], s["Wg"], s["idx"], s["probs"], s["dscores"], s["dprobs"], s["dlogits"], s["dxp"], s["inv"],
                           s["dx_out"], s["dz_out"], s["dWg_out"], s["dbg_out"], s["workspace"])
    return {"dx": s["dx_out"], "dz": s["dz_out"], "dWg": s["dWg_out"], "dbg": s["dbg_out"]}


def _values(codes, scales):
    """The float values of one expert's codes [rows, cols / 2] and scales [rows, cols / 32]."""
    table = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device=DEV)
    rows, half = codes.shape
    code = torch.stack([codes & 15, codes >> 4], -1).reshape(rows, 2 * half)
    return (table[code.int()].reshape(rows, -1, GROUP) * torch.ldexp(torch.ones((), device=DEV), scales.int() - 127)[..., None]
            ).reshape(rows, 2 * half)


def _gelu(u):
    return 0.5 * u * (1.0 + torch.erf(u * math.sqrt(0.5)))


def _gelu_slope(u):
    return 0.5 * (1.0 + torch.erf(u * math.sqrt(0.5))) + u * torch.exp(-0.5 * u * u) / math.sqrt(2.0 * math.pi)


def _run_plain(s):
    case, dt = s["case"], s["dt"]
    T, d, F, E, k, kind = (case[n] for n in ("T", "d", "F", "E", "k", "kind"))
    N = T * k
    if kind == "quantize":
        codes, scales = _quantized(s["W"].reshape(E * F, d))
        return {"codes": codes.reshape(E, F, d // 2), "scales": scales.reshape(E, F, d // GROUP),
                "values": _values(codes, scales).to(dt).reshape(E, F, d)}
    if kind in ("ffn", "ffn_bwd"):
        rows_out, hidden_out = torch.empty((N, d), dtype=dt, device=DEV), torch.empty((N, F), dtype=dt, device=DEV)
        if kind == "ffn":
            x = s["x"][(s["perm"] // k).long()].float()
        for e in range(E):
            lo, hi = s["ends"][e], s["ends"][e + 1]
            if lo == hi:
                continue
            W1, W2 = _values(s["W1"][0][e], s["W1"][1][e]), _values(s["W2"][0][e], s["W2"][1][e])
            if kind == "ffn":
                u = x[lo:hi] @ W1.t()
                if case["bias"]:
                    u = u + s["b1"][e]
                h = _gelu(u) @ W2.t()
                rows_out[lo:hi] = h + s["b2"][e] if case["bias"] else h
                hidden_out[lo:hi] = u
            else:
                du = (s["dh"][lo:hi].float() @ W2) * _gelu_slope(s["u"][lo:hi].float())
                rows_out[lo:hi] = du @ W1
                hidden_out[lo:hi] = du
        a, b = ("h", "u") if kind == "ffn" else ("dx", "du")
        return {a: rows_out, b: hidden_out} if case["keep"] else {a: rows_out}
    inv = s["inv"].long()
    there = (inv >= 0)[:, None]
    if kind == "combine_bwd":
        pairs = s["perm"][:s["rows"]].long()
        dy = s["dy"].float()
        dh = s["scores"].flatten()[pairs][:, None] * dy[pairs // k]
        h = torch.where(there, s["h"][inv.clamp(min=0)].float(), 0.0).reshape(T, k, d)
        return {"dh": dh.to(dt), "dscores": (h * dy[:, None, :]).sum(-1)}
    dz = _plain_dz(s)
    dx = dz @ s["Wg"].float() + torch.where(there, s["dxp"][inv.clamp(min=0)].float(), 0.0).reshape(T, k, d).sum(1)
    dWg = dz.double().t() @ s["x"].double()                    # sums over all tokens
    return {"dx": dx.to(dt), "dz": dz, "dWg": dWg.float(), "dbg": dz.double().sum(0).float()}


def _plain_dz(s):
    """Gradient of the logits: softmax over the experts under the gradient of the probabilities."""
    probs, idx = s["probs"], s["idx"].long()
    g = torch.zeros_like(probs) if s["dprobs"] is None else s["dprobs"].clone()
    ds = s["dscores"]
    if s["case"]["renorm"]:
        picked = torch.gather(probs, 1, idx)
        total = picked.sum(1, keepdim=True)
        ds = (ds - (ds * picked / total).sum(1, keepdim=True)) / total
    g.scatter_add_(1, idx, ds)
    dz = probs * (g - (probs * g).sum(1, keepdim=True))
    return dz if s["dlogits"] is None else dz + s["dlogits"]


# ---- the definition, in double

def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    T, d, F, E, k, kind = (case[n] for n in ("T", "d", "F", "E", "k", "kind"))
    f64 = torch.float64
    if kind == "quantize":
        w = s["W"].reshape(-1, GROUP)
        values = torch.cat([_exact_values(part) for part in w.split(1 << 20)])
        return {"codes": None, "scales": None, "values": values.reshape(E, F, d)}
    if kind in ("ffn", "ffn_bwd"):
        out = {"h" if kind == "ffn" else "dx": torch.empty((T * k, d), dtype=f64, device=DEV)}
        if case["keep"]:
            out["u" if kind == "ffn" else "du"] = torch.empty((T * k, F), dtype=f64, device=DEV)
        for e in range(E):
            lo, hi = s["ends"][e], s["ends"][e + 1]
            if hi == lo:
                continue
            W1, W2 = (_exact_weight(s[n][0][e], s[n][1][e]) for n in ("W1", "W2"))
            if kind == "ffn":
                token = torch.div(s["perm"][lo:hi].long(), k, rounding_mode="floor")
                u = torch.mm(W1, s["x"][token].to(f64).t()).t()
                if case["bias"]:
                    u = u + s["b1"][e].to(f64)
                h = torch.mm(W2, (u * 0.5 * torch.erfc(-u / math.sqrt(2.0))).t()).t()
                out["h"][lo:hi] = h + s["b2"][e].to(f64) if case["bias"] else h
                if case["keep"]:
                    out["u"][lo:hi] = u
            else:
                u = s["u"][lo:hi].to(f64)
                slope = 0.5 * torch.erfc(-u / math.sqrt(2.0)) + u * torch.exp(-u * u / 2.0) * (0.5 * math.sqrt(2.0 / math.pi))
                du = torch.mm(W2.t(), s["dh"][lo:hi].to(f64).t()).t() * slope
                out["dx"][lo:hi] = torch.mm(W1.t(), du.t()).t()
                if case["keep"]:
                    out["du"][lo:hi] = du
        return out
    inv = s["inv"].reshape(T, k).long()
    if kind == "combine_bwd":
        dy, h = s["dy"].to(f64), s["h"].to(f64)
        dh = torch.zeros((s["rows"], d), dtype=f64, device=DEV)
        ds = torch.zeros((T, k), dtype=f64, device=DEV)
        for j in range(k):
            t = (inv[:, j] >= 0).nonzero().flatten()
            r = inv[t, j]
            dh[r] = s["scores"][t, j].to(f64)[:, None] * dy[t]
            ds[t, j] = (h[r] * dy[t]).sum(1)
        return {"dh": dh, "dscores": ds}
    probs, idx, ds = s["probs"].to(f64), s["idx"].long(), s["dscores"].to(f64)
    chosen = torch.zeros((T, k, E), dtype=f64, device=DEV).scatter_(2, idx[..., None], 1.0)
    p = (chosen * probs[:, None, :]).sum(2)
    dz = torch.zeros((T, E), dtype=f64, device=DEV)
    for j in range(k):                                         # ds_j / dz_e by the quotient rule, expert by expert
        if case["renorm"]:
            share = p / p.sum(1, keepdim=True)
            dz += (ds[:, j] * share[:, j])[:, None] * (chosen[:, j] - (chosen * share[..., None]).sum(1))
        else:
            dz += (ds[:, j] * p[:, j])[:, None] * (chosen[:, j] - probs)
    if s["dprobs"] is not None:
        g = s["dprobs"].to(f64)
        dz += probs * g - probs * (probs * g).sum(1, keepdim=True)
    if s["dlogits"] is not None:
        dz += s["dlogits"].to(f64)
    dx = torch.mm(dz, s["Wg"].to(f64))
    for j in range(k):
        t = (inv[:, j] >= 0).nonzero().flatten()
        dx[t] += s["dxp"][inv[t, j]].to(f64)
    return {"dx": dx, "dz": dz, "dWg": torch.mm(dz.t(), s["x"].to(f64)), "dbg": dz.sum(0)}


def _exact_weight(codes, scales):
    signed = torch.tensor([0, 1, 2, 3, 4, 6, 8, 12, 0, -1, -2, -3, -4, -6, -8, -12], dtype=torch.float64, device=DEV)     # halves
    out = torch.empty((codes.shape[0], codes.shape[1] * 2), dtype=torch.float64, device=DEV)
    out[:, 0::2], out[:, 1::2] = signed[(codes % 16).long()], signed[torch.div(codes, 16, rounding_mode="floor").long()]
    return out * torch.repeat_interleave(torch.pow(2.0, scales.to(torch.float64) - 128.0), GROUP, dim=1)


def _exact_values(groups):
    """Nearest code value of every weight in rows of 32: the scale by comparison with 7 times powers of two."""
    w = groups.double()
    largest = w.abs().max(1).values
    exponent = torch.ceil(torch.log2(torch.clamp(largest / 7.0, min=2.0 ** -126)))
    exponent += (largest > 7.0 * torch.pow(2.0, exponent)).double()                # where the logarithm rounded across a power
    exponent -= (largest <= 7.0 * torch.pow(2.0, exponent - 1.0)).double()
    step = torch.pow(2.0, torch.clamp(exponent, min=-126.0))[:, None]
    v = w.abs() / step
    grid = torch.where(v < 2.0, 0.5, torch.where(v < 4.0, 1.0, 2.0))               # spacing of the code values around v
    return torch.sign(w) * torch.clamp(torch.round(v / grid) * grid, max=6.0) * step
