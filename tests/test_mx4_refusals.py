"""Refusals of the 4-bit expert calls and of the gradient calls: before any launch, without a GPU."""
import ctypes

import pytest
import torch

from paper_2411_16786_amd import binding as B

ONE = ctypes.c_void_p(16)       # a non-null dummy address; never dereferenced on these paths


def _ctx(**kw):
    shape = dict(T_max=64, d=64, F=256, E=4, k=2, dtype="bf16")
    shape.update(kw)
    return B.Context(**shape)


def test_quantize_refuses():
    L, c = B.lib(), _ctx()
    for rows, cols in ((-1, 64), (8, 0), (8, 16), (8, 48), (8, -32), (1 << 38, 32), (1 << 62, 64)):
        assert L.moe_quantize_mx4(c._h, ONE, rows, cols, ONE, ONE, None, None) == B.MOE_ERR_SHAPE, (rows, cols)
    for args in ((None, ONE, ONE), (ONE, None, ONE), (ONE, ONE, None)):
        assert L.moe_quantize_mx4(c._h, args[0], 8, 64, args[1], args[2], None, None) == B.MOE_ERR_NULL
    assert b"moe_quantize_mx4" in L.moe_last_error(c._h)
    assert L.moe_quantize_mx4(None, ONE, 8, 64, ONE, ONE, None, None) == B.MOE_ERR_NULL
    assert L.moe_quantize_mx4(c._h, None, 0, 64, None, None, None, None) == B.MOE_OK


def _ffn(c, max_rows=8, n_seg=4, **null):
    names = ("x", "row_pairs", "out_pairs", "offsets", "expert", "W1c", "W1s", "b1", "W2c", "W2s", "b2", "u", "h", "ws")
    a = {n: (None if n in null or n in ("row_pairs", "out_pairs", "b1", "b2", "u") else ONE) for n in names}
    return B.lib().moe_expert_ffn_mx4(c._h if c else None, a["x"], a["row_pairs"], a["out_pairs"], a["offsets"], a["expert"], n_seg, max_rows,
                                      a["W1c"], a["W1s"], a["b1"], a["W2c"], a["W2s"], a["b2"], a["u"], a["h"], a["ws"], None)


def _ffn_backward(c, max_rows=8, n_seg=4, **null):
    names = ("dh", "u", "offsets", "expert", "W1c", "W1s", "W2c", "W2s", "du", "dx", "ws")
    a = {n: (None if n in null or n == "du" else ONE) for n in names}
    return B.lib().moe_expert_ffn_mx4_backward(c._h if c else None, a["dh"], a["u"], a["offsets"], a["expert"], n_seg, max_rows,
                                               a["W1c"], a["W1s"], a["W2c"], a["W2s"], a["du"], a["dx"], a["ws"], None)


@pytest.mark.parametrize("call,required", [(_ffn, ("x", "offsets", "expert", "W1c", "W1s", "W2c", "W2s", "h")),
                                           (_ffn_backward, ("dh", "u", "offsets", "expert", "W1c", "W1s", "W2c", "W2s", "dx"))])
def test_ffn_calls_refuse(call, required):
    c = _ctx()
    assert call(None) == B.MOE_ERR_NULL
    for name in required:
        assert call(c, **{name: True}) == B.MOE_ERR_NULL, name
    assert call(c, ws=True) == B.MOE_ERR_WORKSPACE
    for kw in (dict(max_rows=-1), dict(max_rows=129), dict(n_seg=0), dict(n_seg=1025)):
        assert call(c, **kw) == B.MOE_ERR_SHAPE, kw
    # float rows may be multiples of 16, which is half a scale group
    assert call(_ctx(d=48, dtype="f32")) == B.MOE_ERR_SHAPE
    assert call(_ctx(F=240, dtype="f32")) == B.MOE_ERR_SHAPE
    assert call(_ctx(T_max=1, F=1 << 21)) == B.MOE_ERR_SHAPE
    # a table of so many short segments that a launch would have 2^32 threads
    assert call(_ctx(T_max=512, d=64, F=1 << 20), max_rows=512, n_seg=512) == B.MOE_ERR_SHAPE


def test_combine_backward_refuses():
    L, c = B.lib(), _ctx()
    good = [ONE] * 4 + [8] + [ONE] * 2
    for i in (0, 1, 2, 3, 5, 6):
        bad = list(good)
        bad[i] = None
        assert L.moe_combine_backward(c._h, *bad, None) == B.MOE_ERR_NULL, i
    for T in (-1, 65):
        assert L.moe_combine_backward(c._h, *[ONE] * 4, T, ONE, ONE, None) == B.MOE_ERR_SHAPE
    assert L.moe_combine_backward(c._h, *[None] * 4, 0, None, None, None) == B.MOE_OK
    assert L.moe_combine_backward(None, *good, None) == B.MOE_ERR_NULL


def test_route_backward_refuses():
    L, c = B.lib(), _ctx()
    names = ("x", "Wg", "idx", "probs", "dscores", "dprobs", "dlogits", "dxp", "inv", "T", "dx", "dz", "dWg", "dbg", "ws")

    def call(T=8, **null):
        a = [T if n == "T" else (None if n in null else ONE) for n in names]
        return L.moe_route_backward(c._h, *a, None)

    for missing in (("x",), ("idx",), ("probs",), ("dscores",), ("dx",), ("dxp",), ("inv",)):
        assert call(**{n: True for n in missing}) == B.MOE_ERR_NULL, missing
    assert call(ws=True) == B.MOE_ERR_WORKSPACE
    assert call(T=-1) == B.MOE_ERR_SHAPE and call(T=65) == B.MOE_ERR_SHAPE
    # the dispatch alone gives nothing for the router
    assert call(Wg=True) == B.MOE_ERR_NULL
    assert call(Wg=True, dz=True, dWg=True) == B.MOE_ERR_NULL
    assert call(Wg=True, dz=True, dWg=True, dbg=True, dxp=True, inv=True) == B.MOE_ERR_NULL
    assert call(T=0, Wg=True, dz=True, dWg=True, dbg=True, dxp=True, inv=True) == B.MOE_OK
    assert L.moe_route_backward(None, *[ONE] * 9, 8, *[ONE] * 5, None) == B.MOE_ERR_NULL


def test_binding_refuses_shapes_and_cpu_tensors():
    c = _ctx(T_max=8)
    W = torch.zeros(4, 64, dtype=torch.bfloat16)
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)
    with pytest.raises(ValueError, match="GPU"):
        c.moe_quantize_mx4(W, u8(4, 32), u8(4, 2))
    W1, W2 = (u8(4, 256, 32), u8(4, 256, 2)), (u8(4, 64, 128), u8(4, 64, 8))
    x, i32 = torch.zeros(16, 64, dtype=torch.bfloat16), torch.zeros(5, dtype=torch.int32)
    with pytest.raises(ValueError, match="x_rows"):
        c.moe_expert_ffn_mx4(x[:15], None, None, i32, i32[:4], 16, W1, None, W2, None, None, x, u8(8))
    with pytest.raises(ValueError, match="u_packed"):
        c.moe_expert_ffn_mx4_backward(_Cuda(x), x, i32, i32[:4], 16, W1, W2, None, x, u8(8))          # u has d columns, not F
    with pytest.raises(ValueError, match="dscores"):
        f = torch.zeros(8, 2)
        c.moe_combine_backward(_Cuda(x[:8]), _Cuda(x), _Cuda(i32[:1].repeat(16)), _Cuda(f), _Cuda(x), _Cuda(f[:7]))


class _Cuda:
    """A CPU tensor that says it lives on the GPU: the checks that come before the address is used."""

    def __init__(self, t):
        self.t = t
        self.is_cuda = True

    def __getattr__(self, name):
        return getattr(self.t, name)

    def view(self, *shape):
        return _Cuda(self.t.view(*shape))
