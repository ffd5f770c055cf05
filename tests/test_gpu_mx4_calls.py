"""Calls of the 4-bit experts and the layer's gradients as a program makes them: the timing event."""
import pytest
import torch

from test_gpu_layer_gradients import Layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [3, 600])
@pytest.mark.parametrize("call", ["forward", "backward"])
def test_between_event_is_recorded_between_the_products(call, T):
    L = Layer(T, 256, 512, 4, 2, "bf16", False)
    L.step()
    N, b = T * 2, L.buf
    before, between, after = (torch.cuda.Event(enable_timing=True) for _ in range(3))

    def run():
        if call == "forward":
            L.ctx.moe_expert_ffn_mx4(L.on["x"], b.perm, None, b.offsets, b.seg_expert, N, L.W1, L.on["b1"], L.W2, L.on["b2"], L.u, b.h_packed, b.workspace)
        else:
            L.ctx.moe_expert_ffn_mx4_backward(L.dh, L.u, b.offsets, b.seg_expert, N, L.W1, L.W2, None, L.dxp, b.workspace)

    between.record()                                                # (creates it)
    torch.cuda.synchronize()
    L.ctx.moe_expert_ffn_between_event(between)
    before.record()
    run()
    after.record()
    L.ctx.moe_expert_ffn_between_event(None)
    torch.cuda.synchronize()
    first, second = before.elapsed_time(between), between.elapsed_time(after)
    assert first > 0 and second > 0
    run()                                                           # without the hook the event stays as it is
    torch.cuda.synchronize()
    assert before.elapsed_time(between) == first
