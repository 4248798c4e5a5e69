"""The recurrence's states in one array, before and behind a call, where several CTAs share a sequence."""
import pytest
import torch

import paper_2402_18668_b200 as based
from paper_2402_18668_b200 import binding
from test_gpu_gated_recurrence import draw

pytestmark = pytest.mark.gpu
# one step of a cluster's CTAs, of 2 to 16 of them, and several
SHAPES = [(1, 128, 8), (1, 300, 64), (2, 512, 64), (3, 1000, 72), (1, 1024, 64), (1, 2048, 128), (1, 4099, 64), (2, 9001, 40)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,N,C", SHAPES)
def test_state(B, N, C, dtype):
    x, r, g, rate, h0, _, _ = draw(B, N, C, dtype, seed=30)
    last = torch.empty_like(h0)
    want = based.based_gated_recurrence_forward(x, r, g, rate, state_in=h0, state_out=last)
    for _ in range(20):
        state = h0.clone()
        out = based.based_gated_recurrence_forward(x, r, g, rate, state_in=state, state_out=state)
        assert torch.equal(out, want) and torch.equal(state, last)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,N,C", SHAPES)
def test_gradient_of_the_state(B, N, C, dtype):
    x, r, g, rate, h0, dout, dh = draw(B, N, C, dtype, seed=31)
    out = based.based_gated_recurrence_forward(x, r, g, rate, state_in=h0)
    want = based.based_gated_recurrence_backward(x, r, g, rate, out, dout, h0, dh)
    io = 0 if dtype == "f32" else 1
    need = based.lib().based_gated_recurrence_backward_workspace_bytes(B, N, C, io)
    work = torch.empty(need, device="cuda", dtype=torch.uint8)
    tokens = lambda t: binding.Tokens(t.data_ptr(), N * C, C)
    for _ in range(20):
        state = dh.clone()
        got = [torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty_like(rate), state]
        status = based.lib().based_gated_recurrence_backward(
            tokens(x), tokens(r), tokens(g), rate.data_ptr(), h0.data_ptr(), tokens(out), tokens(dout), state.data_ptr(),
            *(t.data_ptr() for t in got), B, N, C, io, work.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
        assert status == based.BASED_OK
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert based.based_poll_error() == based.BASED_OK
