"""The gated recurrence on large finite inputs: the sequence and its tokens one by one, whichever rates a slab of channels holds."""
import pytest
import torch

import paper_2402_18668_b200 as based
from layers64 import close, half_step, recurrence
from test_gpu_gated_recurrence import channel_max, draw, f64, slack

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [1e30, 1e35])
@pytest.mark.parametrize("fast", [False, True])
@pytest.mark.parametrize("B,N,C", [(2, 70, 96), (1, 1500, 64)])
def test_large_inputs(B, N, C, fast, size, dtype):
    """Rates of at most 0.2, or one of 0.4 in every 16 channels.  The state is below 1 / (1 - a) times the largest input, 1e38."""
    x, r, g, rate, h0, _, _ = draw(B, N, C, dtype, seed=12, rate_lo=0.05, rate_hi=0.2)
    if fast:
        rate[::16] = 0.4
    x, h0 = (x.float() * size).to(x.dtype), h0 * size
    want, a, m, i = recurrence(*f64(x, r, g, rate, h0))
    off = slack(a) * channel_max(want, m * i * x.double(), h0)
    last = torch.empty_like(h0)
    out = based.based_gated_recurrence_forward(x, r, g, rate, state_in=h0, state_out=last)
    close(out, want, off + half_step(x.dtype) * (want.abs() + off), "sequence")
    close(last, want[:, -1], off, "state")
    state = h0.clone()
    for t in range(70):
        y = based.based_gated_recurrence_step(x[:, t], r[:, t], g[:, t], rate, state)
        close(y, want[:, t], off + half_step(x.dtype) * (want[:, t].abs() + off), f"token {t}")
