"""The recurrence's gradients against the definition in 64 bits for slow, ordinary and fast decays.

The kernels take one of two ways by the rates of a slab of channels (64, fp32 32): all of at most 1/4, or not.  Bounds are those of
test_gpu_gated_recurrence.py with the decays' own error: sigmoid(r) is off by 16 U relative at most, so the exponent -rate
sigmoid(r) by 18 U of itself with its roundings, and a by (18 rate + 24) U relative, below 32 U (1 + rate); a^2 by twice that.
With tok >= 64 U of the gradient's own error, 3 tok (1 + rate) covers the terms of dlog a.  Absolutely a is off by less than 16 U
whatever the rate (z exp(-z) <= 1 / e), as for the slow ones, so nothing changes for G and the states.
"""
import pytest
import torch

import paper_2402_18668_b200 as based
from layers64 import U, close, half_step, recurrence, recurrence_grad
from test_gpu_gated_recurrence import channel_max, draw, f64, slack

pytestmark = pytest.mark.gpu


def rates(kind, C):
    lo, hi = {"slow": (1e-3, 0.105), "edge": (0.2, 0.25), "one fast": (1e-3, 0.2), "both sides": (0.02, 0.6), "fast": (3.0, 20.0)}[kind]
    g = torch.Generator(device="cuda").manual_seed(21)
    rate = lo + (hi - lo) * torch.rand(C, generator=g, device="cuda")
    if kind == "one fast":
        rate[5::32] = 0.3
    return rate


def check(x, r, g, rate, start, out, dout, end, got):
    w = recurrence_grad(*f64(x, r, g, rate, start, out, dout, end))
    N = x.shape[1]
    tok, h = slack(w["a"]), half_step(x.dtype)
    G = channel_max(w["G"], dout.double(), end)
    xd, rd = x.double(), rate.double()
    for name, t, factor in (("dx", got[0], w["m"] * w["i"]), ("dg", got[2], w["m"] * xd * w["i"] * (1 - w["i"]))):
        off = 2 * tok * G * factor.abs()
        off = off + (4 * U * G * (w["m"] * xd * w["i"]).abs() if name == "dg" else 0)
        close(t, w[name], off + h * (w[name].abs() + off), name)
    terms = G * ((w["a"] * w["prev"]).abs() + (w["a"] ** 2 / w["m"] * w["i"] * xd).abs())
    dla_off = 3 * tok * (1 + rd) * terms
    off = rd * dla_off * w["s"] * (1 - w["s"]) + 4 * U * rd * w["s"] * terms
    close(got[1], w["dr"], off + h * (w["dr"].abs() + off), "dr")
    close(got[3], w["drate"], (dla_off * w["s"]).sum((0, 1)) + (N / 16 + 32) * U * (terms * w["s"]).sum((0, 1)), "drate")
    if start is not None:
        close(got[4], w["dh0"], tok * G, "dstate_in")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["slow", "edge", "one fast", "both sides", "fast"])
@pytest.mark.parametrize("B,N,C", [(2, 64, 128), (3, 63, 72), (1, 4099, 64), (1, 1, 40)])
def test_backward(B, N, C, kind, dtype):
    x, r, g, _, h0, dout, dh = draw(B, N, C, dtype, seed=20)
    rate = rates(kind, C)
    for start, end in ((None, None), (h0, dh)):
        out = based.based_gated_recurrence_forward(x, r, g, rate, state_in=start)
        check(x, r, g, rate, start, out, dout, end,
              based.based_gated_recurrence_backward(x, r, g, rate, out, dout, state_in=start, dstate_out=end))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_fast_decays_leave_of_a_state(dtype):
    """Without inputs the state is the product of the decays: off by (18 z + 24) U for each, z its exponent, and the products' roundings."""
    N, C = 3, 64
    _, r, g, _, h0, _, _ = draw(2, N, C, dtype, seed=22)
    x, rate, h0 = torch.zeros_like(r), rates("fast", C), h0 * 1e6
    want, a, _, _ = recurrence(*f64(x, r, g, rate, h0))
    rel = ((18 * -torch.log(a) + 24) * U).cumsum(1)
    last = torch.empty_like(h0)
    out = based.based_gated_recurrence_forward(x, r, g, rate, state_in=h0, state_out=last)
    close(out, want, (rel + half_step(x.dtype) * (1 + rel)) * want.abs(), "sequence")
    close(last, want[:, -1], rel[:, -1] * want[:, -1].abs(), "state")
    state = h0.clone()
    for t in range(N):
        y = based.based_gated_recurrence_step(x[:, t], r[:, t], g[:, t], rate, state)
        close(y, want[:, t], (rel[:, t] + half_step(x.dtype) * (1 + rel[:, t])) * want[:, t].abs(), f"token {t}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,N,C", [(2, 203, 64), (1, 3001, 72)])
def test_rates_of_zero_beside_fast_ones(B, N, C, dtype):
    """Of either sign: the state stays as it is to the last bit, and its gradient gathers the outputs' (N sums in fp32 in any order)."""
    x, r, g, _, h0, dout, dh = draw(B, N, C, dtype, seed=23)
    rate = rates("fast", C)
    rate[::8], rate[1::8] = 0.0, -0.0
    still = (rate == 0).nonzero()[:, 0]
    last = torch.empty_like(h0)
    out = based.based_gated_recurrence_forward(x, r, g, rate, state_in=h0, state_out=last)
    assert torch.equal(last[:, still], h0[:, still])
    assert torch.equal(out[..., still], h0[:, None, still].expand(B, N, -1).to(out.dtype))
    dx, _, dg, _, dh0 = based.based_gated_recurrence_backward(x, r, g, rate, out, dout, state_in=h0, dstate_out=dh)
    assert (dx[..., still] == 0).all() and (dg[..., still] == 0).all()
    want = dout.double().sum(1) + dh.double()
    close(dh0[:, still], want[:, still], (N + 1) * U * (dout.double().abs().sum(1) + dh.double().abs())[:, still], "dstate_in")
