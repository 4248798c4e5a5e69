"""The gated recurrence against its definition in 64 bits: sequence, token, backward, and their use together.

Bounds.  Per token the kernel's a = 1 + p and m i x carry a few roundings of fp32 each, and the special functions two steps:
16 U relative covers a sigmoid, a decay or a product of them.  h follows e_t <= a e_{t-1} + 16 U (|h| + |b|), so it is off by at most
32 U max(|h|, |b|) / (1 - max a) over a channel; the joins of runs (12 of them at most) add their own roundings, hence 64.
Results are rounded to the io type once.
"""
import pytest
import torch

import paper_2402_18668_b200 as based
from layers64 import U, close, half_step, recurrence, recurrence_grad
from paper_2402_18668_b200 import autograd as ag

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def draw(B, N, C, dtype, seed=0, rate_lo=0.02, rate_hi=0.6):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x, r, gt, dout = (rnd(B, N, C).to(DT[dtype]) for _ in range(4))
    rate = rate_lo + (rate_hi - rate_lo) * torch.rand(C, generator=g, device="cuda")
    return x, r, gt, rate, rnd(B, C), dout, rnd(B, C)


def f64(*ts):
    return [None if t is None else t.double() for t in ts]


def channel_max(*ts):
    """[C]: the largest absolute value of any of them in a channel."""
    return torch.stack([t.abs().flatten(0, -2).amax(0) for t in ts if t is not None]).amax(0)


def slack(a):
    return 64 * U / (1 - a.flatten(0, -2).amax(0))


SHAPES = [(1, 1, 8), (1, 2, 8), (2, 3, 64), (3, 63, 72), (2, 64, 128), (1, 65, 200), (2, 257, 520), (1, 1000, 1000), (5, 129, 264),
          (1, 4099, 64), (40, 100, 2048), (1, 513, 8)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,N,C", SHAPES)
def test_sequence(B, N, C, dtype):
    x, r, g, rate, h0, _, _ = draw(B, N, C, dtype)
    for start in (None, h0):
        last = torch.full((B, C), 7.0, device="cuda")
        out = based.based_gated_recurrence_forward(x, r, g, rate, state_in=start, state_out=last)
        want, a, m, i = recurrence(*f64(x, r, g, rate, start))
        off = slack(a) * channel_max(want, m * i * x.double(), start)
        close(out, want, off + half_step(x.dtype) * (want.abs() + off), "out")
        close(last, want[:, -1], off, "state")
    assert based.based_poll_error() == based.BASED_OK


@pytest.mark.parametrize("rates", [(0.0, 1e-4), (1e-3, 0.01), (0.2, 0.3), (3.0, 200.0)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rates(rates, dtype):
    """Slow decays (where 1 - a^2 would cancel), those on both sides of the series' range, and none of the past left."""
    x, r, g, rate, h0, dout, dh = draw(2, 200, 96, dtype, rate_lo=rates[0], rate_hi=rates[1])
    rate[3] = rates[0]
    out = based.based_gated_recurrence_forward(x, r, g, rate, state_in=h0)
    want, a, m, i = recurrence(*f64(x, r, g, rate, h0))
    # over N tokens the sum of a^k is at most N, whatever the decay
    per = 64 * U * torch.clamp(1 / (1 - a.flatten(0, 1).amax(0)), max=200.0) * channel_max(want, m * i * x.double(), h0)
    close(out, want, per + half_step(x.dtype) * (want.abs() + per), "out")
    grads = based.based_gated_recurrence_backward(x, r, g, rate, out, dout, h0, dh)
    assert all(torch.isfinite(t).all() for t in grads)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_gates(dtype):
    """Gates far out: open or shut to the last digit, and a NaN stays in its channel and behind its token."""
    x, r, g, rate, h0, dout, dh = draw(1, 150, 64, dtype, seed=2)
    r[0, :, 0], r[0, :, 1], g[0, :, 2], g[0, :, 3] = 80.0, -80.0, 90.0, -90.0
    r[0, 5, 4], g[0, 5, 5] = float("inf"), -float("inf")
    want, a, m, i = recurrence(*f64(x, r, g, rate, h0))
    out = based.based_gated_recurrence_forward(x, r, g, rate, state_in=h0)
    # (a shut gate counts as 2^-59: an m of up to sqrt(2 rate 2^-59) < 2^-28.5 in the place of a smaller one, times x < 8, 150 times)
    off = 64 * U * 150 * channel_max(want, m * i * x.double(), h0) + 2.0 ** -28.5 * 8 * 150
    close(out, want, off + half_step(x.dtype) * (want.abs() + off), "out")
    grads = based.based_gated_recurrence_backward(x, r, g, rate, out, dout, h0, dh)
    assert all(torch.isfinite(t).all() for t in grads)
    x[0, 70, 9], r[0, 80, 10], g[0, 90, 11] = float("nan"), float("nan"), float("nan")
    y = based.based_gated_recurrence_forward(x, r, g, rate, state_in=h0)
    bad = torch.isnan(y[0])
    assert bad[70:, 9].all() and bad[80:, 10].all() and bad[90:, 11].all()
    assert int(bad.sum()) == 80 + 70 + 60
    assert torch.equal(y[0][~bad], out[0][~bad])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,N,C", SHAPES)
def test_backward(B, N, C, dtype):
    x, r, g, rate, h0, dout, dh = draw(B, N, C, dtype, seed=1)
    for start, end in ((None, None), (h0, dh), (h0, None), (None, dh)):
        out = based.based_gated_recurrence_forward(x, r, g, rate, state_in=start)
        got = based.based_gated_recurrence_backward(x, r, g, rate, out, dout, state_in=start, dstate_out=end)
        w = recurrence_grad(*f64(x, r, g, rate, start, out, dout, end))
        # G is off by tok times its channel's largest value, every other factor by 16 U of itself (tok > 64 U)
        tok, h = slack(w["a"]), half_step(x.dtype)
        G = channel_max(w["G"], dout.double(), end)
        xd, rd = x.double(), rate.double()
        for name, t, factor in (("dx", got[0], w["m"] * w["i"]), ("dg", got[2], w["m"] * xd * w["i"] * (1 - w["i"]))):
            off = 2 * tok * G * factor.abs()
            # (1 - i: off by 2 U absolutely)
            off = off + (4 * U * G * (w["m"] * xd * w["i"]).abs() if name == "dg" else 0)
            close(t, w[name], off + h * (w[name].abs() + off), name)
        # dlog a: two terms that may cancel
        dla_off = 2 * tok * G * ((w["a"] * w["prev"]).abs() + (w["a"] ** 2 / w["m"] * w["i"] * xd).abs())
        s1 = w["s"] * (1 - w["s"])
        off = rd * dla_off * s1 + 4 * U * rd * w["s"] * dla_off / (2 * tok)
        close(got[1], w["dr"], off + h * (w["dr"].abs() + off), "dr")
        # (the sum: a chain of N / 16 terms at most, then trees)
        terms = (dla_off / (2 * tok) * w["s"]).sum((0, 1))
        close(got[3], w["drate"], (dla_off * w["s"]).sum((0, 1)) + (N / 16 + 32) * U * terms, "drate")
        if start is None:
            assert got[4] is None
        else:
            close(got[4], w["dh0"], tok * G, "dstate_in")
        again = based.based_gated_recurrence_backward(x, r, g, rate, out, dout, state_in=start, dstate_out=end)
        assert all(torch.equal(a, b) for a, b in zip(got, again) if a is not None)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tokens_follow_the_sequence(dtype):
    """A prompt, then tokens one by one in place: the same as the sequence in one call."""
    B, N, C, k = 3, 70, 136, 9
    x, r, g, rate, h0, _, _ = draw(B, N, C, dtype, seed=3)
    whole = based.based_gated_recurrence_forward(x, r, g, rate, state_in=h0)
    state = h0.clone()
    outs = [based.based_gated_recurrence_forward(*(t[:, :N - k].contiguous() for t in (x, r, g)), rate, state_in=state, state_out=state)]
    for t in range(N - k, N):
        kept = state.clone()
        other = torch.empty_like(state)
        y0 = based.based_gated_recurrence_step(*(z[:, t].contiguous() for z in (x, r, g)), rate, state, state_out=other)
        assert torch.equal(state, kept)
        y = based.based_gated_recurrence_step(*(z[:, t].contiguous() for z in (x, r, g)), rate, state)
        assert torch.equal(y, y0) and torch.equal(state, other)
        outs.append(y[:, None])
    want, a, m, i = recurrence(*f64(x, r, g, rate, h0))
    off = slack(a) * channel_max(want, m * i * x.double(), h0)
    close(torch.cat(outs, 1), want, off + half_step(x.dtype) * (want.abs() + off))
    close(whole, want, off + half_step(x.dtype) * (want.abs() + off))
    close(state, want[:, -1], off)


def test_differences():
    """The autograd node's gradient along random directions against central differences of the definition in 64 bits."""
    B, N, C = 2, 90, 24
    x, r, g, rate, h0, dout, dh = draw(B, N, C, "f32", seed=4)
    leaves = [t.clone().requires_grad_(True) for t in (x, r, g, rate, h0)]
    out, last = ag.gated_recurrence(*leaves)
    ((out * dout).sum() + (last * dh).sum()).backward()
    gen = torch.Generator(device="cuda").manual_seed(5)

    def f(ts):
        y = recurrence(*ts)[0]
        return float((y * dout.double()).sum() + (y[:, -1] * dh.double()).sum())

    base = f64(x, r, g, rate, h0)
    for n, leaf in enumerate(leaves):
        for _ in range(3):
            v = torch.randn(leaf.shape, generator=gen, device="cuda").double() * (0.01 if n == 3 else 1.0)
            e = 1e-5
            up, down = list(base), list(base)
            up[n], down[n] = base[n] + e * v, base[n] - e * v
            slope = (f(up) - f(down)) / (2 * e)
            along = leaf.grad.double() * v
            # the gradient: 64 U / (1 - a) of every term (a < 0.998: below 2e-3 relative, times 1e-2 for random signs); the
            # differences: truncation e^2 and rounding 1e-16 / e of the sum, below 1e-6
            assert abs(slope - float(along.sum())) <= 2e-5 * float(along.abs().sum()) + 1e-5, n


def test_autograd_only_one_output_used_and_no_second_derivative():
    x, r, g, rate, h0, dout, dh = draw(2, 40, 16, "bf16", seed=6)
    leaves = [t.clone().requires_grad_(True) for t in (x, r, g, rate, h0)]
    _, last = ag.gated_recurrence(*leaves)
    a = torch.autograd.grad((last * dh).sum(), leaves)
    want = based.based_gated_recurrence_backward(x, r, g, rate, based.based_gated_recurrence_forward(x, r, g, rate, state_in=h0),
                                                 torch.zeros_like(x), h0, dh)
    assert all(torch.equal(p, q) for p, q in zip(a, want))
    out, _ = ag.gated_recurrence(*leaves)
    with pytest.raises(RuntimeError, match="cannot be differentiated again"):
        torch.autograd.grad(out.float().sum(), leaves, create_graph=True)
    out, last = ag.gated_recurrence(*leaves[:4])            # without a state; inputs that are not contiguous
    y, _ = ag.gated_recurrence(*(t.transpose(1, 2).contiguous().transpose(1, 2) for t in (x, r, g)), rate)
    assert torch.equal(out, y)


def test_streams_graph_and_neighbours():
    """On another stream, captured and replayed with new inputs, and nothing written outside the outputs."""
    B, N, C = 2, 333, 200
    x, r, g, rate, h0, dout, dh = draw(B, N, C, "bf16", seed=7)
    want = based.based_gated_recurrence_forward(x, r, g, rate, state_in=h0)
    room = torch.full((B * N * C + 256,), 3.0, device="cuda", dtype=torch.bfloat16)
    states = torch.full((B * C + 64,), 5.0, device="cuda")
    out, last = room[128:128 + B * N * C].view(B, N, C), states[32:32 + B * C].view(B, C)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    based.based_gated_recurrence_forward(x, r, g, rate, state_in=h0, out=out, state_out=last, stream=s)
    s.synchronize()
    assert torch.equal(out, want)
    assert (room[:128] == 3).all() and (room[128 + B * N * C:] == 3).all() and (states[:32] == 5).all() and (states[32 + B * C:] == 5).all()
    grads = based.based_gated_recurrence_backward(x, r, g, rate, want, dout, h0, dh)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = based.based_gated_recurrence_forward(x, r, g, rate, state_in=h0)
        got = based.based_gated_recurrence_backward(x, r, g, rate, y, dout, h0, dh)
    graph.replay()
    assert torch.equal(y, want) and all(torch.equal(a, b) for a, b in zip(got, grads))
    x.copy_(torch.randn_like(x, dtype=torch.float32))
    graph.replay()
    want = based.based_gated_recurrence_forward(x, r, g, rate, state_in=h0)
    grads = based.based_gated_recurrence_backward(x, r, g, rate, want, dout, h0, dh)
    assert torch.equal(y, want) and all(torch.equal(a, b) for a, b in zip(got, grads))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_views_with_strides(dtype):
    """Slices of a fused projection and of a longer batch, as they lie; the autograd node too."""
    B, N, C = 3, 150, 72
    x, r, g, rate, h0, dout, dh = draw(B, N, C, dtype, seed=8)
    fused = torch.cat([r, g, x], -1)
    longer = torch.nn.functional.pad(dout, (0, 0, 0, 50), value=float("nan"))
    views = (fused[..., 2 * C:], fused[..., :C], fused[..., C:2 * C])
    want = based.based_gated_recurrence_forward(x, r, g, rate, state_in=h0)
    assert torch.equal(based.based_gated_recurrence_forward(*views, rate, state_in=h0), want)
    out = torch.nn.functional.pad(want, (0, 0, 0, 7), value=float("nan"))[:, :N]
    a = based.based_gated_recurrence_backward(x, r, g, rate, want, dout, h0, dh)
    b = based.based_gated_recurrence_backward(*views, rate, out, longer[:, :N], h0, dh)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    leaf = fused.clone().requires_grad_(True)
    y, _ = ag.gated_recurrence(leaf[..., 2 * C:], leaf[..., :C], leaf[..., C:2 * C], rate)
    (d,) = torch.autograd.grad(y, leaf, longer[:, :N])
    c = based.based_gated_recurrence_backward(x, r, g, rate, y.detach(), dout)
    assert torch.equal(d, torch.cat([c[1], c[2], c[0]], -1))
    state = h0.clone()
    one = based.based_gated_recurrence_step(*(v[:, 3] for v in views), rate, state)
    other = h0.clone()
    assert torch.equal(one, based.based_gated_recurrence_step(*(v[:, 3].contiguous() for v in (x, r, g)), rate, other)) and torch.equal(state, other)
    with pytest.raises(ValueError):
        based.based_gated_recurrence_forward(x.transpose(1, 2), r.transpose(1, 2), g.transpose(1, 2), rate)
    with pytest.raises(based.BasedError):                    # the same tokens for every sequence
        based.based_gated_recurrence_forward(x[:1].expand(B, N, C), r, g, rate)


def test_refusals():
    x, r, g, rate, h0, dout, dh = draw(2, 10, 16, "bf16")
    f, s, b = based.based_gated_recurrence_forward, based.based_gated_recurrence_step, based.based_gated_recurrence_backward
    pool = torch.zeros(40, device="cuda")
    one = lambda t: t[:, 0].contiguous()
    V, T, E = ValueError, TypeError, based.BasedError
    for err, call in (
            (V, lambda: f(x, r[:, :9], g, rate)), (V, lambda: f(x, r.float(), g, rate)), (T, lambda: f(x, r, g, rate.double())),
            (V, lambda: f(x, r, g, rate[:8])), (V, lambda: f(x, r, g, rate, state_in=h0[:1])), (V, lambda: f(x, r, g, rate, out=x)),
            # neither the same state nor another one
            (V, lambda: f(x, r, g, rate, state_in=pool[:32].view(2, 16), state_out=pool[4:36].view(2, 16))),
            (V, lambda: f(x.cpu(), r, g, rate)), (T, lambda: f(x.half(), r.half(), g.half(), rate)), (V, lambda: f(one(x), one(r), one(g), rate)),
            (E, lambda: f(*(t[..., :12].contiguous() for t in (x, r, g)), rate[:12].contiguous())),
            (E, lambda: f(*(t[:, :0] for t in (x, r, g)), rate)),
            (V, lambda: s(one(x), one(r), one(g), rate, h0[:1])), (E, lambda: s(one(x), one(r), one(g), rate, None)),
            (V, lambda: s(x, r, g, rate, h0)), (V, lambda: b(x, r, g, rate, x[:, :9].contiguous(), dout)),
            (V, lambda: b(x, r, g, rate, x, dout, h0, dh[:1])), (V, lambda: b(x, r, g, rate, x, dout, workspace=x))):
        with pytest.raises(err):
            call()
    assert based.based_poll_error() == based.BASED_OK
