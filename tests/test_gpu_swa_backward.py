"""The sliding window's backward pass against its definition in 64 bits, and the layers in a row as a model would call them.

Bounds: layers64.window_grad gives, per element, what rounding P and dS once to the io type does (bf16 operands of the tensor cores;
fp32 io rounds them to fp32) and what fp32 sums do; the result is rounded once more.
"""
import pytest
import torch

import paper_2402_18668_b200 as based
from layers64 import U, close, half_step, norm_rotate, recurrence, window, window_grad
from paper_2402_18668_b200 import autograd as ag

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def draw(B, H, L, dtype, seed=0, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(B, H, L, 64, generator=g, device="cuda") * size).to(DT[dtype]) for _ in range(4)]


def check(got, t, w, scale):
    grads, per_h, rest = window_grad(*(x.double() for x in t), w, scale)
    h = half_step(t[0].dtype)
    for name, y, want, a, b in zip(("dq", "dk", "dv"), got, grads, per_h, rest):
        off = h * a + U * b
        # exponentials and products below 2^-126 count as 0: w weights (P, or dS of at most 2 max |dP| scale times as much), each times
        # one of the other factors
        big = max(1.0, *(float(x.abs().max()) for x in t))
        lost = 2.0 ** -126 * w * max(1.0, 2 * 64 * big * big * scale) * big
        close(y, want, off + h * (want.abs() + off) + lost, name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,H,L,w", [(1, 1, 1, 64), (1, 2, 2, 64), (2, 1, 63, 64), (1, 3, 64, 64), (1, 1, 65, 64), (2, 2, 127, 64), (1, 2, 128, 64),
                                     (1, 2, 129, 64), (1, 1, 200, 1), (1, 1, 200, 2), (1, 2, 300, 7), (1, 2, 257, 63), (1, 2, 513, 65),
                                     (2, 3, 384, 128), (1, 2, 700, 100), (1, 1, 1025, 127), (1, 160, 130, 64), (3, 50, 260, 128), (1, 1, 1500, 33),
                                     (2, 20, 1100, 64), (1, 20, 1300, 128)])
def test_against_the_definition(B, H, L, w, dtype):
    t = draw(B, H, L, dtype)
    got = based.swa_backward(*t, window=w)
    check(got, t, w, 0.125)
    assert all(torch.equal(a, b) for a, b in zip(got, based.swa_backward(*t, window=w)))
    assert based.based_poll_error() == based.BASED_OK
    if w == 1 or L == 1:                                     # one key: its weight is 1 whatever its score
        assert (got[0] == 0).all() and (got[1] == 0).all() and torch.equal(got[2], t[3])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale,size", [(0.125, 4.0), (1.0, 2.0), (1e-3, 1.0), (0.125, 0.0)])
def test_scales(scale, size, dtype):
    """Scores far apart (one weight near 1, the others tiny), all alike, and inputs of zero."""
    t = draw(1, 2, 300, dtype, seed=1, size=size)
    check(based.swa_backward(*t, window=64, softmax_scale=scale), t, 64, scale)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_autograd_streams_and_graph(dtype):
    B, H, L, w = 2, 3, 300, 64
    t = draw(B, H, L, dtype, seed=2)
    want = based.swa_backward(*t, window=w)
    leaves = [x.clone().requires_grad_(True) for x in t[:3]]
    out = ag.sliding_window_attention(*leaves, window=w)
    assert torch.equal(out, based.swa_forward(*t[:3], window=w))
    g = t[3].transpose(1, 2).contiguous().transpose(1, 2)    # as it comes back from a projection
    for grad in (t[3], g):
        got = torch.autograd.grad(out, leaves, grad, retain_graph=True)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    with pytest.raises(RuntimeError, match="cannot be differentiated again"):
        torch.autograd.grad(out.float().sum(), leaves, create_graph=True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = based.swa_backward(*t, window=w, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = based.swa_backward(*t, window=w)
    t[0].mul_(0.5)
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(got, based.swa_backward(*t, window=w)))


def test_differences():
    t = draw(1, 2, 150, "f32", seed=3)
    got = based.swa_backward(*t, window=40)
    gen = torch.Generator(device="cuda").manual_seed(4)
    base = [x.double() for x in t]
    for i in range(3):
        v = torch.randn(base[i].shape, generator=gen, device="cuda").double()
        e = 1e-5
        up, down = list(base), list(base)
        up[i], down[i] = base[i] + e * v, base[i] - e * v
        f = lambda x: float((window(x[0], x[1], x[2], 40, 0.125)[0] * base[3]).sum())
        along = got[i].double() * v
        # the differences are good to 1e-8 of the sum's terms; the gradient's terms to about 2000 U (a score's 64 U sum |q k| dominates)
        assert abs((f(up) - f(down)) / (2 * e) - float(along.sum())) <= 1.2e-4 * float(along.abs().sum()) / 10 + 1e-6


def test_many_heads():
    """More heads than a grid has rows are cut into slabs."""
    B, H, L = 1, 65540, 3
    t = draw(B, H, L, "bf16", seed=5)
    got = based.swa_backward(*t, window=2)
    for lo in (0, 65530):
        part = [x[:, lo:lo + 10].contiguous() for x in t]
        check([x[:, lo:lo + 10] for x in got], part, 2, 0.125)


def test_refusals():
    q, k, v, do = draw(1, 2, 70, "bf16")
    f = based.swa_backward
    E, V = based.BasedError, ValueError
    for err, call in ((V, lambda: f(q, k[:, :, :69], v, do)), (V, lambda: f(q, k, v.float(), do)), (V, lambda: f(q, k, v, do[:, :1])),
                      (E, lambda: f(q, k, v, do, window=0)), (E, lambda: f(q, k, v, do, window=129)),
                      (E, lambda: f(*(t[..., :32].contiguous() for t in (q, k, v, do)))), (V, lambda: f(q.cpu(), k, v, do)),
                      (V, lambda: f(q.transpose(2, 3), k, v, do)), (TypeError, lambda: f(q.half(), k.half(), v.half(), do.half())),
                      (V, lambda: f(q, k, v, do, workspace=q))):
        with pytest.raises(err):
            call()
    assert based.based_poll_error() == based.BASED_OK


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layers_in_a_row(dtype):
    """A block as a model would call it: a fused projection, norm and rotation, the sliding window, then the gated recurrence over
    the heads' outputs; its gradients against autograd on the definitions in 64 bits."""
    B, L, H, d, w = 2, 150, 2, 64, 48
    C = H * d
    gen = torch.Generator(device="cuda").manual_seed(6)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    dt = DT[dtype]
    qkv, gates, dout = rnd(B, L, 3 * C).to(dt), rnd(B, L, 2 * C).to(dt), rnd(B, L, C).to(dt)
    wq, wk, rate = 1 + 0.2 * rnd(d), 1 + 0.2 * rnd(d), 0.05 + 0.3 * torch.rand(C, generator=gen, device="cuda")
    freqs = 10000.0 ** (-torch.arange(32, device="cuda", dtype=torch.float64) / 32)

    def run(qkv, gates, wq, wk, rate, own):
        q, k, v = (t.unflatten(-1, (H, d)) for t in qkv.split(C, -1))
        if own:
            q, k = ag.qk_norm_rotate(q, k, wq, wk, freqs)
            x = ag.sliding_window_attention(q, k, v.transpose(1, 2), window=w)
        else:
            pos = torch.arange(L, device="cuda").expand(B, L)
            q, k = (norm_rotate(t, s, freqs, pos, 1e-6, False)[0] for t, s in ((q, wq), (k, wk)))
            x, _ = window(q, k, v.transpose(1, 2), w, 0.125)
        x = x.transpose(1, 2).flatten(2)
        r, g = gates.split(C, -1)
        return ag.gated_recurrence(x, r, g, rate)[0] if own else recurrence(x, r, g, rate)[0]

    a = [t.clone().requires_grad_(True) for t in (qkv, gates, wq, wk, rate)]
    b = [t.double().requires_grad_(True) for t in (qkv, gates, wq, wk, rate)]
    y, z = run(*a, True), run(*b, False)
    ga, gb = torch.autograd.grad(y, a, dout), torch.autograd.grad(z, b, dout.double())
    # every stage rounds its result once (four stages forward, four back), and P and dS too: random roundings of h / sqrt(3) rms each
    # add up to well under 12 h of the whole in the 2-norm
    h = half_step(dt) if dtype == "bf16" else 64 * U
    for p, q in zip((y,) + ga, (z,) + gb):
        assert p.dtype in (dt, torch.float32) and float((p.detach().double() - q.detach()).norm() / q.detach().norm()) <= 12 * h


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_generation_follows_the_sequence(dtype):
    """Token by token: norm and rotation at the sequences' own positions, the window's step on its rolling cache and the recurrence's
    step give what the calls over the whole sequence give."""
    B, L, H, d, w = 3, 90, 2, 64, 32
    C = H * d
    gen = torch.Generator(device="cuda").manual_seed(7)
    dt = DT[dtype]
    qkv, gates = torch.randn(B, L, 3 * C, generator=gen, device="cuda").to(dt), torch.randn(B, L, 2 * C, generator=gen, device="cuda").to(dt)
    rate = 0.05 + 0.3 * torch.rand(C, generator=gen, device="cuda")
    freqs = 10000.0 ** (-torch.arange(32, device="cuda", dtype=torch.float64) / 32)
    q, k, v = (t.unflatten(-1, (H, d)) for t in qkv.split(C, -1))
    yq, yk = based.based_qk_norm_rotate(q, k, freqs=freqs)
    x = based.swa_forward(yq, yk, v.transpose(1, 2).contiguous(), window=w).transpose(1, 2).flatten(2)
    r, g = (t.contiguous() for t in gates.split(C, -1))
    want = based.based_gated_recurrence_forward(x, r, g, rate)
    kc, vc = (torch.zeros(B, H, w, d, device="cuda", dtype=dt) for _ in range(2))
    state = torch.zeros(B, C, device="cuda")
    pos = torch.zeros(B, device="cuda", dtype=torch.int32)
    got = []
    for t in range(L):
        tq, tk = based.based_qk_norm_rotate(q[:, t:t + 1], k[:, t:t + 1], freqs=freqs, positions=pos)
        assert torch.equal(tq[:, :, 0], yq[:, :, t]) and torch.equal(tk[:, :, 0], yk[:, :, t])
        o = based.swa_decode_step_ragged(tq[:, :, 0].contiguous(), tk[:, :, 0].contiguous(), v[:, t].contiguous(), kc, vc, pos)
        got.append(based.based_gated_recurrence_step(o.flatten(1), r[:, t].contiguous(), g[:, t].contiguous(), rate, state))
        pos += 1
    got = torch.stack(got, 1).double()
    # the window's output is rounded in both (from weights that were rounded to bf16 in one), the recurrence's once more
    h = half_step(dt) if dtype == "bf16" else 64 * U
    assert float((got - want.double()).norm() / want.double().norm()) <= 4 * h
