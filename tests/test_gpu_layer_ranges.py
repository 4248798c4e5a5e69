"""The recurrence, the rotation and the window's backward pass where a CTA goes several rounds, under capture through autograd, and two
calls at once.  Bounds are those of the operators' own tests, whose checks are used.
"""
import pytest
import torch

import paper_2402_18668_b200 as based
import test_gpu_norm_rotate as rotation
import test_gpu_swa_backward as sliding
from paper_2402_18668_b200 import autograd as ag

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", [(3, 7001, 3, 1, 32, 8, False, "tokens"), (1, 20011, 2, 1, 256, 128, False, "range"),
                                  (2, 6007, 1, 5, 48, 16, True, "sequences"), (1, 9500, 33, 2, 16, 8, False, "start")])
def test_rotation_in_several_rounds(case, dtype):
    rotation.test_forward_and_backward(*case, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,H,L,w", [(2, 40, 1300, 128), (2, 40, 1283, 64), (1, 3, 5003, 100), (4, 64, 130, 127), (300, 1, 129, 64),
                                     (1, 8, 700, 64), (1, 8, 1100, 60), (2, 4, 290, 128), (1, 8, 700, 128)])
def test_window_in_several_rounds(B, H, L, w, dtype):
    t = sliding.draw(B, H, L, dtype, seed=11)
    got = based.swa_backward(*t, window=w)
    for lo in range(0, B):                                   # a sequence at a time: the definition takes [L,L] of each head
        sliding.check([x[lo:lo + 1] for x in got], [x[lo:lo + 1] for x in t], w, 0.125)
        if lo == 3:
            break
    sliding.check([x[-1:] for x in got], [x[-1:] for x in t], w, 0.125)
    assert all(torch.equal(a, b) for a, b in zip(got, based.swa_backward(*t, window=w)))
    assert based.based_poll_error() == based.BASED_OK


def layers(x, qkv, r, g, rate, wq, freqs):
    """One value of all three layers in a row: qkv [B,L,3,H,64], x, r, g [B,L,H 64]."""
    qh, kh = ag.qk_norm_rotate(qkv[:, :, 0], qkv[:, :, 1], wq, wq, freqs)
    o = ag.sliding_window_attention(qh, kh, qkv[:, :, 2].transpose(1, 2), window=100)
    h, last = ag.gated_recurrence(x + o.transpose(1, 2).flatten(2), r, g, rate)
    return h.float().square().mean() + last.mean()


def leaves(seed, B=2, L=333, H=3):
    rnd = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=rnd, device="cuda")
    t = [n(B, L, H * 64).bfloat16(), n(B, L, 3, H, 64).bfloat16(), n(B, L, H * 64).bfloat16(), n(B, L, H * 64).bfloat16(),
         torch.rand(H * 64, generator=rnd, device="cuda"), 1 + 0.1 * n(64)]
    return [x.requires_grad_(True) for x in t], 100.0 ** -torch.linspace(0, 1, 32, device="cuda", dtype=torch.float64)


def test_backward_under_capture():
    t, freqs = leaves(1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(layers(*t, freqs), t)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = torch.autograd.grad(layers(*t, freqs), t)
    for seed in (1, 2):
        with torch.no_grad():
            for x, y in zip(t, leaves(seed)[0]):
                x.copy_(y)
        graph.replay()
        want = torch.autograd.grad(layers(*t, freqs), t)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert based.based_poll_error() == based.BASED_OK


def test_two_streams_at_once():
    sets = [leaves(s) for s in (3, 4)]
    want = [torch.autograd.grad(layers(*t, f), t) for t, f in sets]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, (t, f) in enumerate(sets):
            with torch.cuda.stream(streams[i]):
                got[i].append(torch.autograd.grad(layers(*t, f), t))
    torch.cuda.synchronize()
    for i in range(2):
        for d in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(d, want[i]))
    assert based.based_poll_error() == based.BASED_OK


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_same_tensor_twice(dtype):
    """One tensor as queries, keys and values, as all gates, and as both halves of the rotation."""
    dt = sliding.DT[dtype]
    t = sliding.draw(2, 3, 200, dtype, seed=5)[0]
    sliding.check(based.swa_backward(t, t, t, t, window=64), [t] * 4, 64, 0.125)
    x = torch.randn(2, 50, 64, device="cuda").to(dt)
    rate = torch.full((64,), 0.5, device="cuda")
    y = based.based_gated_recurrence_forward(x, x, x, rate)
    assert torch.equal(y, based.based_gated_recurrence_forward(x, x.clone(), x.clone(), rate))
    assert all(a is None or torch.equal(a, b) for a, b in zip(based.based_gated_recurrence_backward(x, x, x, rate, y, y),
                                                             based.based_gated_recurrence_backward(x, x.clone(), x.clone(), rate, y, y.clone())))
    q = torch.randn(2, 9, 4, 64, device="cuda").to(dt)
    a, b = based.based_qk_norm_rotate(q, q)
    assert torch.equal(a, b)
