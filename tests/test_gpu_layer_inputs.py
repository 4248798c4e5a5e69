"""The layers' autograd functions take any tensor of their shapes: a start off the 16-byte grid, strides that the kernels cannot take."""
import pytest
import torch

from paper_2402_18668_b200 import autograd as ag

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def shifted(t):
    """The same values, contiguous, one element behind the start of their storage."""
    room = torch.empty(t.numel() + 1, device="cuda", dtype=t.dtype)
    return room[1:].view(t.shape).copy_(t)


def same(f, args, grads, views):
    """f of the views, and their gradients, against f of the tensors themselves."""
    res = []
    for give in (False, True):
        leaves = [None if a is None else a.clone().requires_grad_(True) for a in args]
        ins = [None if a is None else view(a) if give else a for a, view in zip(leaves, views)]
        outs = f(*ins)
        outs = outs if isinstance(outs, tuple) else (outs,)
        gs = [shifted(g) if give else g for g in grads]
        res.append((outs, torch.autograd.grad(outs, [a for a in leaves if a is not None], gs)))
    for a, b in zip(res[0][0] + res[0][1], res[1][0] + res[1][1]):
        assert torch.equal(a, b)


class Shift(torch.autograd.Function):
    """shifted() within a graph."""

    @staticmethod
    def forward(ctx, t):
        return shifted(t)

    @staticmethod
    def backward(ctx, g):
        return g


def odd_rows(t):
    """The same values in rows that lie an odd number of elements apart."""
    return torch.cat([t.flatten(2), t.flatten(2)[..., :3]], -1)[..., :t.shape[2] * t.shape[3]].unflatten(-1, t.shape[2:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_recurrence(dtype):
    n = lambda *s: torch.randn(*s, device="cuda")
    x, r, g, dout = (n(2, 50, 24).to(DT[dtype]) for _ in range(4))
    same(ag.gated_recurrence, [x, r, g, torch.rand(24, device="cuda"), n(2, 24)], [dout, n(2, 24)], [Shift.apply] * 5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("view", [Shift.apply, odd_rows])
def test_rotation(view, dtype):
    n = lambda *s: torch.randn(*s, device="cuda")
    q, k = n(2, 30, 4, 32).to(DT[dtype]), n(2, 30, 2, 32).to(DT[dtype])
    freqs = shifted(100.0 ** -torch.linspace(0, 1, 8, device="cuda", dtype=torch.float64))
    pos = shifted(torch.randint(0, 1000, (2, 30), device="cuda", dtype=torch.int32))
    same(lambda a, b, c, d: ag.qk_norm_rotate(a, b, c, d, freqs, pos), [q, k, 1 + n(32), 1 + n(32)],
         [n(2, 4, 30, 32).to(q.dtype), n(2, 2, 30, 32).to(q.dtype)], [view, view, Shift.apply, Shift.apply])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_window(dtype):
    t = [torch.randn(2, 3, 100, 64, device="cuda").to(DT[dtype]) for _ in range(4)]
    same(lambda q, k, v: ag.sliding_window_attention(q, k, v, window=40), t[:3], t[3:], [Shift.apply] * 3)
