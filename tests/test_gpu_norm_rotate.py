"""The norm of queries and keys with the position rotation against its definition in 64 bits.

Bounds.  The sum of squares of d values, the reciprocal root and two products are off by at most (d / 8 + 8) U relative (partial sums of
d / 8 terms or fewer, then a tree), a sine or cosine by 4 U absolute plus the rounding of the part of a turn, pi U; a turned element
is therefore off by that much of the pair's size.  (d / 8 + 32) U covers them.  Results are rounded once.
"""
import pytest
import torch

import paper_2402_18668_b200 as based
from layers64 import U, close, half_step, norm_rotate
from paper_2402_18668_b200 import autograd as ag

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def draw(B, L, Hq, Hk, d, n, dtype, where, seed=0, fused=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    if fused:
        t = rnd(B, L, (Hq + 2 * Hk) * d).to(DT[dtype])
        q, k = t[..., :Hq * d].unflatten(-1, (Hq, d)), t[..., Hq * d:(Hq + Hk) * d].unflatten(-1, (Hk, d))
    else:
        q, k = rnd(B, L, Hq, d).to(DT[dtype]), rnd(B, L, Hk, d).to(DT[dtype])
    wq, wk = 1 + 0.3 * rnd(d), 1 + 0.3 * rnd(d)
    freqs = 10000.0 ** (-torch.arange(n, device="cuda", dtype=torch.float64) / n) if n else None
    pos, start = None, 0
    at = torch.arange(L, device="cuda").expand(B, L)
    if where == "start":
        start, at = 123456, at + 123456
    elif where == "sequences":
        pos = torch.randint(0, 1 << 20, (B,), generator=g, device="cuda", dtype=torch.int32)
        at = at + pos[:, None]
    elif where == "tokens":
        pos = torch.randint(-5, 1 << 30, (B, L), generator=g, device="cuda", dtype=torch.int32)
        at = pos
    return q, k, wq, wk, freqs, pos, start, at, rnd


CASES = [  # B, L, Hq, Hk, d, n, pairs, where
    (1, 1, 1, 1, 16, 0, False, "range"), (2, 5, 3, 1, 16, 8, False, "tokens"), (2, 5, 3, 1, 16, 8, True, "tokens"),
    (1, 1, 16, 16, 64, 32, False, "sequences"), (128, 1, 16, 16, 64, 32, False, "sequences"), (7, 1, 4, 2, 64, 16, True, "sequences"),
    (3, 100, 8, 2, 112, 56, False, "start"), (2, 33, 5, 5, 128, 64, False, "range"), (2, 33, 5, 5, 128, 32, True, "tokens"),
    (1, 1000, 16, 4, 64, 24, False, "tokens"), (2, 17, 2, 3, 256, 128, False, "range"), (2, 17, 2, 3, 256, 40, True, "start"),
    (1, 9, 2, 2, 48, 24, False, "sequences"), (1, 9, 2, 2, 48, 8, True, "sequences"), (1, 9, 40, 2, 240, 0, False, "range"),
    (1, 7000, 2, 1, 32, 16, False, "range")]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,L,Hq,Hk,d,n,pairs,where", CASES)
def test_forward_and_backward(B, L, Hq, Hk, d, n, pairs, where, dtype):
    q, k, wq, wk, freqs, pos, start, at, rnd = draw(B, L, Hq, Hk, d, n, dtype, where)
    flags = based.BASED_ROTATE_PAIRS if pairs else 0
    eps = 1e-5
    got = based.based_qk_norm_rotate(q, k, wq, wk, freqs, pos, eps=eps, flags=flags, start=start)
    h, c = half_step(q.dtype), (d / 8 + 32) * U
    for y, x, w in zip(got, (q, k), (wq, wk)):
        want, size = norm_rotate(x.double(), w.double(), freqs, at, eps, pairs)
        close(y, want, c * size + h * (want.abs() + c * size), "y")
    # backward: the definition's gradient by autograd in 64 bits
    gq, gk = rnd(B, Hq, L, d).to(q.dtype), rnd(B, Hk, L, d).to(q.dtype)
    grads = based.based_qk_norm_rotate_backward(q, k, gq, gk, wq, wk, freqs, pos, eps=eps, flags=flags, start=start)
    for x, w, g, dx, dw in ((q, wq, gq, grads[0], grads[2]), (k, wk, gk, grads[1], grads[3])):
        xl, wl = x.double().clone().requires_grad_(True), w.double().clone().requires_grad_(True)
        y, _ = norm_rotate(xl, wl, freqs, at, eps, pairs)
        want_x, want_w = torch.autograd.grad(y, (xl, wl), g.double())
        # dx = inv (w e - x inv^2 mean(w e x)): every term to a few c of the row's size of it
        inv = torch.rsqrt((x.double() ** 2).mean(-1, keepdim=True) + eps)
        e = (1.4143 * g.double().abs().amax(-1, keepdim=True)).transpose(1, 2)
        off = 4 * c * inv * e * w.double().abs().max() * (1 + (x.double() * inv).abs())
        close(dx, want_x, off + h * (want_x.abs() + off), "dx")
        # (a thread sums its rows in a chain: at most rows x heads / 128 of them and a block more, then trees)
        terms = (e * (x.double() * inv).abs()).sum((0, 1, 2))
        close(dw, want_w, (4 * c + (x.shape[1] * B * x.shape[2] / 128 + 64) * U) * terms, "dw")
        assert dx.shape == x.shape and dx.is_contiguous()
    again = based.based_qk_norm_rotate_backward(q, k, gq, gk, wq, wk, freqs, pos, eps=eps, flags=flags, start=start)
    assert all(torch.equal(a, b) for a, b in zip(grads, again))
    assert based.based_poll_error() == based.BASED_OK


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layouts_agree(dtype):
    """Slices of a fused projection, contiguous tensors, gradients into slices of one gradient, and tokens one by one."""
    B, L, Hq, Hk, d, n = 3, 21, 4, 2, 64, 32
    q, k, wq, wk, freqs, pos, start, at, rnd = draw(B, L, Hq, Hk, d, n, dtype, "tokens", seed=1)
    a = based.based_qk_norm_rotate(q, k, wq, wk, freqs, pos)
    b = based.based_qk_norm_rotate(q.contiguous(), k.contiguous(), wq, wk, freqs, pos)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    gq, gk = rnd(B, Hq, L, d).to(q.dtype), rnd(B, Hk, L, d).to(q.dtype)
    want = based.based_qk_norm_rotate_backward(q, k, gq, gk, wq, wk, freqs, pos)
    fused = torch.full((B, L, (Hq + 2 * Hk) * d), 9.0, device="cuda", dtype=q.dtype)
    dq, dk = fused[..., :Hq * d].unflatten(-1, (Hq, d)), fused[..., Hq * d:(Hq + Hk) * d].unflatten(-1, (Hk, d))
    got = based.based_qk_norm_rotate_backward(q, k, gq, gk, wq, wk, freqs, pos, dq=dq, dk=dk)
    assert all(torch.equal(x, y) for x, y in zip(got, want)) and torch.equal(dq, want[0]) and torch.equal(dk, want[1])
    assert (fused[..., (Hq + Hk) * d:] == 9).all()
    for t in (0, 7, L - 1):                                  # tokens one by one, at positions of their own
        one = based.based_qk_norm_rotate(q[:, t:t + 1], k[:, t:t + 1], wq, wk, freqs, pos[:, t].contiguous())
        assert all(torch.equal(x[:, :, 0], y[:, :, t]) for x, y in zip(one, a))
    none = based.based_qk_norm_rotate(q, k, None, None, freqs, pos)
    ones = based.based_qk_norm_rotate(q, k, torch.ones(d, device="cuda"), torch.ones(d, device="cuda"), freqs, pos)
    assert all(torch.equal(x, y) for x, y in zip(none, ones))
    g = based.based_qk_norm_rotate_backward(q, k, gq, gk, None, wk, freqs, pos)
    assert g[2] is None and torch.equal(g[3], want[3])


def test_empty_and_unfinite_rows():
    """A row of zeros stays zeros (eps > 0), with a finite gradient; a row that is not finite reaches no other."""
    q, k, wq, wk, freqs, pos, start, at, rnd = draw(2, 12, 4, 4, 64, 32, "bf16", "range", seed=2)
    want = based.based_qk_norm_rotate(q, k, wq, wk, freqs)
    q[0, 3, 1] = 0
    q[1, 5, 2, 7] = float("nan")
    q[1, 6, 2, 7] = float("inf")
    got = based.based_qk_norm_rotate(q, k, wq, wk, freqs)
    assert (got[0][0, 1, 3] == 0).all()
    assert torch.isnan(got[0][1, 2, 5]).all()
    mask = torch.ones(2, 4, 12, dtype=torch.bool, device="cuda")
    mask[0, 1, 3] = mask[1, 2, 5] = mask[1, 2, 6] = False
    assert torch.equal(got[0][mask], want[0][mask]) and torch.equal(got[1], want[1])
    g = torch.randn(2, 4, 12, 64, device="cuda").bfloat16()
    d = based.based_qk_norm_rotate_backward(q, k, g, g, None, None, freqs)
    assert torch.isfinite(d[0].transpose(1, 2)[mask]).all() and torch.isfinite(d[0][0, 3, 1]).all()


def test_autograd_and_graph():
    B, L, H, d, n = 2, 50, 4, 64, 32
    q, k, wq, wk, freqs, pos, start, at, rnd = draw(B, L, H, H, d, n, "bf16", "sequences", seed=3)
    gq, gk = rnd(B, H, L, d).to(q.dtype), rnd(B, H, L, d).to(q.dtype)
    want = based.based_qk_norm_rotate_backward(q, k, gq, gk, wq, wk, freqs, pos)
    proj = torch.cat([q.flatten(2), k.flatten(2)], -1).requires_grad_(True)
    leaves = [wq.clone().requires_grad_(True), wk.clone().requires_grad_(True)]
    yq, yk = ag.qk_norm_rotate(proj[..., :H * d].unflatten(-1, (H, d)), proj[..., H * d:].unflatten(-1, (H, d)), *leaves, freqs, pos)
    torch.autograd.backward([yq, yk], [gq, gk])
    assert torch.equal(proj.grad, torch.cat([want[0].flatten(2), want[1].flatten(2)], -1))
    assert torch.equal(leaves[0].grad, want[2]) and torch.equal(leaves[1].grad, want[3])
    # only the queries' output used; weights that need no gradient
    ql = q.contiguous().requires_grad_(True)
    yq, _ = ag.qk_norm_rotate(ql, k, wq, wk, freqs, pos)
    (dq,) = torch.autograd.grad(yq, ql, gq)
    assert torch.equal(dq, want[0])
    with pytest.raises(RuntimeError, match="cannot be differentiated again"):
        torch.autograd.grad(ag.qk_norm_rotate(ql, k, wq, wk, freqs, pos)[0].float().sum(), ql, create_graph=True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = based.based_qk_norm_rotate(q, k, wq, wk, freqs, pos)
        g = based.based_qk_norm_rotate_backward(q, k, gq, gk, wq, wk, freqs, pos)
    pos.add_(1000)
    q.mul_(0.5)
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(y, based.based_qk_norm_rotate(q, k, wq, wk, freqs, pos)))
    assert all(torch.equal(a, b) for a, b in zip(g, based.based_qk_norm_rotate_backward(q, k, gq, gk, wq, wk, freqs, pos)))


def test_differences():
    """The gradient along random directions against central differences of the definition in 64 bits."""
    B, L, H, d, n = 2, 9, 3, 32, 8
    q, k, wq, wk, freqs, pos, start, at, rnd = draw(B, L, H, H, d, n, "f32", "tokens", seed=4)
    gq, gk = rnd(B, H, L, d), rnd(B, H, L, d)
    got = based.based_qk_norm_rotate_backward(q, k, gq, gk, wq, wk, freqs, pos, flags=based.BASED_ROTATE_PAIRS)
    base = [t.double() for t in (q, k, wq, wk)]

    def f(t):
        return float((norm_rotate(t[0], t[2], freqs, at, 1e-6, True)[0] * gq.double()).sum() +
                     (norm_rotate(t[1], t[3], freqs, at, 1e-6, True)[0] * gk.double()).sum())

    for i in range(4):
        v = rnd(*base[i].shape).double()
        e = 1e-5
        up, down = list(base), list(base)
        up[i], down[i] = base[i] + e * v, base[i] - e * v
        along = got[i].double() * v
        # the differences are good to 1e-8 of the sum's terms, the gradient to 8 (d / 8 + 32) U = 2e-5 of them
        assert abs((f(up) - f(down)) / (2 * e) - float(along.sum())) <= 2e-5 * float(along.abs().sum()) + 1e-6


def test_refusals():
    q, k, wq, wk, freqs, pos, start, at, rnd = draw(2, 6, 4, 2, 64, 32, "bf16", "tokens", fused=False)
    f, b = based.based_qk_norm_rotate, based.based_qk_norm_rotate_backward
    E, V = based.BasedError, ValueError
    gq, gk = q.transpose(1, 2).contiguous(), k.transpose(1, 2).contiguous()
    one = torch.empty(2, 6, 4, 64, device="cuda", dtype=q.dtype)
    for err, call in (
            (V, lambda: f(q, k[:, :5], wq, wk, freqs, pos)), (V, lambda: f(q, k.float(), wq, wk, freqs, pos)),
            (V, lambda: f(q, k, wq[:32], wk, freqs, pos)), (TypeError, lambda: f(q, k, wq.bfloat16(), wk, freqs, pos)),
            (TypeError, lambda: f(q, k, wq, wk, freqs.float(), pos)), (V, lambda: f(q, k, wq, wk, freqs, pos.long())),
            (V, lambda: f(q, k, wq, wk, freqs, pos[:, :5].contiguous())), (V, lambda: f(q, k, wq, wk, freqs, pos, start=3)),
            (E, lambda: f(q, k, wq, wk, freqs, pos, flags=1)), (E, lambda: f(q, k, wq, wk, freqs, pos, eps=-1.0)),
            (E, lambda: f(q, k, wq, wk, freqs, pos, eps=float("nan"))), (E, lambda: f(q, k, wq, wk, freqs[:31].contiguous(), pos)),
            (E, lambda: f(q, k, wq, wk, torch.ones(40, device="cuda", dtype=torch.float64), pos)),
            (E, lambda: f(q[..., :40].contiguous(), k[..., :40].contiguous())), (V, lambda: f(gq, k)),
            (V, lambda: f(q.transpose(1, 2), k.transpose(1, 2))),
            (V, lambda: f(q[..., ::2], k[..., ::2])), (V, lambda: f(q.cpu(), k)), (TypeError, lambda: f(q.half(), k.half())),
            (V, lambda: f(q, k, out_q=q)), (V, lambda: f(q, k, out_q=one.view(2, 4, 6, 64)[:, :3])),
            (V, lambda: f(q, k, out_q=one.view(2, 4, 6, 64), out_k=one.view(-1)[:2 * 2 * 6 * 64].view(2, 2, 6, 64))),
            (V, lambda: b(q, k, q, k)), (V, lambda: b(q, k, gq, gk, dq=q)), (V, lambda: b(q, k, gq, gk, dq=one, dk=one[:, :, 1:3])),
            # a row that starts off the 16-byte grid
            (E, lambda: f(torch.zeros(2, 6, 264, device="cuda", dtype=q.dtype)[..., 1:257].unflatten(-1, (4, 64)), k))):
        with pytest.raises(err):
            call()
    assert based.based_poll_error() == based.BASED_OK
