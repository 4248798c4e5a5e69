"""The gated recurrence, the norm with rotation and the sliding window from their definitions, in 64 bits (torch, any device)."""
import math

import torch

U = 2.0 ** -24                     # half a step of fp32, relative


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def recurrence(x, r, g, rate, h0=None):
    """h [B,N,C], token by token; and a, m, i (fp64)."""
    la = -rate * torch.sigmoid(r)
    a = torch.exp(la)
    m = torch.sqrt(-torch.expm1(2 * la))
    i = torch.sigmoid(g)
    h = torch.zeros_like(x[:, 0]) if h0 is None else h0
    out = []
    for t in range(x.shape[1]):
        h = a[:, t] * h + m[:, t] * i[:, t] * x[:, t]
        out.append(h)
    return torch.stack(out, 1), a, m, i


def recurrence_grad(x, r, g, rate, h0, out, dout, dh):
    """The formulas of the gradient, with the kept output's values, and the size of dr's and drate's terms."""
    _, a, m, i = recurrence(x, r, g, rate, h0)
    s = torch.sigmoid(r)
    up = torch.zeros_like(x[:, 0]) if dh is None else dh
    G = torch.empty_like(x)
    for t in reversed(range(x.shape[1])):
        G[:, t] = dout[:, t] + up
        up = a[:, t] * G[:, t]
    first = torch.zeros_like(x[:, :1]) if h0 is None else h0[:, None]
    prev = torch.cat([first, out[:, :-1]], 1)
    one, two = a * G * prev, a * a / m * G * i * x
    dla = one - two
    return {"dx": G * m * i, "dr": -rate * dla * s * (1 - s), "dg": G * m * x * i * (1 - i), "drate": -(dla * s).sum((0, 1)),
            "dh0": up, "G": G, "a": a, "m": m, "i": i, "s": s, "prev": prev}


def norm_rotate(x, w, freqs, pos, eps, pairs):
    """x [B,L,H,d] -> y [B,H,L,d], and the size of a pair's elements at every element."""
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    if w is not None:
        y = y * w
    size = y.abs()
    if freqs is not None:
        n = freqs.shape[0]
        t = (pos[..., None].double() * freqs)[:, :, None]
        c, s = torch.cos(t), torch.sin(t)
        lo, hi = (y[..., 0:2 * n:2], y[..., 1:2 * n:2]) if pairs else (y[..., :n], y[..., n:2 * n])
        new = (lo * c - hi * s, hi * c + lo * s)
        both = torch.sqrt(lo * lo + hi * hi)
        join = (lambda p: torch.stack(p, -1).flatten(-2)) if pairs else (lambda p: torch.cat(p, -1))
        size = torch.cat([join((both, both)), size[..., 2 * n:]], -1)
        y = torch.cat([join(new), y[..., 2 * n:]], -1)
    return y.transpose(1, 2), size.transpose(1, 2)


def window(q, k, v, w, scale):
    """out and P of the sliding window, [B,H,L,L]."""
    L = q.shape[2]
    i = torch.arange(L, device=q.device)
    seen = (i[None] <= i[:, None]) & (i[None] > i[:, None] - w)
    s = (scale * q @ k.transpose(2, 3)).masked_fill(~seen, -math.inf)
    P = torch.softmax(s, -1)
    return P @ v, P


def window_grad(q, k, v, dout, w, scale):
    """dq, dk, dv; bounds on what rounding P and dS to a type with half step h does to them, per h; and bounds on the
    rest (fp32 sums of 64 products, exponentials), per U."""
    _, P = window(q, k, v, w, scale)
    dP = dout @ v.transpose(2, 3)
    D = (P * dP).sum(-1, keepdim=True)
    dS = scale * P * (dP - D)
    grads = (dS @ k, dS.transpose(2, 3) @ q, P.transpose(2, 3) @ dout)
    per_h = (dS.abs() @ k.abs(), dS.abs().transpose(2, 3) @ q.abs(), P.transpose(2, 3) @ dout.abs())
    # a score is off by 64 U sum |q k|, so a weight by twice scale times the largest of that in its row (its own and its row's sum),
    # relatively, and 64 U more of the exponential and the sum; dP by 64 U sum |dout v|; D by both; then 256 U of the sums over tokens
    rel = 2 * scale * 64 * (q.abs() @ k.abs().transpose(2, 3)).masked_fill(P == 0, 0).amax(-1, keepdim=True) + 64
    dp = 64 * (dout.abs() @ v.abs().transpose(2, 3))
    D_off = (P * (dp + rel * dP.abs())).sum(-1, keepdim=True)
    off = scale * P * (dp + D_off) + dS.abs() * (rel + 256)
    rest = (off @ k.abs(), off.transpose(2, 3) @ q.abs(), (P * (rel + 256)).transpose(2, 3) @ dout.abs())
    return grads, per_h, rest


def close(got, want, bound, what=""):
    """Elementwise, and finite."""
    got = got.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert torch.isfinite(got).all(), what
    over = (got - want).abs() - bound
    assert (over <= 0).all(), (f"{what}: {float((over > 0).double().mean()):.2%} over; worst off by "
                               f"{float(((got - want).abs() / bound.expand_as(want).clamp_min(1e-300)).max()):.2f} bounds")
