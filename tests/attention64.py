"""Decay attention and attention over a paged cache from their definitions, in 64 bits (torch, any device), and bounds on what rounding may
change: every formula is run a second time on absolute values, which gives the size of the terms that it sums."""
import math

import torch

U = 2.0 ** -24                     # half a step of fp32, relative


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def _steps(documents, B, L):
    """Per token [L,B]: whether it counts, and whether the state goes on to it (it is no other document's than the last that counts)."""
    live, keep = torch.ones(L, B, dtype=torch.float64), torch.ones(L, B, dtype=torch.float64)
    if documents is not None:
        for b, row in enumerate(documents.tolist()):
            seen = None
            for t, x in enumerate(row):
                if x < 0:
                    live[t, b] = 0
                else:
                    keep[t, b] = float(seen is None or seen == x)
                    seen = x
    return live, keep


def _fade(rate, live, keep, device):
    """What a token leaves of the state ahead of it, [L,B,H,1,1]; padding leaves it."""
    live, keep = live.to(device)[:, :, None, None, None], keep.to(device)[:, :, None, None, None]
    return torch.where(live > 0, keep * torch.exp(-rate.double())[:, None, None], torch.ones((), dtype=torch.float64, device=device))


def _clean(x, live):
    """[B,H,L,d] -> [L,B,H,d] fp64, rows of padding 0 whatever they hold."""
    x = x.double().permute(2, 0, 1, 3)
    return torch.where(live.to(x.device)[:, :, None, None] > 0, x, torch.zeros((), dtype=torch.float64, device=x.device))


def decay(q, k, v, rate, documents=None, state=None, scale=None):
    """out [B,H,L,d_v], the state behind the last token."""
    B, H, L, dk = q.shape
    scale = dk ** -0.5 if scale is None else scale
    live, keep = _steps(documents, B, L)
    fade = _fade(rate, live, keep, q.device)
    q, k, v = (_clean(x, live) for x in (q, k, v))
    S = torch.zeros(B, H, dk, v.shape[-1], dtype=torch.float64, device=q.device) if state is None else state.double().clone()
    out = torch.empty_like(v)
    for t in range(L):
        S = torch.where(fade[t] > 0, S * fade[t], torch.zeros_like(S)) + k[t][..., None] * v[t][..., None, :]
        out[t] = scale * (q[t][..., None, :] @ S)[..., 0, :]
    return out.permute(1, 2, 0, 3), S


def decay_grad(q, k, v, rate, dout, documents=None, state=None, dstate=None, scale=None):
    """dq, dk, dv, and the gradient of the state before the first token."""
    B, H, L, dk = q.shape
    scale = dk ** -0.5 if scale is None else scale
    live, keep = _steps(documents, B, L)
    fade = _fade(rate, live, keep, q.device)
    q, k, v, do = (_clean(x, live) for x in (q, k, v, dout))
    S = torch.zeros(B, H, dk, v.shape[-1], dtype=torch.float64, device=q.device) if state is None else state.double().clone()
    dq, dk_, dv = torch.empty_like(q), torch.empty_like(q), torch.empty_like(v)
    for t in range(L):
        S = S * fade[t] + k[t][..., None] * v[t][..., None, :]
        dq[t] = scale * (S @ do[t][..., None])[..., 0]
    R = torch.zeros_like(S) if dstate is None else dstate.double().clone()
    for t in reversed(range(L)):
        R = R + scale * q[t][..., None] * do[t][..., None, :]
        dk_[t] = (R @ v[t][..., None])[..., 0]
        dv[t] = (k[t][..., None, :] @ R)[..., 0, :]
        R = R * fade[t]
    live = live.to(q.device)[:, :, None, None]
    return [(x * live).permute(1, 2, 0, 3) for x in (dq, dk_, dv)] + [R]


def decay_bound(size, exact, dtype, d, L):
    """By how much a result of `size` (the formula on absolute values) may be off.  fp32 arithmetic: a product of d terms, one over the up to
    128 tokens of a block, a step of the state per block of 64, weights whose exponent (below 40 where they matter) is rounded twice: each
    worst rounding adds up, twice over for what is formed of both.  bf16 io besides: the scores' or the state's rounding as operands (half a step
    of every term), 2^-15 of what goes into the state, and half a step of the result."""
    bound = 2 * U * (d + 128 + 2 * (L // 64 + 1) + 80) * size
    if dtype == torch.bfloat16:
        u = half_step(dtype)
        bound = bound + (u + 2.0 ** -14) * size * (1 + u) + u * exact.abs()
    else:
        bound = bound + U * exact.abs()
    return bound + 1e-30


def state_bound(size, L):
    """The state is fp32 in either io type, what goes into it has 24 bits (bf16 io: in three parts of 8)."""
    return 2 * U * (128 + 2 * (L // 64 + 1) + 80) * size + 1e-30


def paged(q, k, v, k_pages, v_pages, table, pos, scale=None, cap=0.0, slopes=None, window=0):
    """out [B,Hq,d] in 64 bits, its bound, and the pools with the new tokens in place."""
    B, Hq, d = q.shape
    P, Hk, ps, _ = k_pages.shape
    scale = d ** -0.5 if scale is None else scale
    kp, vp = k_pages.clone(), v_pages.clone()
    out, bound = torch.zeros(B, Hq, d, dtype=torch.float64, device=q.device), torch.zeros(B, Hq, d, dtype=torch.float64, device=q.device)
    u = half_step(q.dtype)
    for b in range(B):
        p = int(pos[b])
        if p < 0:
            continue
        page = int(table[b, p // ps])
        kp[page, :, p % ps], vp[page, :, p % ps] = k[b], v[b]
        lo = max(0, p + 1 - window) if window else 0
        at = table[b, :p // ps + 1].long()
        K = kp[at].transpose(0, 1).reshape(Hk, -1, d)[:, lo:p + 1].double()
        V = vp[at].transpose(0, 1).reshape(Hk, -1, d)[:, lo:p + 1].double()
        Q = q[b].double().view(Hk, Hq // Hk, d)
        s = scale * torch.einsum("hgd,hnd->hgn", Q, K)
        # how far a score may be off: its product's d + 2 roundings, the cap's function, the bias and the step to base 2
        off = U * (d + 4) * scale * torch.einsum("hgd,hnd->hgn", Q.abs(), K.abs())
        if cap:
            s = cap * torch.tanh(s / cap)
            off = off + (1e-6 if q.dtype == torch.bfloat16 else 4 * U) * s.abs()
        if slopes is not None:
            far = slopes.double().view(Hk, -1, 1) * (p - torch.arange(lo, p + 1, device=q.device, dtype=torch.float64))
            s = s - far
            off = off + 2 * U * far
        off = off + 4 * U * s.abs()
        w = torch.softmax(s, -1)
        y = torch.einsum("hgn,hnd->hgd", w, V)
        size = torch.einsum("hgn,hnd->hgd", w * (2 * off + 2 * off.amax(-1, keepdim=True) + 2 * U * (p + 1 - lo + 64) + 2.0 ** -20), V.abs())
        if q.dtype == torch.bfloat16:
            size = size + u * torch.einsum("hgn,hnd->hgd", w, V.abs())
        out[b], bound[b] = y.reshape(Hq, d), (size + u * y.abs() + 1e-30).reshape(Hq, d)
    return out, bound, kp, vp
