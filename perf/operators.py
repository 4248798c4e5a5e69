"""Cases and plain forms of the operators around the mixers: the gated linear recurrence (whole sequence, one token, backward),
the norm of queries and keys with the position rotation (whole sequence, one token, backward) and the backward pass of the
sliding window.

    gated recurrence, per sequence and channel, from h_0 (or 0):
        s = sigmoid(r), a = exp(-rate s), m = sqrt(1 - a^2),     h_t = a_t h_{t-1} + m_t sigmoid(g_t) x_t
    norm and rotation, per token and head, over the head's d elements:
        y = w x / sqrt(mean(x^2) + eps); then the pair j of the first 2 n elements turns by (position freqs[j]):
        (y_lo cos - y_hi sin, y_hi cos + y_lo sin), pairs (j, n + j), or (2 j, 2 j + 1)
    sliding window: query i attends keys max(0, i-w+1) .. i
        P = softmax(scale q k^T), dV = P^T dO, dS = P (dO v^T - rowsum(P (dO v^T))), dQ = scale dS k, dK = scale dS^T q

`own` False: elementary torch operations in fp32 (angles in fp64), rounded once at the end.  `own` True: the framework's calls.
"""
import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_EPS = 1e-6


# ------------------------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # the width of the 1.3B layer (16 heads of 128) over its training batch
        {"name": "recurrence_layer", "op": "rec", "dtype": "bf16", "B": 8, "N": 4096, "C": 2048, "state": False},
        # one long prompt at a width that is no power of two, continued from a state and returning one
        {"name": "recurrence_long", "op": "rec", "dtype": "f32", "B": 1, "N": 32768, "C": 1000, "state": True},
        # one token of the generation batch
        {"name": "recurrence_token", "op": "rec_step", "dtype": "bf16", "B": 128, "C": 2048},
        # the training batch's backward pass
        {"name": "recurrence_grad", "op": "rec_grad", "dtype": "bf16", "B": 8, "N": 4096, "C": 2048, "state": False},
        # a small ragged one, with the gradients of both states
        {"name": "recurrence_grad_odd", "op": "rec_grad", "dtype": "f32", "B": 3, "N": 1111, "C": 1000, "state": True},
        # the window mixer's queries and keys of the 32k-token prompt, out of a fused projection
        {"name": "rotate_prompt", "op": "rot", "dtype": "bf16", "B": 2, "L": 32768, "Hq": 16, "Hk": 16, "d": 64, "n": 32,
         "pairs": False, "positions": "range"},
        # fewer key heads, a wider head of which half turns, packed sequences at far positions
        {"name": "rotate_packed", "op": "rot", "dtype": "f32", "B": 3, "L": 777, "Hq": 16, "Hk": 4, "d": 128, "n": 32,
         "pairs": True, "positions": "tokens"},
        # one token of the generation batch, every sequence at a position of its own
        {"name": "rotate_token", "op": "rot", "dtype": "bf16", "B": 128, "L": 1, "Hq": 16, "Hk": 16, "d": 64, "n": 32,
         "pairs": False, "positions": "sequences"},
        # the 360M layer's training batch
        {"name": "rotate_grad", "op": "rot_grad", "dtype": "bf16", "B": 4, "L": 2048, "Hq": 16, "Hk": 16, "d": 64, "n": 32,
         "pairs": False, "positions": "range"},
        # the sliding window over the 32k-token sequences of the mixer pair
        {"name": "window_grad", "op": "swa_grad", "dtype": "bf16", "B": 2, "H": 16, "L": 32768, "w": 64},
        # the widest window, a length that ends inside a tile
        {"name": "window_grad_wide", "op": "swa_grad", "dtype": "bf16", "B": 3, "H": 16, "L": 1777, "w": 128},
        # fp32, few heads
        {"name": "window_grad_f32", "op": "swa_grad", "dtype": "f32", "B": 1, "H": 16, "L": 1000, "w": 64},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rec", "rec", "rec_step", "rec_grad", "rec_grad", "rot", "rot", "rot", "rot_grad", "swa_grad", "swa_grad", "swa_grad"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "rec_step":
        return {"op": op, "dtype": dtype, "B": _log(rng, 1, 256), "C": 8 * _log(rng, 16, 512)}
    if op in ("rec", "rec_grad"):
        C, N = 8 * _log(rng, 16, 512), _log(rng, 1, 32768)
        most = 1 << 25 if dtype == "f32" else 1 << 26
        N = min(N, most // C)
        B = _log(rng, 1, max(1, min(16, most // (C * N))))
        return {"op": op, "dtype": dtype, "B": B, "N": N, "C": C, "state": rng.random() < 0.5}
    if op in ("rot", "rot_grad"):
        d = rng.choice([16, 32, 64, 64, 64, 112, 128])
        Hk = _log(rng, 1, 16)
        Hq = Hk * rng.choice([1, 1, 2, 4])
        L = 1 if op == "rot" and rng.random() < 0.3 else _log(rng, 1, 32768)
        most = 2 * 32768 * 16 * 64 // (2 if dtype == "f32" else 1)
        B = _log(rng, 1, max(1, min(128 if L < 64 else 8, most // (L * (Hq + Hk) // 2 * d))))
        while B * L * (Hq + Hk) // 2 * d > most:
            L = L // 2
        n = 8 * rng.randint(0, d // 16)
        return {"op": op, "dtype": dtype, "B": B, "L": L, "Hq": Hq, "Hk": Hk, "d": d, "n": n, "pairs": rng.random() < 0.4,
                "positions": rng.choice(["range", "sequences", "tokens"])}
    L, H, w = _log(rng, 2, 32768), _log(rng, 1, 16), rng.choice([64, 64, 128, rng.randint(2, 128)])
    most = 2 * 16 * 32768 if dtype == "bf16" else 1 << 16
    B = _log(rng, 1, max(1, min(8, most // (L * H))))
    while B * L * H > most:
        L = L // 2
    return {"op": op, "dtype": dtype, "B": B, "H": H, "L": L, "w": w}


# ----------------------------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = _DT[case["dtype"]]

    def normal(*shape, dtype=dt):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)

    s = {"op": case["op"]}
    if case["op"].startswith("rec"):
        B, C = case["B"], case["C"]
        lead = (B, C) if case["op"] == "rec_step" else (B, case["N"], C)
        for name in ("x", "r", "g"):
            s[name] = normal(*lead)
        # decays of 0.9 to 0.999 a token where the gate is open
        s["rate"] = -torch.log(0.9 + 0.099 * torch.rand(C, generator=gen, device="cuda"))
        h0 = normal(B, C, dtype=torch.float32)
        s["h0"] = h0 if case["op"] == "rec_step" or case["state"] else None
        s["want_state"] = bool(case.get("state", True))
        if case["op"] == "rec_grad":
            s["dout"] = normal(*lead)
            s["dh"] = normal(B, C, dtype=torch.float32) if case["state"] else None
            s["out"] = _recurrence(s["x"], s["r"], s["g"], s["rate"], s["h0"])[0]
        return s
    if case["op"].startswith("rot"):
        B, L, Hq, Hk, d, n = (case[k] for k in ("B", "L", "Hq", "Hk", "d", "n"))
        fused = normal(B, L, (Hq + 2 * Hk) * d)                 # a layer's projection: queries, keys and values of a token
        s["q"] = fused[..., :Hq * d].unflatten(-1, (Hq, d))
        s["k"] = fused[..., Hq * d:(Hq + Hk) * d].unflatten(-1, (Hk, d))
        s["wq"] = 1 + 0.2 * normal(d, dtype=torch.float32)
        s["wk"] = 1 + 0.2 * normal(d, dtype=torch.float32)
        s["freqs"] = 10000.0 ** (-torch.arange(n, device="cuda", dtype=torch.float64) / max(n, 1)) if n else None
        s["pairs"] = case["pairs"]
        s["positions"] = None
        if case["positions"] == "sequences":
            s["positions"] = torch.randint(0, 1 << 17, (B,), generator=gen, device="cuda", dtype=torch.int32)
        elif case["positions"] == "tokens":
            s["positions"] = torch.randint(0, 1 << 20, (B, L), generator=gen, device="cuda", dtype=torch.int32)
        if case["op"] == "rot_grad":
            s["dq"], s["dk"] = normal(B, Hq, L, d), normal(B, Hk, L, d)
        return s
    shape = (case["B"], case["H"], case["L"], 64)
    for name in ("q", "k", "v", "dout"):
        s[name] = normal(*shape)
    s["w"] = case["w"]
    return s


# ------------------------------------------------------------------------------------------------------------ plain forms
def _doubling(a, b, axis):
    """h_t = a_t h_{t-1} + b_t along an axis, from 0, by doubling; also the running products of a."""
    n, step = a.shape[axis], 1
    a, b = a.clone(), b.clone()
    while step < n:
        tail_a, tail_b = a.narrow(axis, step, n - step), b.narrow(axis, step, n - step)
        new_b = tail_b + tail_a * b.narrow(axis, 0, n - step)
        new_a = tail_a * a.narrow(axis, 0, n - step)
        tail_b.copy_(new_b)
        tail_a.copy_(new_a)
        step *= 2
    return a, b


def _scan(a, b, h0):
    """The same over [B,N,C] from h0: inside blocks of 64 tokens, over the blocks' ends, and the two joined."""
    B, N, C = a.shape
    T = 64
    full = -(-N // T) * T
    if full != N:
        a = torch.cat([a, a.new_ones(B, full - N, C)], 1)
        b = torch.cat([b, b.new_zeros(B, full - N, C)], 1)
    A, H = _doubling(a.view(B, -1, T, C), b.view(B, -1, T, C), 2)
    ends_a, ends_h = _doubling(A[:, :, -1], H[:, :, -1], 1)
    if h0 is None:
        h0 = a.new_zeros(B, C)
    ends = ends_h + ends_a * h0[:, None]
    before = torch.cat([h0[:, None], ends[:, :-1]], 1)
    return (H + A * before[:, :, None]).view(B, full, C)[:, :N]


def _gates(x, r, g, rate):
    x, r, g = x.float(), r.float(), g.float()
    s, i = torch.sigmoid(r), torch.sigmoid(g)
    la = -rate * s
    return x, s, i, torch.exp(la), torch.sqrt(-torch.expm1(2 * la))


def _recurrence(x, r, g, rate, h0):
    xf, s, i, a, m = _gates(x, r, g, rate)
    h = _scan(a, m * i * xf, h0)
    return h.to(x.dtype), h[:, -1].clone()


def _recurrence_step(x, r, g, rate, h0):
    xf, s, i, a, m = _gates(x, r, g, rate)
    h = a * h0 + m * i * xf
    return h.to(x.dtype), h


def _recurrence_grad(x, r, g, rate, h0, out, dout, dh):
    dt = x.dtype
    xf, s, i, a, m = _gates(x, r, g, rate)
    do = dout.float()
    if dh is None:
        dh = torch.zeros_like(do[:, 0])
    # E_t = a_t (dout_t + E_{t+1}), from E_{N+1} = dh: what reaches the state before token t
    E = _scan(a.flip(1), (a * do).flip(1), dh).flip(1)
    G = do + torch.cat([E[:, 1:], dh[:, None]], 1)
    first = torch.zeros_like(do[:, :1]) if h0 is None else h0[:, None]
    prev = torch.cat([first, out[:, :-1].float()], 1)
    dla = a * G * prev - a * a / m * (G * i * xf)
    grads = [(G * m * i).to(dt), (-rate * dla * s * (1 - s)).to(dt), (G * m * xf * i * (1 - i)).to(dt), (-dla * s).sum((0, 1))]
    if h0 is not None:
        grads.append(E[:, 0])
    return grads


def _angles(freqs, positions, B, L):
    """cos, sin [B,L,1,n] in fp32, the angles taken in fp64."""
    p = torch.arange(L, device="cuda", dtype=torch.float64).expand(B, L)
    if positions is not None:
        p = positions.double() if positions.dim() == 2 else p + positions.double()[:, None]
    t = p[..., None, None] * freqs
    return torch.cos(t).float(), torch.sin(t).float()


def _turn(y, cos, sin, pairs, back=False):
    n = cos.shape[-1]
    head, rest = y[..., :2 * n], y[..., 2 * n:]
    lo, hi = (head[..., 0::2], head[..., 1::2]) if pairs else (head[..., :n], head[..., n:])
    if back:
        sin = -sin
    lo, hi = lo * cos - hi * sin, hi * cos + lo * sin
    head = torch.stack([lo, hi], -1).flatten(-2) if pairs else torch.cat([lo, hi], -1)
    return torch.cat([head, rest], -1)


def _rotate(x, w, freqs, positions, pairs):
    xf = x.float()
    y = xf * torch.rsqrt(xf.square().mean(-1, keepdim=True) + _EPS) * w
    if freqs is not None:
        y = _turn(y, *_angles(freqs, positions, x.shape[0], x.shape[1]), pairs)
    return y.to(x.dtype).transpose(1, 2).contiguous()


def _rotate_grad(x, dy, w, freqs, positions, pairs):
    xf, dy = x.float(), dy.float().transpose(1, 2)
    if freqs is not None:
        dy = _turn(dy, *_angles(freqs, positions, x.shape[0], x.shape[1]), pairs, back=True)
    inv = torch.rsqrt(xf.square().mean(-1, keepdim=True) + _EPS)
    xn = xf * inv
    dn = dy * w
    dx = inv * (dn - xn * (dn * xn).mean(-1, keepdim=True))
    return dx.to(x.dtype).contiguous(), (dy * xn).sum((0, 1, 2))


def _window_grad(q, k, v, dout, w):
    B, H, L, d = q.shape
    T = max(w, 32)
    nb = -(-L // T)
    scale = d ** -0.5

    def rows(x):                                            # [BH, nb, T, d]
        return torch.nn.functional.pad(x.float().reshape(B * H, L, d), (0, 0, 0, nb * T - L)).view(B * H, nb, T, d)

    def under(x):                                           # the block before and the block: [BH, nb, 2T, d]
        x = rows(x)
        return torch.cat([torch.nn.functional.pad(x, (0, 0, 0, 0, 1, 0))[:, :-1], x], 2)

    def add_up(x):                                          # its transpose, back to [B, H, L, d]
        y = x[:, :, T:] + torch.nn.functional.pad(x[:, 1:, :T], (0, 0, 0, 0, 0, 1))
        return y.reshape(B, H, nb * T, d)[:, :, :L].to(q.dtype).contiguous()

    qb, ob, kb, vb = rows(q), rows(dout), under(k), under(v)
    i = torch.arange(T, device=q.device)[:, None]
    j = torch.arange(2 * T, device=q.device)[None] - T
    first = torch.arange(nb, device=q.device)[:, None, None] * T
    seen = (j <= i) & (j > i - w) & (first + j >= 0)
    P = (qb @ kb.transpose(2, 3) * scale).masked_fill(~seen, -math.inf)
    P = torch.exp(P - P.amax(-1, keepdim=True))
    P = P / P.sum(-1, keepdim=True)
    dP = ob @ vb.transpose(2, 3)
    dS = P * (dP - (P * dP).sum(-1, keepdim=True)) * scale
    dq = (dS @ kb).reshape(B, H, nb * T, d)[:, :, :L].to(q.dtype).contiguous()
    return dq, add_up(dS.transpose(2, 3) @ qb), add_up(P.transpose(2, 3) @ ob)


# ------------------------------------------------------------------------------------------------------------------- runs
def run(s):
    op = s["op"]
    if own:
        import paper_2402_18668_b200 as based

        if op == "rec":
            state = torch.empty(s["x"].shape[0], s["x"].shape[2], device="cuda") if s["want_state"] else None
            out = based.based_gated_recurrence_forward(s["x"], s["r"], s["g"], s["rate"], state_in=s["h0"], state_out=state)
            return [out, state] if s["want_state"] else [out]
        if op == "rec_step":
            state = torch.empty_like(s["h0"])
            out = based.based_gated_recurrence_step(s["x"], s["r"], s["g"], s["rate"], s["h0"], state_out=state)
            return [out, state]
        if op == "rec_grad":
            grads = based.based_gated_recurrence_backward(s["x"], s["r"], s["g"], s["rate"], s["out"], s["dout"],
                                                          state_in=s["h0"], dstate_out=s["dh"])
            return [x for x in grads if x is not None]
        flags = based.BASED_ROTATE_PAIRS if s.get("pairs") else 0
        if op == "rot":
            return list(based.based_qk_norm_rotate(s["q"], s["k"], s["wq"], s["wk"], s["freqs"], s["positions"], eps=_EPS,
                                                   flags=flags))
        if op == "rot_grad":
            return list(based.based_qk_norm_rotate_backward(s["q"], s["k"], s["dq"], s["dk"], s["wq"], s["wk"], s["freqs"],
                                                            s["positions"], eps=_EPS, flags=flags))
        return list(based.swa_backward(s["q"], s["k"], s["v"], s["dout"], window=s["w"]))
    if op == "rec":
        out, state = _recurrence(s["x"], s["r"], s["g"], s["rate"], s["h0"])
        return [out, state] if s["want_state"] else [out]
    if op == "rec_step":
        return list(_recurrence_step(s["x"], s["r"], s["g"], s["rate"], s["h0"]))
    if op == "rec_grad":
        return _recurrence_grad(s["x"], s["r"], s["g"], s["rate"], s["h0"], s["out"], s["dout"], s["dh"])
    if op == "rot":
        more = (s["freqs"], s["positions"], s["pairs"])
        return [_rotate(s["q"], s["wq"], *more), _rotate(s["k"], s["wk"], *more)]
    if op == "rot_grad":
        more = (s["freqs"], s["positions"], s["pairs"])
        (dq, dwq), (dk, dwk) = _rotate_grad(s["q"], s["dq"], s["wq"], *more), _rotate_grad(s["k"], s["dk"], s["wk"], *more)
        return [dq, dk, dwq, dwk]
    return list(_window_grad(s["q"], s["k"], s["v"], s["dout"], s["w"]))


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"].startswith("rec"):
        n, states = case["B"] * case.get("N", 1) * case["C"], case["B"] * case["C"] * 4
        if case["op"] == "rec_grad":       # x r g out dout -> dx dr dg (and the states' gradients), rate, drate
            return {"bytes": 8 * n * e + (3 * states if case["state"] else 0) + 8 * case["C"], "flops": 40 * n}
        with_states = 2 * states if case.get("state", True) else 0
        return {"bytes": 4 * n * e + with_states + 4 * case["C"], "flops": 20 * n}
    if case["op"].startswith("rot"):
        n = case["B"] * case["L"] * (case["Hq"] + case["Hk"]) * case["d"]
        pos = 4 * case["B"] * {"range": 0, "sequences": 1, "tokens": case["L"]}[case["positions"]]
        small = 8 * case["d"] + 8 * case["n"] + pos
        return {"bytes": 3 * n * e + 2 * small if case["op"] == "rot_grad" else 2 * n * e + small,
                "flops": (16 if case["op"] == "rot_grad" else 7) * n}
    n, L, w = case["B"] * case["H"], case["L"], case["w"]
    seen = L * w - w * (w - 1) // 2 if L >= w else L * (L + 1) // 2
    return {"bytes": 7 * n * L * 64 * e, "flops": n * seen * 64 * 10}


# ------------------------------------------------------------------------------------------- the definitions, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    D = {k: t.double() if isinstance(t, torch.Tensor) and t.is_floating_point() else t for k, t in s.items()}
    if op.startswith("rec"):
        a = torch.exp(-D["rate"] / (1 + torch.exp(-D["r"])))
        i = 1 / (1 + torch.exp(-D["g"]))
        m = torch.sqrt(1 - a * a)
        if op == "rec_step":
            h = a * D["h0"] + m * i * D["x"]
            return [h, h]
        N = a.shape[1]
        zero = torch.zeros_like(a[:, 0])
        if op == "rec":
            b, out, h = m * i * D["x"], torch.empty_like(a), zero if D["h0"] is None else D["h0"]
            for t in range(N):
                h = torch.addcmul(b[:, t], a[:, t], h)
                out[:, t] = h
            return [out, h] if s["want_state"] else [out]
        # G_t: the gradient of h_t, from the last token back
        G, up = torch.empty_like(a), zero if D["dh"] is None else D["dh"]
        for t in reversed(range(N)):
            up = D["dout"][:, t] + up
            G[:, t] = up
            up = a[:, t] * up
        prev = torch.cat([(zero if D["h0"] is None else D["h0"])[:, None], D["out"][:, :-1]], 1)
        da = G * prev - G * i * D["x"] * a / m                 # of a, through a h and through m = sqrt(1 - a^2)
        gate = 1 / (1 + torch.exp(-D["r"]))
        dlog = da * a
        grads = [G * m * i, dlog * -D["rate"] * gate * (1 - gate), G * m * D["x"] * i * (1 - i), -(dlog * gate).sum((0, 1))]
        return grads + ([up] if s["h0"] is not None else [])
    if op.startswith("rot"):
        B, L, n = case["B"], case["L"], case["n"]
        pos = torch.arange(L, device="cuda").repeat(B, 1)
        if case["positions"] == "sequences":
            pos = pos + s["positions"].long()[:, None]
        elif case["positions"] == "tokens":
            pos = s["positions"].long()

        def forward(x, w):
            y = x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + _EPS) * w
            if n:
                z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), pos[:, :, None] * s["freqs"])[:, :, None]
                pair = y[..., :2 * n].unflatten(-1, (n, 2)) if case["pairs"] else y[..., :2 * n].unflatten(-1, (2, n)).transpose(-1, -2)
                turned = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * z)
                if not case["pairs"]:
                    turned = turned.transpose(-1, -2)
                y = torch.cat([turned.flatten(-2), y[..., 2 * n:]], -1)
            return y.transpose(1, 2)

        if op == "rot":
            return [forward(D["q"], D["wq"]), forward(D["k"], D["wk"])]
        leaves = [D[k].detach().clone().requires_grad_(True) for k in ("q", "k", "wq", "wk")]
        outs = [forward(leaves[0], leaves[2]), forward(leaves[1], leaves[3])]
        return list(torch.autograd.grad(outs, leaves, [D["dq"], D["dk"]]))
    # the window by distance: entry t of a row is the key t tokens back
    q, k, v, do, w = D["q"], D["k"], D["v"], D["dout"], min(case["w"], case["L"])
    L = case["L"]
    S = torch.full((w,) + q.shape[:3], -math.inf, dtype=torch.float64, device="cuda")
    dP = torch.zeros_like(S)
    for t in range(w):
        S[t, :, :, t:] = (q[:, :, t:] * k[:, :, :L - t]).sum(-1) / 8
        dP[t, :, :, t:] = (do[:, :, t:] * v[:, :, :L - t]).sum(-1)
    P = torch.softmax(S, 0)
    dS = P * (dP - (P * dP).sum(0)) / 8
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(q)
    for t in range(w):
        dq[:, :, t:] += dS[t, :, :, t:, None] * k[:, :, :L - t]
        dk[:, :, :L - t] += dS[t, :, :, t:, None] * q[:, :, t:]
        dv[:, :, :L - t] += P[t, :, :, t:, None] * do[:, :, t:]
    return [dq, dk, dv]
