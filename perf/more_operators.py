"""Cases and plain forms of two more mixers: linear attention with a decay per head (prompts, single tokens, backward) and
softmax attention of one new token over a paged key-value cache (with the copy of a prompt into its pages).

    decay attention, per sequence and head, from S_0 (or 0), a = exp(-rate of the head):
        S_t = a S_{t-1} + k_t v_t^T,     o_t = scale q_t S_t
    a token whose document is negative is padding: it is passed over (its output is 0); a token of another document than the
    token before it starts from an empty state
    paged attention: the new key and value of sequence b go to position pos_b; token j lies in row j % page_size of page
    page_table[b, j / page_size].  Over the keys j = max(0, pos_b - window + 1) .. pos_b:
        s_j = cap tanh(scale q . k_j / cap) - slope (pos_b - j),  o = sum_j softmax(s)_j v_j;   pos_b < 0: no token, o = 0

`own` False: elementary torch operations in fp32, rounded once at the end.  `own` True: the framework's calls.
"""
import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # the 1.3B layer's training batch: 16 heads of 128
        {"name": "decay_layer", "op": "decay", "dtype": "bf16", "B": 8, "H": 16, "L": 4096, "dk": 128, "dv": 128,
         "layout": "heads", "documents": "none", "state": False},
        # the mixer pair's 32k-token sequences, documents packed one behind the other, as projections leave them
        {"name": "decay_packed", "op": "decay", "dtype": "bf16", "B": 2, "H": 16, "L": 32768, "dk": 64, "dv": 64,
         "layout": "tokens", "documents": "packed", "state": False},
        # a ragged prompt in fp32, continued from a state and returning one, widths that fill no tile
        {"name": "decay_prompt_f32", "op": "decay", "dtype": "f32", "B": 3, "H": 5, "L": 1111, "dk": 40, "dv": 72,
         "layout": "heads", "documents": "padded", "state": True},
        # one token of the generation batch
        {"name": "decay_token", "op": "decay_step", "dtype": "bf16", "B": 128, "H": 16, "dk": 128, "dv": 128},
        # one token of one sequence: the latency of a call
        {"name": "decay_token_one", "op": "decay_step", "dtype": "f32", "B": 1, "H": 16, "dk": 64, "dv": 64},
        # the 1.3B layer's backward pass
        {"name": "decay_grad_layer", "op": "decay_grad", "dtype": "bf16", "B": 8, "H": 16, "L": 4096, "dk": 128, "dv": 128,
         "layout": "heads", "documents": "none", "state": False},
        # a small ragged one in fp32 with packed documents and the gradients of both states
        {"name": "decay_grad_f32", "op": "decay_grad", "dtype": "f32", "B": 2, "H": 4, "L": 777, "dk": 64, "dv": 64,
         "layout": "heads", "documents": "packed", "state": True},
        # generation: 32 sequences of unequal lengths up to 8192, 16 query heads on 4 cached ones
        {"name": "paged_batch", "op": "paged", "dtype": "bf16", "B": 32, "Hq": 16, "Hk": 4, "d": 128, "page": 16, "least": 700,
         "most": 8192, "cap": 0.0, "slopes": False, "window": 0},
        # one sequence of 131072 tokens: the cache's length is all there is to split
        {"name": "paged_long", "op": "paged", "dtype": "bf16", "B": 1, "Hq": 16, "Hk": 16, "d": 64, "page": 64, "least": 131072,
         "most": 131072, "cap": 0.0, "slopes": False, "window": 0},
        # a few short ones in fp32: capped scores, a bias by distance, a window, pages that end inside any tile
        {"name": "paged_small_f32", "op": "paged", "dtype": "f32", "B": 3, "Hq": 6, "Hk": 2, "d": 64, "page": 24, "least": 90,
         "most": 1000, "cap": 20.0, "slopes": True, "window": 512},
        # prompts of unequal lengths copied into their pages
        {"name": "pages_prompts", "op": "pages", "dtype": "bf16", "B": 16, "H": 4, "L": 4096, "d": 128, "page": 16, "least": 300},
        # one odd prompt in fp32
        {"name": "pages_prompt_f32", "op": "pages", "dtype": "f32", "B": 1, "H": 2, "L": 333, "d": 64, "page": 24, "least": 333},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["decay", "decay", "decay", "decay_grad", "decay_grad", "decay_step", "paged", "paged", "paged", "pages"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op.startswith("decay"):
        dk, dv = rng.choice([16, 32, 64, 64, 96, 128, 128, 8 * rng.randint(1, 16)]), rng.choice([16, 64, 64, 112, 128, 128, 8 * rng.randint(1, 16)])
        H = _log(rng, 1, 32)
        if op == "decay_step":
            return {"op": op, "dtype": dtype, "B": _log(rng, 1, min(256, (1 << 25) // (H * dk * dv))), "H": H, "dk": dk, "dv": dv}
        most = (1 << (26 if dtype == "bf16" else 23)) // max(dk, dv, 32)           # tokens times heads
        L = min(_log(rng, 1, 32768), most // H)
        B = _log(rng, 1, max(1, min(16, most // (H * L))))
        return {"op": op, "dtype": dtype, "B": B, "H": H, "L": L, "dk": dk, "dv": dv, "layout": rng.choice(["heads", "tokens"]),
                "documents": rng.choice(["none", "packed", "padded"]), "state": rng.random() < 0.5}
    page, d = rng.choice([8, 16, 24, 64, 128]), rng.choice([32, 64, 64, 128, 128])
    Hk = _log(rng, 1, 16)
    if op == "pages":
        L = min(_log(rng, 1, 8192), (1 << 25) // (Hk * d))
        B = _log(rng, 1, max(1, min(32, (1 << 25) // (Hk * L * d))))
        return {"op": op, "dtype": dtype, "B": B, "H": Hk, "L": L, "d": d, "page": page, "least": rng.randint(1, L)}
    most = min(_log(rng, 1, 131072), (1 << (27 if dtype == "bf16" else 25)) // (Hk * d))
    B = _log(rng, 1, max(1, min(64, (1 << (27 if dtype == "bf16" else 25)) // (Hk * most * d))))
    return {"op": op, "dtype": dtype, "B": B, "Hq": Hk * rng.choice([1, 1, 2, 4, 5, 8]), "Hk": Hk, "d": d, "page": page,
            "least": rng.randint(1, most), "most": most, "cap": rng.choice([0.0, 0.0, 30.0]), "slopes": rng.random() < 0.4,
            "window": rng.choice([0, 0, _log(rng, 1, 4096)])}


# ----------------------------------------------------------------------------------------------------------------- inputs
def _lengths(B, least, most):
    """Lengths spread evenly over least .. most, in no order; one sequence has `most`."""
    return [most - int((most - least) * ((0.6180339887498949 * b) % 1.0)) for b in range(B)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    dt = _DT[case["dtype"]]

    def normal(*shape, dtype=dt):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)

    s = {"op": case["op"]}
    if case["op"].startswith("decay"):
        B, H, dk, dv = (case[k] for k in ("B", "H", "dk", "dv"))
        s["rate"] = torch.exp2(-8.0 * torch.arange(1, H + 1, device="cuda", dtype=torch.float32) / H)      # 0.004 to 0.7
        if case["op"] == "decay_step":
            s["q"], s["k"], s["v"], s["state"] = normal(B, H, dk), normal(B, H, dk), normal(B, H, dv), normal(B, H, dk, dv, dtype=torch.float32)
            return s
        L = case["L"]

        def heads(d):
            return normal(B, H, L, d) if case["layout"] == "heads" else normal(B, L, H, d).transpose(1, 2)

        s["q"], s["k"], s["v"] = heads(dk), heads(dk), heads(dv)
        s["documents"] = None
        if case["documents"] == "packed":                       # a new document after about 1000 tokens
            s["documents"] = (torch.rand(B, L, generator=gen, device="cuda") < 0.001).cumsum(1).int()
        elif case["documents"] == "padded":                     # sequences of unequal lengths, padded behind
            lengths = torch.randint(1, L + 1, (B, 1), generator=gen, device="cuda")
            s["documents"] = torch.where(torch.arange(L, device="cuda") < lengths, 0, -1).int()
        s["state"] = normal(B, H, dk, dv, dtype=torch.float32) if case["state"] else None
        if case["op"] == "decay_grad":
            s["dout"] = heads(dv)
            s["dstate"] = normal(B, H, dk, dv, dtype=torch.float32) if case["state"] else None
        return s
    B, page, d = case["B"], case["page"], case["d"]
    if case["op"] == "pages":
        H, L, counts = case["H"], case["L"], _lengths(B, case["least"], case["L"])
        first = [(37 * b + 5) % (3 * page) for b in range(B)]  # behind what the sequence holds already
        used, Hk = [-(-(f + n) // page) for f, n in zip(first, counts)], H
        s["k"], s["v"] = normal(B, H, L, d), normal(B, H, L, d)
        s["pos"], s["counts"] = torch.tensor(first, dtype=torch.int32).cuda(), torch.tensor(counts, dtype=torch.int32).cuda()
    else:
        Hk, lengths = case["Hk"], _lengths(B, case["least"], case["most"])
        used = [-(-n // page) for n in lengths]
        s["q"], s["k"], s["v"] = normal(B, case["Hq"], d), normal(B, Hk, d), normal(B, Hk, d)
        s["pos"] = torch.tensor(lengths, dtype=torch.int32).cuda() - 1
        s["cap"], s["window"] = case["cap"], case["window"]
        s["slopes"] = torch.exp2(-8.0 * torch.arange(1, case["Hq"] + 1, device="cuda", dtype=torch.float32) / case["Hq"]) if case["slopes"] else None
    # the pool has a few pages that nobody uses; a sequence's pages lie anywhere in it
    table, order, at = torch.zeros(B, max(used), dtype=torch.int32), torch.randperm(sum(used) + 5, generator=host).int(), 0
    for b, n in enumerate(used):
        table[b, :n] = order[at:at + n]
        at += n
    s["table"] = table.cuda()
    s["k_pages"], s["v_pages"] = normal(sum(used) + 5, Hk, page, d), normal(sum(used) + 5, Hk, page, d)
    return s


# ------------------------------------------------------------------------------------------------------------ plain forms
_T = 128


def _blocks(x, fill=0.0):
    """[B,H,L,d] -> [B,H,n,T,d] in fp32, the last block filled up."""
    B, H, L, d = x.shape
    n = -(-L // _T)
    return torch.nn.functional.pad(x.float(), (0, 0, 0, n * _T - L), value=fill).reshape(B, H, n, _T, d)


def _places(documents, B, L):
    """Per token: how many tokens up to it are no padding, which document they are in (counted), and whether it is one."""
    if documents is None:
        valid = torch.ones(B, L, dtype=torch.bool, device="cuda")
        run = torch.zeros(B, L, dtype=torch.int64, device="cuda")
    else:
        valid = documents >= 0
        t = torch.arange(L, device="cuda").expand(B, L)
        last = torch.where(valid, t, -1).cummax(1).values       # the last token that counts, up to each
        before = torch.nn.functional.pad(last[:, :-1], (1, 0), value=-1)
        new = valid & (before >= 0) & (documents.gather(1, before.clamp(min=0)) != documents)
        run = new.cumsum(1)
    return valid.cumsum(1), run, valid


def _decay(x, y, z, rate, places, state, back):
    """sum over the tokens j up to each (back: from each on) of a^|distance| (x_t . y_j) z_j, and a^.. x_t state; the state
    behind all tokens (before them)."""
    B, H, L, _ = x.shape
    count, run, valid = places
    n = -(-L // _T)
    pad = n * _T - L
    count = torch.cat([count, count[:, -1:].expand(B, pad)], 1).reshape(B, 1, n, _T)
    run = torch.cat([run, run[:, -1:].expand(B, pad)], 1).reshape(B, 1, n, _T)
    valid = torch.nn.functional.pad(valid, (0, pad)).reshape(B, 1, n, _T)
    # counts and documents at the blocks' borders: before each block, and behind it
    c1, d1 = count[..., -1], run[..., -1]
    c0, d0 = torch.nn.functional.pad(c1[..., :-1], (1, 0)), torch.nn.functional.pad(d1[..., :-1], (1, 0))
    X, Y, Z = _blocks(x), _blocks(y), _blocks(z)

    def faded(steps, same):
        return torch.exp(-rate.view(1, H, *[1] * (steps.dim() - 2)) * steps.clamp(min=0).float()) * same

    i, j = (count[..., None], run[..., None], valid[..., None]), (count[..., None, :], run[..., None, :], valid[..., None, :])
    t = torch.arange(_T, device="cuda")
    seen = (t[:, None] <= t if back else t[:, None] >= t) & i[2] & j[2] & (i[1] == j[1])
    inside = ((X @ Y.transpose(3, 4)) * faded((i[0] - j[0]).abs(), seen)) @ Z
    if back:
        give = faded(count - c0[..., None], valid & (run == d0[..., None]))          # a block's tokens to the state before it
        take = faded(c1[..., None] - count, valid & (run == d1[..., None]))
        cross = faded(c0[..., None, :] - c1[..., None], (d0[..., None, :] == d1[..., None])) * torch.ones(n, n, device="cuda").triu(1)
        whole = faded(c1[..., -1:] - c1, d1[..., -1:] == d1)
        ends = faded(c0, d0 == 0), faded(c1[..., -1:], d1[..., -1:] == 0)
    else:
        give = faded(c1[..., None] - count, valid & (run == d1[..., None]))          # to the state behind it
        take = faded(count - c0[..., None], valid & (run == d0[..., None]))
        cross = faded(c0[..., None] - c1[..., None, :], (d0[..., None] == d1[..., None, :])) * torch.ones(n, n, device="cuda").tril(-1)
        whole = faded(c0, d0 == 0)
        ends = faded(c1[..., -1:] - c1, d1[..., -1:] == d1), faded(c1[..., -1:], d1[..., -1:] == 0)
    own_state = (Y * give[..., None]).transpose(3, 4) @ Z                            # [B,H,n,d,e]
    flat = own_state.flatten(3)
    states = (cross @ flat).view_as(own_state)
    if state is not None:
        states = states + whole[..., None, None] * state[:, :, None]
    out = inside + take[..., None] * (X @ states)
    last = (ends[0][..., None, :] @ flat).view(B, H, *own_state.shape[3:])
    if state is not None:
        last = last + ends[1][..., None] * state
    return out.reshape(B, H, n * _T, -1)[:, :, :L], last


def _decay_forward(s):
    q, k, v = s["q"], s["k"], s["v"]
    out, last = _decay(q, k, v, s["rate"], _places(s["documents"], q.shape[0], q.shape[2]), s["state"], False)
    return [(out * q.shape[-1] ** -0.5).to(v.dtype).contiguous()] + ([last] if s["state"] is not None else [])


def _decay_grad(s):
    q, k, v, do, scale = s["q"], s["k"], s["v"], s["dout"], s["q"].shape[-1] ** -0.5
    places = _places(s["documents"], q.shape[0], q.shape[2])
    turned = lambda t: None if t is None else t.transpose(2, 3)  # noqa: E731
    dstate = None if s["dstate"] is None else s["dstate"] / scale
    dq, _ = _decay(do, v, k, s["rate"], places, turned(s["state"]), False)
    dk, _ = _decay(v, do, q, s["rate"], places, turned(dstate), True)
    dv, first = _decay(k, q, do, s["rate"], places, dstate, True)
    grads = [(g * scale).to(q.dtype).contiguous() for g in (dq, dk, dv)]
    return grads + ([first * scale] if s["state"] is not None else [])


def _decay_step(s):
    state = torch.exp(-s["rate"]).view(1, -1, 1, 1) * s["state"] + s["k"].float()[..., None] * s["v"].float()[..., None, :]
    out = (s["q"].float()[..., None, :] @ state)[..., 0, :] * s["q"].shape[-1] ** -0.5
    return [out.to(s["v"].dtype), state]


def _paged(s):
    q, kp, vp, table, pos = s["q"], s["k_pages"], s["v_pages"], s["table"].long(), s["pos"].long()
    (B, Hq, d), (_, Hk, page, _) = q.shape, kp.shape
    at = table.gather(1, (pos // page)[:, None])[:, 0]
    kp[at, :, pos % page] = s["k"]
    vp[at, :, pos % page] = s["v"]
    n = table.shape[1] * page
    K = kp[table].transpose(1, 2).reshape(B, Hk, 1, n, d).float()
    V = vp[table].transpose(1, 2).reshape(B, Hk, 1, n, d).float()
    S = (K @ q.float().view(B, Hk, Hq // Hk, d, 1)).view(B, Hq, n) * d ** -0.5
    back = pos[:, None] - torch.arange(n, device="cuda")
    if s["cap"]:
        S = s["cap"] * torch.tanh(S / s["cap"])
    if s["slopes"] is not None:
        S = S - s["slopes"][:, None] * back[:, None].float()
    seen = (back >= 0) & (back < s["window"]) if s["window"] else back >= 0
    S = S.masked_fill(~seen[:, None], -math.inf)
    P = torch.exp(S - S.amax(-1, keepdim=True))
    P = P / P.sum(-1, keepdim=True)
    out = P.view(B, Hk, Hq // Hk, 1, n) @ V
    return [out.view(B, Hq, d).to(q.dtype), kp, vp]


def _pages(s):
    k, v, kp, vp = s["k"], s["v"], s["k_pages"], s["v_pages"]
    page, L = kp.shape[2], k.shape[2]
    b, t = torch.nonzero(torch.arange(L, device="cuda") < s["counts"][:, None], as_tuple=True)
    where = s["pos"].long()[b] + t
    at = s["table"].long()[b, where // page]
    kp[at, :, where % page] = k[b, :, t]
    vp[at, :, where % page] = v[b, :, t]
    return [kp, vp]


# ------------------------------------------------------------------------------------------------------------------- runs
def run(s):
    op = s["op"]
    if own:
        import paper_2402_18668_b200 as based

        if op == "decay":
            last = torch.empty_like(s["state"]) if s["state"] is not None else None
            out = based.based_decay_attention_forward(s["q"], s["k"], s["v"], s["rate"], documents=s["documents"], state_in=s["state"],
                                                      state_out=last)
            return [out] if last is None else [out, last]
        if op == "decay_step":
            state = torch.empty_like(s["state"])
            return [based.based_decay_attention_step(s["q"], s["k"], s["v"], s["rate"], s["state"], state_out=state), state]
        if op == "decay_grad":
            grads = based.based_decay_attention_backward(s["q"], s["k"], s["v"], s["rate"], s["dout"], documents=s["documents"],
                                                         state_in=s["state"], dstate_out=s["dstate"])
            return [x for x in grads if x is not None]
        if op == "paged":
            out = based.paged_decode_step(s["q"], s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["pos"], softcap=s["cap"],
                                          slopes=s["slopes"], window=s["window"])
            return [out, s["k_pages"], s["v_pages"]]
        based.paged_cache_write(s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["pos"], counts=s["counts"])
        return [s["k_pages"], s["v_pages"]]
    return {"decay": _decay_forward, "decay_step": _decay_step, "decay_grad": _decay_grad, "paged": _paged, "pages": _pages}[op](s)


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"].startswith("decay"):
        B, H, dk, dv = (case[k] for k in ("B", "H", "dk", "dv"))
        states = B * H * dk * dv * 4
        if case["op"] == "decay_step":
            return {"bytes": 2 * states + 2 * B * H * (dk + dv) * e + 4 * H, "flops": 5 * B * H * dk * dv}
        n, T = B * H * case["L"], min(case["L"], 64)
        ids = 4 * B * case["L"] if case["documents"] != "none" else 0
        # the least of the two forms: token by token through the state, or in blocks of T with the pairs inside them
        one = n * min(4 * dk * dv, 2 * dk * dv + 2 * dk * dv // T + (dk + dv) * T)
        if case["op"] == "decay_grad":                           # q k v dout -> dq dk dv (and the states')
            return {"bytes": n * (4 * dk + 3 * dv) * e + ids + 4 * H + (3 * states if case["state"] else 0), "flops": 3 * one}
        return {"bytes": n * (2 * dk + 2 * dv) * e + ids + 4 * H + (2 * states if case["state"] else 0), "flops": one}
    if case["op"] == "pages":
        tokens = sum(_lengths(case["B"], case["least"], case["L"]))
        return {"bytes": 4 * tokens * case["H"] * case["d"] * e + 4 * tokens // case["page"] + 8 * case["B"], "flops": 0}
    lengths = _lengths(case["B"], case["least"], case["most"])
    keys = sum(min(n, case["window"]) if case["window"] else n for n in lengths)
    row, B = case["d"] * e, case["B"]
    return {"bytes": 2 * keys * case["Hk"] * row + 2 * B * (case["Hq"] + case["Hk"]) * row + 4 * keys // case["page"] + 4 * B,
            "flops": 4 * keys * case["Hq"] * case["d"]}


# ------------------------------------------------------------------------------------------- the definitions, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    D = {k: t.double() if isinstance(t, torch.Tensor) and t.is_floating_point() else t for k, t in s.items()}
    op = case["op"]
    if op == "pages":
        kp, vp = D["k_pages"], D["v_pages"]
        for b in range(case["B"]):
            for i in range(0, int(s["counts"][b])):
                if case["B"] * case["L"] > 20000:
                    return None                                  # (copies: the plain form's are these values)
                p = int(s["pos"][b]) + i
                kp[int(s["table"][b, p // case["page"]]), :, p % case["page"]] = D["k"][b, :, i]
                vp[int(s["table"][b, p // case["page"]]), :, p % case["page"]] = D["v"][b, :, i]
        return [kp, vp]
    if op == "paged":
        out = torch.zeros_like(D["q"])
        group, page = case["Hq"] // case["Hk"], case["page"]
        for b in range(case["B"]):
            p = int(s["pos"][b])
            at = s["table"][b, :p // page + 1].long()
            K = s["k_pages"][at].transpose(0, 1).reshape(case["Hk"], -1, case["d"])[:, :p + 1].double()
            V = s["v_pages"][at].transpose(0, 1).reshape(case["Hk"], -1, case["d"])[:, :p + 1].double()
            K[:, p], V[:, p] = D["k"][b], D["v"][b]
            lo = max(0, p + 1 - case["window"]) if case["window"] else 0
            x = torch.einsum("hgd,hnd->hgn", D["q"][b].view(-1, group, case["d"]), K[:, lo:]) / math.sqrt(case["d"])
            if case["cap"]:
                x = case["cap"] * torch.tanh(x / case["cap"])
            if case["slopes"]:
                x = x - D["slopes"].view(-1, group, 1) * (p - torch.arange(lo, p + 1, device="cuda", dtype=torch.float64))
            out[b] = torch.einsum("hgn,hnd->hgd", torch.softmax(x, -1), V[:, lo:]).reshape(-1, case["d"])
        return [out, None, None]
    scale = 1 / math.sqrt(case["dk"])
    a = torch.exp(-D["rate"])[:, None, None]
    if op == "decay_step":
        S = a * D["state"] + torch.einsum("bhi,bhj->bhij", D["k"], D["v"])
        return [torch.einsum("bhi,bhij->bhj", D["q"], S) * scale, S]
    # token by token
    B, H, L, dk, dv = (case[k] for k in ("B", "H", "L", "dk", "dv"))
    if B * H * L * dk * dv > 1 << 33 or L > 40000:
        return None
    q, k, v = (D[n].permute(2, 0, 1, 3).contiguous() for n in ("q", "k", "v"))
    ids = torch.zeros(B, L, dtype=torch.int64) if s["documents"] is None else s["documents"].long().cpu()
    keep, live, seen = torch.ones(L, B), torch.ones(L, B), [None] * B     # whether the state goes on to a token; whether it is one
    for b, row in enumerate(ids.tolist()):
        for t, x in enumerate(row):
            if x < 0:
                live[t, b] = 0
            else:
                keep[t, b] = float(seen[b] is None or seen[b] == x)
                seen[b] = x
    live, keep = live.double().cuda()[:, :, None, None, None], keep.double().cuda()[:, :, None, None, None]
    fade = torch.where(live > 0, keep * a, torch.ones_like(a))            # [L,B,H,1,1]
    S = torch.zeros(B, H, dk, dv, dtype=torch.float64, device="cuda") if s["state"] is None else D["state"].clone()
    k = k * live[..., 0]
    if op == "decay":
        out = torch.empty(L, B, H, dv, dtype=torch.float64, device="cuda")
        for t in range(L):
            S.mul_(fade[t]).add_(k[t][..., None] * v[t][..., None, :])
            out[t] = (q[t][..., None, :] @ S)[..., 0, :]
        out = (out * live[..., 0] * scale).permute(1, 2, 0, 3)
        return [out] + ([S] if s["state"] is not None else [])
    do = D["dout"].permute(2, 0, 1, 3).contiguous() * live[..., 0] * scale
    dq, dk_, dv_ = torch.empty_like(q), torch.empty_like(q), torch.empty_like(v)
    for t in range(L):
        S.mul_(fade[t]).add_(k[t][..., None] * v[t][..., None, :])
        dq[t] = (S @ do[t][..., None])[..., 0]
    R = torch.zeros(B, H, dk, dv, dtype=torch.float64, device="cuda") if s["dstate"] is None else D["dstate"].clone()
    for t in reversed(range(L)):
        R.add_(q[t][..., None] * do[t][..., None, :])
        dk_[t] = (R @ v[t][..., None])[..., 0]
        dv_[t] = (k[t][..., None, :] @ R)[..., 0, :]
        R.mul_(fade[t])
    grads = [g.permute(1, 2, 0, 3) for g in (dq, dk_ * live[..., 0], dv_)]
    return grads + ([R] if s["state"] is not None else [])
