"""Attention of one new token over a paged cache, and the copy of prompts into its pages, against the definition in 64 bits."""
import pytest
import torch

import attention64 as ref

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def based():
    import paper_2402_18668_b200 as based
    based.based_poll_error()
    return based


def normal(gen, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=gen, device="cuda").to(dtype)


def cache(gen, pos, Hk, ps, d, dtype, layout="heads", spare=3, wide=2):
    """Pools whose unused rows hold NaN, a table with shuffled pages and entries of no page behind them."""
    B = len(pos)
    used = [max(p, 0) // ps + 1 for p in pos]
    total = sum(used) + spare
    shape = (total, Hk, ps, d) if layout == "heads" else (total, ps, Hk, d)
    kp, vp = (torch.full(shape, float("nan"), device="cuda", dtype=dtype) for _ in range(2))
    if layout != "heads":
        kp, vp = kp.transpose(1, 2), vp.transpose(1, 2)
    table = torch.full((B, max(used) + wide), -7, dtype=torch.int32)
    order = torch.randperm(total, generator=torch.Generator().manual_seed(1))
    at = 0
    for b, n in enumerate(used):
        ids = order[at:at + n]
        at += n
        table[b, :n] = ids.int()
        for x in (kp, vp):
            rows = normal(gen, Hk, max(pos[b], 0), d, dtype=dtype)
            for i in range(0, max(pos[b], 0), ps):
                piece = rows[:, i:i + ps]
                x[int(ids[i // ps]), :, :piece.shape[1]] = piece
    return kp, vp, table.cuda()


def check(based, gen, dtype, pos, Hq, Hk, d, ps, layout="heads", cap=0.0, slopes=False, window=0, scale=0.0, **kw):
    kp, vp, table = cache(gen, pos, Hk, ps, d, dtype, layout, **kw)
    B = len(pos)
    q, k, v = normal(gen, B, Hq, d, dtype=dtype), normal(gen, B, Hk, d, dtype=dtype), normal(gen, B, Hk, d, dtype=dtype)
    sl = torch.rand(Hq, generator=gen, device="cuda") if slopes else None
    at = torch.tensor(pos, dtype=torch.int32, device="cuda")
    want, bound, kw_, vw_ = ref.paged(q, k, v, kp, vp, table, at, scale if scale > 0 else None, cap, sl, window)
    out = based.paged_decode_step(q, k, v, kp, vp, table, at, softmax_scale=scale, softcap=cap, slopes=sl, window=window)
    assert torch.isfinite(out).all() and out.dtype == dtype
    over = (out.double() - want).abs() - bound
    assert over.max() <= 0, f"{over.max()} over the bound"
    # the new tokens are in their places, everything else is as it was
    assert torch.equal(kp.nan_to_num(7.0), kw_.nan_to_num(7.0)) and torch.equal(vp.nan_to_num(7.0), vw_.nan_to_num(7.0))
    assert based.based_poll_error() == 0


POS = [[0], [15], [16], [63, 64, 65], [-1, 5, 200], [0, 1, 2, 3, 4, 5, 6, 7], [900, 3, 31, -1, 512], [2500]]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("pos", POS, ids=str)
def test_lengths(based, dtype, pos):
    gen = torch.Generator(device="cuda").manual_seed(len(pos))
    check(based, gen, DTYPES[dtype], pos, 4, 2, 64, 16)
    check(based, gen, DTYPES[dtype], pos, 3, 3, 128, 24)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("heads", [(1, 1), (8, 1), (5, 1), (12, 4), (17, 1), (40, 2), (64, 2)], ids=str)
@pytest.mark.parametrize("d", [8, 64, 72, 128])
def test_heads_and_widths(based, dtype, heads, d):
    gen = torch.Generator(device="cuda").manual_seed(d)
    check(based, gen, DTYPES[dtype], [130, 37], *heads, d, 32)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("ps", [1, 3, 8, 16, 48, 100, 128])
@pytest.mark.parametrize("layout", ["heads", "tokens"])
def test_pages(based, dtype, ps, layout):
    gen = torch.Generator(device="cuda").manual_seed(ps)
    check(based, gen, DTYPES[dtype], [777, 99], 4, 2, 64, ps, layout=layout)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("window", [0, 1, 16, 17, 64, 500, 5000])
@pytest.mark.parametrize("cap,slopes", [(0.0, False), (5.0, False), (0.0, True), (1000.0, True)])
def test_scores(based, dtype, window, cap, slopes):
    gen = torch.Generator(device="cuda").manual_seed(window + 1)
    check(based, gen, DTYPES[dtype], [1100, 3, 260], 6, 2, 64, 16, window=window, cap=cap, slopes=slopes, scale=0.3)


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_many_sequences(based, dtype):
    gen = torch.Generator(device="cuda").manual_seed(17)
    check(based, gen, DTYPES[dtype], [(37 * i) % 90 - 1 for i in range(300)], 2, 1, 64, 16)
    check(based, gen, DTYPES[dtype], [(997 * i) % 3000 for i in range(20)], 8, 2, 128, 64)


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_one_long_sequence(based, dtype):
    gen = torch.Generator(device="cuda").manual_seed(18)
    check(based, gen, DTYPES[dtype], [40000], 2, 1, 64, 64)
    check(based, gen, DTYPES[dtype], [12345], 16, 2, 128, 16, cap=30.0, slopes=True)


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_tables_longer_than_the_sequences(based, dtype):
    """How the work is cut goes by the tables' length as well: with more outputs than joins, hardly any tokens, none at all, one token for all CTAs."""
    gen = torch.Generator(device="cuda").manual_seed(25)
    check(based, gen, DTYPES[dtype], [(37 * i) % 330 - 30 for i in range(300)], 4, 2, 64, 16, wide=120)
    check(based, gen, DTYPES[dtype], [70 if i % 401 == 5 else -1 for i in range(1300)], 1, 1, 64, 16, wide=120)
    check(based, gen, DTYPES[dtype], [-1] * 3, 4, 2, 64, 16, wide=120)
    check(based, gen, DTYPES[dtype], [-1] * 600, 2, 1, 64, 16, wide=120)
    check(based, gen, DTYPES[dtype], [0], 2, 1, 128, 16, wide=500)
    check(based, gen, DTYPES[dtype], [65, 0, 4000], 6, 2, 64, 16, wide=500, window=64)
    check(based, gen, DTYPES[dtype], [(61 * i) % 900 for i in range(40)], 2, 1, 64, 16)                # 900 tokens at most: nothing is cut


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_sequences_that_share_pages(based, dtype):
    """Two sequences with one prompt, whose whole pages they share; each has a last page of its own."""
    gen = torch.Generator(device="cuda").manual_seed(26)
    kp, vp, table = cache(gen, [1500], 2, 16, 64, DTYPES[dtype])
    kp, vp = torch.cat([kp, kp]), torch.cat([vp, vp])
    both = table.expand(2, -1).clone()
    both[1, 1500 // 16] += kp.shape[0] // 2
    q, k, v = normal(gen, 2, 4, 64, dtype=DTYPES[dtype]), normal(gen, 2, 2, 64, dtype=DTYPES[dtype]), normal(gen, 2, 2, 64, dtype=DTYPES[dtype])
    pos = torch.tensor([1500, 1500], dtype=torch.int32, device="cuda")
    want, bound, kw, vw = ref.paged(q, k, v, kp, vp, both, pos, None, 0.0, None, 0)
    out = based.paged_decode_step(q, k, v, kp, vp, both, pos)
    assert ((out.double() - want).abs() <= bound).all()
    assert torch.equal(kp.nan_to_num(7.0), kw.nan_to_num(7.0)) and torch.equal(vp.nan_to_num(7.0), vw.nan_to_num(7.0))


def test_offsets_past_32_bits(based):
    """A pool of more than 2^32 elements, of which the pages at its end are used."""
    free, _ = torch.cuda.mem_get_info()
    if free < 40 << 30:
        pytest.skip("no room for a pool of 17 GB")
    gen = torch.Generator(device="cuda").manual_seed(19)
    Hk, ps, d = 2, 64, 128
    pages = (1 << 32) // (Hk * ps * d) + 40
    kp, vp = (torch.empty(pages, Hk, ps, d, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    for x in (kp, vp):
        x[-40:] = normal(gen, 40, Hk, ps, d, dtype=torch.bfloat16)
    table = (torch.arange(12, device="cuda", dtype=torch.int32) * 3 + pages - 40)[None]
    pos = torch.tensor([700], device="cuda", dtype=torch.int32)
    q, k, v = normal(gen, 1, 4, d, dtype=torch.bfloat16), normal(gen, 1, Hk, d, dtype=torch.bfloat16), normal(gen, 1, Hk, d, dtype=torch.bfloat16)
    want, bound, *_ = ref.paged(q, k, v, kp[-40:], vp[-40:], table - (pages - 40), pos)
    out = based.paged_decode_step(q, k, v, kp, vp, table, pos)
    assert ((out.double() - want).abs() <= bound).all()
    row = table[0, 700 // ps].item()
    assert torch.equal(kp[row, :, 700 % ps], k[0])


def test_extreme_scores(based):
    """One key far above the rest; scores of hundreds either way; a value that is infinite stays in its own sequence."""
    for dtype in DTYPES.values():
        gen = torch.Generator(device="cuda").manual_seed(20)
        kp, vp, table = cache(gen, [300, 300], 1, 16, 64, dtype)
        q, k, v = normal(gen, 2, 2, 64, dtype=dtype) * 30, normal(gen, 2, 1, 64, dtype=dtype) * 30, normal(gen, 2, 1, 64, dtype=dtype)
        pos = torch.tensor([300, 300], dtype=torch.int32, device="cuda")
        want, bound, *_ = ref.paged(q, k, v, kp, vp, table, pos)
        out = based.paged_decode_step(q, k, v, kp, vp, table, pos)
        assert torch.isfinite(out).all() and ((out.double() - want).abs() <= bound).all()
        vp[int(table[0, 3])] = float("inf")
        again = based.paged_decode_step(q, k, v, kp, vp, table, pos)
        assert torch.equal(again[1], out[1])


def test_pages_out_of_range(based):
    """Pages that are not in the pool are not touched, read as zeros, and reported."""
    for dtype in DTYPES.values():
        gen = torch.Generator(device="cuda").manual_seed(23)
        for bad in (-1, 1 << 30, 10 ** 6):
            kp, vp, table = cache(gen, [100, 100], 2, 16, 64, dtype)
            q, k, v = normal(gen, 2, 2, 64, dtype=dtype), normal(gen, 2, 2, 64, dtype=dtype), normal(gen, 2, 2, 64, dtype=dtype)
            pos = torch.tensor([100, 100], dtype=torch.int32, device="cuda")
            fine = based.paged_decode_step(q, k, v, kp, vp, table, pos)
            assert based.based_poll_error() == 0
            table[0, 2] = bad                                  # inside
            out = based.paged_decode_step(q, k, v, kp, vp, table, pos)
            assert based.based_poll_error() == 1 and based.based_poll_error() == 0
            assert torch.isfinite(out).all() and torch.equal(out[1], fine[1])
            table[0, 6] = bad                                  # and the new token's
            k_before = kp.clone()
            based.paged_decode_step(q, -k, v, kp, vp, table, pos)
            assert based.based_poll_error() == 1
            k_before[int(table[1, 6]), :, 100 % 16] = -k[1]
            assert torch.equal(kp.nan_to_num(7.0), k_before.nan_to_num(7.0))
        pos[0] = 10 ** 9                                       # past what the table can hold
        out = based.paged_decode_step(q, k, v, kp, vp, table, pos)
        assert based.based_poll_error() == 1 and not out[0].any()
        counts = torch.tensor([5, 200], dtype=torch.int32, device="cuda")
        pos = torch.tensor([0, 0], dtype=torch.int32, device="cuda")
        rows = normal(gen, 2, 2, 200, 64, dtype=dtype)
        based.paged_cache_write(rows, rows, kp, vp, table, pos, counts)      # the second is longer than its pages
        assert based.based_poll_error() == 1


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("layout", ["heads", "tokens"])
@pytest.mark.parametrize("ps,d", [(1, 8), (16, 64), (24, 128), (128, 72)])
def test_write(based, dtype, layout, ps, d):
    dtype = DTYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(ps)
    H, L, first, counts = 3, 150, [0, 7, 40, -1, 5], [150, 0, 100, 150, 500]
    shape = (60 if ps > 16 else 1000 // ps, H, ps, d)
    kp, vp = normal(gen, *shape, dtype=dtype), normal(gen, *shape, dtype=dtype)
    if layout == "tokens":
        kp, vp = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (kp, vp))
    n = 200 // ps + 2
    table = torch.randperm(shape[0], generator=torch.Generator().manual_seed(2))[:len(first) * n] if shape[0] >= len(first) * n else None
    if table is None:
        kp, vp = (normal(gen, len(first) * n, *shape[1:], dtype=dtype) for _ in range(2))
        table = torch.randperm(len(first) * n)
    table = table.view(len(first), n).int().cuda()
    k, v = normal(gen, len(first), L, H, d, dtype=dtype).transpose(1, 2), normal(gen, len(first), H, L, d, dtype=dtype)
    kw, vw = kp.clone(), vp.clone()
    for b, (f, c) in enumerate(zip(first, counts)):
        for t in range(min(c, L) if f >= 0 else 0):
            page = int(table[b, (f + t) // ps])
            kw[page, :, (f + t) % ps], vw[page, :, (f + t) % ps] = k[b, :, t], v[b, :, t]
    pos = torch.tensor(first, dtype=torch.int32, device="cuda")
    based.paged_cache_write(k, v, kp, vp, table, pos, torch.tensor(counts, dtype=torch.int32, device="cuda"))
    assert torch.equal(kp, kw) and torch.equal(vp, vw)
    pos.clamp_(min=0)
    based.paged_cache_write(k, v, kp, vp, table, pos)           # all of them
    assert based.based_poll_error() == 0
    assert torch.equal(kp[int(table[3, 20 // ps]), :, 20 % ps], k[3, :, 20])


def test_prompt_and_generation_of_a_hybrid_stack(based):
    """A padded batch through a layer of each kind: decay attention keeps a state, the exact layer its pages; then token by token, captured."""
    gen = torch.Generator(device="cuda").manual_seed(30)
    B, H, Hk, d, ps, lengths, T = 3, 4, 2, 64, 16, [70, 33, 5], 20
    dt = torch.bfloat16
    rate = torch.exp(-torch.rand(H, generator=gen, device="cuda") * 4)
    L = max(lengths)
    ids = torch.where(torch.arange(L)[None] < torch.tensor(lengths)[:, None], 0, -1).int().cuda()
    ql, kl, vl = (normal(gen, B, H, L, d, dtype=dt) for _ in range(3))
    kx, vx = normal(gen, B, Hk, L, d, dtype=dt), normal(gen, B, Hk, L, d, dtype=dt)
    state = torch.empty(B, H, d, d, device="cuda")
    based.based_decay_attention_forward(ql, kl, vl, rate, documents=ids, state_out=state)
    n = (L + T) // ps + 1
    kp, vp = (torch.zeros(B * n, Hk, ps, d, device="cuda", dtype=dt) for _ in range(2))
    table = torch.randperm(B * n, generator=torch.Generator().manual_seed(3)).view(B, n).int().cuda()
    pos = torch.zeros(B, dtype=torch.int32, device="cuda")
    counts = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    based.paged_cache_write(kx, vx, kp, vp, table, pos, counts)
    pos.copy_(counts)
    steps = [[normal(gen, T, B, h, d, dtype=dt) for h in (H, H, H, H, Hk, Hk)]][0]
    tok = [x[0].clone() for x in steps]
    start = (state.clone(), kp.clone(), vp.clone(), pos.clone())

    def layer():
        y = based.based_decay_attention_step(tok[0], tok[1], tok[2], rate, state)
        z = based.paged_decode_step(tok[3], tok[4], tok[5], kp, vp, table, pos)
        pos.add_(1)
        return y, z
    eager = []
    for t in range(T):
        for a, x in zip(tok, steps):
            a.copy_(x[t])
        eager.append([o.clone() for o in layer()])
    for x, y in zip((state, kp, vp, pos), start):
        x.copy_(y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, z = layer()
    for x, s in zip((state, kp, vp, pos), start):
        x.copy_(s)
    for t in range(T):
        for a, x in zip(tok, steps):
            a.copy_(x[t])
        graph.replay()
        assert torch.equal(y, eager[t][0]) and torch.equal(z, eager[t][1])
    assert based.based_poll_error() == 0
    b = 1                                                       # one sequence from the definitions, at the last token
    whole = [torch.cat([p[b:b + 1, :, :lengths[b]], s[:, b].transpose(0, 1)[None]], 2) for p, s in zip((ql, kl, vl), steps)]
    want, _ = ref.decay(*whole, rate)
    size, _ = ref.decay(*(x.abs() for x in whole), rate)
    assert ((y[b].double() - want[0, :, -1]).abs() <= ref.decay_bound(size, want, dt, d, 100)[0, :, -1]).all()
    K = torch.cat([kx[b, :, :lengths[b]], steps[4][:, b].transpose(0, 1)], 1)[None]
    V = torch.cat([vx[b, :, :lengths[b]], steps[5][:, b].transpose(0, 1)], 1)[None]
    one = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    want, bound, *_ = ref.paged(steps[3][-1, b:b + 1], K[:, :, -1], V[:, :, -1], K, V, one, torch.tensor([K.shape[2] - 1], device="cuda"))
    assert ((z[b].double() - want[0]).abs() <= bound[0]).all()


def test_refusals(based):
    q, k = torch.zeros(2, 4, 64, device="cuda"), torch.zeros(2, 2, 64, device="cuda")
    kp, vp = torch.zeros(10, 2, 16, 64, device="cuda"), torch.zeros(10, 2, 16, 64, device="cuda")
    table, pos = torch.zeros(2, 4, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    f = based.paged_decode_step
    for bad, error in ((dict(q=q[:, :3].contiguous()), RuntimeError), (dict(k=k[:1]), ValueError), (dict(k_pages=kp.bfloat16(), v_pages=vp.bfloat16()), ValueError),
                       (dict(v_pages=vp[:5]), ValueError), (dict(page_table=table.long()), ValueError), (dict(page_table=table[:1]), ValueError),
                       (dict(pos=pos.long()), TypeError), (dict(pos=pos[:1]), ValueError), (dict(slopes=torch.zeros(3, device="cuda")), ValueError),
                       (dict(window=-1), RuntimeError), (dict(softcap=-1.0), RuntimeError), (dict(softcap=float("nan")), RuntimeError),
                       (dict(out=q), ValueError), (dict(k_pages=kp, v_pages=kp), ValueError), (dict(q=q.cpu()), ValueError),
                       (dict(page_table=torch.zeros(2, 8, dtype=torch.int32, device="cuda")[:, :4]), ValueError),
                       (dict(pos=torch.zeros(4, dtype=torch.int32, device="cuda")[::2]), ValueError)):
        with pytest.raises(error):
            f(**{**dict(q=q, k=k, v=k.clone(), k_pages=kp, v_pages=vp, page_table=table, pos=pos), **bad})
    rows = torch.zeros(2, 2, 8, 64, device="cuda")
    for bad, error in ((dict(v=rows[:, :, :5]), ValueError), (dict(k=rows[..., :32], v=rows[..., :32]), ValueError), (dict(counts=pos.long()), TypeError),
                       (dict(k=kp[:2, :, :8], v=rows), ValueError), (dict(k_pages=kp, v_pages=kp), ValueError)):
        with pytest.raises(error):
            based.paged_cache_write(**{**dict(k=rows, v=rows.clone(), k_pages=kp, v_pages=vp, page_table=table, pos=pos), **bad})
    assert based.based_poll_error() == 0


def test_same_results_again_on_any_stream(based):
    gen = torch.Generator(device="cuda").manual_seed(31)
    kp, vp, table = cache(gen, [5000, 77], 2, 16, 128, torch.bfloat16)
    q, k, v = normal(gen, 2, 8, 128, dtype=torch.bfloat16), normal(gen, 2, 2, 128, dtype=torch.bfloat16), normal(gen, 2, 2, 128, dtype=torch.bfloat16)
    pos = torch.tensor([5000, 77], dtype=torch.int32, device="cuda")
    first = based.paged_decode_step(q, k, v, kp, vp, table, pos)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = [based.paged_decode_step(q, k, v, kp, vp, table, pos, stream=s) for s in streams for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(o, first) for o in outs)
