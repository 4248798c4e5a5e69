"""Linear attention with a decay per head: prompts, single tokens and gradients against the definition in 64 bits."""
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


def heads(gen, B, H, L, d, dtype, layout):
    """[B,H,L,d] contiguous, the heads of a projection, or slices of a fused one."""
    if layout == "heads":
        return normal(gen, B, H, L, d, dtype=dtype)
    if layout == "tokens":
        return normal(gen, B, L, H, d, dtype=dtype).transpose(1, 2)
    return normal(gen, B, L, 3, H, d + 8, dtype=dtype)[:, :, 1, :, :d].transpose(1, 2)


def rates(gen, H):
    return torch.exp(torch.rand(H, generator=gen, device="cuda") * 5.5 - 5.5)          # 0.004 to 1


def documents(gen, B, L, kind):
    if kind == "none":
        return None
    ids = (torch.rand(B, L, generator=gen, device="cuda") < 0.02).cumsum(1).int()
    if kind == "one":
        return torch.full_like(ids, 7)
    if kind == "packed":
        return ids
    t = torch.arange(L, device="cuda")
    if kind == "right":
        return torch.where(t < torch.randint(0, L + 1, (B, 1), generator=gen, device="cuda"), 3, -1).int()
    if kind == "left":
        return torch.where(t >= torch.randint(0, L + 1, (B, 1), generator=gen, device="cuda"), 0, -5).int()
    assert kind == "holes"
    return torch.where(torch.rand(B, L, generator=gen, device="cuda") < 0.3, -1, ids).int()


def close(got, want, bound):
    assert torch.isfinite(got).all()
    over = (got.double() - want).abs() - bound
    assert over.max() <= 0, f"{over.max()} over the bound, {(over > 0).sum()} of {over.numel()}"


def check_forward(based, gen, dtype, B, H, L, dk, dv, layout="heads", docs="none", with_state=True, scale=0.0):
    q, k, v = heads(gen, B, H, L, dk, dtype, layout), heads(gen, B, H, L, dk, dtype, layout), heads(gen, B, H, L, dv, dtype, layout)
    rate, ids = rates(gen, H), documents(gen, B, L, docs)
    state = normal(gen, B, H, dk, dv) if with_state else None
    last = torch.full((B, H, dk, dv), float("nan"), device="cuda") if with_state else None
    out = based.based_decay_attention_forward(q, k, v, rate, documents=ids, state_in=state, state_out=last, scale=scale)
    s = scale if scale > 0 else None
    want, S = ref.decay(q, k, v, rate, ids, state, s)
    size, T = ref.decay(q.abs(), k.abs(), v.abs(), rate, ids, None if state is None else state.abs(), s)
    assert out.shape == (B, H, L, dv) and out.dtype == dtype
    close(out, want, ref.decay_bound(size, want, dtype, dk, L))
    if with_state:
        close(last, S, ref.state_bound(T, L))
    assert based.based_poll_error() == 0


def check_backward(based, gen, dtype, B, H, L, dk, dv, layout="heads", docs="none", with_state=True):
    q, k, v = heads(gen, B, H, L, dk, dtype, layout), heads(gen, B, H, L, dk, dtype, layout), heads(gen, B, H, L, dv, dtype, layout)
    do = heads(gen, B, H, L, dv, dtype, layout)
    rate, ids = rates(gen, H), documents(gen, B, L, docs)
    state, ds = (normal(gen, B, H, dk, dv), normal(gen, B, H, dk, dv)) if with_state else (None, None)
    got = based.based_decay_attention_backward(q, k, v, rate, do, documents=ids, state_in=state, dstate_out=ds)
    want = ref.decay_grad(q, k, v, rate, do, ids, state, ds)
    size = ref.decay_grad(q.abs(), k.abs(), v.abs(), rate, do.abs(), ids, None if state is None else state.abs(), None if ds is None else ds.abs())
    for g, w, z, d in zip(got[:3], want, size, (dv, dv, dk)):
        close(g, w, ref.decay_bound(z, w, dtype, d, L))
    if with_state:
        close(got[3], want[3], ref.state_bound(size[3], L))
    else:
        assert got[3] is None
    assert based.based_poll_error() == 0


SIZES = [(1, 1, 1, 8, 8), (2, 3, 2, 16, 24), (1, 2, 63, 64, 64), (2, 1, 64, 40, 72), (1, 2, 65, 128, 128), (3, 2, 128, 64, 128),
         (1, 1, 129, 128, 64), (2, 2, 333, 96, 120), (1, 3, 700, 32, 16)]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward(based, dtype, size):
    gen = torch.Generator(device="cuda").manual_seed(sum(size))
    for with_state in (True, False):
        check_forward(based, gen, DTYPES[dtype], *size, with_state=with_state)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_backward(based, dtype, size):
    gen = torch.Generator(device="cuda").manual_seed(sum(size) + 1)
    for with_state in (True, False):
        check_backward(based, gen, DTYPES[dtype], *size, with_state=with_state)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("docs", ["one", "packed", "right", "left", "holes"])
@pytest.mark.parametrize("L", [1, 127, 500])
def test_documents(based, dtype, docs, L):
    gen = torch.Generator(device="cuda").manual_seed(L)
    check_forward(based, gen, DTYPES[dtype], 3, 2, L, 64, 64, docs=docs)
    check_backward(based, gen, DTYPES[dtype], 3, 2, L, 64, 48, docs=docs)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("layout", ["tokens", "fused"])
def test_layouts(based, dtype, layout):
    gen = torch.Generator(device="cuda").manual_seed(5)
    check_forward(based, gen, DTYPES[dtype], 2, 3, 200, 64, 96, layout=layout, docs="packed", scale=0.25)
    check_backward(based, gen, DTYPES[dtype], 2, 3, 200, 64, 96, layout=layout)


@pytest.mark.parametrize("docs", ["none", "packed", "holes"])
def test_many_heads(based, docs):
    """More heads than SMs: tiles of all columns where no state is returned, and a backward pass of its own for the one that returns one."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    for with_state in (True, False):
        check_forward(based, gen, torch.bfloat16, 16, 16, 300, 128, 128, docs=docs, with_state=with_state)
        check_backward(based, gen, torch.bfloat16, 16, 16, 512, 128, 128, docs=docs, with_state=with_state)
        check_backward(based, gen, torch.bfloat16, 16, 16, 257, 64, 120, docs=docs, with_state=with_state, layout="tokens")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("docs", ["none", "packed", "holes"])
def test_long_in_segments(based, dtype, docs):
    """Few heads, many blocks: the sequence is cut into segments, whose states are added up."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    check_forward(based, gen, DTYPES[dtype], 1, 2, 3000, 64, 128, docs=docs)
    check_backward(based, gen, DTYPES[dtype], 1, 2, 2500, 128, 64, docs=docs)


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_rates(based, dtype):
    """No decay, one so slow that a segment's state matters to the end, one that leaves nothing of a token's neighbour, an infinite one."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    rate = torch.tensor([0.0, 1e-5, 0.7, 60.0, float("inf")], device="cuda")
    for L in (100, 2500):
        q, k, v = (normal(gen, 1, 5, L, 64, dtype=DTYPES[dtype]) for _ in range(3))
        state = normal(gen, 1, 5, 64, 64)
        last = torch.empty_like(state)
        out = based.based_decay_attention_forward(q, k, v, rate, state_in=state, state_out=last)
        want, S = ref.decay(q, k, v, rate, None, state)
        size, T = ref.decay(q.abs(), k.abs(), v.abs(), rate, None, state.abs())
        close(out, want, ref.decay_bound(size, want, DTYPES[dtype], 64, L))
        close(last, S, ref.state_bound(T, L))
        grads = based.based_decay_attention_backward(q, k, v, rate, v, state_in=state, dstate_out=state)
        want = ref.decay_grad(q, k, v, rate, v, None, state, state)
        size = ref.decay_grad(q.abs(), k.abs(), v.abs(), rate, v.abs(), None, state.abs(), state.abs())
        for g, w, z in zip(grads[:3], want, size):
            close(g, w, ref.decay_bound(z, w, DTYPES[dtype], 64, L))


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_rates_that_leave_nothing(based, dtype):
    """A rate without bound: every token is on its own."""
    gen = torch.Generator(device="cuda").manual_seed(30)
    q, k, v = (normal(gen, 1, 2, 300, 64, dtype=DTYPES[dtype]) for _ in range(3))
    rate = torch.tensor([float("inf"), 3e38], device="cuda")
    last = torch.empty(1, 2, 64, 64, device="cuda")
    out = based.based_decay_attention_forward(q, k, v, rate, state_in=torch.ones(1, 2, 64, 64, device="cuda"), state_out=last)
    score = (q.double() * k.double()).sum(-1, keepdim=True) / 8
    eps = torch.finfo(DTYPES[dtype]).eps
    # the score's sum of 64 products, its rounding and the output's; nothing of another token
    bound = (q.double() * k.double()).abs().sum(-1, keepdim=True) / 8 * v.double().abs() * 64 * 2.0**-24 + 1.01 * eps * (score * v.double()).abs() + 1e-30
    assert ((out.double() - score * v.double()).abs() <= bound).all()
    want = k[:, :, -1, :, None].double() * v[:, :, -1, None, :].double()
    assert ((last.double() - want).abs() <= want.abs() * 2.0**-20 + 1e-30).all()
    state = torch.ones(1, 2, 64, 64, device="cuda")
    based.based_decay_attention_step(q[:, :, -1].contiguous(), k[:, :, -1].contiguous(), v[:, :, -1].contiguous(), rate, state)
    assert ((state.double() - want).abs() <= want.abs() * 2.0**-20 + 1e-30).all()


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_padding_may_hold_anything(based, dtype):
    gen = torch.Generator(device="cuda").manual_seed(4)
    B, H, L, d = 2, 2, 300, 64
    ids = documents(gen, B, L, "holes")
    ids[0, 128:256] = -1                                        # a whole block, and the tail
    ids[1, 200:] = -1
    q, k, v, do = (normal(gen, B, H, L, d, dtype=DTYPES[dtype]) for _ in range(4))
    rate = rates(gen, H)
    bad = [x.clone() for x in (q, k, v, do)]
    pad = (ids < 0)[:, None, :, None].expand(B, H, L, d)
    for x, value in zip(bad, (float("nan"), float("inf"), -float("inf"), float("nan"))):
        x[pad] = value
    state = normal(gen, B, H, d, d)
    for a, b in zip(based.based_decay_attention_backward(*bad[:3], rate, bad[3], documents=ids, state_in=state),
                    based.based_decay_attention_backward(q, k, v, rate, do, documents=ids, state_in=state)):
        assert torch.equal(a, b)
    x, y = torch.empty_like(state), torch.empty_like(state)
    out = based.based_decay_attention_forward(*bad[:3], rate, documents=ids, state_in=state, state_out=x)
    assert torch.equal(out, based.based_decay_attention_forward(q, k, v, rate, documents=ids, state_in=state, state_out=y)) and torch.equal(x, y)
    assert not out[pad].any()


def test_a_dropped_state_may_hold_anything(based):
    """A document that starts at a sequence's second token leaves nothing of an infinite state to it."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    for dtype in DTYPES.values():
        q, k, v = (normal(gen, 1, 1, 400, 64, dtype=dtype) for _ in range(3))
        ids = torch.ones(1, 400, dtype=torch.int32, device="cuda")
        ids[0, 0] = 0
        state = torch.full((1, 1, 64, 64), float("inf"), device="cuda")
        last = torch.empty_like(state)
        out = based.based_decay_attention_forward(q, k, v, rates(gen, 1), documents=ids, state_in=state, state_out=last)
        assert torch.isfinite(out[:, :, 1:]).all() and torch.isfinite(last).all()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("size", [(1, 1, 8, 8), (3, 2, 128, 128), (2, 5, 64, 120), (4, 4, 40, 72), (70, 3, 16, 64)], ids=str)
def test_step(based, dtype, size):
    B, H, dk, dv = size
    dtype = DTYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(sum(size))
    q, k, v, state = normal(gen, B, H, dk, dtype=dtype), normal(gen, B, H, dk, dtype=dtype), normal(gen, B, H, dv, dtype=dtype), normal(gen, B, H, dk, dv)
    rate = rates(gen, H)
    want, S = ref.decay(q[:, :, None], k[:, :, None], v[:, :, None], rate, None, state)
    size_, T = ref.decay(q.abs()[:, :, None], k.abs()[:, :, None], v.abs()[:, :, None], rate, None, state.abs())
    new = torch.empty_like(state)
    kept = state.clone()
    out = based.based_decay_attention_step(q, k, v, rate, state, state_out=new)
    assert torch.equal(state, kept)
    bound = 2 * ref.U * (dk + 8) * size_ + ref.half_step(dtype) * want.abs() + 1e-30
    close(out, want[:, :, 0], bound[:, :, 0])
    close(new, S, 8 * ref.U * T)
    assert torch.equal(based.based_decay_attention_step(q, k, v, rate, state), out) and torch.equal(state, new)        # in place


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_prompt_then_tokens(based, dtype):
    """A padded prompt, a second piece of it, then token by token: as one definition over all of it."""
    dtype = DTYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(8)
    B, H, d, lengths = 3, 2, 64, [200, 131, 1]
    rate = rates(gen, H)
    ids = torch.full((B, 200), -1, dtype=torch.int32, device="cuda")
    for b, n in enumerate(lengths):
        ids[b, :n] = 0
    parts = [[normal(gen, B, H, n, d, dtype=dtype) for _ in range(3)] for n in (200, 70)]
    state, later = torch.empty(B, H, d, d, device="cuda"), torch.empty(B, H, d, d, device="cuda")
    based.based_decay_attention_forward(*parts[0], rate, documents=ids, state_out=state)
    out = [based.based_decay_attention_forward(*parts[1], rate, state_in=state, state_out=later)]
    steps = [[normal(gen, B, H, d, dtype=dtype) for _ in range(3)] for _ in range(5)]
    out += [based.based_decay_attention_step(*s, rate, later)[:, :, None] for s in steps]
    out = torch.cat(out, 2)
    for b, n in enumerate(lengths):
        whole = [torch.cat([p[b:b + 1, :, :n], r[b:b + 1]] + [s[i][b:b + 1, :, None] for s in steps], 2) for i, (p, r) in enumerate(zip(*parts))]
        want, S = ref.decay(*whole, rate)
        size, T = ref.decay(*(x.abs() for x in whole), rate)
        close(out[b:b + 1], want[:, :, n:], ref.decay_bound(size, want, dtype, d, 300)[:, :, n:])
        close(later[b:b + 1], S, 2 * ref.state_bound(T, 300))


def test_gradients_against_differences(based):
    """A function of the outputs and the last state, changed a little along a direction in every input."""
    from paper_2402_18668_b200.autograd import decay_attention
    gen = torch.Generator(device="cuda").manual_seed(2)
    B, H, L, dk, dv = 2, 2, 150, 24, 40
    ids, rate = documents(gen, B, L, "packed"), rates(gen, H)
    x = [normal(gen, B, H, L, dk), normal(gen, B, H, L, dk), normal(gen, B, H, L, dv), normal(gen, B, H, dk, dv)]
    a, b = normal(gen, B, H, L, dv), normal(gen, B, H, dk, dv)
    leaves = [t.clone().requires_grad_() for t in x]
    out, last = decay_attention(*leaves[:3], rate, documents=ids, state=leaves[3])
    ((a * out).sum() + (b * last).sum()).backward()

    def f(step, which, direction):
        y = [t.double() + (step * direction if i == which else 0) for i, t in enumerate(x)]
        o, s = ref.decay(*y[:3], rate, ids, y[3])
        return float((a.double() * o).sum() + (b.double() * s).sum())
    for i, leaf in enumerate(leaves):
        direction = normal(gen, *leaf.shape).double()
        # (the function is linear in each input: a difference has no error but its rounding)
        slope = (f(1.0, i, direction) - f(-1.0, i, direction)) / 2
        assert abs(float((leaf.grad.double() * direction).sum()) - slope) <= 1e-4 * float((leaf.grad.double() * direction).abs().sum())


def test_autograd_forms(based):
    from paper_2402_18668_b200.autograd import decay_attention
    gen = torch.Generator(device="cuda").manual_seed(12)
    q, k, v = (normal(gen, 2, 70, 2, 64, dtype=torch.bfloat16).transpose(1, 2).requires_grad_() for _ in range(3))
    rate = rates(gen, 2)
    out, last = decay_attention(q, k, v, rate)
    out.float().sum().backward()                               # the state's gradient is not there, an expanded one of the output is
    dq = q.grad.clone()
    want = based.based_decay_attention_backward(q.detach(), k.detach(), v.detach(), rate, torch.ones_like(v))
    assert torch.equal(dq, want[0]) and torch.equal(v.grad, want[2])
    out, last = decay_attention(q, k, v, rate)
    last.sum().backward()                                      # and the other way round
    want, none = decay_attention(q, k, v, rate, return_state=False)
    assert none is None and ((want - out).abs() <= 2**-6 * out.abs() + 2**-6 * out.abs().max()).all()     # (their roundings differ)
    for x in (q, k, v):
        x.grad = None
    want.float().sum().backward()
    assert torch.equal(q.grad, dq)
    odd = torch.randn(2, 2, 70, 65, device="cuda")[..., 1:].bfloat16()
    assert odd[..., 1:9].data_ptr() % 16                       # rows that the kernels cannot read as they lie are copied
    decay_attention(odd[..., 1:9], odd[..., 2:10], odd[..., :64], rate)
    out, _ = decay_attention(q, k, v, rate)
    with pytest.raises(RuntimeError, match="differentiated again"):
        torch.autograd.grad(out.float().sum(), q, create_graph=True)
    with pytest.raises(ValueError, match="constants"):
        decay_attention(q, k, v, rate.clone().requires_grad_())


def test_refusals(based):
    q = torch.zeros(2, 2, 10, 64, device="cuda", dtype=torch.bfloat16)
    rate, state = torch.zeros(2, device="cuda"), torch.zeros(2, 2, 64, 64, device="cuda")
    f = based.based_decay_attention_forward
    for bad in (dict(q=q[..., :60], k=q[..., :60]), dict(v=q[..., :60]), dict(q=q[:, :, :0], k=q[:, :, :0], v=q[:, :, :0])):
        with pytest.raises(based.BasedError if hasattr(based, "BasedError") else RuntimeError):
            f(**{**dict(q=q, k=q, v=q, rate=rate), **bad})
    with pytest.raises(ValueError):
        f(q, q[:, :, :5], q, rate)
    with pytest.raises(TypeError):
        f(q.half(), q.half(), q.half(), rate)
    with pytest.raises(ValueError):
        f(q, q, q, rate[:1])
    with pytest.raises(TypeError):
        f(q, q, q, rate.double())
    with pytest.raises(TypeError):
        f(q, q, q, rate, documents=torch.zeros(2, 10, device="cuda", dtype=torch.int64))
    with pytest.raises(ValueError):
        f(q, q, q, rate, documents=torch.zeros(2, 9, device="cuda", dtype=torch.int32))
    with pytest.raises(ValueError):
        f(q, q, q, rate, state_in=state[:1])
    with pytest.raises(ValueError, match="overlaps"):
        f(q, q, q, rate, state_in=state, state_out=state)
    with pytest.raises(ValueError, match="overlaps"):
        f(q, q, q, rate, out=q)
    with pytest.raises(RuntimeError):
        f(q.transpose(2, 3)[..., :10].transpose(2, 3)[:, :, :, 1:57], q[..., :56], q, rate)      # rows from no 16-byte boundary
    with pytest.raises(ValueError):
        based.based_decay_attention_step(q[:, :, 0], q[:, :, 0], q[:, :, 0], rate, state[:, :, :32].contiguous())
    assert based.based_poll_error() == 0


def test_streams_and_capture(based):
    gen = torch.Generator(device="cuda").manual_seed(21)
    q, k, v = (normal(gen, 1, 2, 2000, 64, dtype=torch.bfloat16) for _ in range(3))
    rate, state, ids = rates(gen, 2), normal(gen, 1, 2, 64, 64), documents(gen, 1, 2000, "packed")
    last = torch.empty_like(state)
    want = based.based_decay_attention_forward(q, k, v, rate, documents=ids, state_in=state, state_out=last)
    S = last.clone()
    grads = based.based_decay_attention_backward(q, k, v, rate, v, documents=ids, state_in=state)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [based.based_decay_attention_forward(q, k, v, rate, documents=ids, state_in=state, state_out=torch.empty_like(state), stream=s) for s in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            o = based.based_decay_attention_forward(q, k, v, rate, documents=ids, state_in=state, state_out=last)
            d = based.based_decay_attention_backward(q, k, v, rate, v, documents=ids, state_in=state)
        graphs.append((g, o, d))
    last.zero_()
    for g, _, _ in graphs + graphs:
        g.replay()
    torch.cuda.synchronize()
    for _, o, d in graphs:
        assert torch.equal(o, want) and torch.equal(last, S) and all(torch.equal(x, y) for x, y in zip(d, grads))
    assert based.based_poll_error() == 0


def test_same_results_again(based):
    gen = torch.Generator(device="cuda").manual_seed(22)
    q, k, v = (normal(gen, 4, 8, 900, 128, dtype=torch.bfloat16) for _ in range(3))
    rate = rates(gen, 8)
    first = based.based_decay_attention_backward(q, k, v, rate, v)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first[:3], based.based_decay_attention_backward(q, k, v, rate, v)[:3]))


def test_captured_training_step(based):
    """Forward and backward pass in one graph, replayed on other inputs."""
    from paper_2402_18668_b200.autograd import decay_attention

    def leaves(seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        t = [normal(gen, 2, 300, 2, 64, dtype=torch.bfloat16).transpose(1, 2) for _ in range(3)] + [normal(gen, 2, 2, 64, 64)]
        return [x.requires_grad_() for x in t], rates(gen, 2), documents(gen, 2, 300, "holes")

    def step(t, rate, ids):
        out, last = decay_attention(*t[:3], rate, documents=ids, state=t[3])
        return torch.autograd.grad(out.float().square().sum() + last.square().sum(), t)

    t, rate, ids = leaves(1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(t, rate, ids)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(t, rate, ids)
    for seed in (1, 2):
        with torch.no_grad():
            new, r, d = leaves(seed)
            for x, y in zip(t + [rate, ids], new + [r, d]):
                x.copy_(y)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, step(t, rate, ids)))
    assert based.based_poll_error() == 0


@pytest.fixture
def room():
    torch.cuda.empty_cache()
    yield torch.cuda.mem_get_info()[0]
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("layout", ["heads", "tokens"])
def test_offsets_past_32_bits(based, room, dtype, layout):
    """Inputs of more than 2^31 elements: the last head's outputs and gradients are those of the head alone."""
    H, L, d = 33, 1 << 20, 64
    if room < 8 * H * L * d * torch.finfo(DTYPES[dtype]).bits // 8:
        pytest.skip("no room for seven tensors of 2.2e9 elements")
    gen = torch.Generator(device="cuda").manual_seed(33)
    rate = torch.full((H,), 0.01, device="cuda")

    def tensor():
        x = torch.zeros((1, H, L, d) if layout == "heads" else (1, L, H, d), device="cuda", dtype=DTYPES[dtype])
        x = x if layout == "heads" else x.transpose(1, 2)
        x[:, -1] = normal(gen, 1, L, d, dtype=DTYPES[dtype])
        return x
    q, k, v = tensor(), tensor(), tensor()
    one = [x[:, -1:].contiguous() for x in (q, k, v)]
    eps = torch.finfo(DTYPES[dtype]).eps

    def same(a, b):
        # two divisions into segments: the roundings of a state to bf16 (of its sums in fp32), some ten that count, each at most eps / 2 of outputs of this size
        return (a[:, -1:].float() - b.float()).abs().max() <= 10 * max(eps, 2.0**-20) * b.float().abs().max()
    out = based.based_decay_attention_forward(q, k, v, rate)
    assert same(out, based.based_decay_attention_forward(*one, rate[:1]))
    assert not out[:, :-1].any()
    del out
    if layout == "heads":
        grads = based.based_decay_attention_backward(q, k, v, rate, v)
        for a, b in zip(grads[:3], based.based_decay_attention_backward(*one, rate[:1], one[2])[:3]):
            assert same(a, b)
    assert based.based_poll_error() == 0
