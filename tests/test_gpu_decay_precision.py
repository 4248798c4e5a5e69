"""Decay attention to the precision that it promises: inputs of one sign, where no term hides another's rounding, and the size of the errors
where signs are mixed."""
import pytest
import torch

import attention64 as ref

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
# (B, H, L, d_k, d_v): few heads, cut into segments; tiles of 64 and of 128 columns; more heads than SMs; widths that fill no tile
SIZES = [(1, 2, 3000, 64, 64), (1, 2, 3000, 128, 128), (2, 2, 333, 96, 120), (16, 16, 512, 128, 128), (16, 16, 300, 64, 128), (1, 1, 8000, 64, 128)]


def inputs(dtype, size, one_sign):
    B, H, L, dk, dv = size
    gen = torch.Generator(device="cuda").manual_seed(sum(size))

    def normal(*shape):
        x = torch.randn(shape, generator=gen, device="cuda")
        return x.abs() if one_sign else x
    q, k, v, do = (normal(B, H, L, d).to(dtype) for d in (dk, dk, dv, dv))
    # no decay, hardly any, some: the state is what counts
    return q, k, v, do, torch.tensor([0.0, 1e-5, 0.002, 0.01], device="cuda").repeat(H)[:H], normal(B, H, dk, dv), normal(B, H, dk, dv)


def within(got, want, bound):
    assert torch.isfinite(got).all()
    over = (got.double() - want).abs() - bound
    assert over.max() <= 0, f"{((got.double() - want).abs() / bound).max()} of the bound"


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("states", [False, True])
def test_one_sign(dtype, size, states):
    """The formula on absolute values is the formula: a term that is 1 % short, or 8 bits of a faded key in place of 16, shows."""
    import paper_2402_18668_b200 as based
    dt = DTYPES[dtype]
    q, k, v, do, rate, state, dstate = inputs(dt, size, True)
    L, dk, dv = size[2:]
    last = torch.empty_like(state) if states else None
    out = based.based_decay_attention_forward(q, k, v, rate, state_in=state if states else None, state_out=last)
    want, S = ref.decay(q, k, v, rate, None, state if states else None)
    within(out, want, ref.decay_bound(want, want, dt, dk, L))
    if states:
        within(last, S, ref.state_bound(S, L))
    grads = based.based_decay_attention_backward(q, k, v, rate, do, state_in=state if states else None, dstate_out=dstate if states else None)
    want = ref.decay_grad(q, k, v, rate, do, None, state if states else None, dstate if states else None)
    for g, w, d in zip(grads[:3], want, (dv, dv, dk)):
        within(g, w, ref.decay_bound(w, w, dt, d, L))
    if states:
        within(grads[3], want[3], ref.state_bound(want[3], L))
    assert based.based_poll_error() == 0


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("states", [False, True])
def test_size_of_the_errors(size, states):
    """bf16, mixed signs: every term is rounded once as an operand (score or state) and the result once, each by an even spread over +- u of the
    value at most, u / sqrt(3) in the mean of squares.  The terms' roundings are independent and so are their signs, so the squares add up to 2/3 u^2
    of the outputs' square; 5 % for the 16 bits of a faded key (2^-8 u) and for the sample."""
    import paper_2402_18668_b200 as based
    q, k, v, do, rate, state, dstate = inputs(torch.bfloat16, size, False)
    out = based.based_decay_attention_forward(q, k, v, rate, state_in=state if states else None)
    grads = based.based_decay_attention_backward(q, k, v, rate, do, state_in=state if states else None, dstate_out=dstate if states else None)
    want = [ref.decay(q, k, v, rate, None, state if states else None)[0]]
    want += ref.decay_grad(q, k, v, rate, do, None, state if states else None, dstate if states else None)[:3]
    u = ref.half_step(torch.bfloat16)
    for name, g, w in zip(("out", "dq", "dk", "dv"), (out, *grads[:3]), want):
        for h in range(size[1] if size[1] < 4 else 4):
            off = ((g[:, h].double() - w[:, h]).square().mean() / w[:, h].square().mean()).sqrt()
            assert off <= 1.05 * (2 / 3) ** 0.5 * u, f"{name}, head {h}: {off / u} u"


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("L", [100, 2500])
def test_gradient_of_the_state_by_rate(dtype, L):
    import paper_2402_18668_b200 as based
    gen = torch.Generator(device="cuda").manual_seed(7)
    rate = torch.tensor([0.0, 1e-5, 0.7, 60.0, float("inf")], device="cuda")
    q, k, v, do = (torch.randn(1, 5, L, 64, generator=gen, device="cuda").to(DTYPES[dtype]) for _ in range(4))
    state, dstate = (torch.randn(1, 5, 64, 64, generator=gen, device="cuda") for _ in range(2))
    got = based.based_decay_attention_backward(q, k, v, rate, do, state_in=state, dstate_out=dstate)[3]
    want = ref.decay_grad(q, k, v, rate, do, None, state, dstate)[3]
    size = ref.decay_grad(q.abs(), k.abs(), v.abs(), rate, do.abs(), None, state.abs(), dstate.abs())[3]
    within(got, want, ref.state_bound(size, L))


@pytest.fixture
def room():
    torch.cuda.empty_cache()
    yield torch.cuda.mem_get_info()[0]
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("layout", ["heads", "tokens"])
def test_past_32_bits_element_by_element(room, dtype, layout):
    """Inputs of more than 2^31 elements and of one sign: the last head's results are those of the head alone, each within its bound of the formula
    (which is the result itself), so that the two are within twice that of each other."""
    import paper_2402_18668_b200 as based
    dt = DTYPES[dtype]
    H, L, d = 33, 1 << 20, 64
    if room < 8 * H * L * d * torch.finfo(dt).bits // 8:
        pytest.skip("no room for seven tensors of 2.2e9 elements")
    gen = torch.Generator(device="cuda").manual_seed(34)
    rate = torch.full((H,), 0.01, device="cuda")

    def tensor():
        x = torch.zeros((1, H, L, d) if layout == "heads" else (1, L, H, d), device="cuda", dtype=dt)
        x = x if layout == "heads" else x.transpose(1, 2)
        x[:, -1] = torch.randn(1, L, d, generator=gen, device="cuda").abs().to(dt)
        return x
    q, k, v = tensor(), tensor(), tensor()
    one = [x[:, -1:].contiguous() for x in (q, k, v)]

    def same(a, b):
        a, b = a[:, -1:].double(), b.double()
        # (a little more, for b in place of the exact value; blocks past some 3000 tokens back weigh nothing at this rate)
        return ((a - b).abs() <= 2.02 * ref.decay_bound(b, b, dt, d, 4096)).all()
    out = based.based_decay_attention_forward(q, k, v, rate)
    assert same(out, based.based_decay_attention_forward(*one, rate[:1])) and out[:, -1].min() > 0
    assert not out[:, :-1].any()
    del out
    grads = based.based_decay_attention_backward(q, k, v, rate, v)
    for a, b in zip(grads[:3], based.based_decay_attention_backward(*one, rate[:1], one[2])[:3]):
        assert same(a, b) and not a[:, :-1].any()
    assert based.based_poll_error() == 0
