"""Decay attention with a rate that is not a number: everything that it fades is not one either, the other heads are as without."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def inputs(dtype, B, H, L, dk, dv):
    gen = torch.Generator(device="cuda").manual_seed(L)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")
    q, k, v, do = normal(B, H, L, dk), normal(B, H, L, dk), normal(B, H, L, dv), normal(B, H, L, dv)
    rate = torch.linspace(0.01, 0.5, H, device="cuda")
    broken = rate.clone()
    broken[1] = float("nan")
    return [x.to(dtype) for x in (q, k, v, do)], rate, broken, normal(B, H, dk, dv), normal(B, H, dk, dv)


def others(x):
    return torch.cat([x[:, :1], x[:, 2:]], 1)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("size", [(2, 3, 1, 64, 64), (1, 3, 100, 64, 64), (1, 3, 2500, 64, 128), (20, 9, 300, 128, 128)], ids=str)
@pytest.mark.parametrize("states", [False, True])
@pytest.mark.parametrize("documents", [False, True])
def test_prompt_and_gradients(dtype, size, states, documents):
    import paper_2402_18668_b200 as based
    (q, k, v, do), rate, broken, state, dstate = inputs(DTYPES[dtype], *size)
    B, H, L, dk, dv = size
    ids = torch.zeros(B, L, dtype=torch.int32, device="cuda") if documents else None
    res = []
    for r in (rate, broken):
        last = torch.zeros_like(state) if states else None
        out = based.based_decay_attention_forward(q, k, v, r, documents=ids, state_in=state if states else None, state_out=last)
        grads = based.based_decay_attention_backward(q, k, v, r, do, documents=ids, state_in=state if states else None,
                                                     dstate_out=dstate if states else None)
        res.append([out, last, *grads])
    for a, b in zip(*res):
        if a is not None:
            assert torch.isfinite(a).all() and torch.equal(others(a), others(b))
    out, last, dq, dk_, dv_, dstate_in = (None if x is None else x[:, 1] for x in res[1])
    # S_0 = a S + k v^T; the last token's R is not faded yet, so that its gradients are what they are
    assert torch.isnan(out).all() and torch.isnan(dq).all() and torch.isnan(dk_[:, :-1]).all() and torch.isnan(dv_[:, :-1]).all()
    if states:
        assert torch.isnan(last).all() and torch.isnan(dstate_in).all()
    assert based.based_poll_error() == 0


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_step(dtype):
    import paper_2402_18668_b200 as based
    (q, k, v, _), rate, broken, state, _ = inputs(DTYPES[dtype], 2, 3, 1, 64, 40)
    q, k, v = (x[:, :, 0].contiguous() for x in (q, k, v))
    new = [torch.empty_like(state) for _ in range(2)]
    out = [based.based_decay_attention_step(q, k, v, r, state, state_out=s) for r, s in zip((rate, broken), new)]
    assert torch.isnan(out[1][:, 1]).all() and torch.isnan(new[1][:, 1]).all()
    assert torch.equal(others(out[0]), others(out[1])) and torch.equal(others(new[0]), others(new[1]))
