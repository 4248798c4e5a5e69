"""A decay that leaves nothing of a state drops it whatever it holds, in a prompt and in a step alike."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("dk,dv", [(64, 64), (40, 72), (128, 128)])
def test_step_as_a_prompt_of_one_token(dtype, value, dk, dv):
    import paper_2402_18668_b200 as based
    dt = DTYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(dk)
    B, H = 2, 4
    q, k, v = (torch.randn(B, H, d, generator=gen, device="cuda").to(dt) for d in (dk, dk, dv))
    rate = torch.tensor([float("inf"), 3e38, 1000.0, 0.1], device="cuda")
    state = torch.randn(B, H, dk, dv, generator=gen, device="cuda")
    state[:, :, 3, 5] = value
    state[:, 1] = value
    last, new = torch.empty_like(state), torch.empty_like(state)
    prompt = based.based_decay_attention_forward(q[:, :, None], k[:, :, None], v[:, :, None], rate, state_in=state, state_out=last)[:, :, 0]
    step = based.based_decay_attention_step(q, k, v, rate, state, state_out=new)
    outer = k.double()[..., None] * v.double()[..., None, :]
    score = (q.double() * k.double()).sum(-1, keepdim=True) / dk ** 0.5
    terms = (q.double() * k.double()).abs().sum(-1, keepdim=True) / dk ** 0.5 * v.double().abs()
    # the outer product's rounding (the prompt's bf16 parts hold 24 bits); a sum of dk products, the score's or the state's rounding, the output's
    eps = torch.finfo(dt).eps
    for out, S in ((prompt, last), (step, new)):
        assert ((S[:, :3].double() - outer[:, :3]).abs() <= outer[:, :3].abs() * 2.0 ** -20 + 1e-30).all()
        assert ((out[:, :3].double() - score[:, :3] * v[:, :3].double()).abs()
                <= terms[:, :3] * (dk * 2.0 ** -23 + eps) + eps * (score * v.double()).abs()[:, :3] + 1e-30).all()
        assert not torch.isfinite(out[:, 3]).all() and not torch.isfinite(S[:, 3, 3, 5]).any()
    kept = state.clone()
    assert torch.equal(based.based_decay_attention_step(q, k, v, rate, kept)[:, :3], step[:, :3]) and torch.equal(kept[:, :3], new[:, :3])
    assert based.based_poll_error() == 0
