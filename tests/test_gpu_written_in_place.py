"""What a call writes in the caller's tensors counts as a change in place: a graph that saved one of them refuses its backward pass."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def based():
    import paper_2402_18668_b200 as based
    return based


def f32(*shape):
    return torch.randn(*shape, device="cuda")


def bf16(*shape):
    return f32(*shape).bfloat16()


def calls(based):
    """name -> (the call, the tensors of the caller's that it writes)."""
    B, H, L, d, ps = 1, 2, 5, 64, 16
    rate, state, last = torch.rand(H, device="cuda"), f32(B, H, d, d), f32(B, H, d, d)
    q, k, v, out = (bf16(B, H, L, d) for _ in range(4))
    qt, kt, vt, outt = (bf16(B, H, d) for _ in range(4))
    kp, vp = bf16(3, H, ps, d), bf16(3, H, ps, d)
    table, pos = torch.zeros(B, 1, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    x, xo, xt, xto, xs, xl, xr = bf16(B, L, 32), bf16(B, L, 32), bf16(B, 32), bf16(B, 32), f32(B, 32), f32(B, 32), torch.rand(32, device="cuda")
    lq, lk, lv, lo = bf16(B, H, L, 16), bf16(B, H, L, 16), bf16(B, H, L, 64), bf16(B, H, L, 64)
    lqt, lkt, lvt, lot = bf16(B, H, 16), bf16(B, H, 16), bf16(B, H, 64), bf16(B, H, 64)
    kv, z = based.new_state(B, H, 64)
    kvs, zs = based.new_state(B, H, 64, sym=True)
    kc, vc = bf16(B, H, 64, d), bf16(B, H, 64, d)
    h, b2, cs, cc, cg, co = f32(3, 64), f32(64), bf16(B, 2, 64), bf16(B, 64), bf16(B, 64), bf16(B, 64)
    rq, rk, ro_q, ro_k = bf16(B, L, H, d), bf16(B, L, H, d), bf16(B, H, L, d), bf16(B, H, L, d)
    return {
        "decay, prompt": (lambda: based.based_decay_attention_forward(q, k, v, rate, out=out, state_out=last), (out, last)),
        "decay, step": (lambda: based.based_decay_attention_step(qt, kt, vt, rate, state, out=outt), (state, outt)),
        "decay, step, state_out": (lambda: based.based_decay_attention_step(qt, kt, vt, rate, state, state_out=last), (last,)),
        "paged, step": (lambda: based.paged_decode_step(qt, kt, vt, kp, vp, table, pos, out=outt), (outt, kp, vp)),
        "paged, prompt": (lambda: based.paged_cache_write(q, k, kp, vp, table, pos), (kp, vp)),
        "recurrence, prompt": (lambda: based.based_gated_recurrence_forward(x, x, x, xr, state_in=xs, out=xo, state_out=xl), (xo, xl)),
        "recurrence, step": (lambda: based.based_gated_recurrence_step(xt, xt, xt, xr, xs, out=xto), (xs, xto)),
        "rotation": (lambda: based.based_qk_norm_rotate(rq, rk, out_q=ro_q, out_k=ro_k), (ro_q, ro_k)),
        "prefill": (lambda: based.based_prefill(lq, lk, lv, out=lo, kv_state=kv, z_state=z), (lo, kv, z)),
        "prefill, state": (lambda: based.based_prefill_state(lk, lv, kv, z), (kv, z)),
        "decode": (lambda: based.based_decode_step(lqt, lkt, lvt, kv, z, out=lot), (kv, z, lot)),
        "state, symmetric": (lambda: based.based_state_to_sym(kv, z, kvs, zs), (kvs, zs)),
        "state, whole": (lambda: based.based_state_from_sym(kvs, zs, kv, z), (kv, z)),
        "window": (lambda: based.swa_forward(q, k, v, out=out), (out,)),
        "window, step": (lambda: based.swa_decode_step(qt, kt, vt, kc, vc, 3, out=outt), (kc, vc, outt)),
        "convolution, step": (lambda: based.baseconv_gate_step(cc, cg, h, b2, cs, out=co), (cs, co)),
    }


def test_every_call_counts(based):
    for name, (call, writes) in calls(based).items():
        before = [t._version for t in writes]
        call()
        assert all(t._version > n for t, n in zip(writes, before)), name
    assert based.based_poll_error() == 0


def test_a_saved_state_that_a_step_overwrites(based):
    from paper_2402_18668_b200 import autograd as ag
    q, k, v = (bf16(1, 2, 70, 64).requires_grad_() for _ in range(3))
    rate, state = torch.rand(2, device="cuda"), f32(1, 2, 64, 64)
    out, _ = ag.decay_attention(q, k, v, rate, state=state)
    token = [x.detach()[:, :, 0].contiguous() for x in (q, k, v)]
    based.based_decay_attention_step(*token, rate, state)
    with pytest.raises(RuntimeError, match="inplace"):
        out.float().sum().backward()
    x = bf16(1, 70, 32).requires_grad_()
    state = f32(1, 32)
    out, _ = ag.gated_recurrence(x, x, x, torch.rand(32, device="cuda"), state)
    t = x.detach()[:, 0].contiguous()
    based.based_gated_recurrence_step(t, t, t, torch.rand(32, device="cuda"), state)
    with pytest.raises(RuntimeError, match="inplace"):
        out.float().sum().backward()


def test_a_view_of_a_saved_pool(based):
    """The pages of one layer's pool are a slice of all layers'."""
    pool = bf16(2, 2, 3, 2, 16, 64)
    weight = torch.ones((), device="cuda", dtype=torch.bfloat16, requires_grad=True)
    y = (pool * weight).sum()
    q, table, pos = bf16(1, 2, 64), torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    based.paged_decode_step(q, q, q, pool[1, 0], pool[1, 1], table, pos)
    with pytest.raises(RuntimeError, match="inplace"):
        y.backward()


def test_tensors_of_inference_mode(based):
    with torch.inference_mode():
        inside = calls(based)
    for name, (call, _) in inside.items():
        call()
    with torch.inference_mode():
        for call, _ in calls(based).values():
            call()
    assert based.based_poll_error() == 0
