"""Tensors that lie in each other's gaps share nothing: one pool for keys and values, an output beside its inputs in a fused buffer."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def pools(kind, pages, H, ps, d, dtype):
    """Keys and values [pages,H,page_size,d] out of one allocation."""
    if kind == "page":
        kv = torch.zeros(pages, 2, H, ps, d, device="cuda", dtype=dtype)
        return kv, kv[:, 0], kv[:, 1]
    if kind == "tokens":
        kv = torch.zeros(pages, 2, ps, H, d, device="cuda", dtype=dtype)
        return kv, kv[:, 0].transpose(1, 2), kv[:, 1].transpose(1, 2)
    if kind == "head":
        kv = torch.zeros(pages, ps, H, 2, d, device="cuda", dtype=dtype)
        return kv, kv[..., 0, :].transpose(1, 2), kv[..., 1, :].transpose(1, 2)
    kv = torch.zeros(pages, ps, H, 2 * d, device="cuda", dtype=dtype)
    return kv, kv[..., :d].transpose(1, 2), kv[..., d:].transpose(1, 2)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("kind", ["page", "tokens", "head", "row"])
def test_one_pool_for_keys_and_values(dtype, kind):
    import paper_2402_18668_b200 as based
    dt = DTYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(3)
    B, Hq, Hk, d, ps, L = 3, 4, 2, 64, 16, 90
    n = L // ps + 2
    table = torch.randperm(B * n, generator=torch.Generator().manual_seed(1)).view(B, n).int().cuda()
    pos, counts = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.tensor([90, 3, 64], dtype=torch.int32, device="cuda")
    rows = [torch.randn(B, Hk, L, d, generator=gen, device="cuda").to(dt) for _ in range(2)]
    q, k, v = (torch.randn(B, h, d, generator=gen, device="cuda").to(dt) for h in (Hq, Hk, Hk))
    kv, kp, vp = pools(kind, B * n, Hk, ps, d, dt)
    apart = [torch.zeros(B * n, Hk, ps, d, device="cuda", dtype=dt) for _ in range(2)]
    outs = []
    for K, V in ((kp, vp), apart):
        based.paged_cache_write(*rows, K, V, table, pos, counts)
        outs.append(based.paged_decode_step(q, k, v, K, V, table, counts))
    assert torch.equal(outs[0], outs[1]) and torch.equal(kp, apart[0]) and torch.equal(vp, apart[1])
    with pytest.raises(ValueError, match="two outputs overlap"):
        based.paged_decode_step(q, k, v, kp, kp, table, counts)
    assert based.based_poll_error() == 0


def test_pools_that_do_overlap():
    """One row, or a part of one, in both."""
    import paper_2402_18668_b200 as based
    B, H, d, ps = 1, 2, 64, 16
    q, table, pos = torch.zeros(B, H, d, device="cuda"), torch.zeros(B, 1, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    kv = torch.zeros(5, 3, H, ps, d, device="cuda")
    flat = kv.view(-1)
    page = 2 * H * ps * d
    for at in (0, 4, ps * d, H * ps * d - 4, H * ps * d + 4, page, -4 + page):           # from the start of the first pool, in floats
        k, v = flat.as_strided((2, H, ps, d), (page, ps * d, d, 1), 0), flat.as_strided((2, H, ps, d), (page, ps * d, d, 1), at)
        with pytest.raises(ValueError, match="two outputs overlap"):
            based.paged_decode_step(q, q, q, k, v, table, pos)
        with pytest.raises(ValueError, match="two outputs overlap"):
            based.paged_cache_write(q[:, :, None], q[:, :, None], k, v, table, pos)
    assert based.based_poll_error() == 0


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_output_beside_its_inputs(dtype):
    """q, k, v and the output as slices of one buffer [B,L,4,H,d]."""
    import paper_2402_18668_b200 as based
    dt = DTYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(4)
    B, L, H, d = 2, 200, 3, 64
    buf = torch.randn(B, L, 4, H, d, generator=gen, device="cuda").to(dt)
    kept = buf.clone()
    q, k, v, out = (buf[:, :, i].transpose(1, 2) for i in range(4))
    rate = torch.linspace(0.01, 0.5, H, device="cuda")
    want = based.based_decay_attention_forward(q, k, v, rate)
    based.based_decay_attention_forward(q, k, v, rate, out=out)
    assert torch.equal(out, want) and torch.equal(buf[:, :, :3], kept[:, :, :3])
    for bad in (q, k, v, buf.view(B, L, 4 * H, d)[:, :, 2 * H + 1:3 * H + 1].transpose(1, 2)):
        with pytest.raises(ValueError, match="overlaps"):
            based.based_decay_attention_forward(q, k, v, rate, out=bad)
    assert based.based_poll_error() == 0
