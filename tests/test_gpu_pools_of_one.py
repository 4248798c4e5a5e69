"""Paged cache: dimensions of size 1 have strides that mean nothing, and may differ between the pools."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", [(5, 1, 16, 64), (1, 2, 128, 64), (80, 2, 1, 64), (1, 1, 128, 64)], ids=str)
def test_strides_of_dimensions_of_one(dtype, shape):
    import paper_2402_18668_b200 as based
    gen = torch.Generator(device="cuda").manual_seed(1)
    pages, H, ps, d = shape
    n = min(pages, -(-70 // ps))
    table = torch.arange(n, dtype=torch.int32, device="cuda")[None]
    pos, L = torch.tensor([n * ps - 1], dtype=torch.int32, device="cuda"), n * ps - 1
    rows = [torch.randn(1, H, L, d, generator=gen, device="cuda").to(dtype) for _ in range(2)]
    q, k, v = (torch.randn(1, h, d, generator=gen, device="cuda").to(dtype) for h in (2 * H, H, H))
    kp, vp = torch.zeros(shape, device="cuda", dtype=dtype), torch.zeros(shape, device="cuda", dtype=dtype)
    odd = [8 if size == 1 else stride for size, stride in zip(shape, kp.stride())]
    vo = torch.zeros_like(vp).as_strided(shape, odd)
    assert vo.stride() != kp.stride()
    outs = []
    for values in (vp, vo):
        based.paged_cache_write(*rows, kp, values, table, torch.zeros_like(pos))
        outs.append(based.paged_decode_step(q, k, v, kp, values, table, pos))
    assert torch.equal(outs[0], outs[1]) and torch.equal(vp, vo) and outs[0].float().abs().max() > 0
    if H > 1 and ps > 1:
        with pytest.raises(ValueError, match="one layout"):
            based.paged_decode_step(q, k, v, kp, torch.zeros(pages, ps, H, d, device="cuda", dtype=dtype).transpose(1, 2), table, pos)
    assert based.based_poll_error() == 0
