"""Attention over a paged cache at the last positions that its tables can hold, just below 2^31."""
import pytest
import torch

import attention64 as ref

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
PAGE, PAGES = 2 * 9 * 7 * 11, 31 * 151 * 331           # 2^31 - 2 tokens


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("window", [1, 5, 100, 2000])
@pytest.mark.parametrize("back", [1, 2, 14, 15, 16, 17, 65])
def test_last_positions(dtype, window, back):
    """A window makes them cheap to reach: the pool holds the last pages alone."""
    import paper_2402_18668_b200 as based
    assert PAGE * PAGES == 2**31 - 2
    dt = DTYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(back)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda").to(dt)
    B, Hq, Hk, d, last = 2, 4, 2, 64, 3
    kp, vp = normal(B * last, Hk, PAGE, d), normal(B * last, Hk, PAGE, d)
    table = torch.full((B, PAGES), -1, dtype=torch.int32, device="cuda")
    table[:, -last:] = torch.arange(B * last, dtype=torch.int32, device="cuda").view(B, last)
    pos = torch.full((B,), 2**31 - 2 - back, dtype=torch.int32, device="cuda")
    q, k, v = normal(B, Hq, d), normal(B, Hk, d), normal(B, Hk, d)
    slopes = torch.linspace(0.01, 0.1, Hq, device="cuda")
    # the same with the pages ahead of the last ones cut off: distances stay
    want, bound, kw, vw = ref.paged(q, k, v, kp, vp, table[:, -last:], pos - (PAGES - last) * PAGE, None, 30.0, slopes, window)
    out = based.paged_decode_step(q, k, v, kp, vp, table, pos, softcap=30.0, slopes=slopes, window=window)
    assert ((out.double() - want).abs() <= bound).all()
    assert torch.equal(kp, kw) and torch.equal(vp, vw)
    assert based.based_poll_error() == 0


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_prompt_up_to_the_last_position(dtype):
    """A copy that ends at the last token; what would lie behind it is reported and goes nowhere."""
    import paper_2402_18668_b200 as based
    dt = DTYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(1)
    H, d, L = 2, 64, 100
    kp, vp = (torch.zeros(1, H, PAGE, d, device="cuda", dtype=dt) for _ in range(2))
    table = torch.full((1, PAGES), -1, dtype=torch.int32, device="cuda")
    table[0, -1] = 0
    k, v = (torch.randn(1, H, L, d, generator=gen, device="cuda").to(dt) for _ in range(2))
    pos = torch.full((1,), 2**31 - 2 - L, dtype=torch.int32, device="cuda")
    based.paged_cache_write(k, v, kp, vp, table, pos)
    assert based.based_poll_error() == 0
    assert torch.equal(kp[0, :, -L:], k[0]) and torch.equal(vp[0, :, -L:], v[0]) and not kp[0, :, :-L].any()
    before = kp.clone()
    based.paged_cache_write(-k, v, kp, vp, table, pos + 40)
    assert based.based_poll_error() == 1
    before[0, :, PAGE - L + 40:] = -k[0, :, :L - 40]
    assert torch.equal(kp, before)
