"""Attention over a paged cache: a score that is not a number is not lost, whether scores are capped or not."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("where", ["key", "first key", "new key", "query"])
@pytest.mark.parametrize("n", [200, 3000])
def test_nan_shows(dtype, cap, bias, where, n):
    """In a key: all query heads of its key head; in a query: that head; everything else has the same bits as without."""
    import paper_2402_18668_b200 as based
    dt = DTYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(n)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda").to(dt)
    B, Hq, Hk, d, ps = 2, 6, 2, 64, 16
    pages = -(-n // ps)
    kp, vp = normal(B * pages, Hk, ps, d), normal(B * pages, Hk, ps, d)
    table = torch.arange(B * pages, dtype=torch.int32, device="cuda").view(B, pages)
    pos = torch.full((B,), n - 1, dtype=torch.int32, device="cuda")
    q, k, v = normal(B, Hq, d), normal(B, Hk, d), normal(B, Hk, d)
    slopes = torch.linspace(0.01, 0.5, Hq, device="cuda") if bias else None

    def call():
        return based.paged_decode_step(q, k, v, kp, vp, table, pos, softcap=cap, slopes=slopes)
    want = call()
    assert torch.isfinite(want).all()
    hit = torch.zeros(B, Hq, dtype=torch.bool, device="cuda")
    if where == "query":
        q[1, 4, 3] = float("nan")
        hit[1, 4] = True
    else:
        if where == "new key":
            k[1, 1, 5] = float("nan")
        else:
            at = n // 2 if where == "key" else 0
            kp[int(table[1, at // ps]), 1, at % ps, 5] = float("nan")
        hit[1, 3:] = True
    got = call()
    assert torch.isnan(got[hit]).all()
    assert torch.equal(got[~hit], want[~hit])
    assert based.based_poll_error() == 0
