"""The rotation's backward pass with one weight alone, on a stream of the caller's: what it writes besides the gradients that it returns
lies in memory that nobody else is given meanwhile."""
import pytest
import torch

import paper_2402_18668_b200 as based

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("which", ["q", "k"])
def test_one_weight_on_another_stream(which):
    B, L, H, d = 1, 40, 2, 64
    q, k = (torch.randn(B, L, H, d, device="cuda").bfloat16() for _ in range(2))
    gq, gk = (torch.randn(B, H, L, d, device="cuda").bfloat16() for _ in range(2))
    w = 1 + 0.1 * torch.randn(d, device="cuda")
    wq, wk = (w, None) if which == "q" else (None, w)
    want = based.based_qk_norm_rotate_backward(q, k, gq, gk, wq, wk)
    both = based.based_qk_norm_rotate_backward(q, k, gq, gk, w if which == "q" else torch.ones_like(w), torch.ones_like(w) if which == "q" else w)
    assert (want[2] is None) == (which == "k") and (want[3] is None) == (which == "q")
    assert all(a is None or torch.equal(a, b) for a, b in zip(want, both))
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(40_000_000)                        # the call's kernels run after what follows on the current stream
    got = based.based_qk_norm_rotate_backward(q, k, gq, gk, wq, wk, stream=s)
    later = [torch.full((d,), 7.0, device="cuda") for _ in range(64)]
    torch.cuda.synchronize()
    assert all((t == 7).all() for t in later)
    assert all(a is None or torch.equal(a, b) for a, b in zip(got, want))
