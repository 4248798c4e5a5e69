"""Integers that do not fit the library's 32 bits are refused, not cut: a window of 2^32 + 64 is none of 64."""
import pytest
import torch

import paper_2402_18668_b200 as based
from paper_2402_18668_b200 import autograd as ag

BEYOND = (2**31, -2**31 - 1, 2**32 + 64, 2**70)


@pytest.mark.parametrize("x", BEYOND)
def test_autograd(x):
    q = torch.zeros(1, 1, 4, 64)
    for call in (lambda: ag.sliding_window_attention(q, q, q, window=x), lambda: ag.qk_norm_rotate(q, q, start=x),
                 lambda: ag.qk_norm_rotate(q, q, flags=x)):
        with pytest.raises(ValueError, match="32 bits"):
            call()


@pytest.mark.gpu
@pytest.mark.parametrize("x", BEYOND)
def test_calls(x):
    q = torch.zeros(1, 1, 4, 64, device="cuda")
    for call in (lambda: based.swa_forward(q, q, q, window=x), lambda: based.swa_backward(q, q, q, q, window=x),
                 lambda: based.based_qk_norm_rotate(q, q, start=x), lambda: based.based_qk_norm_rotate(q, q, flags=x),
                 lambda: based.based_qk_norm_rotate_backward(q, q, q, q, start=x),
                 lambda: based.swa_decode_step(q[:, :, 0], q[:, :, 0], q[:, :, 0], torch.zeros(1, 1, 64, 64, device="cuda"),
                                               torch.zeros(1, 1, 64, 64, device="cuda"), x)):
        with pytest.raises(ValueError, match="32 bits"):
            call()


def test_the_largest_integer_goes_on():
    q = torch.zeros(1, 1, 4, 64)
    for x in (2**31 - 1, -2**31):
        with pytest.raises(ValueError, match="CUDA"):
            ag.sliding_window_attention(q, q, q, window=x)
