"""torch.autograd glue for the mixers and the layers around them (training-time use).

`linear_attention(q, k, v)` returns based_prefill's output from the empty state (fp32: up to rounding, from the
tensor-core form of the pass where that is the faster and the device has room for its scratch) and, under
autograd, routes the output gradient through based_prefill_backward (with the saved forward
output, which lets the bf16 path merge two of its passes).  The node itself is native
(csrc_host/native.cpp), so neither direction waits for the interpreter; both run in the library's
kernels.

The layers' functions take tensors however they lie: what the kernels can read as it lies is not copied (contiguous ones, and slices of a
fused projection whose rows start on 16-byte boundaries), anything else is.

A backward pass can be captured into a CUDA graph under torch's own rule for that: no eager graph of the same leaves may be alive
(their gradients would be accumulated on the stream that it was built on, which the capture refuses with an error).
"""
from __future__ import annotations

from . import binding as _b


def linear_attention(q, k, v, numerator_only: bool = False):
    """Causal Taylor linear attention of q, k [B,H,L,16] and v [B,H,L,d_v] (bf16 or fp32, CUDA),
    differentiable with respect to q, k and v."""
    return _b.native().linear_attention(q, k, v, _b.BASED_NUMERATOR_ONLY if numerator_only else 0)


def sliding_window_attention(q, k, v, window: int = 64, softmax_scale: float = 0.0):
    """swa_forward of q, k, v [B,H,L,64], differentiable with respect to them (swa_backward)."""
    return _b.native().sliding_window(q, k, v, int(window), float(softmax_scale))


def qk_norm_rotate(q, k, q_weight=None, k_weight=None, freqs=None, positions=None, eps: float = 1e-6, flags: int = 0,
                   start: int = 0):
    """based_qk_norm_rotate, differentiable with respect to q, k and the weights: projections [B,L,H,d] -> what the mixers
    take, [B,H,L,d]."""
    return _b.native().qk_norm_rotate(q, k, q_weight, k_weight, freqs, positions, float(eps), int(flags), int(start))


def gated_recurrence(x, r, g, rate, state=None):
    """based_gated_recurrence_forward, differentiable with respect to x, r, g [B,N,C], rate [C] and state [B,C].  Returns
    (out, the state behind the last token), both differentiable."""
    return _b.native().gated_recurrence(x, r, g, rate, state)


def decay_attention(q, k, v, rate, documents=None, state=None, scale: float = 0.0, return_state: bool = True):
    """based_decay_attention_forward, differentiable with respect to q, k [B,H,L,d_k], v [B,H,L,d_v] and state [B,H,d_k,d_v]; the
    rates [H] are constants (one that requires a gradient is refused).  Returns (out, the state behind the last token), both
    differentiable; with return_state=False (out, None), which in bf16 takes up to half the time and may differ in the last bits of out."""
    return _b.native().decay_attention(q, k, v, rate, documents, state, float(scale), int(return_state))
