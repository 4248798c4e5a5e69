"""Argument checks of the recurrence's, the norm-and-rotation's and the window backward's C entry points: host only."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2402_18668_b200 import build
    build.build()
    from paper_2402_18668_b200 import binding
    return binding.lib()


def P(i):
    return ctypes.c_void_p(0x10000 * (i + 1))      # aligned, never read: the checks fail first


U = ctypes.c_void_p(0x8008)
INVALID, UNSUPPORTED, ALIGNMENT, WORKSPACE = 1, 2, 3, 6


def T(p, batch=128, token=16):
    from paper_2402_18668_b200.binding import Tokens
    return Tokens(p, batch, token)


def test_recurrence(lib):
    def f(x=P(0), r=P(1), g=P(2), rate=P(3), si=None, out=P(4), so=None, B=2, N=8, C=16, io=1, batch=128, token=16):
        return lib.based_gated_recurrence_forward(T(x, batch, token), T(r), T(g), rate, si, out, so, B, N, C, io, None)
    for k in ("x", "r", "g", "rate", "out"):
        assert f(**{k: None}) == INVALID
        assert f(**{k: U}) == ALIGNMENT
    assert f(si=U) == ALIGNMENT and f(so=U) == ALIGNMENT
    assert f(B=0) == f(N=0) == f(C=0) == f(N=-1) == f(io=2) == INVALID
    assert f(C=12) == f(token=20, batch=160) == f(batch=132) == f(io=0, batch=130) == UNSUPPORTED
    assert f(token=8) == f(batch=120) == f(batch=0) == f(batch=-128) == f(token=-16) == INVALID
    assert f(out=P(0)) == f(out=P(1)) == f(out=P(2)) == f(so=P(3)) == f(so=P(4)) == f(si=P(4)) == INVALID
    assert f(B=2**31 - 1, N=2, C=2**31 - 8) == f(N=2**31 - 1) == UNSUPPORTED
    s = lib.based_gated_recurrence_step
    assert s(T(P(0)), T(P(1)), T(P(2)), P(3), None, P(4), P(5), 1, 16, 1, None) == INVALID
    assert s(T(P(0)), T(P(1)), T(P(2)), P(3), P(5), P(4), None, 1, 16, 1, None) == INVALID
    assert s(T(P(0)), T(P(1)), T(P(2)), P(3), P(5), P(4), P(5), 1, 20, 1, None) == UNSUPPORTED


def test_recurrence_backward(lib):
    need = lib.based_gated_recurrence_backward_workspace_bytes(2, 8, 16, 1)
    assert need >= 2 * 16 * 4
    assert lib.based_gated_recurrence_backward_workspace_bytes(0, 8, 16, 1) == 0

    def f(ws=P(20), bytes_=need, B=2, N=8, C=16, io=1, **kw):
        names = ("x", "r", "g", "rate", "si", "out", "dout", "dso", "dx", "dr", "dg", "drate", "dsi")
        a = {n: P(i) for i, n in enumerate(names)} | kw
        a |= {n: T(a[n]) for n in ("x", "r", "g", "out", "dout")}
        return lib.based_gated_recurrence_backward(*(a[n] for n in names), B, N, C, io, ws, bytes_, None)
    for k in ("x", "r", "g", "rate", "out", "dout", "dx", "dr", "dg", "drate"):
        assert f(**{k: None}) == INVALID
        assert f(**{k: U}) == ALIGNMENT
    assert f(dsi=U) == f(dso=U) == f(ws=U) == ALIGNMENT
    assert f(ws=None) == f(bytes_=need - 1) == WORKSPACE
    assert f(dx=P(0)) == f(dr=P(8)) == f(drate=P(20)) == f(dg=P(7)) == f(dg=P(5)) == INVALID
    assert f(C=4) == UNSUPPORTED and f(io=3) == INVALID and f(N=0) == INVALID and f(N=9) == INVALID


def test_norm_rotate(lib):
    def f(q=P(0), k=P(1), sq=128, sk=128, wq=P(2), wk=P(3), fr=P(4), pos=P(5), per=1, start=0, oq=P(6), ok=P(7), B=1, L=8, Hq=2, Hk=2,
          d=64, n=32, eps=1e-6, io=1, flags=0):
        return lib.based_qk_norm_rotate(q, k, sq, sk, wq, wk, fr, pos, per, start, oq, ok, B, L, Hq, Hk, d, n, eps, io, flags, None)
    for k in ("q", "k", "oq", "ok"):
        assert f(**{k: None}) == INVALID
        assert f(**{k: U}) == ALIGNMENT
    assert f(wq=U) == f(wk=U) == f(fr=ctypes.c_void_p(0x1004)) == f(pos=ctypes.c_void_p(0x1002)) == ALIGNMENT
    assert f(B=0) == f(L=0) == f(Hq=0) == f(Hk=0) == f(d=0) == f(n=-8) == f(io=5) == f(flags=1) == f(eps=-1.0) == f(eps=float("nan")) == INVALID
    assert f(fr=None) == f(n=0) == f(per=2) == f(sq=64) == f(sk=127) == INVALID
    assert f(d=40, sq=80, sk=80) == f(d=272, sq=544, sk=544) == f(n=12) == f(n=40) == f(sq=130) == f(B=2**16, L=2**15) == UNSUPPORTED
    assert f(oq=P(0)) == f(ok=P(1)) == f(ok=P(6)) == f(oq=P(3)) == INVALID


def test_norm_rotate_backward(lib):
    need = lib.based_qk_norm_rotate_backward_workspace_bytes(1, 8, 2, 2, 64, 1)
    assert need >= 2 * 64 * 4 and lib.based_qk_norm_rotate_backward_workspace_bytes(1, 8, 2, 2, 40, 1) == 0

    def f(q=P(0), k=P(1), wq=P(2), gq=P(8), gk=P(9), dq=P(10), dk=P(11), sdq=128, sdk=128, dwq=P(12), dwk=P(13), ws=P(14), bytes_=need, d=64):
        return lib.based_qk_norm_rotate_backward(q, k, 128, 128, wq, P(3), P(4), None, 0, 0, gq, gk, dq, dk, sdq, sdk, dwq, dwk, 1, 8, 2, 2,
                                                 d, 32, 1e-6, 1, 0, ws, bytes_, None)
    for k in ("q", "k", "gq", "gk", "dq", "dk"):
        assert f(**{k: None}) == INVALID
        assert f(**{k: U}) == ALIGNMENT
    assert f(dwq=None) == f(dwk=None) == f(dwk=P(12)) == f(dq=P(11)) == f(dq=P(8)) == f(dwq=P(2)) == f(sdq=64) == INVALID
    assert f(sdk=130) == UNSUPPORTED and f(d=40) == UNSUPPORTED
    assert f(ws=None) == f(bytes_=need - 4) == WORKSPACE
    assert f(dwq=U) == f(ws=U) == ALIGNMENT


def test_swa_backward(lib):
    need = lib.swa_backward_workspace_bytes(1, 2, 70, 64, 0)
    assert lib.swa_backward_workspace_bytes(1, 2, 70, 129, 1) == 0

    def f(q=P(0), k=P(1), v=P(2), do=P(3), dq=P(4), dk=P(5), dv=P(6), L=70, d=64, w=64, io=0, ws=P(7), bytes_=need):
        return lib.swa_backward(q, k, v, do, dq, dk, dv, 1, 2, L, d, w, 0.0, io, ws, bytes_, None)
    for k in ("q", "k", "v", "do", "dq", "dk", "dv"):
        assert f(**{k: None}) == INVALID
        assert f(**{k: U}) == ALIGNMENT
    assert f(L=0) == f(w=0) == f(io=2) == f(dq=P(0)) == f(dk=P(4)) == f(dv=P(3)) == f(dv=P(7)) == INVALID
    assert f(d=32) == f(w=129) == UNSUPPORTED
    assert need == 0 or f(ws=None) == f(bytes_=need - 1) == WORKSPACE


def test_host_tensors_are_refused():
    import torch
    import paper_2402_18668_b200 as based
    from paper_2402_18668_b200 import autograd as ag
    with pytest.raises(ValueError, match="CUDA"):
        based.based_gated_recurrence_forward(*(torch.zeros(1, 2, 8) for _ in range(3)), torch.zeros(8))
    with pytest.raises(ValueError, match="dimensions"):
        based.based_gated_recurrence_step(*(torch.zeros(1, 2, 8) for _ in range(3)), torch.zeros(8), torch.zeros(1, 8))
    with pytest.raises(ValueError, match="CUDA"):
        based.based_qk_norm_rotate(torch.zeros(1, 2, 2, 64), torch.zeros(1, 2, 2, 64))
    with pytest.raises(ValueError, match="CUDA"):
        based.swa_backward(*(torch.zeros(1, 1, 4, 64) for _ in range(4)))
    for call in (lambda: ag.sliding_window_attention(*(torch.zeros(1, 1, 4, 64) for _ in range(3))),
                 lambda: ag.qk_norm_rotate(torch.zeros(1, 2, 2, 64), torch.zeros(1, 2, 2, 64)),
                 lambda: ag.gated_recurrence(*(torch.zeros(1, 2, 8) for _ in range(3)), torch.zeros(8))):
        with pytest.raises(ValueError, match="CUDA"):
            call()
