"""Argument checks of decay attention's and the paged cache's C entry points: host only."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2402_18668_b200 import build
    build.build()
    from paper_2402_18668_b200 import binding
    return binding.lib()


def P(i):
    return ctypes.c_void_p(0x100000 * (i + 1))     # aligned, never read: the checks fail first


U = ctypes.c_void_p(0x100008)
INVALID, UNSUPPORTED, ALIGNMENT, WORKSPACE = 1, 2, 3, 6


def V(p, batch=2 * 300 * 64, head=300 * 64, token=64):
    from paper_2402_18668_b200.binding import Heads
    return Heads(p, batch, head, token)


def test_decay_forward(lib):
    bytes_of = lib.based_decay_attention_workspace_bytes
    need = bytes_of(2, 2, 300, 64, 64, 1, 1)
    assert need > 0 and bytes_of(0, 2, 300, 64, 64, 1, 1) == bytes_of(2, 2, 300, 63, 64, 1, 1) == bytes_of(2, 2, 300, 64, 136, 1, 1) == 0

    def f(q=P(0), k=P(1), v=P(2), rate=P(3), docs=P(4), si=P(5), out=P(6), so=P(7), B=2, H=2, L=300, dk=64, dv=64, scale=0.0, io=1, ws=P(8), n=1 << 40,
          q_=None, out_=None):
        return lib.based_decay_attention_forward(q_ or V(q), V(k), V(v), rate, docs, si, out_ or V(out), so, B, H, L, dk, dv, scale, io, ws, n, None)
    for x in ("q", "k", "v", "rate", "out"):
        assert f(**{x: None}) == INVALID
        assert f(**{x: U}) == ALIGNMENT
    assert f(si=U) == f(so=U) == f(ws=U) == f(docs=ctypes.c_void_p(0x100002)) == ALIGNMENT
    assert f(B=0) == f(H=-1) == f(L=0) == f(dk=0) == f(dv=-8) == f(io=2) == INVALID
    assert f(dk=60) == f(dv=136) == f(dk=256) == f(L=2**31 - 1) == f(B=2**20, H=2**12) == UNSUPPORTED
    assert f(out=P(0)) == f(out=P(5)) == f(so=P(5)) == f(so=P(2)) == f(out=P(7)) == f(out=P(8)) == f(so=P(8)) == INVALID
    assert f(q_=V(P(0), token=56)) == f(q_=V(P(0), head=0)) == f(q_=V(P(0), batch=-64)) == INVALID
    assert f(q_=V(P(0), token=68)) == f(q_=V(P(0), token=1 << 38)) == UNSUPPORTED
    assert f(out_=V(P(6), head=64, token=64)) == f(out_=V(P(6), batch=64)) == INVALID         # rows over each other
    assert f(n=need - 1) == f(ws=None) == WORKSPACE
    assert f(scale=1e-30) == f(scale=1e30) == f(scale=float("inf")) == UNSUPPORTED


def test_decay_step(lib):
    def f(q=P(0), k=P(1), v=P(2), rate=P(3), si=P(4), out=P(5), so=P(6), B=2, H=2, dk=64, dv=64, io=1, scale=0.0):
        return lib.based_decay_attention_step(q, k, v, rate, si, out, so, B, H, dk, dv, scale, io, None)
    for x in ("q", "k", "v", "rate", "si", "out", "so"):
        assert f(**{x: None}) == INVALID
        assert f(**{x: U}) == ALIGNMENT
    assert f(B=0) == f(H=0) == f(dk=0) == f(io=7) == f(out=P(0)) == f(out=P(4)) == f(out=P(6)) == f(so=P(0)) == f(so=P(3)) == INVALID
    assert f(dk=12) == f(dv=136) == f(B=2**16, H=2**16) == f(scale=1e-30) == f(scale=float("inf")) == UNSUPPORTED


def test_decay_backward(lib):
    need = lib.based_decay_attention_backward_workspace_bytes(2, 2, 300, 64, 64, 1, 1)
    assert need > 0
    names = ("q", "k", "v", "rate", "docs", "si", "do", "dso", "dq", "dk", "dv", "dsi")
    views = {"q", "k", "v", "do", "dq", "dk", "dv"}

    def f(n=need, ws=P(20), B=2, io=1, d_k=64, scale=0.0, **kw):
        a = {x: P(i) for i, x in enumerate(names)} | kw
        a |= {x: V(a[x]) for x in views}
        return lib.based_decay_attention_backward(*(a[x] for x in names), B, 2, 300, d_k, 64, scale, io, ws, n, None)
    for x in ("q", "k", "v", "rate", "do", "dq", "dk", "dv"):
        assert f(**{x: None}) == INVALID
        assert f(**{x: U}) == ALIGNMENT
    assert f(si=U) == f(dso=U) == f(dsi=U) == f(ws=U) == ALIGNMENT
    assert f(dq=P(0)) == f(dk=P(9 - 1)) == f(dv=P(6)) == f(dsi=P(5)) == f(dsi=P(7)) == f(dv=P(20)) == f(B=0) == f(io=3) == INVALID
    assert f(d_k=60) == f(scale=1e-30) == f(scale=1e30) == UNSUPPORTED
    assert f(ws=None) == f(n=need - 1) == WORKSPACE


def test_paged(lib):
    from paper_2402_18668_b200.binding import Pages
    bytes_of = lib.based_paged_decode_step_workspace_bytes
    need = bytes_of(2, 4, 2, 64, 16, 100, 1)
    assert need > 0 and bytes_of(2, 3, 2, 64, 16, 100, 1) == bytes_of(2, 4, 2, 60, 16, 100, 1) == bytes_of(2, 4, 2, 64, 16, 2**30, 1) == 0

    def C(k=P(10), v=P(11), page=2 * 16 * 64, head=16 * 64, token=64, pages=50, size=16):
        return Pages(k, v, page, head, token, pages, size)

    def f(q=P(0), k=P(1), v=P(2), c=None, table=P(3), pos=P(4), slopes=P(5), out=P(6), B=2, Hq=4, Hk=2, d=64, mp=100, window=0, cap=0.0, io=1, ws=P(7), n=need, scale=0.0):
        return lib.based_paged_decode_step(q, k, v, c or C(), table, pos, slopes, out, B, Hq, Hk, d, mp, window, scale, cap, io, ws, n, None)

    def w(k=P(0), v=P(1), c=None, table=P(3), pos=P(4), counts=P(5), B=2, H=2, L=300, d=64, mp=100, io=1):
        return lib.based_paged_cache_write(V(k), V(v), c or C(), table, pos, counts, B, H, L, d, mp, io, None)
    for x in ("q", "k", "v", "table", "pos", "out"):
        assert f(**{x: None}) == INVALID
    for x in ("k", "v", "table", "pos"):
        assert w(**{x: None}) == INVALID
    for x in ("q", "k", "v", "out", "ws"):
        assert f(**{x: U}) == ALIGNMENT
    assert f(table=ctypes.c_void_p(0x100002)) == f(pos=ctypes.c_void_p(0x100001)) == f(slopes=ctypes.c_void_p(0x100002)) == w(counts=ctypes.c_void_p(0x100002)) == w(k=U) == ALIGNMENT
    for g in (f, w):
        assert g(B=0) == g(d=0) == g(mp=0) == g(io=2) == INVALID
        assert g(d=60) == g(d=136) == g(mp=2**30) == UNSUPPORTED
        assert g(c=C(k=None)) == g(c=C(v=P(10))) == g(c=C(pages=0)) == g(c=C(size=0)) == g(c=C(token=32)) == g(c=C(head=64)) == g(c=C(page=16 * 64)) == INVALID
        assert g(c=C(token=68)) == g(c=C(page=1 << 41)) == UNSUPPORTED
        assert g(c=C(k=U)) == ALIGNMENT
    assert f(Hq=3) == f(Hk=0) == f(window=-1) == f(cap=-1.0) == f(cap=float("nan")) == f(out=P(0)) == f(out=P(10)) == f(out=P(7)) == f(ws=P(10)) == INVALID
    assert f(n=need - 1) == f(ws=None) == WORKSPACE
    assert f(cap=float("inf")) == f(cap=1e-30) == f(scale=1e-30) == f(scale=float("inf")) == UNSUPPORTED
    assert w(L=0) == w(k=P(10)) == w(v=P(11)) == INVALID
    assert w(L=2**31 - 1) == w(B=2**18, H=2**13) == UNSUPPORTED


def test_host_tensors_are_refused():
    import torch
    import paper_2402_18668_b200 as based
    from paper_2402_18668_b200 import autograd as ag
    x, rate = torch.zeros(1, 2, 4, 64), torch.zeros(2)
    ints = torch.zeros(1, 4, dtype=torch.int32)
    for call in (lambda: based.based_decay_attention_forward(x, x, x, rate), lambda: based.based_decay_attention_backward(x, x, x, rate, x),
                 lambda: based.based_decay_attention_step(x[:, :, 0], x[:, :, 0], x[:, :, 0], rate, torch.zeros(1, 2, 64, 64)),
                 lambda: ag.decay_attention(x, x, x, rate), lambda: based.paged_decode_step(x[:, :, 0], x[:, :, 0], x[:, :, 0], x, x, ints, ints[:, 0]),
                 lambda: based.paged_cache_write(x, x, x, x, ints, ints[:, 0])):
        with pytest.raises(ValueError, match="CUDA"):
            call()
