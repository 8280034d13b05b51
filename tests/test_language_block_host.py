"""Refusals of the language-model block's calls, and their workspace sizes: nothing is launched, no GPU is needed."""
import ctypes as C

import pytest
import torch

import paper_2111_11124_amd as m
from paper_2111_11124_amd._ffi import AttentionIn, AttentionMask, AttentionOut

P = 0x10000
BIG = 1 << 40


@pytest.fixture(scope="module")
def L():
    return m.lib()


def heads(**kw):
    base = dict(T=10, Hq=4, Hk=2, Hv=2, D=64, rot=64, interleaved=False, sections=None, eps=1e-6)
    return m.QkvHeads(**{**base, **kw})


def fwd(L, h, x=P, row=512, gq=P, gk=P, freq=P, pos=P, al=P, be=P, lam=0.9, y=2 * P, rstd=P, q=P, mode=0, ws=P, size=BIG, dt=m.F16):
    return L.mesa_qkv_norm_rope_fwd_q(x, row, h, gq, gk, freq, pos, al, be, lam, y, rstd, q, mode, 0, 0, ws, size, dt, None)


def bwd(L, h, q=P, gq=P, gk=P, freq=P, pos=P, al=P, be=P, rstd=P, dy=P, dx=2 * P, row=384, dgq=P, dgk=P, ws=P, size=BIG, dt=m.F16):
    return L.mesa_qkv_norm_rope_bwd_q(q, h, gq, gk, freq, pos, al, be, rstd, dy, dx, row, dgq, dgk, ws, size, dt, None)


def test_projection_refusals(L):
    bad, no, room = m.ERR_INVALID_ARG, m.ERR_UNSUPPORTED, m.ERR_WORKSPACE
    for kw in (dict(T=-1), dict(Hq=0, Hk=0), dict(Hv=-1), dict(D=0), dict(rot=-2), dict(rot=66), dict(rot=31), dict(sections=[31]), dict(sections=[40, -8]), dict(eps=-1.0),
               dict(eps=float("nan"))):
        assert fwd(L, heads(**kw), row=1 << 20) == bad and bwd(L, heads(**kw), row=1 << 20) == bad, kw
        assert m.qkv_norm_rope_fwd_q_workspace_bytes(heads(**kw)) == 0
    for kw in (dict(D=60, rot=32), dict(D=264, rot=32), dict(rot=24), dict(Hq=600), dict(T=1 << 31)):
        assert fwd(L, heads(**kw), row=1 << 20) == no and bwd(L, heads(**kw), row=1 << 20) == no, kw
    h = heads()
    for kw in (dict(x=None), dict(x=P + 8), dict(row=510), dict(row=504), dict(gq=None), dict(gk=None), dict(freq=None), dict(pos=None), dict(al=None), dict(be=None), dict(lam=1.5),
               dict(lam=float("nan")), dict(y=None), dict(y=P), dict(y=P + 4), dict(rstd=None), dict(q=None), dict(q=P + 8), dict(mode=2), dict(dt=3)):
        assert fwd(L, h, **kw) == bad, kw
    assert fwd(L, h, ws=None) == room and fwd(L, h, size=16) == room
    assert fwd(L, heads(T=0), x=None, y=None, q=None) == m.OK
    for kw in (dict(q=None), dict(gq=None), dict(freq=None), dict(rstd=None), dict(dy=None), dict(dx=None), dict(dx=2 * P + 8), dict(row=376), dict(row=388), dict(dgq=None), dict(dgk=None),
               dict(al=None), dict(dx=P, row=512), dict(dt=-1)):
        assert bwd(L, h, **kw) == bad, kw
    assert bwd(L, h, ws=None) == room and bwd(L, h, size=16) == room
    assert L.mesa_qkv_norm_rope_recompute_q(P, h, P, P, P, P, P, P, None, P, m.F16, None) == bad
    assert L.mesa_qkv_norm_rope_recompute_q(None, h, P, P, P, P, P, P, P, P, m.F16, None) == bad
    assert L.mesa_qkv_norm_rope_recompute_q(P, heads(rot=24), P, P, P, P, P, P, P, P, m.F16, None) == no
    assert m.qkv_norm_rope_fwd_q_workspace_bytes(heads(T=100000)) >= 2 * 8 * 4


def shape(**kw):
    return m.Attention(**{**dict(B=2, Nq=10, Nk=12, Hq=4, Hk=2, D=64, scale=0.125, cap=0.0), **kw})


def view(data=P, batch=4096, token=256, head=64, al=None, be=None):
    return AttentionIn(data, batch, token, head, al, be)


def out(data=P, batch=4096, token=256, head=64):
    return AttentionOut(data, batch, token, head)


def attend(L, a, q=None, k=None, v=None, o=None, lse=P, mask=None, ws=P, size=BIG, dt=m.F16):
    return L.mesa_attention_fwd(a, q or view(), k or view(), v or view(), o or out(), lse, mask or AttentionMask(), ws, size, dt, None)


def attend_bwd(L, a, q=None, k=None, v=None, o=None, lse=P, do=None, dq=None, dk=None, dv=None, mask=None, ws=P, size=BIG, dt=m.F16):
    return L.mesa_attention_bwd_q(a, q or view(), k or view(), v or view(), o or view(), lse, do or view(), dq or out(), dk or out(), dv or out(), mask or AttentionMask(), ws, size, dt,
                                  None)


def test_attention_refusals(L):
    bad, no, room = m.ERR_INVALID_ARG, m.ERR_UNSUPPORTED, m.ERR_WORKSPACE
    for kw in (dict(B=-1), dict(Nq=-1), dict(Nk=-1), dict(Hk=0), dict(Hq=3), dict(D=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(cap=-1.0),
               dict(cap=float("nan")), dict(cap=float("inf"))):
        assert attend(L, shape(**kw)) == bad and attend_bwd(L, shape(**kw)) == bad, kw
    for kw in (dict(scale=1e38), dict(scale=1e30, cap=1e-10)):
        assert attend(L, shape(**kw)) == bad and attend_bwd(L, shape(**kw)) == bad, kw
    for kw in (dict(D=60), dict(D=136), dict(D=256), dict(cap=257.0)):
        assert attend(L, shape(**kw)) == no and attend_bwd(L, shape(**kw)) == no, kw
        assert m.attention_bwd_q_workspace_bytes(shape(**kw)) == 0
    for kw in (dict(Nq=1 << 29, D=128), dict(Nk=1 << 28, D=64), dict(Nq=1 << 28, Hq=32), dict(B=1 << 24), dict(B=1 << 29, Hq=1 << 29, Hk=1 << 29)):
        assert attend(L, shape(**kw)) == no and attend_bwd(L, shape(**kw)) == no, kw
        assert m.attention_bwd_q_workspace_bytes(shape(**kw)) == 0 and m.attention_fwd_workspace_bytes(shape(**kw)) == 0
    a = shape()
    assert attend(L, a, dt=m.F32) == no and attend_bwd(L, a, dt=m.F32) == no and attend(L, a, dt=7) == bad
    wrong = (dict(data=P + 8), dict(data=None), dict(token=252), dict(head=60), dict(batch=4), dict(token=-8), dict(token=1 << 23), dict(head=1 << 30))
    for kw in wrong:
        for n in ("q", "k", "v"):
            assert attend(L, a, **{n: view(**kw)}) == bad and attend_bwd(L, a, **{n: view(**kw)}) == bad, (n, kw)
        assert attend(L, a, o=out(**kw)) == bad, kw
        for n in ("o", "do"):
            assert attend_bwd(L, a, **{n: view(**kw)}) == bad, (n, kw)
        for n in ("dq", "dk", "dv"):
            assert attend_bwd(L, a, **{n: out(**kw)}) == bad, (n, kw)
    coded = view(al=P, be=P)
    assert attend(L, a, q=coded) == bad and attend_bwd(L, a, o=coded) == bad and attend_bwd(L, a, do=coded) == bad
    assert attend_bwd(L, a, v=view(al=P)) == bad and attend_bwd(L, a, v=view(be=P)) == bad and attend_bwd(L, a, v=view(data=P + 4, al=P, be=P)) == bad
    assert attend(L, a, lse=None) == bad and attend_bwd(L, a, lse=None) == bad
    assert attend(L, a, mask=AttentionMask(P, None, None, None)) == bad and attend_bwd(L, a, mask=AttentionMask(None, P, None, None)) == bad
    assert attend(L, a, mask=AttentionMask(P + 2, P, None, None)) == bad
    few = shape(B=1, Nq=1, Nk=100000, Hq=1, Hk=1)
    assert m.attention_fwd_workspace_bytes(few) > 0
    assert attend(L, few, ws=None) == room and attend(L, few, size=m.attention_fwd_workspace_bytes(few) - 1) == room
    assert attend_bwd(L, a, ws=None) == room and attend_bwd(L, a, size=m.attention_bwd_q_workspace_bytes(a, False, False, False) - 1) == room
    assert m.attention_bwd_q_workspace_bytes(a, False, False, True) >= m.attention_bwd_q_workspace_bytes(a, False, False, False) + 2 * 12 * 2 * 64 * 2
    assert attend(L, shape(B=0)) == m.OK and attend(L, shape(Nq=0)) == m.OK and attend_bwd(L, shape(B=0)) == m.OK and attend_bwd(L, shape(Nq=0, Nk=0)) == m.OK


def test_results_in_an_operands_place_are_refused(L):
    a, ws = shape(), 64 * P
    far = {n: k * P for k, n in enumerate(("q", "k", "v", "o", "do"), 2)}
    for n in ("q", "k", "v"):
        assert attend(L, a, **{x: view(far[x]) for x in ("q", "k", "v")}, o=out(far[n]), ws=ws) == m.ERR_INVALID_ARG, n
    res = dict(dq=out(10 * P), dk=out(11 * P), dv=out(12 * P))
    for r in res:
        for n in far:
            assert attend_bwd(L, a, **{x: view(far[x]) for x in far}, **dict(res, **{r: out(far[n])}), ws=ws) == m.ERR_INVALID_ARG, (r, n)
        for n in res:
            if n != r:
                assert attend_bwd(L, a, **{x: view(far[x]) for x in far}, **dict(res, **{r: res[n]}), ws=ws) == m.ERR_INVALID_ARG, (r, n)


def test_bounds_refusals(L):
    f = lambda lo=P, hi=2 * P, B=2, Nq=5, Nk=7, w=0, kv=None, doc=None: L.mesa_attention_bounds(lo, hi, B, Nq, Nk, 1, w, kv, None, None, doc, None)  # noqa: E731
    bad, no = m.ERR_INVALID_ARG, m.ERR_UNSUPPORTED
    assert f(lo=None) == bad and f(hi=None) == bad and f(hi=P) == bad and f(lo=P + 2) == bad and f(B=-1) == bad and f(Nq=-1) == bad and f(Nk=-1) == bad and f(w=-1) == bad
    assert f(kv=P + 1) == bad and f(doc=P + 2) == bad and f(Nq=1 << 30) == no and f(Nk=1 << 30) == no and f(B=1 << 36, Nq=1 << 10) == no
    assert f(B=0) == m.OK and f(Nq=0) == m.OK


def test_the_binding_refuses_what_does_not_fit():
    a = m.Attention(1, 2, 2, 1, 1, 16, 1.0)
    x = torch.zeros(1, 2, 1, 16, dtype=torch.float16)
    with pytest.raises(ValueError):
        m.mesa_attention_fwd(a, x, x, x, x, torch.zeros(1, 1, 2))            # not on a device
    with pytest.raises(ValueError):
        m.QkvHeads(1, 1, 1, 1, 16, sections=[1, 2, 3, 4, 5])
    with pytest.raises(ValueError):
        m.mesa_attention_bounds(torch.zeros(2, 3, dtype=torch.int32), torch.zeros(3, 2, dtype=torch.int32), 4, True)
    assert C.sizeof(m.Attention) == 56 and C.sizeof(m.QkvHeads) == 96
