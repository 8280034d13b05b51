"""Attention over intervals of keys: the intervals, the forward and the backward from codes, against 64-bit forms with the bounds
that their roundings give (language_block.py)."""
import math

import pytest
import torch

import paper_2111_11124_amd as m
from tests.language_block import U, attention, attention_bwd, dequantize, intervals, seen_matrix

pytestmark = pytest.mark.gpu
MD = {torch.float16: m.F16, torch.bfloat16: m.BF16}
DEV = "cuda"


def lists(B, Nq, Nk, causal=False, window=0, docs=0, prefix=False, pad=False, start=None, seed=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda lo, hi: torch.randint(lo, hi + 1, (B,), generator=g, dtype=torch.int32)  # noqa: E731
    out = dict(causal=causal, window=window)
    if pad:
        out["kv_len"] = r(0, Nk)
    if start is not None:
        out["q_start"] = torch.full((B,), start, dtype=torch.int32) if isinstance(start, int) else r(*start)
    if prefix:
        out["prefix"] = r(-1, Nk + 2)
    if docs:
        cut = (torch.rand(B, Nk, generator=g) < docs / Nk).int()
        out["doc"] = torch.cumsum(cut * torch.randint(1, 3, (B, Nk), generator=g), 1).int() - 5
    return out


@pytest.mark.parametrize("B,Nq,Nk,kw", [
    (1, 1, 1, {}), (3, 5, 5, dict(causal=True)), (2, 70, 70, dict(causal=True, window=9)), (2, 70, 70, dict(window=9)), (4, 33, 90, dict(causal=True, pad=True)),
    (4, 90, 33, dict(causal=True)), (5, 65, 65, dict(causal=True, prefix=True, pad=True)), (3, 300, 300, dict(docs=7)), (3, 300, 300, dict(causal=True, docs=40, prefix=True, window=30)),
    (4, 40, 100, dict(causal=True, docs=5, pad=True, start=(-20, 90))), (2, 7, 0, {}), (2, 1, 513, dict(causal=True, docs=500)), (2, 300, 300, dict(window=1)),
    (3, 20, 50, dict(start=(-30, 60), window=5, docs=3, pad=True)),
    # documents within, across and over several of the stretches that a workgroup takes
    (2, 3000, 3000, dict(docs=3)), (1, 2500, 5000, dict(causal=True, docs=900, pad=True)), (2, 2049, 2049, dict(docs=1500, causal=True)),
    (2, 1500, 4000, dict(docs=2, start=(-700, 3500), window=600))])
def test_bounds(B, Nq, Nk, kw):
    l = lists(B, Nq, Nk, **kw)
    seen = seen_matrix(Nq, Nk, B, **l)
    lo, hi = (torch.full((B, Nq), -7, dtype=torch.int32, device=DEV) for _ in range(2))
    m.mesa_attention_bounds(lo, hi, Nk, l["causal"], l["window"], **{k: v.to(DEV) for k, v in l.items() if torch.is_tensor(v)})
    wlo, whi = intervals(seen) if Nk else (torch.zeros(B, Nq, dtype=torch.int32),) * 2
    assert torch.equal(lo.cpu(), wlo) and torch.equal(hi.cpu(), whi)


def test_what_lies_behind_the_keys_is_not_looked_at():
    """a padded batch whose padding carries a number of its own, below the documents'"""
    B, N = 3, 5000
    n = torch.tensor([4100, 700, 1], dtype=torch.int32)
    doc = torch.cumsum((torch.rand(B, N, generator=torch.Generator().manual_seed(4)) < 0.002).int(), 1).int()
    clean = doc.clone()
    for b in range(B):
        doc[b, n[b]:] = -100
    lo, hi, wlo, whi = (torch.empty(B, N, dtype=torch.int32, device=DEV) for _ in range(4))
    start = torch.zeros(B, dtype=torch.int32, device=DEV)
    m.mesa_attention_bounds(lo, hi, N, False, kv_len=n.to(DEV), q_start=start, doc=doc.to(DEV))
    m.mesa_attention_bounds(wlo, whi, N, False, kv_len=n.to(DEV), q_start=start, doc=clean.to(DEV))
    assert torch.equal(lo, wlo) and torch.equal(hi, whi) and (hi[0, :4100] > lo[0, :4100]).all()


def test_bounds_stay_within_the_keys_whatever_the_lists_hold():
    B, Nq, Nk = 6, 50, 40
    g = torch.Generator().manual_seed(1)
    wild = lambda *s: torch.randint(-2**31, 2**31 - 1, s, generator=g, dtype=torch.int64).int().to(DEV)  # noqa: E731
    lo, hi = (torch.full((B, Nq), -7, dtype=torch.int32, device=DEV) for _ in range(2))
    for kv, st, pr, dc in ((wild(B), wild(B), wild(B), wild(B, Nk)), (None, None, wild(B), wild(B, Nk)), (wild(B).abs(), None, None, None)):
        m.mesa_attention_bounds(lo, hi, Nk, True, 3, kv_len=kv, q_start=st, prefix=pr, doc=dc)
        assert (lo >= 0).all() and (hi <= Nk).all() and (lo <= hi).all()


def tensors(B, Nq, Nk, Hq, Hk, D, dtype, layout, seed):
    g = torch.Generator().manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    q = rand(B, Nq, Hq, D) * torch.exp(0.3 * rand(Hq, 1))
    k = rand(B, Nk, Hk, D) * torch.exp(0.3 * rand(Hk, 1))
    v, do = rand(B, Nk, Hk, D) + 0.3 * rand(Hk, D), rand(B, Nq, Hq, D)
    q, k, v, do = (t.to(dtype).to(DEV) for t in (q, k, v, do))
    if layout == "bhnd":
        q, k, v, do = (t.transpose(1, 2).contiguous().transpose(1, 2) for t in (q, k, v, do))
    elif layout == "packed" and Nq == Nk:
        x = torch.cat([q, k, v, torch.full_like(v[:, :, :1], math.nan)], 2).contiguous()
        q, k, v = x[:, :, :Hq], x[:, :, Hq:Hq + Hk], x[:, :, Hq + Hk:Hq + 2 * Hk]
    return q, k, v, do


def like(t):
    return torch.full_like(t, math.nan)      # keeps a permuted layout


def check(got, want, bound, what):
    d = (got.to(torch.float64) - want).abs()
    assert torch.isfinite(got).all(), what
    worst = (d / bound.clamp_min(1e-300)).max() if d.numel() else 0
    assert (d <= bound).all(), (what, float(worst))


def forward(a, q, k, v, lo, hi, slopes, start, lse=None):
    o = torch.full((a.B, a.Nq, a.Hq, a.D), math.nan, dtype=q.dtype, device=DEV)
    lse = torch.full((a.B, a.Hq, a.Nq), math.nan, device=DEV)
    size = m.attention_fwd_workspace_bytes(a, MD[q.dtype])
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV) if size else None
    m.mesa_attention_fwd(a, q, k, v, o, lse, ws, lo, hi, slopes, start)
    return o, lse


CASES = [  # B, Nq, Nk, Hq, Hk, D, mask, cap, bias, layout
    (1, 1, 1, 1, 1, 8, {}, 0, False, "bnhd"),
    (2, 3, 7, 2, 1, 16, dict(causal=True), 0, True, "bnhd"),
    (2, 197, 197, 3, 3, 64, {}, 0, False, "bhnd"),
    (1, 130, 130, 8, 2, 32, dict(causal=True), 20.0, False, "packed"),
    (2, 65, 129, 6, 2, 80, dict(causal=True, pad=True), 0, True, "bnhd"),
    (3, 300, 300, 4, 2, 64, dict(causal=True, docs=6, pad=True), 0, True, "packed"),
    (2, 257, 257, 7, 1, 128, dict(causal=True, prefix=True), 30.0, True, "packed"),
    (2, 200, 200, 5, 5, 96, dict(window=33), 0, False, "bhnd"),
    (1, 513, 513, 2, 2, 128, dict(causal=True, window=100), 0, False, "bnhd"),
    (2, 700, 700, 2, 1, 104, dict(docs=9), 5.0, False, "packed"),
    (3, 90, 33, 2, 2, 64, dict(causal=True), 0, False, "bnhd"),          # queries before the first key see nothing
    (2, 40, 100, 4, 2, 128, dict(causal=True, docs=5, pad=True, start=(-20, 90)), 0, True, "bnhd"),
    (1, 1000, 1000, 1, 1, 64, {}, 0, False, "bnhd"),
    # more heads to a key head than a tile has rows, and not a multiple of it; widths that end within a piece of either tile
    (1, 70, 70, 40, 1, 64, dict(causal=True), 0, False, "bnhd"),
    (2, 21, 37, 66, 2, 24, dict(causal=True, docs=3), 10.0, True, "bnhd"),
    (1, 130, 130, 33, 1, 120, dict(window=20, pad=True), 0, False, "bnhd"),
    (1, 200, 200, 5, 1, 72, {}, 0, False, "packed"),
    # capped scores over many keys
    (1, 530, 530, 4, 2, 72, dict(causal=True, prefix=True), 15.0, True, "packed"),
    (1, 150, 700, 2, 1, 64, dict(causal=True, window=90), 30.0, False, "bnhd"),
    (1, 150, 600, 2, 1, 64, dict(causal=True), 256.0, False, "bnhd"),
    # few workgroups and long walks: keys and rows are dealt out in the backward
    (1, 911, 911, 2, 2, 96, dict(causal=True), 30.0, True, "packed"),
    (2, 801, 1001, 3, 1, 64, dict(causal=True, docs=3, pad=True), 0, False, "bhnd"),
    (1, 800, 790, 2, 1, 128, dict(window=50), 0, True, "bnhd"),
    (1, 60, 900, 16, 1, 40, {}, 0, False, "bnhd"),
]
FEW = [  # few rows over many keys: the keys are shared out
    (1, 1, 5000, 8, 1, 128, dict(causal=True), 0, False, "bnhd"),
    (3, 1, 2311, 6, 3, 64, dict(causal=True, pad=True, start=(0, 2310)), 30.0, True, "bhnd"),
    (1, 5, 3000, 12, 2, 80, dict(causal=True, docs=3), 0, True, "bnhd"),
    (1, 64, 4100, 4, 1, 128, dict(causal=True), 0, False, "bnhd"),
    (2, 33, 2050, 2, 1, 64, dict(window=300), 0, False, "bnhd"),
    (1, 600, 2100, 10, 2, 40, dict(causal=True), 30.0, False, "bnhd"),   # many rows to a join of few splits, and of many
    (1, 131, 2500, 33, 1, 80, dict(causal=True, docs=4), 0, True, "bhnd"),
]


def problem(case, dtype, seed=0):
    B, Nq, Nk, Hq, Hk, D, mask, cap, bias, layout = case
    l = lists(B, Nq, Nk, seed=seed, **mask)
    seen = (seen_matrix(Nq, Nk, B, **l) if mask else torch.ones(B, Nq, Nk, dtype=torch.bool)).to(DEV)   # no lists: every key for every query
    start = l.get("q_start", torch.full((B,), Nk - Nq, dtype=torch.int32)).to(DEV)
    lo, hi = (t.to(DEV) for t in intervals(seen.cpu())) if mask else (None, None)
    slopes = (2.0 ** -torch.linspace(1, 8, Hq)).to(DEV) if bias else None
    a = m.Attention(B, Nq, Nk, Hq, Hk, D, D**-0.5, cap)
    return a, tensors(B, Nq, Nk, Hq, Hk, D, dtype, layout, seed), seen, start, lo, hi, slopes, (start if "q_start" in l else None)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("case", CASES + FEW)
def test_forward(case, dtype):
    a, (q, k, v, _), seen, start, lo, hi, slopes, q_start = problem(case, dtype)
    o, lse = forward(a, q, k, v, lo, hi, slopes, q_start)
    want, wlse, bound = attention(q, k, v, a.scale, a.cap, slopes, start, seen)
    check(o, want, bound, "o")
    some = torch.isfinite(wlse)
    assert torch.equal(torch.isfinite(lse), some) and (lse[~some] == -math.inf).all()
    # E32 in every score, binary32 sums and logarithm
    assert ((lse.double() - wlse)[some].abs() <= E_LSE + 2.0**-21 * wlse[some].abs()).all()


E_LSE = 1e-4


def quantized(x, dt):
    """codes of (B, N, heads, D), one (alpha, beta) per head, in x's own layout, and their de-quantized values"""
    h = x.shape[2]
    r = x.float().transpose(0, 2).reshape(h, -1)
    mn, mx = 0.95 * r.amin(1), 0.95 * r.amax(1)
    alpha, beta = (mx - mn).contiguous(), mn.contiguous()
    q = ((x.float() - beta[:, None]) * (255 / alpha)[:, None]).round().clamp(0, 255).sub(128).to(torch.int8)
    return (q, alpha, beta), dequantize(q, alpha, beta, dt)


def backward(a, q, k, v, o, lse, do, lo, hi, slopes, start, layouts=None):
    coded = [not torch.is_tensor(t) for t in (q, k, v)]
    dq = torch.full((a.B, a.Nq, a.Hq, a.D), math.nan, dtype=do.dtype, device=DEV)
    wide = torch.full((a.B, a.Nk, 2 * a.Hk + 1, a.D), 3.0, dtype=do.dtype, device=DEV)
    dk, dv = wide[:, :, :a.Hk], wide[:, :, a.Hk:2 * a.Hk]
    ws = torch.full((m.attention_bwd_q_workspace_bytes(a, *coded, MD[do.dtype]),), 0xFF, dtype=torch.uint8, device=DEV)
    m.mesa_attention_bwd_q(a, q, k, v, o, lse, do, dq, dk, dv, ws, lo, hi, slopes, start)
    assert (wide[:, :, 2 * a.Hk:] == 3.0).all()
    return dq, dk, dv


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("codes", ["", "v", "qkv"])
@pytest.mark.parametrize("case", CASES + [(1, 900, 100, 4, 1, 64, {}, 0, False, "bnhd"), (1, 600, 140, 3, 1, 128, dict(window=400), 0, True, "bnhd")])
def test_backward(case, codes, dtype):
    a, (q, k, v, do), seen, start, lo, hi, slopes, q_start = problem(case, dtype, 1)
    o, lse = forward(a, q, k, v, lo, hi, slopes, q_start)
    given, used = {}, {}
    for n, t in (("q", q), ("k", k), ("v", v)):
        given[n], used[n] = quantized(t, dtype) if n in codes else (t, t)
    got = backward(a, given["q"], given["k"], given["v"], o, lse, do, lo, hi, slopes, q_start)
    want, bound = attention_bwd(used["q"], used["k"], used["v"], o, lse, do, a.scale, a.cap, slopes, start, seen)
    for g, w, b, n in zip(got, want, bound, ("dq", "dk", "dv")):
        check(g, w, b, n)
    again = backward(a, given["q"], given["k"], given["v"], o, lse, do, lo, hi, slopes, q_start)
    assert all(torch.equal(x, y) for x, y in zip(got, again))


@pytest.mark.parametrize("power", [-16, -8, 8])
def test_backward_binary16_gradients_of_any_size(power):
    """small and large upstream gradients lose nothing: as a power of two goes in it comes out, subnormal results aside"""
    a, (q, k, v, do), seen, start, lo, hi, slopes, _ = problem((1, 300, 300, 2, 1, 64, dict(causal=True), 0, False, "bnhd"), torch.float16, 4)
    o, lse = forward(a, q, k, v, lo, hi, None, None)
    do = (do.float() * 2.0**power).half()
    got = backward(a, q, k, v, o, lse, do, lo, hi, None, None)
    want, bound = attention_bwd(q, k, v, o, lse, do, a.scale, 0, None, start, seen)
    for g, w, b, n in zip(got, want, bound, ("dq", "dk", "dv")):
        check(g, w, b, n)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("junk", [math.nan, math.inf, -math.inf, 60000.0])
def test_what_nobody_sees_does_not_matter(junk, dtype):
    B, N, Hq, Hk, D = 2, 300, 4, 2, 64
    a = m.Attention(B, N, N, Hq, Hk, D, D**-0.5)
    q, k, v, do = tensors(B, N, N, Hq, Hk, D, dtype, "bnhd", 5)
    # documents with gaps between them and padding behind: rows of the gaps see nothing and are seen by none
    seen = torch.zeros(B, N, N, dtype=torch.bool)
    for b, spans in enumerate([[(0, 40), (41, 130), (150, 259)], [(3, 64), (64, 70), (100, 101)]]):
        for x, y in spans:
            seen[b, x:y, x:y] = torch.ones(y - x, y - x).tril().bool()
    lo, hi = (t.to(DEV) for t in intervals(seen))
    seen = seen.to(DEV)
    dead = ~seen.any(-1)
    for t in (q, k, v, do):
        t[dead] = junk
    start = torch.zeros(B, dtype=torch.int32, device=DEV)
    o, lse = forward(a, q, k, v, lo, hi, None, None)
    want, wlse, bound = attention(q, k, v, a.scale, 0, None, start, seen)
    check(o, want, bound, "o")
    assert (o[dead] == 0).all() and (lse.transpose(1, 2)[dead] == -math.inf).all()
    o[dead] = junk
    got = backward(a, q, k, v, o, lse, do, lo, hi, None, None)
    want, bound = attention_bwd(q, k, v, o, lse, do, a.scale, 0, None, start, seen)
    for g, w, b, n in zip(got, want, bound, ("dq", "dk", "dv")):
        check(g, w, b, n)
        assert (g[dead] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("Nq,Nk", [(100, 300), (3, 4000), (50, 600)])
def test_what_is_not_a_number_stays_so(Nq, Nk, cap, dtype):
    """a query that is not a number, and one that sees a key that is none: o and lse are none there, and as they were in other rows"""
    a = m.Attention(1, Nq, Nk, 2, 1, 64, 0.125, cap)
    q, k, v, _ = tensors(1, Nq, Nk, 2, 1, 64, dtype, "bnhd", 9)
    lo = torch.zeros(1, Nq, dtype=torch.int32, device=DEV)
    hi = torch.full_like(lo, Nk - 100)
    hi[0, 2] = Nk
    o, lse = forward(a, q, k, v, lo, hi, None, None)
    q[0, 1, 0, 5] = math.nan
    k[0, Nk - 50, 0, 3] = math.nan
    got, glse = forward(a, q, k, v, lo, hi, None, None)
    bad = torch.zeros(1, Nq, 2, dtype=torch.bool, device=DEV)
    bad[0, 1, 0] = True
    bad[0, 2] = True
    assert torch.isnan(got[bad]).all() and torch.equal(got[~bad], o[~bad])
    bad = bad.transpose(1, 2)
    assert torch.isnan(glse[bad]).all() and torch.equal(glse[~bad], lse[~bad])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("Nk", [130, 530])
def test_infinite_scores_meet_the_cap(Nk, dtype):
    """tanh of 3e4 / 8 / 20 is one in 64 bits already, so an infinity in that place changes nothing"""
    a = m.Attention(1, 70, Nk, 2, 1, 64, 0.125, 20.0)
    q, k, v, _ = tensors(1, 70, Nk, 2, 1, 64, dtype, "bnhd", 10)
    q[..., 7] = q[..., 7].sign() + (q[..., 7] == 0)
    for sign in (1, -1):
        k[0, 77, 0, 7] = sign * 3e4
        want = forward(a, q, k, v, None, None, None, None)
        k[0, 77, 0, 7] = sign * math.inf
        got = forward(a, q, k, v, None, None, None, None)
        assert all(torch.equal(g, w) for g, w in zip(got, want)) and torch.isfinite(got[0]).all()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("junk", [math.nan, math.inf])
def test_a_gradient_that_is_no_number_stays_with_what_it_meets(junk, dtype):
    """two documents of which one has an infinity in its gradient: the other one's gradients are what they were without"""
    a = m.Attention(1, 192, 192, 2, 1, 64, 0.125)
    q, k, v, do = tensors(1, 192, 192, 2, 1, 64, dtype, "bnhd", 11)
    lo = torch.tensor([[0] * 64 + [64] * 128], dtype=torch.int32, device=DEV)
    hi = torch.tensor([[64] * 64 + [192] * 128], dtype=torch.int32, device=DEV)
    seen = torch.zeros(1, 192, 192, dtype=torch.bool, device=DEV)
    seen[0, :64, :64] = True
    seen[0, 64:, 64:] = True
    o, lse = forward(a, q, k, v, lo, hi, None, None)
    want, bound = attention_bwd(q, k, v, o, lse, do, a.scale, 0, None, torch.zeros(1, dtype=torch.int32, device=DEV), seen)
    do[0, 20, 1, 9] = junk
    for g, w, b, n in zip(backward(a, q, k, v, o, lse, do, lo, hi, None, None), want, bound, ("dq", "dk", "dv")):
        check(g[:, 64:], w[:, 64:], b[:, 64:], n)
        assert not torch.isfinite(g[:, 20 if n == "dq" else slice(0, 64)]).all(), n


def test_intervals_beyond_the_keys_are_cut():
    a = m.Attention(1, 70, 50, 2, 2, 32, 0.3)
    q, k, v, _ = tensors(1, 70, 50, 2, 2, 32, torch.float16, "bnhd", 6)
    lo = torch.randint(-2**31, 40, (1, 70), dtype=torch.int64).int().to(DEV)
    hi = torch.randint(10, 2**31 - 1, (1, 70), dtype=torch.int64).int().to(DEV)
    cut = forward(a, q, k, v, lo.clamp(0, 50), hi.clamp(0, 50), None, None)
    got = forward(a, q, k, v, lo, hi, None, None)
    assert torch.equal(cut[0], got[0]) and torch.equal(cut[1], got[1])


def test_large_scores():
    """scores of hundreds: one key takes a row, nothing overflows"""
    for dtype in (torch.float16, torch.bfloat16):
        a = m.Attention(1, 100, 300, 2, 1, 64, 4.0)
        q, k, v, do = tensors(1, 100, 300, 2, 1, 64, dtype, "bnhd", 7)
        seen = torch.ones(1, 100, 300, dtype=torch.bool, device=DEV)
        start = torch.zeros(1, dtype=torch.int32, device=DEV)
        o, lse = forward(a, q, k, v, None, None, None, None)
        want, wlse, bound = attention(q, k, v, 4.0, 0, None, start, seen)
        # scores of up to 64 * 4 * |q||k| products: 128 * 2^-24 of their sum, up to 1e3, is 1e-2 in p at worst where rows are undecided
        check(o, want, bound + 2e-2 * v.abs().max(), "o")
        assert ((lse.double() - wlse).abs() <= 1e-4 + 2.0**-20 * wlse.abs()).all()
        for g in backward(a, q, k, v, o, lse, do, None, None, None, None):
            assert torch.isfinite(g).all()


def test_no_keys_and_no_queries():
    f16 = dict(dtype=torch.float16, device=DEV)
    a = m.Attention(2, 3, 0, 2, 1, 16, 1.0)
    o, lse = torch.ones(2, 3, 2, 16, **f16), torch.ones(2, 2, 3, device=DEV)
    kv = torch.empty(2, 0, 1, 16, **f16)
    m.mesa_attention_fwd(a, torch.ones(2, 3, 2, 16, **f16), kv, kv, o, lse)
    assert (o == 0).all() and (lse == -math.inf).all()
    dq = torch.ones(2, 3, 2, 16, **f16)
    m.mesa_attention_bwd_q(a, torch.ones(2, 3, 2, 16, **f16), kv, kv, o, lse, torch.ones_like(o), dq, kv.clone(), kv.clone(), None)
    assert (dq == 0).all()
    a = m.Attention(2, 0, 3, 2, 1, 16, 1.0)
    e, x = torch.empty(2, 0, 2, 16, **f16), torch.ones(2, 3, 1, 16, **f16)
    m.mesa_attention_fwd(a, e, x, x, e.clone(), torch.empty(2, 2, 0, device=DEV))
    dk, dv = torch.ones_like(x), torch.ones_like(x)
    m.mesa_attention_bwd_q(a, e, x, x, e, torch.empty(2, 2, 0, device=DEV), e, e.clone(), dk, dv, None)
    assert (dk == 0).all() and (dv == 0).all()


def test_offsets_past_32_bits():
    """keys and values whose rows lie 8 MB apart: 700 of them span more than 4 GB"""
    N, D, step = 700, 64, (1 << 22) - 264
    big = torch.empty(N * step + 4096, dtype=torch.bfloat16, device=DEV)
    a = m.Attention(1, 40, N, 2, 1, D, D**-0.5)
    q, k, v, do = tensors(1, 40, N, 2, 1, D, torch.bfloat16, "bnhd", 8)
    far = []
    for n, t in enumerate((k, v)):
        w = big[n * 1024:].as_strided((1, N, 1, D), (0, step, 64, 1), n * 1024)
        w.copy_(t)
        far.append(w)
    o, lse = forward(a, q, *far, None, None, None, None)
    o1, lse1 = forward(a, q, k, v, None, None, None, None)
    assert torch.equal(o, o1) and torch.equal(lse, lse1)
    got, want = (backward(a, q, *kv, o, lse, do, None, None, None, None) for kv in (far, (k, v)))
    assert all(torch.equal(x, y) for x, y in zip(got, want))
