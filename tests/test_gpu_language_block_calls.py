"""The language-model block's calls as a training step makes them: one after the other, marshalled either way, on other streams,
captured into a graph and replayed, with two workspaces at once."""
import math

import pytest
import torch

import paper_2111_11124_amd as m
from paper_2111_11124_amd import _ffi
from tests.language_block import F8, U, angles, seen_matrix, turn

pytestmark = pytest.mark.gpu
DEV = "cuda"
MD = {torch.float16: m.F16, torch.bfloat16: m.BF16}


class Block:
    """one attention layer of B x N tokens: what it keeps, its forward and its backward"""

    def __init__(self, B, N, Hq, Hk, D, dtype, cap=0.0, seed=0, docs=0, axes=(None,)):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.B, self.N, self.Hq, self.Hk, self.D = dtype, B, N, Hq, Hk, D
        T, H = B * N, Hq + 2 * Hk
        self.heads = m.QkvHeads(T, Hq, Hk, Hk, D, eps=1e-5)
        self.plan = m.Attention(B, N, N, Hq, Hk, D, D**-0.5, cap)
        # multiples of 1/32 between -4 and 127/32: the codes of an interval [-4, 255/32 - 4] hold them exactly, and so does every storage type
        self.x = (torch.randint(-128, 128, (T, H * D), generator=g).float() / 32).to(dtype).to(DEV)
        self.est = torch.empty(2, H, device=DEV)
        self.gamma = [(1 + 0.2 * torch.randn(D, generator=g)).to(dtype).to(DEV) for _ in range(2)]
        self.freq = (100.0 ** -torch.linspace(0, 1, D // 2)).to(DEV)
        self.pos = torch.arange(N, dtype=torch.int32).repeat(B)[None].contiguous().to(DEV)
        self.doc = torch.cumsum((torch.rand(B, N, generator=g) < docs / N).int(), 1).int().to(DEV) if docs else None
        self.do = torch.randn(B, N, Hq, D, generator=g).to(dtype).to(DEV)
        e = lambda *s, dt=dtype: torch.empty(*s, dtype=dt, device=DEV)  # noqa: E731
        n = Hq + Hk
        self.y, self.again, self.dy = e(T, n, D), e(T, n, D), e(B, N, n, D)
        self.rstd, self.lse = e(T, n, dt=torch.float32), e(B, Hq, N, dt=torch.float32)
        self.q, self.o, self.dqkv = e(T, H, D, dt=torch.int8), e(B, N, Hq, D), e(T, H * D)
        self.dgamma = [e(D, dt=torch.float32) for _ in range(2)]
        self.lo, self.hi = e(B, N, dt=torch.int32), e(B, N, dt=torch.int32)
        md = MD[dtype]
        size = max(m.qkv_norm_rope_fwd_q_workspace_bytes(self.heads, md), m.qkv_norm_rope_bwd_q_workspace_bytes(self.heads, md), m.attention_fwd_workspace_bytes(self.plan, md),
                   m.attention_bwd_q_workspace_bytes(self.plan, False, False, True, md))
        self.ws = e(size, dt=torch.uint8)

    def step(self):
        B, N, Hq, Hk, D = self.B, self.N, self.Hq, self.Hk, self.D
        self.est[0].fill_(255 / 32)
        self.est[1].fill_(-4.0)
        norm = (self.heads, *self.gamma, self.freq, self.pos)
        m.mesa_attention_bounds(self.lo, self.hi, N, True, doc=self.doc)
        est = self.est.clone()
        m.mesa_qkv_norm_rope_fwd_q(self.x, *norm, est[0], est[1], 0.9, self.y, self.rstd, self.q, self.ws, m.ROUND_NEAREST_EVEN)
        y = self.y.view(B, N, Hq + Hk, D)
        v = self.x.view(B, N, -1, D)[:, :, Hq + Hk:]
        m.mesa_attention_fwd(self.plan, y[:, :, :Hq], y[:, :, Hq:], v, self.o, self.lse, self.ws, self.lo, self.hi)
        # backward: queries and keys from the codes, values as codes
        m.mesa_qkv_norm_rope_recompute_q(self.q, *norm, self.est[0], self.est[1], self.rstd, self.again)
        z = self.again.view(B, N, Hq + Hk, D)
        vq = (self.q.view(B, N, -1, D)[:, :, Hq + Hk:], self.est[0][Hq + Hk:], self.est[1][Hq + Hk:])
        dv = self.dqkv.view(B, N, -1, D)[:, :, Hq + Hk:]
        m.mesa_attention_bwd_q(self.plan, z[:, :, :Hq], z[:, :, Hq:], vq, self.o, self.lse, self.do, self.dy[:, :, :Hq], self.dy[:, :, Hq:], dv, self.ws, self.lo, self.hi)
        m.mesa_qkv_norm_rope_bwd_q(self.q, *norm, self.est[0], self.est[1], self.rstd, self.dy.view(-1, Hq + Hk, D), self.dqkv, *self.dgamma, self.ws)

    def results(self):
        return [t.clone() for t in (self.o, self.lse, self.q, self.dqkv, *self.dgamma)]

    def exact(self, x, gq, gk):
        """the output in 64 bits"""
        B, N, Hq, Hk, D = self.B, self.N, self.Hq, self.Hk, self.D
        h = x.view(B * N, -1, D)
        z = h[:, :Hq + Hk]
        z = z * (z.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * torch.cat([gq.expand(Hq, -1), gk.expand(Hk, -1)])
        z = turn(z, *angles(self.pos, self.freq, [D // 2]), False).view(B, N, Hq + Hk, D)
        q, k, v = z[:, :, :Hq], z[:, :, Hq:], h[:, Hq + Hk:].reshape(B, N, Hk, D)
        k, v = (t.repeat_interleave(Hq // Hk, 2).transpose(1, 2) for t in (k, v))
        s = torch.matmul(q.transpose(1, 2), k.transpose(-1, -2).contiguous()) * self.plan.scale
        if self.plan.cap:
            s = self.plan.cap * torch.tanh(s / self.plan.cap)
        seen = seen_matrix(N, N, B, True, doc=None if self.doc is None else self.doc.cpu()).to(DEV)
        return torch.matmul(s.masked_fill(~seen[:, None], -math.inf).softmax(-1), v.contiguous()).transpose(1, 2)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("kw", [dict(B=2, N=77, Hq=4, Hk=2, D=64), dict(B=1, N=300, Hq=3, Hk=1, D=128, cap=20.0), dict(B=2, N=150, Hq=2, Hk=2, D=32, docs=4)])
def test_a_training_step(kw, dtype):
    """values on the codes' grid: the saved codes are exact, so the backward is the gradient of the forward itself"""
    b = Block(dtype=dtype, **kw)
    b.step()
    x, gq, gk = (t.to(F8).requires_grad_() for t in (b.x, *b.gamma))
    o = b.exact(x, gq, gk)
    o.backward(b.do.to(F8))
    rel = lambda got, want: float((got.to(F8) - want).norm() / want.norm())  # noqa: E731
    # roundings on the way to a result, each off by at most u in the 2-norm of what it rounds: y (twice: q and k), p, o; and for the gradients
    # ds, delta's o, dq or dk, dx as well.  Twice their number for how the softmax passes them on (scores of order one to four).
    u = U[dtype]
    assert rel(b.o, o.detach()) <= 8 * u
    # x is -4 .. 4, so gradients of queries and keys are not small against those of values
    assert rel(b.dqkv, x.grad) <= 16 * u
    for got, want in zip(b.dgamma, (gq.grad, gk.grad)):
        assert rel(got, want) <= 16 * u
    # and against differences of the forward, along one direction
    d = torch.randn(b.x.shape, generator=torch.Generator().manual_seed(1), dtype=F8).to(DEV)
    e = 1e-5
    with torch.no_grad():
        num = ((b.exact(x + e * d, gq, gk) - b.exact(x - e * d, gq, gk)) * b.do.to(F8)).sum() / (2 * e)
    # an error of that norm against a direction drawn apart from it: six standard deviations of their product
    assert abs(float(num - (b.dqkv.to(F8) * d).sum())) <= 16 * u * float(b.dqkv.to(F8).norm() * d.norm()) / d.numel()**0.5 * 6 + 1e-6


def test_native_and_general_marshalling_make_the_same_calls(monkeypatch):
    b = Block(2, 90, 4, 2, 64, torch.float16, docs=3)
    seen = []
    native = _ffi._fast
    assert not isinstance(native, _ffi._General)

    class Watch:
        def __getattr__(self, name):
            def call(*args):
                r = getattr(native, name)(*args)
                seen.append((name, r))
                return r
            return call

    monkeypatch.setattr(_ffi, "_fast", Watch())
    b.step()
    want = b.results()
    assert sorted(seen) == [(n, 0) for n in ("attention_bounds", "attention_bwd_q", "attention_fwd", "qkv_norm_rope_bwd_q", "qkv_norm_rope_fwd_q", "qkv_norm_rope_recompute_q")]
    monkeypatch.setattr(_ffi, "_fast", _ffi._General())
    b.step()
    assert all(torch.equal(x, y) for x, y in zip(b.results(), want))


@pytest.mark.parametrize("general", [False, True])
def test_tensors_that_do_not_fit_are_refused(general, monkeypatch):
    if general:
        monkeypatch.setattr(_ffi, "_fast", _ffi._General())
    b = Block(1, 8, 2, 1, 32, torch.float16)
    y = b.y.view(1, 8, 3, 32)
    q, k, v = y[:, :, :2], y[:, :, 2:], b.x.view(1, 8, 4, 32)[:, :, 3:]
    for bad in (dict(q=q.float()), dict(q=q[:, :7]), dict(k=k.transpose(1, 3)), dict(v=v.cpu()), dict(o=b.o.to(torch.bfloat16)), dict(lse=b.lse[:, :1]), dict(lo=b.lo.long()),
                dict(lo=b.lo[:, :4].contiguous(), hi=b.hi)):
        args = {**dict(q=q, k=k, v=v, o=b.o, lse=b.lse, lo=None, hi=None), **bad}
        with pytest.raises((ValueError, m.MesaError)):
            m.mesa_attention_fwd(b.plan, args["q"], args["k"], args["v"], args["o"], args["lse"], b.ws, args["lo"], args["hi"])
    with pytest.raises(m.MesaError):
        m.mesa_attention_fwd(b.plan, q, k, v, b.o, b.lse, b.ws, b.lo, None)      # one of the two lists
    with pytest.raises(ValueError):
        m.mesa_qkv_norm_rope_recompute_q(b.q[:7], b.heads, *b.gamma, b.freq, b.pos, *b.est, b.rstd, b.again)
    with pytest.raises(ValueError):
        m.mesa_qkv_norm_rope_bwd_q(b.q, b.heads, *b.gamma, b.freq, b.pos, *b.est, b.rstd, b.dy.view(8, 3, 32), b.dqkv.t(), *b.dgamma, b.ws)


def test_on_other_streams_with_workspaces_of_their_own():
    blocks = [Block(2, 200, 4, 1, 64, torch.bfloat16, seed=k, docs=3) for k in range(2)]
    want = []
    for b in blocks:
        b.step()
        want.append(b.results())
    for b in blocks:
        b.o.zero_(), b.dqkv.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in blocks]
    for _ in range(3):
        for b, s in zip(blocks, streams):
            with torch.cuda.stream(s):
                b.step()
    torch.cuda.synchronize()
    for b, w in zip(blocks, want):
        assert all(torch.equal(x, y) for x, y in zip(b.results(), w))


@pytest.mark.parametrize("kw", [dict(B=2, N=130, Hq=4, Hk=2, D=64, dtype=torch.float16), dict(B=1, N=700, Hq=4, Hk=1, D=128, dtype=torch.bfloat16, cap=30.0)])
def test_captured_and_replayed(kw):
    b = Block(**kw)
    other = (torch.randint(-128, 128, b.x.shape, generator=torch.Generator().manual_seed(9)).float() / 32).to(b.dtype).to(DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b.step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.step()
    first = b.x.clone()
    for x in (other, first, other):
        b.x.copy_(x)
        b.step()
        torch.cuda.synchronize()
        want = b.results()
        b.o.zero_(), b.dqkv.zero_(), b.lse.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(b.results(), want))
