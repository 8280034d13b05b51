"""The packed query/key/value projection's forward, recomputation and backward against 64-bit forms; codes and estimates bit for
bit against the calls that they stand for."""
import pytest
import torch

import paper_2111_11124_amd as m
from tests.language_block import F8, U, angles, dequantize, turn

pytestmark = pytest.mark.gpu
MD = {torch.float16: m.F16, torch.bfloat16: m.BF16, torch.float32: m.F32}
EPS = 1e-5
CASES = [  # T, Hq, Hk, Hv, D, rot, interleaved, sections, norm, row padding
    (1, 4, 2, 2, 64, 64, False, None, True, 0),
    (1, 1, 0, 0, 8, 8, True, None, True, 0),
    (33, 3, 1, 1, 32, 32, False, (7, 6, 3), True, 16),
    (197, 6, 6, 6, 64, 32, True, (5, 0, 6, 5), True, 0),
    (70, 5, 5, 0, 80, 80, False, None, True, 8),
    (1031, 7, 1, 2, 128, 64, False, None, True, 0),
    (2100, 2, 1, 1, 256, 256, False, None, True, 0),
    (65, 3, 2, 1, 104, 26, True, None, True, 0),
    (40, 9, 3, 3, 96, 96, False, None, False, 24),
    (129, 2, 2, 2, 64, 0, False, (0,), True, 0),
    (1, 300, 100, 112, 16, 16, False, None, True, 0),
]


def make(case, dtype, seed=0):
    T, Hq, Hk, Hv, D, rot, inter, sections, norm, pad = case
    g = torch.Generator().manual_seed(seed)
    H = Hq + Hk + Hv
    x = torch.randn(T, H, D, generator=g) * torch.exp(0.5 * torch.randn(H, 1, generator=g)) + 0.3 * torch.randn(H, D, generator=g)
    wide = torch.full((T, H * D + pad), float("nan"), dtype=dtype)
    wide[:, :H * D] = x.reshape(T, -1).to(dtype)
    xs = wide[:, :H * D].reshape(T, H, D).float()
    mn, mx = 0.9 * xs.amin((0, 2)), 0.9 * xs.amax((0, 2))
    s = dict(heads=m.QkvHeads(T, Hq, Hk, Hv, D, rot, inter, sections, EPS), wide=wide.cuda(), alpha=(mx - mn).cuda(), beta=mn.cuda())
    s["gamma"] = [(1 + 0.3 * torch.randn(D, generator=g)).to(dtype).cuda() if norm else None for _ in range(2)]
    axes = s["heads"].axes
    s["pos"] = torch.randint(-50, 200000, (axes, T), generator=g, dtype=torch.int32).cuda()
    s["freq"] = (10000.0 ** (-torch.arange(rot // 2) / max(1, rot // 2))).float().cuda()
    s["sections"] = list(s["heads"].section)[:axes]
    s["dy"] = torch.randn(T, Hq + Hk, D, generator=g).to(dtype).cuda()
    return s


def forward(s, dtype, mode=m.ROUND_STOCHASTIC, seed=7, offset=3):
    h = s["heads"]
    n, H = h.Hq + h.Hk, h.Hq + h.Hk + h.Hv
    y = torch.full((h.T, n, h.D), float("nan"), dtype=dtype, device="cuda")
    rstd = torch.full((h.T, n), float("nan"), device="cuda") if s["gamma"][0] is not None else None
    q = torch.zeros(h.T, H, h.D, dtype=torch.int8, device="cuda")
    a, b = s["alpha"].clone(), s["beta"].clone()
    ws = torch.empty(m.qkv_norm_rope_fwd_q_workspace_bytes(h, MD[dtype]), dtype=torch.uint8, device="cuda")
    m.mesa_qkv_norm_rope_fwd_q(s["wide"], h, *s["gamma"], s["freq"], s["pos"], a, b, 0.9, y, rstd, q, ws, mode, seed, offset)
    return y, rstd, q, a, b


def gains(s):
    h = s["heads"]
    if s["gamma"][0] is None:
        return torch.ones(h.Hq + h.Hk, h.D, dtype=F8, device="cuda")
    return torch.cat([s["gamma"][0].to(F8).expand(h.Hq, -1), s["gamma"][1].to(F8).expand(h.Hk, -1)])


def off(z, f32):
    """z's binary32 arithmetic: a few roundings relative to the pair of elements that a result mixes (their sizes' sum bounds it)"""
    return f32 * (z.abs().amax(-1, keepdim=True) * 2)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("mode", [m.ROUND_NEAREST_EVEN, m.ROUND_STOCHASTIC])
def test_forward(case, dtype, mode):
    s = make(case, dtype)
    h = s["heads"]
    n, H = h.Hq + h.Hk, h.Hq + h.Hk + h.Hv
    y, rstd, q, a, b = forward(s, dtype, mode)
    x = s["wide"][:, :H * h.D].contiguous()
    a1, b1, q1 = s["alpha"].clone(), s["beta"].clone(), torch.zeros_like(q)
    lay = (h.T, H, h.D)
    ws = torch.empty(m.workspace_bytes(m.OP_UPDATE_RUNNING_PARAMS, *lay), dtype=torch.uint8, device="cuda")
    m.mesa_quantize_update_fused(x, lay, a1, b1, 0.9, q1, ws, mode, 7, 3)
    assert torch.equal(q, q1) and torch.equal(a, a1) and torch.equal(b, b1)
    z = x.reshape(h.T, H, h.D)[:, :n].to(F8)
    if rstd is not None:
        r = (z.square().mean(-1) + EPS).rsqrt()
        assert ((rstd.to(F8) - r).abs() <= (h.D + 8) * 2.0**-24 * r).all()      # a sum of D squares, three roundings more
        z = z * r[..., None] * gains(s)
    want = turn(z, *angles(s["pos"], s["freq"], s["sections"]), bool(h.interleaved)) if h.rot else z
    # binary32: D + 16 roundings; angles: reduced to 2^-25 turns, 2e-7 of a pair's size, and 2^-53 of 2^18 radians and more turns
    assert ((y.to(F8) - want).abs() <= U[dtype] * want.abs() + off(z, (h.D + 16) * 2.0**-24 + 4e-7) + 2.0**-24).all()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("case", CASES)
def test_recompute_and_backward(case, dtype):
    s = make(case, dtype, 1)
    h = s["heads"]
    n = h.Hq + h.Hk
    y, rstd, q, _, _ = forward(s, dtype, m.ROUND_NEAREST_EVEN)
    norm = rstd is not None
    again = torch.full_like(y, float("nan"))
    m.mesa_qkv_norm_rope_recompute_q(q, h, *s["gamma"], s["freq"], s["pos"], s["alpha"], s["beta"], rstd, again)
    hat = dequantize(q, s["alpha"], s["beta"])[:, :n]
    r = rstd.to(F8)[..., None] if norm else torch.ones(h.T, n, 1, dtype=F8, device="cuda")
    unit, gain = hat * r, gains(s)
    cs = angles(s["pos"], s["freq"], s["sections"])
    spin = (lambda t, c, sn: turn(t, c, sn, bool(h.interleaved))) if h.rot else (lambda t, c, sn: t)
    want = spin(unit * gain, *cs)
    span = ((s["alpha"].abs() + s["beta"].abs())[:n, None] * r).amax()           # x_hat is a difference of values of this size
    f32 = 2.0**-20 * span + 4e-7 * unit.abs().amax(-1, keepdim=True)
    assert ((again.to(F8) - want).abs() <= U[dtype] * want.abs() + 4 * f32 * gain.abs().amax() + 2.0**-24).all()

    wide = torch.full((h.T, n * h.D + 64), 3.0, dtype=dtype, device="cuda")
    dgq, dgk = (torch.full((h.D,), float("nan"), device="cuda") if norm else None for _ in range(2))
    ws = torch.empty(m.qkv_norm_rope_bwd_q_workspace_bytes(h, MD[dtype]), dtype=torch.uint8, device="cuda")
    args = (q, h, *s["gamma"], s["freq"], s["pos"], s["alpha"], s["beta"], rstd)
    m.mesa_qkv_norm_rope_bwd_q(*args, s["dy"], wide, dgq, dgk, ws)
    assert (wide[:, n * h.D:] == 3.0).all()                                      # beyond the heads: left as it was
    dx = wide[:, :n * h.D].reshape(h.T, n, h.D)
    g = spin(s["dy"].to(F8), cs[0], -cs[1])
    gmax = g.abs().amax(-1, keepdim=True)
    if not norm:
        assert ((dx.to(F8) - g).abs() <= U[dtype] * g.abs() + 1e-6 * gmax + 2.0**-24).all()
    else:
        u = g * gain
        mean = (u * unit).mean(-1, keepdim=True)
        want = r * (u - unit * mean)
        size = r * (u.abs().amax(-1, keepdim=True) * (1 + unit.abs().amax(-1, keepdim=True) * unit.abs().mean(-1, keepdim=True)))
        rel = (h.D + 40) * 2.0**-24 + 4 * f32
        assert ((dx.to(F8) - want).abs() <= U[dtype] * want.abs() + rel * size * (1 + unit.abs().amax()) + 2.0**-24).all()
        for got, part in ((dgq, slice(0, h.Hq)), (dgk, slice(h.Hq, n))):
            t = (g * unit)[:, part]
            want = t.sum((0, 1))
            # fixed-order binary32 sums in parts of at most 32 tokens x heads, then 1024 parts
            bound = t.abs().sum((0, 1)) * (1200 * 2.0**-24) + 2 * (g.abs()[:, part] * f32[:, part] if h.Hq and part.stop > part.start else g.abs()[:, part]).sum((0, 1))
            assert ((got.to(F8) - want).abs() <= bound + 1e-30).all()
    if n * h.D % 8 == 0:                                                          # in place, and the same again
        flat = s["dy"].clone()
        m.mesa_qkv_norm_rope_bwd_q(*args, flat, flat, dgq, dgk, ws)
        assert torch.equal(flat, dx)


def test_gradients_are_differences_of_the_forward():
    """central differences of the 64-bit forward at x_hat, along one direction for x and along each gain"""
    case = (5, 2, 1, 0, 16, 16, False, (3, 5), True, 0)
    s = make(case, torch.float32, 2)
    h = s["heads"]
    n = h.Hq + h.Hk
    hat = dequantize(forward(s, torch.float32, m.ROUND_NEAREST_EVEN)[2], s["alpha"], s["beta"])[:, :n]
    cs = angles(s["pos"], s["freq"], s["sections"])
    f = lambda x, gain: (turn(x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * gain, *cs, False) * s["dy"].to(F8)).sum()  # noqa: E731
    rstd = (hat.square().mean(-1) + EPS).rsqrt().float()
    q = forward(s, torch.float32, m.ROUND_NEAREST_EVEN)[2]
    dx, dgq, dgk = torch.empty(h.T, n, h.D, device="cuda"), torch.empty(h.D, device="cuda"), torch.empty(h.D, device="cuda")
    ws = torch.empty(m.qkv_norm_rope_bwd_q_workspace_bytes(h, m.F32), dtype=torch.uint8, device="cuda")
    m.mesa_qkv_norm_rope_bwd_q(q, h, *s["gamma"], s["freq"], s["pos"], s["alpha"], s["beta"], rstd, s["dy"], dx, dgq, dgk, ws)
    d = torch.randn(hat.shape, generator=torch.Generator().manual_seed(3), dtype=F8).cuda()
    gain, e = gains(s), 1e-5
    num = (f(hat + e * d, gain) - f(hat - e * d, gain)) / (2 * e)
    assert abs(float(num - (dx.to(F8) * d).sum())) <= 1e-5 * float((dx.to(F8) * d).abs().sum())
    dg = torch.zeros_like(gain)
    dg[:h.Hq] = d[0, 0]
    num = (f(hat, gain + e * dg) - f(hat, gain - e * dg)) / (2 * e)
    assert abs(float(num - (dgq.to(F8) * d[0, 0]).sum())) <= 1e-5 * float((dgq.to(F8) * d[0, 0]).abs().sum())


def test_no_tokens():
    h = m.QkvHeads(0, 2, 1, 1, 32)
    dev = dict(device="cuda")
    ws = torch.empty(1 << 16, dtype=torch.uint8, **dev)
    gam, freq, pos = torch.ones(32, dtype=torch.float16, **dev), torch.ones(16, **dev), torch.zeros(1, 0, dtype=torch.int32, **dev)
    est = torch.ones(2, 4, **dev)
    e = torch.empty(0, 4, 32, dtype=torch.float16, **dev)
    q = torch.empty(0, 4, 32, dtype=torch.int8, **dev)
    rstd = torch.empty(0, 3, **dev)
    m.mesa_qkv_norm_rope_fwd_q(torch.empty(0, 128, dtype=torch.float16, **dev), h, gam, gam, freq, pos, est[0], est[1], 0.9, e, rstd, q, ws)
    assert (est == 1).all()
    dgq, dgk = torch.full((32,), 5.0, **dev), torch.full((32,), 5.0, **dev)
    m.mesa_qkv_norm_rope_bwd_q(q, h, gam, gam, freq, pos, est[0], est[1], rstd, e[:, :3].contiguous(), torch.empty(0, 96, dtype=torch.float16, **dev), dgq, dgk, ws)
    assert (dgq == 0).all() and (dgk == 0).all()
