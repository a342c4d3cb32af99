"""The update operators against their definitions in 64 bits.

Tolerances count roundings, u = 2^-24 being half a step of float32 and half(dt) half a
step of the output's type, each bound taken elementwise from the reference's own
magnitudes:

* log-probs: an exponential's argument (s - m) log2 e carries 5 u |s - m| (difference,
  two constants, two products) and the hardware's exp2 2 u; a sum of n = V / 512 + 32
  running additions n u.  So |d lse| <= u (5 E_p|s - m| + n + 4 + 2 |lse| + 2 |m|), and
  likewise for the others, see _logprob_bounds.
* q/k: the angle is reduced in 64 bits and rounded once, 2 pi 2^-25 < 2^-22; sums of
  squares run over 16 products and 3 exchanges; all of it below 2^-20 of |x1| + |x2|.
* attention: a score carries (hd + 4) u sum |q||k| scale, which is its probability's
  relative error; bf16 probabilities and score gradients are rounded once more, 2^-8, and
  the probabilities in the score gradients may be of 11 bits.
* AdamW: fewer than 32 operations per element.
"""
import itertools
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DEV = "cuda:0"
BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64


def _half(dt):
    return torch.finfo(dt).eps / 2


def _within(got, ref, tol, what):
    got = got.to(F64)
    assert got.shape == ref.shape, what
    assert torch.isfinite(got).all(), what
    bad = (got - ref).abs() - tol
    assert float(bad.max()) <= 0 if bad.numel() else True, (
        what, float((got - ref).abs().max()), float((bad).max()), int((bad > 0).sum()))


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _say(*a):
    print(*a, flush=True)


# ------------------------------------------------------------------ log-probs

def _logprob_inputs(R, V, dt, seed, pad=0, spread=2.5):
    g = _gen(seed)
    z = (spread * torch.randn((R, V + pad), generator=g, device=DEV)).to(dt)[:, :V]
    zr = (z.float() + 0.3 * torch.randn((R, V), generator=g, device=DEV)).to(dt)
    tok = torch.randint(0, V, (R,), generator=g, device=DEV, dtype=torch.int32)
    gl = torch.randn((R,), generator=g, device=DEV)
    gk = torch.randn((R,), generator=g, device=DEV)
    return z, zr, tok, gl, gk


def _scores64(z, T, eos, b):
    s = z.to(F64).clone()
    if eos >= 0:
        s[:, eos] += b
    return s / T


def _logprob_check(z, zr, tok, gl, gk, T, eos, b, br, call_fwd, call_bwd, dt):
    """Both passes against the definition; returns nothing."""
    V = z.shape[1]
    s = _scores64(z, T, eos, b)
    live = (tok >= 0) & (tok < V)
    y = tok.clamp(0, V - 1).long()[:, None]
    m = s.amax(1)
    lp = s.log_softmax(1)
    lse = s.logsumexp(1)
    p = lp.exp()
    away = torch.where(p > 0, p * (s - m[:, None]).abs(), torch.zeros_like(p)).sum(1)
    n = V / 512 + 32
    t_lse = U * (5 * away + n + 4 + 2 * lse.abs() + 2 * m.abs())
    logp = lp.gather(1, y)[:, 0]
    zero = torch.zeros_like(lse)
    r = call_fwd()
    _within(r["lse"], torch.where(live, lse, zero), t_lse, "lse")
    _within(r["logp"], torch.where(live, logp, zero), t_lse + U * (4 * logp.abs() + 4 * (lse - m)), "logp")
    kl = diff = None
    if zr is not None:
        q = _scores64(zr, T, eos, br)
        mr = q.amax(1)
        diff = lse - q.logsumexp(1)
        pr = q.softmax(1)
        awayr = torch.where(pr > 0, pr * (q - mr[:, None]).abs(), torch.zeros_like(pr)).sum(1)
        t_diff = U * (5 * (away + awayr) + 2 * n + 8 + 2 * diff.abs() + 4 * (m - mr).abs())
        d = torch.where(p > 0, s - q, torch.zeros_like(s))
        kl = (p * d).sum(1) - diff
        t_kl = t_diff + U * ((n + 8) * (p * d.abs()).sum(1) + 5 * (p * d.abs() * (s - m[:, None]).abs().clamp(max=1e3)).sum(1)
                             + 5 * away * (p * d.abs()).sum(1) + 2 * kl.abs())
        _within(r["lse_diff"], torch.where(live, diff, zero), t_diff, "lse_diff")
        _within(r["kl"], torch.where(live, kl, zero), t_kl, "kl")
    if call_bwd is None:
        return r
    grad = call_bwd(r)
    hot = torch.zeros_like(p).scatter_(1, y, 1.0)
    gl64 = gl.to(F64)[:, None]
    want = gl64 * (hot - p)
    arg = torch.where(p > 0, lp.abs(), torch.zeros_like(lp))
    rel = t_lse[:, None] + U * (2 * s.abs().clamp(max=1e3) + 3 * arg + 12)
    size = gl64.abs() * (p + hot)
    if gk is not None and zr is not None:
        gk64 = gk.to(F64)[:, None]
        want = want + gk64 * p * (d - diff[:, None] - kl[:, None])
        size = size + gk64.abs() * p * (d.abs() + diff.abs()[:, None] + kl.abs()[:, None])
        extra = gk64.abs() * p * (t_diff + t_kl)[:, None]
    else:
        extra = torch.zeros_like(p)
    want = torch.where(live[:, None], want / T, torch.zeros_like(want))
    # below the smallest normal of the type, results may be flushed
    tol = (size * rel + extra) / T + _half(dt) * want.abs() + 2.0 ** -126
    _within(grad, want, tol, "grad")
    assert (grad[~live] == 0).all()
    return r


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("R,V", [(1, 1), (3, 2), (5, 7), (1, 8), (9, 63), (2, 2047), (7, 2048), (3, 2049), (1, 4097),
                                 (2, 32001), (1, 151936), (1030, 513), (1100, 5003)])
def test_logprob(R, V, dt):
    """Rows of a wave, of a workgroup, cut into parts; odd lengths; with reference,
    temperature and EOS biases; rows left out (token -1 or past the vocabulary)."""
    from paper_2606_28166_amd import engine as E
    _say("logprob", R, V, dt)
    z, zr, tok, gl, gk = _logprob_inputs(R, V, dt, R * 7 + V)
    if R > 2:
        tok[0], tok[R // 2] = -1, V
    for T, eos in ((1.0, -1), (0.6, V - 1)):
        o = dict(temperature=T, eos_id=eos, eos_bias=2.25, eos_bias_ref=-1.5)
        # T is a float in the call
        T64 = float(torch.tensor(T, dtype=F32))
        _logprob_check(z, zr, tok, gl, gk, T64, eos, 2.25, -1.5, lambda: E.token_logprob(z, tok, ref=zr, **o),
                       lambda r: E.token_logprob_backward(z, tok, r, gl, g_kl=gk, ref=zr, **o), dt)
        _logprob_check(z, None, tok, gl, None, T64, eos, 2.25, 0.0, lambda: E.token_logprob(z, tok, **o),
                       lambda r: E.token_logprob_backward(z, tok, r, gl, **o), dt)


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
def test_logprob_strides_and_place(dt):
    """Rows inside a wider array, an odd stride, and a gradient that takes the logits'
    place; the columns beside the vocabulary are left alone."""
    from paper_2606_28166_amd import engine as E
    R, V, pad = 6, 4099, 14
    z, zr, tok, gl, gk = _logprob_inputs(R, V, dt, 3, pad=pad)
    whole = z._base
    before = whole.clone()
    r = _logprob_check(z, zr, tok, gl, gk, 1.0, -1, 0.0, 0.0, lambda: E.token_logprob(z, tok, ref=zr),
                       lambda r: E.token_logprob_backward(z, tok, r, gl, g_kl=gk, ref=zr), dt)
    g = E.token_logprob_backward(z, tok, r, gl, g_kl=gk, ref=zr)
    assert torch.equal(whole, before)
    g2 = E.token_logprob_backward(z, tok, r, gl, g_kl=gk, ref=zr, out=z)
    assert g2.data_ptr() == whole.data_ptr()
    assert torch.equal(whole[:, :V], g) and torch.equal(whole[:, V:], before[:, V:])


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("V", [300, 9000])
def test_logprob_masked_entries(dt, V):
    """Entries of -inf and of the type's lowest value, in the logits and in the
    reference; a row of nothing but the lowest value is uniform."""
    from paper_2606_28166_amd import engine as E
    low = torch.finfo(dt).min
    z, zr, tok, gl, gk = _logprob_inputs(5, V, dt, V)
    tok.fill_(3)
    z[0, V // 2:] = -math.inf
    zr[0, V // 2:] = -math.inf
    z[1, V // 2:] = low
    zr[1, V // 2:] = low
    z[2, 5:] = -math.inf                       # the reference has mass where the senior has none
    z[3] = low
    zr[3] = low
    zr[4, 0] = zr[4, 1]
    _logprob_check(z, zr, tok, gl, gk, 1.0, -1, 0.0, 0.0, lambda: E.token_logprob(z, tok, ref=zr),
                   lambda r: E.token_logprob_backward(z, tok, r, gl, g_kl=gk, ref=zr), dt)
    # the senior has mass where the reference has none: infinite divergence, and a gradient
    # of the log-prob alone is not touched by it
    z, zr, tok, gl, gk = _logprob_inputs(2, V, dt, V + 1)
    zr[0, 7] = -math.inf
    gk.zero_()
    r = E.token_logprob(z, tok, ref=zr)
    assert float(r["kl"][0]) == math.inf and math.isfinite(float(r["kl"][1]))
    g = E.token_logprob_backward(z, tok, r, gl, g_kl=gk, ref=zr)
    assert torch.equal(g, E.token_logprob_backward(z, tok, r, gl))
    # a row of nothing but the lowest value is uniform, its gradient too, also in the logits' place
    z, zr, tok, gl, gk = _logprob_inputs(3, V, dt, V + 2)
    z[1] = low
    tok.fill_(2)
    r = E.token_logprob(z, tok)
    assert abs(float(r["logp"][1]) + math.log(V)) <= 4 * U * math.log(V)
    want = float(gl[1]) * (torch.nn.functional.one_hot(torch.tensor(2), V).to(DEV).to(F64) - 1.0 / V)
    for out in (None, z):
        _within(E.token_logprob_backward(z, tok, r, gl, out=out)[1], want, (_half(dt) + 8 * U) * want.abs(), "grad")
    # rows without a distribution
    z, zr, tok, gl, gk = _logprob_inputs(2, V, dt, V + 1)
    z[0] = -math.inf
    z[1, 1] = math.nan
    r = E.token_logprob(z, tok)
    assert float(r["lse"][0]) == -math.inf and torch.isnan(r["logp"]).all() and torch.isnan(r["lse"][1])
    # a row without gradient is not read
    gl.zero_()
    assert (E.token_logprob_backward(z, tok, r, gl) == 0).all()


def test_logprob_gradient_by_differences():
    """float32: the gradient of sum(g logp + k kl) against central differences of the
    definition in 64 bits, with temperature and the rollout's EOS bias."""
    from paper_2606_28166_amd import engine as E
    R, V, T, eos, b, br = 4, 37, 0.7, 5, 1.5, -0.5
    z, zr, tok, gl, gk = _logprob_inputs(R, V, F32, 2)
    kw = dict(temperature=T, eos_id=eos, eos_bias=b, eos_bias_ref=br)
    f = E.token_logprob(z, tok, ref=zr, **kw)
    got = E.token_logprob_backward(z, tok, f, gl, g_kl=gk, ref=zr, **kw).cpu().double()
    x, q = z.cpu().double(), _scores64(zr.cpu(), T, eos, br).log_softmax(1)
    y, wl, wk = tok.cpu().long()[:, None], gl.cpu().double(), gk.cpu().double()

    def loss(x):
        lp = _scores64(x, T, eos, b).log_softmax(1)
        return float((wl * lp.gather(1, y)[:, 0] + wk * (lp.exp() * (lp - q)).sum(1)).sum())

    step = 1e-5
    flat = x.view(-1)
    for at in range(flat.numel()):
        keep = float(flat[at])
        flat[at] = keep + step
        up = loss(x)
        flat[at] = keep - step
        down = loss(x)
        flat[at] = keep
        assert abs((up - down) / (2 * step) - float(got.view(-1)[at])) <= 1e-4, at


def test_logprob_far_rows():
    """Rows whose offset passes 2^31 elements."""
    from paper_2606_28166_amd import engine as E
    V, ld = 1000, 1 << 21
    whole = torch.zeros((1100, ld), dtype=BF, device=DEV)      # 2.3e9 elements
    z = whole[:, :V]
    z[-1] = (2 * torch.randn((V,), generator=_gen(2), device=DEV)).to(BF)
    tok = torch.full((1100,), -1, dtype=torch.int32, device=DEV)
    tok[-1] = 5
    gl = torch.ones(1100, device=DEV)
    r = E.token_logprob(z, tok)
    want = z[-1:].double().log_softmax(1)
    assert abs(float(r["logp"][-1]) - float(want[0, 5])) <= 1e-5
    g = E.token_logprob_backward(z, tok, r, gl, out=z)
    hot = torch.zeros(V, dtype=F64, device=DEV)
    hot[5] = 1
    _within(g[-1], hot - want[0].exp(), _half(BF) * (hot - want[0].exp()).abs() + 1e-6, "grad")


# ------------------------------------------------------------------ q/k norm and rotation

def _qk_reference(qkv, pos, nq, nkv, theta, eps, gq, gk, dq, dk):
    """Outputs, gradients and the magnitudes their bounds are taken from, in 64 bits."""
    N, hd = qkv.shape[0], qkv.shape[1] // (nq + 2 * nkv)
    h = hd // 2
    x = qkv.to(F64).view(N, nq + 2 * nkv, hd)
    th = float(torch.tensor(theta, dtype=F32))
    ep = float(torch.tensor(eps, dtype=F32))
    ang = pos.to(F64)[:, None] * torch.tensor([th ** (-2.0 * i / hd) for i in range(h)], dtype=F64, device=DEV)
    c, s = ang.cos()[:, None], ang.sin()[:, None]
    out = []
    for part, gain, dy in ((x[:, :nq], gq, dq), (x[:, nq:nq + nkv], gk, dk)):
        g = torch.ones(hd, dtype=F64, device=DEV) if gain is None else gain.to(F64)
        r = torch.ones_like(part[..., :1]) if gain is None else (part.square().mean(-1, keepdim=True) + ep).rsqrt()
        n = part * r * g
        y = torch.cat([n[..., :h] * c - n[..., h:] * s, n[..., h:] * c + n[..., :h] * s], -1)
        size = (n[..., :h].abs() + n[..., h:].abs()).repeat(1, 1, 2)
        d = dy.to(F64)
        dn = torch.cat([d[..., :h] * c + d[..., h:] * s, d[..., h:] * c - d[..., :h] * s], -1)
        dsize = (d[..., :h].abs() + d[..., h:].abs()).repeat(1, 1, 2)
        t, ts = dn * g, dsize * g.abs()
        if gain is None:
            dx, xs, dg, gs = dn, dsize, None, None
        else:
            dx = r * (t - part * r * r * (t * part).mean(-1, keepdim=True))
            xs = r * (ts + part.abs() * r * r * (ts * part.abs()).mean(-1, keepdim=True))
            dg = (dn * part * r).sum((0, 1))
            gs = (dsize * part.abs() * r).sum((0, 1))
        out.append((y, size, dx, xs, dg, gs))
    return out


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("nq,nkv,hd,N,far", [(4, 2, 32, 1, 3), (2, 1, 32, 77, 100), (1, 1, 64, 5, 1 << 20),
                                             (16, 4, 64, 33, 4000), (6, 3, 64, 130, 9), (32, 8, 128, 19, 100000),
                                             (16, 8, 128, 257, 8703), (5, 5, 128, 3, 1 << 30), (64, 1, 128, 4, 50)])
@pytest.mark.parametrize("norm", [True, False], ids=["norm", "plain"])
def test_qk_norm_rope(nq, nkv, hd, N, far, dt, norm):
    from paper_2606_28166_amd import engine as E
    _say("qk", nq, nkv, hd, N, dt, norm)
    g = _gen(N + hd)
    cols = (nq + 2 * nkv) * hd
    wide = torch.randn((N, cols + 32), generator=g, device=DEV).to(dt)
    qkv = wide[:, :cols]
    pos = torch.randint(-far, far + 1, (N,), generator=g, device=DEV, dtype=torch.int32)
    pos[0] = far
    gq, gk = [(1 + 0.3 * torch.randn((hd,), generator=g, device=DEV)) if norm else None for _ in range(2)]
    dq = torch.randn((N, nq, hd), generator=g, device=DEV).to(dt)
    dk = torch.randn((N, nkv + 1, hd), generator=g, device=DEV).to(dt)[:, :nkv]      # strided rows
    theta, eps = 1.0e6, 1.0e-6
    ref = _qk_reference(qkv, pos, nq, nkv, theta, eps, gq, gk, dq, dk)
    f = E.qk_norm_rope(qkv, pos, nq, nkv, theta, eps, q_gain=gq, k_gain=gk)
    for name, (y, size, *_) in zip(("q", "k"), ref):
        _within(f[name], y, 2.0 ** -20 * size + _half(dt) * y.abs(), name)
    assert torch.equal(f["v"], qkv[:, (nq + nkv) * hd:].reshape(N, nkv, hd))
    mark = torch.full_like(wide, 7.0)
    b = E.qk_norm_rope_backward(qkv, pos, dq, dk, theta, eps, q_gain=gq, k_gain=gk, dqkv=mark[:, :cols])
    d = mark[:, :cols].reshape(N, nq + 2 * nkv, hd)
    for name, part, (_, _, dx, xs, _, _) in (("dq", d[:, :nq], ref[0]), ("dk", d[:, nq:nq + nkv], ref[1])):
        _within(part, dx, 2.0 ** -19 * xs + _half(dt) * dx.abs(), name)
    assert (mark[:, (nq + nkv) * hd:] == 7.0).all()            # value columns and the padding beside the rows
    if norm:
        for name, (*_, dg, gs) in zip(("dq_gain", "dk_gain"), ref):
            _within(b[name], dg, (2.0 ** -19 + U * (N * (nq + nkv) / 64 + 160)) * gs, name)
    else:
        assert b["dq_gain"] is None and b["dk_gain"] is None
    fresh = E.qk_norm_rope_backward(qkv, pos, dq, dk, theta, eps, q_gain=gq, k_gain=gk)
    assert torch.equal(fresh["dqkv"][:, :(nq + nkv) * hd], mark[:, :(nq + nkv) * hd])
    assert (fresh["dqkv"][:, (nq + nkv) * hd:] == 0).all()


def test_qk_gradient_by_differences():
    """float32: the gradients of sum(wq q) + sum(wk k) against central differences of the
    definition in 64 bits."""
    from paper_2606_28166_amd import engine as E
    nq, nkv, hd, N, theta, eps = 2, 1, 32, 3, 1e4, 1e-6
    g = _gen(6)
    qkv = torch.randn((N, (nq + 2 * nkv) * hd), generator=g, device=DEV)
    pos = torch.tensor([0, 5, 1000], dtype=torch.int32, device=DEV)
    gq, gk = (1 + 0.3 * torch.randn((hd,), generator=g, device=DEV) for _ in range(2))
    wq, wk = torch.randn((N, nq, hd), generator=g, device=DEV), torch.randn((N, nkv, hd), generator=g, device=DEV)
    b = E.qk_norm_rope_backward(qkv, pos, wq, wk, theta, eps, q_gain=gq, k_gain=gk)
    x = [t.cpu().double().contiguous() for t in (qkv, gq, gk)]
    w = torch.cat([wq, wk], 1).cpu().double()
    a = pos.cpu().double()[:, None] * float(theta) ** (-2.0 * torch.arange(hd // 2, dtype=F64) / hd)
    cos, sin = a.cos()[:, None], a.sin()[:, None]

    def loss(qkv, gq, gk):
        h = qkv[:, :(nq + nkv) * hd].reshape(N, nq + nkv, hd)
        n = h / (h.pow(2).mean(2, keepdim=True) + eps).sqrt() * torch.cat([gq.expand(nq, hd), gk.expand(nkv, hd)])
        u, v = n[..., :hd // 2], n[..., hd // 2:]
        return float((torch.cat([u * cos - v * sin, v * cos + u * sin], 2) * w).sum())

    step = 1e-5
    for which, name in enumerate(("dqkv", "dq_gain", "dk_gain")):
        flat = x[which].view(-1)
        for at in range(0, flat.numel(), 7):
            keep = float(flat[at])
            flat[at] = keep + step
            up = loss(*x)
            flat[at] = keep - step
            down = loss(*x)
            flat[at] = keep
            # the value columns' gradient is 0, as the loss does not read them
            assert abs((up - down) / (2 * step) - float(b[name].reshape(-1)[at])) <= 1e-4, (name, at)


def test_qk_no_rows_clears_the_gains():
    from paper_2606_28166_amd import engine as E
    z = torch.zeros((0, 8 * 64), dtype=BF, device=DEV)
    p = torch.zeros(0, dtype=torch.int32, device=DEV)
    one = torch.ones(64, device=DEV)
    b = E.qk_norm_rope_backward(z, p, torch.zeros((0, 4, 64), dtype=BF, device=DEV),
                                torch.zeros((0, 2, 64), dtype=BF, device=DEV), 1e6, 1e-6, q_gain=one, k_gain=one)
    assert (b["dq_gain"] == 0).all() and (b["dk_gain"] == 0).all()


# ------------------------------------------------------------------ attention

def _attention_reference(q, k, v, dout, offs, scale):
    """out, lse, dq, dk, dv and their elementwise error bounds, in 64 bits."""
    N, nq, hd = q.shape
    nkv, dt = k.shape[1], q.dtype
    G = nq // nkv
    # a bf16 probability and score gradient is rounded once more; float32 ones are not
    e_p = _half(BF) if dt == BF else 4 * U
    # the P in dS may pass from wave to wave in float16 (of 2^15 P, so no subnormals that count):
    # half a step is 2^-11 of it, and (1 + 2^-8)(1 + 2^-11) - 1 <= 2^-8 + 2^-11 + 2^-19
    e_s = e_p + (2.0 ** -11 + 2.0 ** -19 if dt == BF else 0.0)
    h = _half(dt)
    zero = lambda x: torch.zeros(x.shape, dtype=F64, device=DEV)      # noqa: E731
    ref = {n: zero(x) for n, x in (("out", q), ("dq", q), ("dk", k), ("dv", k))}
    tol = {n: zero(x) for n, x in (("out", q), ("dq", q), ("dk", k), ("dv", k))}
    ref["lse"] = torch.zeros((nq, N), dtype=F64, device=DEV)
    tol["lse"] = torch.zeros((nq, N), dtype=F64, device=DEV)
    for a, b in zip(offs[:-1], offs[1:]):
        n = b - a
        if n <= 0:
            continue
        see = torch.ones((n, n), dtype=torch.bool, device=DEV).tril()
        for i in range(nq):
            j = i // G
            Q, K, V, D = (x.to(F64) for x in (q[a:b, i], k[a:b, j], v[a:b, j], dout[a:b, i]))
            s = torch.where(see, Q @ K.t().contiguous() * scale, torch.full((n, n), -math.inf, dtype=F64, device=DEV))
            es = torch.where(see, (Q.abs() @ K.abs().t().contiguous()) * scale, torch.zeros_like(s)) * (hd + 8) * U
            lse = s.logsumexp(1)
            p = s.softmax(1)
            worst = es.amax(1, keepdim=True)
            rel = es + worst + U * (n + 16 + 4 * torch.where(see, (s - lse[:, None]).abs(), torch.zeros_like(s)))
            o = p @ V
            to = (p * (rel + e_p + n * U)) @ V.abs() + h * o.abs()
            ref["out"][a:b, i], tol["out"][a:b, i] = o, to
            ref["lse"][i, a:b] = lse
            tol["lse"][i, a:b] = worst[:, 0] + U * (n + 16 + 4 * lse.abs())
            dp = D @ V.t().contiguous()
            edp = (hd + 4) * U * (D.abs() @ V.abs().t().contiguous())
            # dout . out uses the output as it was rounded
            de = (D.abs() * to).sum(1, keepdim=True) + hd * U * (D * o).abs().sum(1, keepdim=True)
            delta = (D * o).sum(1, keepdim=True)
            ds = p * (dp - delta)
            eds = p * (edp + de + rel * (dp - delta).abs()) + (e_s + 2 * U) * ds.abs()
            more = n * U
            ref["dq"][a:b, i] = ds @ K * scale
            tol["dq"][a:b, i] = (eds + more * ds.abs()) @ K.abs() * scale + h * ref["dq"][a:b, i].abs()
            ref["dk"][a:b, j] += ds.t().contiguous() @ Q * scale
            tol["dk"][a:b, j] += (eds + G * more * ds.abs()).t().contiguous() @ Q.abs() * scale
            ref["dv"][a:b, j] += p.t().contiguous() @ D
            tol["dv"][a:b, j] += (p * (rel + e_p + G * more)).t().contiguous() @ D.abs()
    for n in ("dk", "dv"):
        tol[n] += h * ref[n].abs() + h * tol[n]
    for n in tol:
        tol[n] += 1e-30
    return ref, tol


def _attention_inputs(N, nq, nkv, hd, dt, seed):
    g = _gen(seed)
    q = (1.5 * torch.randn((N, nq, hd), generator=g, device=DEV)).to(dt)
    k = (1.5 * torch.randn((N, nkv, hd), generator=g, device=DEV)).to(dt)
    qkv = torch.randn((N, (nq + 2 * nkv) * hd), generator=g, device=DEV).to(dt)
    v = qkv[:, (nq + nkv) * hd:].view(N, nkv, hd)
    dout = torch.randn((N, nq, hd), generator=g, device=DEV).to(dt)
    return q, k, v, dout


LENS = {
    "single": [1], "pair": [1, 2], "empty": [0, 5, 0, 0, 3, 0], "edges": [31, 32, 33, 63, 64, 65, 1],
    "tiles": [127, 128, 129, 0, 191, 257], "many": [(7 * i) % 23 for i in range(150)], "long": [1037],
    "few": [1100, 0, 1, 1503],
}


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("nq,nkv,hd", [(4, 2, 32), (16, 4, 64), (8, 1, 128), (3, 3, 64), (6, 2, 32), (1, 1, 128)])
@pytest.mark.parametrize("lens", list(LENS), ids=list(LENS))
def test_attention(lens, nq, nkv, hd, dt):
    """Sequences of none, one and many positions, at the tiles' edges, for groups of 1,
    2, 3, 4 and 8 heads; rows of no sequence keep what they held."""
    from paper_2606_28166_amd import engine as E
    _say("attention", lens, nq, nkv, hd, dt)
    n = LENS[lens]
    lead, tail = (3, 5) if lens != "single" else (0, 0)         # rows before the first and behind the last sequence
    offs = list(itertools.accumulate([lead] + n))
    N = offs[-1] + tail
    q, k, v, dout = _attention_inputs(N, nq, nkv, hd, dt, N + nq)
    scale = float(torch.tensor(hd ** -0.5, dtype=F32))
    ref, tol = _attention_reference(q, k, v, dout, offs, scale)
    o = torch.tensor(offs, dtype=torch.int32, device=DEV)
    mark = torch.full_like(q, 7.0)
    f = E.attention(q, k, v, o, out=mark)
    rows = slice(offs[0], offs[-1])
    _within(f["out"][rows], ref["out"][rows], tol["out"][rows], "out")
    _within(f["lse"][:, rows], ref["lse"][:, rows], tol["lse"][:, rows], "lse")
    assert (mark[:offs[0]] == 7.0).all() and (mark[offs[-1]:] == 7.0).all()
    dqkv = torch.full((N, (nq + 2 * nkv) * hd), 7.0, dtype=dt, device=DEV)
    dq, dk = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    dv = dqkv[:, (nq + nkv) * hd:].view(N, nkv, hd)
    b = E.attention_backward(dout, q, k, v, f["out"], f["lse"], o, dq=dq, dk=dk, dv=dv)
    for name in ("dq", "dk", "dv"):
        _within(b[name][rows], ref[name][rows], tol[name][rows], name)
        assert (b[name][:offs[0]] == 7.0).all() and (b[name][offs[-1]:] == 7.0).all(), name
    assert (dqkv[:, :(nq + nkv) * hd] == 7.0).all()
    again = E.attention_backward(dout, q, k, v, f["out"], f["lse"], o)
    for name in ("dq", "dk", "dv"):
        assert torch.equal(again[name][rows], b[name][rows]), name


@pytest.mark.parametrize("nq,nkv,hd", [(8, 4, 128), (16, 4, 64), (4, 2, 32)])
@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
def test_attention_of_many_short_sequences(nq, nkv, hd, dt):
    """A group's heads in one workgroup (enough tiles of keys), sequences found by length
    (64 of them) and by their offsets (65); rows of no sequence hold NaN and reach nothing."""
    from paper_2606_28166_amd import engine as E
    for n in (64, 65):
        _say("attention, many", n, nq, nkv, hd, dt)
        offs = list(itertools.accumulate([2] + [(53 * i) % 131 for i in range(n)]))
        N = offs[-1] + 7
        q, k, v, dout = _attention_inputs(N, nq, nkv, hd, dt, n)
        for x in (q, k, v, dout):
            x[:2] = math.nan
            x[offs[-1]:] = math.nan
        scale = float(torch.tensor(hd ** -0.5, dtype=F32))
        ref, tol = _attention_reference(q, k, v, dout, offs, scale)
        o = torch.tensor(offs, dtype=torch.int32, device=DEV)
        rows = slice(offs[0], offs[-1])
        f = E.attention(q, k, v, o, out=torch.full_like(q, math.nan))
        _within(f["out"][rows], ref["out"][rows], tol["out"][rows], "out")
        _within(f["lse"][:, rows], ref["lse"][:, rows], tol["lse"][:, rows], "lse")
        b = E.attention_backward(dout, q, k, v, f["out"], f["lse"], o)
        for name in ("dq", "dk", "dv"):
            _within(b[name][rows], ref[name][rows], tol[name][rows], name)


def test_attention_gradient_by_differences():
    """float32: the gradient of sum(w out) against central differences of the
    definition in 64 bits."""
    from paper_2606_28166_amd import engine as E
    N, nq, nkv, hd = 9, 2, 1, 32
    q, k, v, w = _attention_inputs(N, nq, nkv, hd, F32, 4)
    offs = [0, 4, 9]
    o = torch.tensor(offs, dtype=torch.int32, device=DEV)
    f = E.attention(q, k, v, o)
    got = E.attention_backward(w, q, k, v, f["out"], f["lse"], o)

    def loss(q, k, v):
        total = 0.0
        for a, b in zip(offs[:-1], offs[1:]):
            for i in range(nq):
                s = (q[a:b, i] @ k[a:b, 0].t()) * hd ** -0.5
                s = s.masked_fill(~torch.ones_like(s, dtype=torch.bool).tril(), -math.inf)
                total = total + (s.softmax(1) @ v[a:b, 0] * w[a:b, i].cpu().double()).sum()
        return float(total)

    x = [t.cpu().double().contiguous() for t in (q, k, v)]
    step = 1e-5
    for which, name in enumerate(("dq", "dk", "dv")):
        flat = x[which].view(-1)
        for at in range(0, flat.numel(), 37):
            keep = float(flat[at])
            flat[at] = keep + step
            up = loss(*x)
            flat[at] = keep - step
            down = loss(*x)
            flat[at] = keep
            # differences are off by the third derivative times step^2 and by 2^-53 |loss| / step
            assert abs((up - down) / (2 * step) - float(got[name].reshape(-1)[at])) <= 1e-4, (name, at)


@pytest.mark.parametrize("offs", [[0, 5, 1 << 30], [-7, 40, 40], [70, 80], [9, 3, 50], [-5, -2, 0]])
def test_attention_offsets_outside_are_clamped(offs):
    """Offsets before, behind and out of order: clamped to the rows there are."""
    from paper_2606_28166_amd import engine as E
    N, nq, nkv, hd = 64, 4, 2, 64
    q, k, v, dout = _attention_inputs(N, nq, nkv, hd, BF, 8)
    o = torch.tensor(offs, dtype=torch.int32, device=DEV)
    f = E.attention(q, k, v, o)
    f["lse"].clamp_(-100, 100).nan_to_num_(0.0)                 # rows of no sequence were not written
    f["out"].nan_to_num_(0.0)
    E.attention_backward(dout, q, k, v, f["out"], f["lse"], o)
    torch.cuda.synchronize()
    if offs == [0, 5, 1 << 30]:
        ref, tol = _attention_reference(q, k, v, dout, [0, 5, N], float(torch.tensor(hd ** -0.5, dtype=F32)))
        _within(f["out"], ref["out"], tol["out"], "out")


def test_attention_far_rows():
    """Rows whose offset passes 2^31 elements: a short sequence at the end of a large array."""
    from paper_2606_28166_amd import engine as E
    nq = nkv = 1
    hd, N, ld = 64, 1060, 1 << 21
    big = torch.zeros((N, ld), dtype=BF, device=DEV)
    q = big[:, :hd].view(N, 1, hd)
    q[-40:] = torch.randn((40, 1, hd), generator=_gen(1), device=DEV).to(BF)
    k = big[:, 64:128].view(N, 1, hd)
    k[-40:] = torch.randn((40, 1, hd), generator=_gen(2), device=DEV).to(BF)
    offs = [N - 40, N]
    o = torch.tensor(offs, dtype=torch.int32, device=DEV)
    f = E.attention(q, k, k, o)
    dq = big[:, 128:192].view(N, 1, hd)
    b = E.attention_backward(q, q, k, k, f["out"], f["lse"], o, dq=dq)
    ref, tol = _attention_reference(q[-40:], k[-40:], k[-40:], q[-40:], [0, 40], float(torch.tensor(hd ** -0.5, dtype=F32)))
    _within(f["out"][-40:], ref["out"], tol["out"], "out")
    for name in ("dq", "dk", "dv"):
        _within(b[name][-40:], ref[name], tol[name], name)
    assert (dq[:-40] == 0).all()


# ------------------------------------------------------------------ AdamW

def _adamw_reference(w, g, m, v, t, lr, b1, b2, eps, decay, c):
    x = c * g
    m = b1 * m + (1 - b1) * x
    v = b2 * v + (1 - b2) * x * x
    move = (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + eps)
    return w * (1 - lr * decay) - lr * move, m, v, lr * move


@pytest.mark.parametrize("master", [True, False], ids=["master", "in place"])
@pytest.mark.parametrize("max_norm", [0.0, 0.5])
@pytest.mark.parametrize("sizes", [[1], [0, 3, 7, 8, 9], [8191, 8192, 8193, 40000], [(13 * i) % 301 for i in range(230)]],
                         ids=["one", "small", "chunks", "many"])
def test_adamw(sizes, max_norm, master):
    """Tensors of no elements up to several chunks, more than one launch holds, both
    types, several steps; the arenas' padding is left alone."""
    from paper_2606_28166_amd import engine as E
    _say("adamw", len(sizes), max_norm, master)
    g = _gen(len(sizes) + sum(sizes))
    types = [BF if i % 2 else F32 for i in range(len(sizes))]
    params = [torch.randn((n,), generator=g, device=DEV).mul_(0.02).to(dt) for n, dt in zip(sizes, types)]
    decay = [0.1 * (i % 3) for i in range(len(sizes))]
    b1, b2, eps, lr = 0.9, 0.999, 1e-8, 1e-2
    opt = E.AdamW(params, betas=(b1, b2), eps=eps, weight_decay=decay, max_norm=max_norm, master=master)
    w = [p.double() for p in params]
    ms = [torch.zeros_like(x) for x in w]
    vs = [torch.zeros_like(x) for x in w]
    slack = [torch.zeros_like(x) for x in w]
    sizes_m = [torch.zeros_like(x) for x in w]
    inside = torch.zeros(opt.elems, dtype=torch.bool, device=DEV)
    for o, n in zip(opt.offsets, sizes):
        inside[o:o + n] = True
    pads = (opt.m, opt.v) + ((opt.master,) if master else ())
    for x in pads:
        x[~inside] = 7.0
    for t in (1, 2, 3):
        grads = [torch.randn((n,), generator=g, device=DEV).mul_(0.1).to(F32 if i % 3 else BF) for i, n in enumerate(sizes)]
        norm = opt.step(grads, lr)
        n64 = torch.sqrt(sum((x.double() ** 2).sum() for x in grads))
        c = min(1.0, max_norm / (float(n64) + 1e-6)) if max_norm else 1.0
        if max_norm:
            assert abs(float(norm) - float(n64)) <= 2 * U * float(n64)
        else:
            assert norm is None
        for i, (n, o) in enumerate(zip(sizes, opt.offsets)):
            w[i], ms[i], vs[i], move = _adamw_reference(w[i], grads[i].double(), ms[i], vs[i], t, lr, b1, b2, eps,
                                                        decay[i], c)
            # a step's roundings are 3 u of |b1 m| and 4 u of |(1 - b1) c g|, and m may cancel: with
            # S = b1 S + (1 - b1) |c g| >= |m|, the error e <= b1 e + 4 u S is at most 4 t u S
            sizes_m[i] = b1 * sizes_m[i] + (1 - b1) * c * grads[i].double().abs()
            size_m = sizes_m[i]
            _within(opt.m[o:o + n], ms[i], 8 * t * U * size_m, "m")
            _within(opt.v[o:o + n], vs[i], 8 * t * U * vs[i].abs(), "v")
            slack[i] += 32 * t * U * (lr * size_m / (1 - b1 ** t)) / ((vs[i] / (1 - b2 ** t)).sqrt() + eps) + \
                32 * U * move.abs() + 4 * U * (w[i].abs() + move.abs())
            if not master and types[i] == BF:
                slack[i] += _half(BF) * (w[i].abs() + slack[i])
                _within(params[i], w[i], slack[i], "weights")
            else:
                if master:
                    _within(opt.master[o:o + n], w[i], slack[i], "master")
                    assert torch.equal(params[i], opt.master[o:o + n].to(types[i]))
                else:
                    _within(params[i], w[i], slack[i], "weights")
    for x in pads:
        assert (x[~inside] == 7.0).all()


def test_adamw_norm_of_extreme_gradients():
    """Squares of 1e30 overflow float32, squares of 1e-30 vanish in it; the norm does neither."""
    from paper_2606_28166_amd import engine as E
    for size in (1e30, 1e-30):
        p = [torch.zeros(1000, device=DEV)]
        opt = E.AdamW(p, max_norm=1.0)
        norm = opt.step([torch.full((1000,), size, device=DEV)], 1e-3)
        want = float(torch.tensor(size, dtype=F32)) * math.sqrt(1000)
        assert abs(float(norm) - want) <= 2 * U * want


def test_adamw_resumes_and_repeats():
    """A state handed to a new optimizer continues; two runs agree bit for bit."""
    from paper_2606_28166_amd import engine as E

    def run(split):
        g = _gen(9)
        p = [torch.randn((n,), generator=g, device=DEV).to(BF) for n in (5, 9000, 33)]
        opt = E.AdamW(p, weight_decay=0.1, max_norm=1.0)
        for t in range(4):
            if t == split:
                opt = E.AdamW(p, weight_decay=0.1, max_norm=1.0, state=opt.state())
            opt.step([torch.randn(x.shape, generator=g, device=DEV).to(BF) for x in p], 1e-3)
        return p + [opt.m, opt.v, opt.master]

    a, b = run(2), run(9)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_adamw_of_trainable_weights():
    """Weights that require gradients: the state stays free of any autograd graph, and the
    step equals that of plain tensors."""
    from paper_2606_28166_amd import engine as E

    def run(make):
        g = _gen(3)
        p = [make(torch.randn(s, generator=g, device=DEV).to(BF)) for s in ((40, 30), (7,))]
        opt = E.AdamW(p, max_norm=1.0, weight_decay=0.1)
        for x in p:
            x.grad = torch.randn(x.shape, generator=g, device=DEV).to(BF)
        opt.step([x.grad for x in p], 1e-2)
        return p, opt

    plain, a = run(lambda x: x)
    train, b = run(lambda x: torch.nn.Parameter(x))
    assert b.master.grad_fn is None and not b.master.requires_grad and all(x.requires_grad for x in train)
    for x, y in zip(plain + [a.m, a.v, a.master], train + [b.m, b.v, b.master]):
        assert torch.equal(x, y.detach())


def test_adamw_refuses_weights_it_cannot_update():
    """Weights that share memory would be written by two workgroups at once; a weight moved
    since the last step is followed, unless it no longer is what the step can write."""
    from paper_2606_28166_amd import engine as E
    w = torch.zeros(64, device=DEV)
    for params in ([w, w], [w, w[32:]], [w[:40], w[39:]], [w[1:2], w, w[:0]]):
        with pytest.raises(ValueError):
            E.AdamW(params)
    E.AdamW([w[:32], w[32:], w[:0], w[:0]])
    a, b = torch.zeros((8, 8), device=DEV), torch.zeros(5, device=DEV)
    opt = E.AdamW([a, b])
    grads = [torch.ones_like(a), torch.ones_like(b)]
    opt.step(grads, 1e-3)
    a.data = a.data.clone()
    opt.step(grads, 1e-3)
    assert (a == a[0, 0]).all() and float(a[0, 0]) < -1.5e-3
    kept, steps = a.data, opt.steps
    for moved in (kept.t(), kept[:1, :1].expand(8, 8), kept.cpu(), kept.double(), kept.flatten()):
        a.data = moved
        with pytest.raises(ValueError):
            opt.step(grads, 1e-3)
    a.data = kept
    b.data = kept.view(-1)[3:8]                                 # now within the other weight
    with pytest.raises(ValueError):
        opt.step(grads, 1e-3)
    assert opt.steps == steps
    for state in (dict(opt.state(), m=None), dict(opt.state(), v=opt.v[:64])):
        with pytest.raises(ValueError):
            E.AdamW([a, torch.zeros(5, device=DEV)], state=state)


def test_workspaces_given():
    """A given workspace is used where it is large enough and contiguous, replaced otherwise."""
    from paper_2606_28166_amd import engine as E
    z, zr, tok, _, _ = _logprob_inputs(2, 40000, F32, 1)
    want = E.token_logprob(z, tok, ref=zr)
    for ws in (torch.full((1 << 16,), 255, dtype=torch.uint8, device=DEV),
               torch.full((1,), 255, dtype=torch.uint8, device=DEV).expand(1 << 16),
               torch.full((1 << 17,), 255, dtype=torch.uint8, device=DEV)[::2],
               torch.full((3,), 255, dtype=torch.uint8, device=DEV)):
        keep = ws.clone()
        got = E.token_logprob(z, tok, ref=zr, workspace=ws)
        assert all(torch.equal(got[n], want[n]) for n in want)
        assert torch.equal(ws, keep) != (ws.is_contiguous() and ws.numel() > 1000)


# ------------------------------------------------------------------ streams, graphs, several at once

def _all_ops(seed):
    """Every operator once on the current stream; a flat list of outputs."""
    from paper_2606_28166_amd import engine as E
    z, zr, tok, gl, gk = _logprob_inputs(5, 33000, BF, seed)
    q, k, v, dout = _attention_inputs(300, 8, 2, 64, BF, seed)
    offs = torch.tensor([0, 100, 101, 300], dtype=torch.int32, device=DEV)
    qkv = torch.randn((300, 12 * 64), generator=_gen(seed), device=DEV).to(BF)
    pos = torch.arange(300, dtype=torch.int32, device=DEV)
    gain = torch.rand((64,), generator=_gen(seed), device=DEV)
    params = [torch.randn((n,), generator=_gen(seed), device=DEV) for n in (100, 9000)]
    grads = [torch.randn((n,), generator=_gen(seed + 1), device=DEV) for n in (100, 9000)]
    opt = E.AdamW(params, max_norm=1.0)

    def run():
        r = E.token_logprob(z, tok, ref=zr)
        g = E.token_logprob_backward(z, tok, r, gl, g_kl=gk, ref=zr)
        n = E.qk_norm_rope(qkv, pos, 8, 2, 1e6, 1e-6, q_gain=gain, k_gain=gain)
        f = E.attention(q, k, v, offs)
        b = E.attention_backward(dout, q, k, v, f["out"], f["lse"], offs)
        nb = E.qk_norm_rope_backward(qkv, pos, n["q"], n["k"], 1e6, 1e-6, q_gain=gain, k_gain=gain)
        return [r["logp"], r["lse"], r["kl"], r["lse_diff"], g, n["q"], n["k"], f["out"], f["lse"], b["dq"], b["dk"],
                b["dv"], nb["dqkv"], nb["dq_gain"], nb["dk_gain"]]

    return run, opt, params, grads


def test_update_graph_replays():
    """Captured and replayed several times with eager work between: every replay
    equals the eager result."""
    run, opt, params, grads = _all_ops(5)
    want = [x.clone() for x in run()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for _ in range(4):
        for x in got:
            x.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
        assert all(torch.equal(x, y) for x, y in zip(run(), want))


def test_attention_graph_of_other_offsets():
    """The offsets are read on the device: one captured call serves other lengths in the
    same rows."""
    from paper_2606_28166_amd import engine as E
    N, nq, nkv, hd = 500, 8, 2, 64
    q, k, v, dout = _attention_inputs(N, nq, nkv, hd, BF, 21)
    offs = torch.tensor([0, 100, 101, 500], dtype=torch.int32, device=DEV)

    def run():
        f = E.attention(q, k, v, offs)
        return f, E.attention_backward(dout, q, k, v, f["out"], f["lse"], offs)

    run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f, b = run()
    for to in ([0, 500, 500, 500], [0, 0, 1, 500], [0, 250, 499, 500], [0, 100, 101, 500]):
        offs.copy_(torch.tensor(to, dtype=torch.int32))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        ff, bb = run()
        for x, y in ((f, ff), (b, bb)):
            assert all(torch.equal(x[n], y[n]) for n in x), to


def test_update_on_two_streams():
    """Two streams at once, neither the default one."""
    runs = [_all_ops(s)[0] for s in (11, 12)]
    want = [[x.clone() for x in r()] for r in runs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    got = [[], []]
    for _ in range(3):
        for i, (r, st) in enumerate(zip(runs, streams)):
            with torch.cuda.stream(st):
                got[i] = r()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_adamw_graph_replays():
    """A captured step repeats that step, its number included."""
    from paper_2606_28166_amd import engine as E
    _, opt, params, grads = _all_ops(6)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = opt.step(grads, 1e-3)
    _, _, q, _ = _all_ops(6)
    other = E.AdamW(q, max_norm=1.0)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        other.steps = 0
        n2 = other.step(grads, 1e-3)
        torch.cuda.synchronize()
        assert torch.equal(norm, n2) and all(torch.equal(a, b) for a, b in zip(params, q))
        assert torch.equal(opt.m, other.m) and torch.equal(opt.v, other.v)
