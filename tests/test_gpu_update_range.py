"""Log-probs of rows whose scores are large in magnitude: everything finite that the type holds,
and the temperatures that make ordinary logits large.

The bounds count roundings, u = 2^-24, and none of them grows with an offset that a row's scores
share.  With s the scores, m their maximum, p the probabilities, d = s - s' and E the mean under p:

* an exponential's argument is off by 5 u |s - m| (difference, two constants, 1 / T, a product), the
  exponential by 4 u; eight of them are summed in float32, 8 u, the rest in 64 bits: a log of
  their sum is off by u (5 E|s - m| + 12).
* logp: that, u (|s_y - m|) for 1 / T and u |logp| for the result; lse_diff: both models', and 2 u of itself; lse: 2 u
  of itself.
* kl: both models' sums, a weight's error times d - E d, u (5 E|s - m||d - E d| + 12 E|d - E d|), and 3 u
  of itself.  Where no score passes 2^10 ln 2 eight differences and eight weights are summed in float32,
  a product and eight additions, and eight additions: 17 u E|d|.
"""
import math

import pytest
import torch

from tests.test_gpu_update import BF, F32, F64, U, _half, _logprob_inputs, _say, _scores64, _within

pytestmark = pytest.mark.gpu

# (base of the logits, of the reference's, temperature): every pair of signs, far beyond 2^30, the type's ends
ROWS = [(1e6, 1e6, 1.0), (-1e6, 1e6, 1.0), (1e9, -1e9, 1.0), (-1e9, 0.0, 1.0), (0.0, -1e9, 1.0), (1e10, 1e10, 1.0),
        (-1e10, -1e10, 1.0), (-7e10, 3.0, 1.0), (3.0, 7e10, 1.0), (3e12, 3e12, 1.0), (-1e20, -1e20, 1.0),
        (2.5e38, 2.5e38, 1.0), (1e4, 1e4, 1.0), (-3e5, 2e5, 1.0), (1.0, 1.0, 1e-3), (1.0, 1.0, 1e-9), (1e4, -1e4, 1e-6)]


def _inputs(R, V, dt, base, base_ref, seed):
    z, zr, tok, gl, gk = _logprob_inputs(R, V, dt, seed)
    z = (z.float() + base).to(dt)
    zr = (zr.float() + base_ref).to(dt)
    z[0], zr[0] = base, base_ref                           # a uniform row
    tok[0] = V - 1
    return z, zr, tok, gl, gk


def _moments(s):
    """Maximum, log of the sum against it (at large offsets a log-sum-exp loses digits in 64 bits too), probabilities."""
    m = s.amax(1)
    logsum = (s - m[:, None]).exp().sum(1).log()
    return m, logsum, (s - m[:, None] - logsum[:, None]).exp()


def _forward_check(r, z, zr, tok, T):
    s = _scores64(z, T, -1, 0.0)
    y = tok.long()[:, None]
    m, logsum, p = _moments(s)
    logp = s.gather(1, y)[:, 0] - m - logsum
    t_sum = U * (5 * (p * (s - m[:, None]).abs()).sum(1) + 12)
    _within(r["logp"], logp, t_sum + U * ((s.gather(1, y)[:, 0] - m).abs() + logp.abs()), "logp")
    _within(r["lse"], m + logsum, t_sum + 2 * U * (m + logsum).abs() + 2 * U * m.abs(), "lse")
    if zr is None:
        return
    q = _scores64(zr, T, -1, 0.0)
    n, logsum_r, pr = _moments(q)
    t_ref = U * (5 * (pr * (q - n[:, None]).abs()).sum(1) + 12)
    diff = (m - n) + (logsum - logsum_r)
    _within(r["lse_diff"], diff, t_sum + t_ref + 2 * U * diff.abs() + U * (m - n).abs(), "lse_diff")
    # the KL without the models' offsets: d against the maxima's difference
    d = (s - m[:, None]) - (q - n[:, None])
    mean = (p * d).sum(1, keepdim=True)
    kl = mean[:, 0] - (logsum - logsum_r)
    away = (d - mean).abs()
    tol = t_sum + t_ref + U * ((p * away * (5 * (s - m[:, None]).abs() + 12)).sum(1) + 3 * kl.abs())
    near = torch.maximum(m.abs(), n.abs()) <= 1024 * math.log(2.0)
    tol = tol + torch.where(near, 17 * U * (p * (s - q).abs()).sum(1), torch.zeros_like(tol))
    if T != 1.0:                                           # the scores here are rounded to 64 bits
        tol = tol + 2.0 ** -52 * (m.abs() + n.abs())
    _within(r["kl"], kl, tol, "kl")


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("R,V", [(5, 1000), (3, 40000), (1030, 2600)], ids=["waves", "parts", "whole"])
def test_logprob_of_large_rows(R, V, dt):
    """Rows of a wave, in parts and of a workgroup; uniform and spread, with and without a reference."""
    from paper_2606_28166_amd import engine as E
    for i, (base, base_ref, T) in enumerate(ROWS + [(torch.finfo(dt).max, torch.finfo(dt).max, 1.0),
                                                    (torch.finfo(dt).min, 1.0, 1.0)]):
        _say("logprob, large", R, V, dt, base, base_ref, T)
        z, zr, tok, _, _ = _inputs(R, V, dt, base, base_ref, i)
        # 1 / T as the call rounds it
        T64 = 1.0 / float(1.0 / torch.tensor(T, dtype=F32))
        _forward_check(E.token_logprob(z, tok, ref=zr, temperature=T), z, zr, tok, T64)
        _forward_check(E.token_logprob(z, tok, temperature=T), z, None, tok, T64)


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
def test_logprob_of_large_rows_beside_masked_entries(dt):
    """Large rows with entries of -inf and of the type's lowest value, in either model."""
    from paper_2606_28166_amd import engine as E
    low = torch.finfo(dt).min
    for V in (700, 20000):
        z, zr, tok, _, _ = _inputs(6, V, dt, 1e6, -1e6, V)
        tok.fill_(1)
        want = E.token_logprob(z[:, :100].contiguous(), tok, ref=zr[:, :100].contiguous())
        for a, b in ((-math.inf, -math.inf), (low, low), (-math.inf, -1.3e6), (low, -1.3e6)):
            z[:, 100:], zr[:, 100:] = a, b
            r = E.token_logprob(z, tok, ref=zr)
            ref = E.token_logprob(z.float(), tok, ref=zr.float())
            assert torch.isfinite(r["kl"]).all() and torch.isfinite(r["logp"]).all()
            # the masked entries add nothing: the same sums as without them, in another order
            for n in ("logp", "lse", "lse_diff", "kl"):
                size = want[n].abs() + 40
                assert ((r[n] - want[n]).abs() <= 32 * U * size).all(), (n, V, a, b)
                assert ((r[n] - ref[n]).abs() <= 32 * U * size).all(), (n, V, a, b)


# The gradient takes p = e^(s - lse) from the float32 lse, which is off by at most u |lse|, up to a log-sum-exp (and a
# mean difference of the models' scores) of this much: 2^-12 in bf16, a sixteenth of half a step, 2^-16 in float32.
# Other rows are summed anew.
GRAD_LIMIT = {BF: 4096.0, F32: 256.0}


def _gradient_check(grad, z, zr, tok, gl, gk, T, dt):
    """grad = (g ([v = y] - p) + k p (d - E d)) / T.  p is off by the argument, 5 u of |s - lse| or |s - m|, the
    exponential and the sum; where lse is taken, by u |lse|.  The terms carry 4 roundings of their sizes, d - E d
    where it is formed from lse_diff + kl 4 of each part and what those are off by."""
    s = _scores64(z, T, -1, 0.0)
    m, logsum, p = _moments(s)
    lse, depth = m + logsum, (s - m[:, None]).abs()
    e_sum = 5 * (p * depth).sum(1) + 12
    hot = torch.zeros_like(p).scatter_(1, tok.long()[:, None], 1.0)
    g = gl.to(F64)[:, None]
    want, size = g * (hot - p), g.abs() * (hot + p)
    taken = lse.abs() < 1.01 * GRAD_LIMIT[dt]
    extra, flushed = torch.zeros_like(p), g.abs().expand_as(p).clone()
    if zr is not None:
        q = _scores64(zr, T, -1, 0.0)
        n, logsum_r, pr = _moments(q)
        d = (s - m[:, None]) - (q - n[:, None])
        mean = (p * d).sum(1, keepdim=True)
        away = (d - mean).abs()
        shift = mean[:, 0] + (m - n)
        taken &= shift.abs() < 1.01 * GRAD_LIMIT[dt]
        k = gk.to(F64)[:, None]
        want = want + k * p * (d - mean)
        size = size + k.abs() * p * away
        e_mean = (p * away * (5 * depth + 12)).sum(1)
        diff = (m - n) + logsum - logsum_r
        kl = mean[:, 0] - (logsum - logsum_r)
        parts = 17 * (p * (s - q).abs()).sum(1) + 2 * diff.abs() + 5 * kl.abs() + 4 * shift.abs() + 2 * e_sum + \
            10 * (pr * (q - n[:, None]).abs()).sum(1) + 24
        extra = U * k.abs() * p * (e_mean[:, None] + torch.where(taken[:, None], parts[:, None] + 4 * (s - q).abs(),
                                                                torch.zeros_like(p)))
        flushed += k.abs() * away
    rel = U * (5 * depth + 5 * (s - m[:, None] - logsum[:, None]).abs() + 16 + e_sum[:, None] +
               torch.where(taken, lse.abs(), torch.zeros_like(lse))[:, None])
    tol = (size * rel + extra + 2.0 ** -126 * flushed) / T + _half(dt) * want.abs() / T + 2.0 ** -126
    _within(grad, want / T, tol, "grad")


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("R,V", [(5, 1000), (3, 40000)])
def test_logprob_gradient_of_large_rows(R, V, dt):
    """The same rows and some near the limit, with and without a reference, also in the logits' place."""
    from paper_2606_28166_amd import engine as E
    near = [(1.0, 1.0, 1.0), (100.0, -100.0, 1.0), (230.0, 231.0, 1.0), (-260.0, 1.0, 1.0), (2.0, 2.0, 0.02),
            (1.0, 300.0, 1.0), (4000.0, 4000.0, 1.0), (-4200.0, 4.0, 1.0), (1e5, 1e5, 1.0), (1.0, 1.0, 1e-4)]
    for i, (base, base_ref, T) in enumerate(near + ROWS + [(torch.finfo(dt).max, torch.finfo(dt).max, 1.0)]):
        _say("gradient, large", R, V, dt, base, base_ref, T)
        z, zr, tok, gl, gk = _inputs(R, V, dt, base, base_ref, i)
        T64 = 1.0 / float(1.0 / torch.tensor(T, dtype=F32))
        keep = z.clone()
        f = E.token_logprob(z, tok, ref=zr, temperature=T)
        a = E.token_logprob_backward(z, tok, f, gl, g_kl=gk, ref=zr, temperature=T)
        _gradient_check(a, z, zr, tok, gl, gk, T64, dt)
        b = E.token_logprob_backward(z, tok, f, gl, temperature=T)
        _gradient_check(b, z, None, tok, gl, None, T64, dt)
        assert torch.equal(z, keep)
        assert torch.equal(E.token_logprob_backward(z, tok, f, gl, g_kl=gk, ref=zr, temperature=T, out=z), a)


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
def test_logprob_gradient_at_the_smallest_temperatures(dt):
    """1 / T^2 passes float32: models that agree everywhere have a KL of 0 and no gradient of it."""
    from paper_2606_28166_amd import engine as E
    for T in (1e-19, 1e-25, 4e-39):
        for V in (50, 9000):
            z, _, tok, gl, gk = _inputs(3, V, dt, 0.0, 0.0, V)
            z.fill_(0.0)
            gl.mul_(0.25)                                    # g / T stays in the type
            f = E.token_logprob(z, tok, ref=z.clone(), temperature=T)
            assert (f["kl"] == 0).all() and (f["lse_diff"] == 0).all()
            g = E.token_logprob_backward(z, tok, f, gl, g_kl=gk, ref=z.clone(), temperature=T)
            hot = torch.zeros((3, V), dtype=F64, device=z.device).scatter_(1, tok.long()[:, None], 1.0)
            want = gl.to(F64)[:, None] * (hot - 1.0 / V) * float(1.0 / torch.tensor(T, dtype=F32))
            _within(g, want, (_half(dt) + 64 * U) * want.abs(), "grad")


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
def test_logprob_at_the_largest_temperatures(dt):
    """1 / T is subnormal: every row is uniform, and no output is lost to it."""
    from paper_2606_28166_amd import engine as E
    for T in (1e38, 3.4e38):
        for R, V in ((3, 50), (2, 40000), (1030, 2600)):
            z, zr, tok, gl, gk = _inputs(R, V, dt, 1.0, -2.0, V)
            f = E.token_logprob(z, tok, ref=zr, temperature=T)
            one = torch.ones(R, dtype=F64, device=z.device)
            _within(f["logp"], -math.log(V) * one, 16 * U * math.log(V) * one, "logp")
            _within(f["lse"], math.log(V) * one, 16 * U * math.log(V) * one, "lse")
            for name in ("kl", "lse_diff"):
                _within(f[name], 0 * one, 32 * U * one, name)
            g = E.token_logprob_backward(z, tok, f, gl, g_kl=gk, ref=zr, temperature=T)
            # at most |g| / T, which is about the smallest normal number
            assert torch.isfinite(g).all() and float(g.float().abs().max()) <= 4 * 2.0 ** -126
