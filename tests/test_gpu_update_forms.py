"""Attention in every form its launches take, against the definition in 64 bits, and offsets outside the rows.

Attention's bounds are those of test_gpu_update.py (a score carries (hd + 8) u scale sum |q||k|, which is its
probability's relative error; bf16 probabilities and score gradients are rounded once more, 2^-8; dout . out takes
the output as it was rounded), with one difference: 11 bits of the probabilities count only where they pass from
wave to wave in float16, in dK of bf16 heads of 64 and 128: 2^-11 + 2^-19 beside the 2^-8 of dS.  dQ, and dK
of heads of 32, do without."""
import itertools
import math

import pytest
import torch

from tests.test_gpu_update import BF, DEV, F32, F64, LENS, U, _attention_inputs, _gen, _half, _say, _within
from tests.update_forms import FORMS

pytestmark = pytest.mark.gpu


def _reference(q, k, v, dout, offs, scale):
    """out, lse, dq, dk, dv and their elementwise bounds, in 64 bits, a head of a sequence at a time."""
    N, nq, hd = q.shape
    nkv, dt = k.shape[1], q.dtype
    G, h = nq // nkv, _half(dt)
    e_p = _half(BF) if dt == BF else 4 * U
    passed = 2.0 ** -11 + 2.0 ** -19 if dt == BF and hd >= 64 else 0.0
    ref = {n: torch.zeros(x.shape, dtype=F64, device=DEV) for n, x in
           (("out", q), ("dq", q), ("dk", k), ("dv", k), ("lse", q[..., 0].t()))}
    tol = {n: torch.zeros_like(x) for n, x in ref.items()}
    for a, b in zip(offs[:-1], offs[1:]):
        n = b - a
        if n <= 0:
            continue
        past = torch.ones((n, n), dtype=torch.bool, device=DEV).triu(1)
        for i in range(nq):
            j = i // G
            Q, K, V, D = (x.to(F64).contiguous() for x in (q[a:b, i], k[a:b, j], v[a:b, j], dout[a:b, i]))
            s = (Q @ K.t().contiguous() * scale).masked_fill_(past, -math.inf)
            es = ((Q.abs() @ K.abs().t().contiguous()) * (scale * (hd + 8) * U)).masked_fill_(past, 0.0)
            lse, p = s.logsumexp(1), s.softmax(1)
            worst = es.amax(1, keepdim=True)
            rel = es + worst + U * (n + 16) + 4 * U * (s - lse[:, None]).abs().masked_fill_(past, 0.0)
            o = p @ V
            to = (p * (rel + e_p + n * U)) @ V.abs() + h * o.abs()
            ref["out"][a:b, i], tol["out"][a:b, i] = o, to
            ref["lse"][i, a:b], tol["lse"][i, a:b] = lse, worst[:, 0] + U * (n + 16 + 4 * lse.abs())
            dp = D @ V.t().contiguous()
            off = dp - (D * o).sum(1, keepdim=True)
            e_off = (hd + 4) * U * (D.abs() @ V.abs().t().contiguous()) + (D.abs() * to).sum(1, keepdim=True) + \
                hd * U * (D * o).abs().sum(1, keepdim=True)
            ds = p * off
            eds = p * (e_off + rel * off.abs()) + (e_p + 2 * U) * ds.abs()
            ref["dq"][a:b, i] = ds @ K * scale
            tol["dq"][a:b, i] = (eds + n * U * ds.abs()) @ K.abs() * scale + h * ref["dq"][a:b, i].abs()
            ref["dk"][a:b, j] += ds.t().contiguous() @ Q * scale
            tol["dk"][a:b, j] += (eds + (passed + G * n * U) * ds.abs()).t().contiguous() @ Q.abs() * scale
            ref["dv"][a:b, j] += p.t().contiguous() @ D
            tol["dv"][a:b, j] += (p * (rel + e_p + G * n * U)).t().contiguous() @ D.abs()
    for n in ("dk", "dv"):
        tol[n] += h * ref[n].abs() + h * tol[n]
    for n in tol:
        tol[n] += 1e-30
    return ref, tol


def _check(lens, nq, nkv, hd, dt, lead=4, tail=5):
    from paper_2606_28166_amd import engine as E
    offs = list(itertools.accumulate([lead] + lens))
    N = offs[-1] + tail
    q, k, v, dout = _attention_inputs(N, nq, nkv, hd, dt, N + hd)
    ref, tol = _reference(q, k, v, dout, offs, float(torch.tensor(hd ** -0.5, dtype=F32)))
    o = torch.tensor(offs, dtype=torch.int32, device=DEV)
    f = E.attention(q, k, v, o)
    f.update(E.attention_backward(dout, q, k, v, f["out"], f["lse"], o))
    for name in ("out", "lse", "dq", "dk", "dv"):
        _within(f[name], ref[name], tol[name], name)        # rows of no sequence: 0 of 1e-30
    again = E.attention(q, k, v, o)
    again.update(E.attention_backward(dout, q, k, v, again["out"], again["lse"], o))
    for name in f:
        assert torch.equal(f[name], again[name]), name


@pytest.mark.parametrize("name", list(FORMS))
def test_attention_form(name):
    lens, nq, nkv, hd, bf16, _, _ = FORMS[name]
    _say("attention form", name)
    _check(lens, nq, nkv, hd, BF if bf16 else F32)


@pytest.mark.parametrize("nq,nkv,hd", [(4, 2, 32), (16, 4, 64), (8, 1, 128), (3, 3, 64), (1, 1, 128)])
@pytest.mark.parametrize("lens", ["edges", "tiles", "long", "few"])
def test_attention_gradients_in_their_own_bits(lens, nq, nkv, hd):
    """bf16: dQ, and dK of heads of 32, within the bound without 11 bits."""
    _say("attention, own bits", lens, nq, nkv, hd)
    _check(LENS[lens], nq, nkv, hd, BF)


@pytest.mark.parametrize("offs", [[0, 5, 1 << 30], [-7, 40, 40], [70, 80], [-5, -2, 0], [-(1 << 31), 3, 64], [64, 64]])
@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
def test_attention_clamps_offsets(offs, dt):
    """Every result of offsets that lie outside the rows: that of the clamped ones."""
    from paper_2606_28166_amd import engine as E
    N, nq, nkv, hd = 64, 4, 2, 64
    q, k, v, dout = _attention_inputs(N, nq, nkv, hd, dt, 8)
    clamped = [min(max(x, 0), N) for x in offs]
    ref, tol = _reference(q, k, v, dout, clamped, float(torch.tensor(hd ** -0.5, dtype=F32)))
    live = torch.zeros(N, dtype=torch.bool, device=DEV)
    live[clamped[0]:clamped[-1]] = True
    o = torch.tensor(offs, dtype=torch.int32, device=DEV)
    f = E.attention(q, k, v, o, out=torch.full_like(q, 7.0))
    f.update(E.attention_backward(dout, q, k, v, f["out"], f["lse"], o,
                                  **{n: torch.full_like(q if n == "dq" else k, 7.0) for n in ("dq", "dk", "dv")}))
    for name in ("out", "dq", "dk", "dv"):
        assert (f[name][~live] == 7.0).all(), name
        _within(f[name][live], ref[name][live], tol[name][live], name)
    _within(f["lse"], ref["lse"], tol["lse"], "lse")


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("nq,nkv,hd", [(2, 1, 32), (4, 1, 64), (2, 2, 128)])
def test_attention_of_large_scores(nq, nkv, hd, dt):
    """Scores of 2^19 and -2^19, exact in float32: the keys of the higher score share a query's probability.  Forward
    they are exact; backward a probability comes from the float32 log-sum-exp, whose exponent is off by 7 roundings
    of 2^19 log2 e at most: 0.32, a factor of 1.25."""
    from paper_2606_28166_amd import engine as E
    n = 150
    g = _gen(hd)
    x = 2.0 ** 19 / (hd * 0.125)                              # scale hd q k = 2^19 with scale 1 / 8
    side = (torch.rand((n,), generator=g, device=DEV) < 0.5).float() * 2 - 1
    side[0] = 1
    q = torch.full((n, nq, hd), 1.0, device=DEV).to(dt)
    k = (side * x)[:, None, None].expand(n, nkv, hd).to(dt).contiguous()
    v = torch.randn((n, nkv, hd), generator=g, device=DEV).to(dt)
    dout = torch.randn((n, nq, hd), generator=g, device=DEV).to(dt)
    o = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    f = E.attention(q, k, v, o, scale=0.125)
    p = ((side > 0)[None] & torch.ones((n, n), dtype=torch.bool, device=DEV).tril()).to(F64)
    p = p / p.sum(1, keepdim=True)
    for h in range(nq):
        V = v[:, h * nkv // nq].to(F64)
        out = p @ V
        _within(f["out"][:, h], out, (2 * _half(dt) + 200 * U) * (p @ V.abs()), "out")
        want = 2.0 ** 19 + (p > 0).sum(1).to(F64).log()
        _within(f["lse"][h], want, 3 * U * want, "lse")
    b = E.attention_backward(dout, q, k, v, f["out"], f["lse"], o, scale=0.125)
    bound = {name: torch.zeros(t.shape, dtype=F64, device=DEV) for name, t in (("dq", q), ("dk", k), ("dv", v))}
    for h in range(nq):
        j = h * nkv // nq
        D, V = dout[:, h].to(F64), v[:, j].to(F64)
        dp = D @ V.t().contiguous()
        off = 1.3 * p * (dp.abs() + (D * (p @ V)).sum(1, keepdim=True).abs() + 0.1 * (D.abs() * (p @ V.abs())).sum(1, keepdim=True))
        bound["dq"][:, h] = off @ k[:, j].to(F64).abs() * 0.125
        bound["dk"][:, j] += off.t().contiguous() @ q[:, h].to(F64).abs() * 0.125
        bound["dv"][:, j] += 1.3 * p.t().contiguous() @ D.abs()
    for name in bound:
        _within(b[name], torch.zeros_like(bound[name]), bound[name] + 1e-30, name)      # finite, and of the terms' size
