"""The q/k backward pass and the optimizer at the sizes where their work spreads over several rounds of
workgroups or several launches, against the definitions in 64 bits."""
import math

import pytest
import torch

from tests.test_gpu_update import BF, DEV, F32, U, _adamw_reference, _gen, _half, _qk_reference, _say, _within

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ q/k backward over several rounds

@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("nq,nkv,hd,N", [(16, 8, 128, 4097), (16, 8, 128, 9001), (32, 8, 64, 5003), (1, 1, 32, 140001),
                                         (5, 5, 128, 20011)])
def test_qk_backward_of_many_rows(nq, nkv, hd, N, dt):
    """More rows than the 1024 workgroups take in one round, with a remainder."""
    from paper_2606_28166_amd import engine as E
    _say("qk backward, many rows", nq, nkv, hd, N, dt)
    g = _gen(N)
    qkv = torch.randn((N, (nq + 2 * nkv) * hd), generator=g, device=DEV).to(dt)
    pos = torch.randint(0, 5000, (N,), generator=g, device=DEV, dtype=torch.int32)
    gq, gk = [1 + 0.3 * torch.randn((hd,), generator=g, device=DEV) for _ in range(2)]
    # a mean that does not vanish, so that rows left out or taken twice show in the gains' sums
    dq = (1 + torch.randn((N, nq, hd), generator=g, device=DEV)).to(dt)
    dk = (1 + torch.randn((N, nkv, hd), generator=g, device=DEV)).to(dt)
    ref = _qk_reference(qkv, pos, nq, nkv, 1e6, 1e-6, gq, gk, dq, dk)
    b = E.qk_norm_rope_backward(qkv, pos, dq, dk, 1e6, 1e-6, q_gain=gq, k_gain=gk)
    d = b["dqkv"].view(N, nq + 2 * nkv, hd)
    for name, part, (_, _, dx, xs, _, _) in (("dq", d[:, :nq], ref[0]), ("dk", d[:, nq:nq + nkv], ref[1])):
        _within(part, dx, 2.0 ** -19 * xs + _half(dt) * dx.abs(), name)
    for name, (*_, dg, gs) in zip(("dq_gain", "dk_gain"), ref):
        # a lane adds at most N (nq + nkv) / 64 terms, a workgroup 128 lanes, workgroups in 64 bits
        _within(b[name], dg, (2.0 ** -19 + U * (N * (nq + nkv) / 64 + 160)) * gs, name)


# ------------------------------------------------------------------ AdamW over several launches, the factor from memory

@pytest.mark.parametrize("max_norm", [0.5, 1e9], ids=["clipped", "below"])
@pytest.mark.parametrize("sizes", [[5_000_001], [3] * 95 + [4_300_000, 77, 8193] + [(31 * i) % 500 for i in range(120)]],
                         ids=["one", "launches"])
def test_adamw_of_more_than_512_chunks(sizes, max_norm):
    """A clipping factor read from memory, sums of squares that cross launches."""
    from paper_2606_28166_amd import engine as E
    assert sum(-(-n // 8192) for n in sizes) > 512
    g = _gen(len(sizes))
    types = [BF if i % 2 else F32 for i in range(len(sizes))]
    params = [torch.randn((n,), generator=g, device=DEV).mul_(0.02).to(t) for n, t in zip(sizes, types)]
    b1, b2, eps, lr, decay = 0.9, 0.999, 1e-8, 1e-2, 0.1
    opt = E.AdamW(params, betas=(b1, b2), eps=eps, weight_decay=decay, max_norm=max_norm, master=True)
    w = [p.double() for p in params]
    state = [(torch.zeros_like(x), torch.zeros_like(x)) for x in w]
    for t in (1, 2):
        # sizes of their own, so that a tensor's sum taken twice or not at all shows in the norm
        grads = [(torch.randn((n,), generator=g, device=DEV) * (0.1 + 0.01 * (i % 7))).to(F32 if i % 3 else BF)
                 for i, n in enumerate(sizes)]
        norm = opt.step(grads, lr)
        n64 = math.sqrt(sum(float((x.double() ** 2).sum()) for x in grads))
        assert abs(float(norm) - n64) <= 2 * U * n64
        c = min(1.0, max_norm / (n64 + 1e-6))
        assert (c < 1.0) == (max_norm < 1)
        for i, (n, o) in enumerate(zip(sizes, opt.offsets)):
            m, v = state[i]
            size_m = b1 * m.abs() + (1 - b1) * c * grads[i].double().abs()
            w[i], m, v, move = _adamw_reference(w[i], grads[i].double(), m, v, t, lr, b1, b2, eps, decay, c)
            state[i] = (m, v)
            # fewer than 32 operations per element and step; m may cancel, so its error is of its terms' size
            _within(opt.m[o:o + n], m, 16 * t * U * size_m + 16 * U * m.abs(), "m")
            _within(opt.v[o:o + n], v, 16 * t * U * v, "v")
            tol = 32 * t * U * (lr * size_m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + eps) + \
                32 * t * U * lr + 8 * t * U * (w[i].abs() + move.abs())
            _within(opt.master[o:o + n], w[i], tol, "master")
            assert torch.equal(params[i], opt.master[o:o + n].to(types[i]))
