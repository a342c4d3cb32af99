"""Rows that belong to no sequence: 0 in the outputs that the binding allocates, so that sums over all
rows (the gains' gradients, a projection's weight gradient) are those of the sequences' rows; as they
were in outputs that the caller gives."""
import itertools
import math

import pytest
import torch

from tests.test_gpu_update import BF, DEV, F32, _attention_inputs, _gen, _say

pytestmark = pytest.mark.gpu

# a few tiles, one long sequence (the keys shared by the waves, the keys' pass in parts), many short ones, none but rows
CASES = {"short": [3, 0, 33], "long": [1300], "many": [(29 * i) % 61 for i in range(80)], "empty": [0, 0],
         "wide": [700, 40, 650]}


def _leave_nan(*tensors):
    """Memory of these sizes that the allocator hands out next holds NaN."""
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    held = [torch.full_like(t, math.nan) for t in tensors]
    torch.cuda.synchronize()
    del held


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("nq,nkv,hd", [(4, 2, 32), (16, 4, 64), (4, 1, 128), (32, 8, 128)])
@pytest.mark.parametrize("lens", list(CASES))
def test_attention_rows_of_no_sequence(lens, nq, nkv, hd, dt):
    from paper_2606_28166_amd import engine as E
    _say("rows of no sequence", lens, nq, nkv, hd, dt)
    offs = list(itertools.accumulate([5] + CASES[lens]))
    N = offs[-1] + 70
    q, k, v, dout = _attention_inputs(N, nq, nkv, hd, dt, N)
    o = torch.tensor(offs, dtype=torch.int32, device=DEV)
    live = torch.zeros(N, dtype=torch.bool, device=DEV)
    live[offs[0]:offs[-1]] = True
    for x in (q, k, v, dout):
        x[~live] = math.nan                                  # not read
    mark = torch.full_like(q, 7.0)
    given = E.attention(q, k, v, o, out=mark)
    assert (mark[~live] == 7.0).all() and (given["lse"][:, ~live] == 0).all()
    _leave_nan(q, given["lse"])
    f = E.attention(q, k, v, o)
    assert (f["out"][~live] == 0).all() and (f["lse"][:, ~live] == 0).all()
    assert torch.equal(f["out"][live], mark[live]) and torch.equal(f["lse"], given["lse"])
    _leave_nan(q, k, v)
    b = E.attention_backward(dout, q, k, v, f["out"], f["lse"], o)
    for name in ("dq", "dk", "dv"):
        assert (b[name][~live] == 0).all(), name
    # some given, some not
    for names in (("dq",), ("dk",), ("dv",), ("dq", "dk", "dv")):
        mine = {n: torch.full_like(q if n == "dq" else k, 7.0) for n in names}
        _leave_nan(q, k, v)
        c = E.attention_backward(dout, q, k, v, f["out"], f["lse"], o, **mine)
        for n in ("dq", "dk", "dv"):
            assert torch.equal(c[n][live], b[n][live]) and (c[n][~live] == (7.0 if n in names else 0.0)).all(), (names, n)


def test_attention_without_sequences():
    from paper_2606_28166_amd import engine as E
    q, k, v, dout = _attention_inputs(40, 4, 2, 64, BF, 1)
    o = torch.tensor([9], dtype=torch.int32, device=DEV)
    _leave_nan(q, k, v)
    f = E.attention(q, k, v, o)
    b = E.attention_backward(dout, q, k, v, f["out"], f["lse"], o)
    for x in (f["out"], f["lse"], b["dq"], b["dk"], b["dv"]):
        assert (x == 0).all()


def test_padded_batch_has_the_gradients_of_its_sequences():
    """The chain over a batch with padding rows against the same chain without them."""
    from paper_2606_28166_amd import engine as E
    nq, nkv, hd, lead, n, tail = 8, 2, 64, 3, 150, 40
    N = lead + n + tail
    g = _gen(4)
    qkv = torch.randn((N, (nq + 2 * nkv) * hd), generator=g, device=DEV)
    x = torch.randn((N, 96), generator=g, device=DEV)
    pos = torch.arange(N, dtype=torch.int32, device=DEV)
    gains = [1 + 0.3 * torch.randn((hd,), generator=g, device=DEV) for _ in range(2)]
    dout = torch.randn((N, nq, hd), generator=g, device=DEV)

    def chain(rows, offs):
        o = torch.tensor(offs, dtype=torch.int32, device=DEV)
        kw = dict(q_gain=gains[0], k_gain=gains[1])
        h = qkv[rows].contiguous()
        r = E.qk_norm_rope(h, pos[rows].contiguous(), nq, nkv, 1e6, 1e-6, **kw)
        _leave_nan(r["q"], r["k"], r["k"])
        f = E.attention(r["q"], r["k"], r["v"], o)
        b = E.attention_backward(dout[rows].contiguous(), r["q"], r["k"], r["v"], f["out"], f["lse"], o)
        d = E.qk_norm_rope_backward(h, pos[rows].contiguous(), b["dq"], b["dk"], 1e6, 1e-6, **kw)
        d["dqkv"][:, (nq + nkv) * hd:] = b["dv"].flatten(1)
        return [d["dq_gain"], d["dk_gain"], x[rows].t() @ d["dqkv"], f["out"].flatten(1).t() @ x[rows]]

    padded = chain(slice(0, N), [lead, lead + 100, lead + n])
    alone = chain(slice(lead, lead + n), [0, 100, n])
    for a, b in zip(padded, alone):
        # the same terms in another order, 190 rows of 8 heads at most: 1600 roundings of 2^-24 of their sizes' sum
        assert torch.isfinite(a).all() and float((a - b).norm()) <= 1e-4 * float(b.norm())
