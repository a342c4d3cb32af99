"""Tensors of the caller's that a call writes: autograd learns of it, so a graph that saved one of them
refuses its backward pass instead of taking the new values."""
import pytest
import torch

from tests.test_gpu_update import DEV, F32, _attention_inputs, _gen, _logprob_inputs

pytestmark = pytest.mark.gpu


def _graph_of(t):
    """A scalar whose graph saved t."""
    x = torch.ones_like(t, requires_grad=True)
    return (x * t).sum()


def test_adamw_weights():
    from paper_2606_28166_amd import engine as E
    w = torch.nn.Parameter(torch.randn((8, 8), generator=_gen(1), device=DEV))
    b = torch.zeros(3, device=DEV)
    opt = E.AdamW([w, b], max_norm=1.0)
    grads = [torch.ones_like(w), torch.ones_like(b)]
    y = (torch.ones((2, 8), device=DEV, requires_grad=True) @ w).sum()
    y.backward(retain_graph=True)
    opt.step(grads, 1e-3)
    with pytest.raises(RuntimeError, match="inplace"):
        y.backward()
    # a graph of the new weights runs; a refused step has written nothing
    y = (torch.ones((2, 8), device=DEV, requires_grad=True) @ w).sum()
    with pytest.raises(ValueError):
        opt.step(grads[:1], 1e-3)
    y.backward()
    # weights made in inference mode have no version
    with torch.inference_mode():
        v = torch.zeros(5, device=DEV)
        E.AdamW([v]).step([torch.ones_like(v)], 1e-3)
    assert float(v[0]) < 0


def test_outputs_that_are_given():
    from paper_2606_28166_amd import engine as E
    z, _, tok, gl, _ = _logprob_inputs(3, 50, F32, 1)
    f = E.token_logprob(z, tok)
    y, keep = _graph_of(z), _graph_of(z.clone())
    E.token_logprob_backward(z, tok, f, gl)
    y.backward(retain_graph=True)                           # z was read only
    E.token_logprob_backward(z, tok, f, gl, out=z)
    with pytest.raises(RuntimeError, match="inplace"):
        y.backward()
    keep.backward()

    q, k, v, dout = _attention_inputs(20, 4, 2, 32, F32, 2)
    o = torch.tensor([0, 20], dtype=torch.int32, device=DEV)
    out, dq, dk, dv = torch.empty_like(q), torch.empty_like(q), torch.empty_like(k), torch.empty_like(k)
    inputs = [_graph_of(x) for x in (q, k, v, dout)]
    y = _graph_of(out)
    f = E.attention(q, k, v, o, out=out)
    with pytest.raises(RuntimeError, match="inplace"):
        y.backward()
    graphs = [_graph_of(x) for x in (dq, dk, dv)]
    E.attention_backward(dout, q, k, v, f["out"], f["lse"], o, dq=dq, dk=dk, dv=dv)
    for y in graphs:
        with pytest.raises(RuntimeError, match="inplace"):
            y.backward()

    qkv = torch.randn((20, 8 * 32), generator=_gen(3), device=DEV)
    pos, one = torch.arange(20, dtype=torch.int32, device=DEV), torch.ones(32, device=DEV)
    for gains in ({}, dict(q_gain=one, k_gain=one)):
        d = torch.zeros_like(qkv)
        y, keep = _graph_of(d), _graph_of(qkv)
        E.qk_norm_rope_backward(qkv, pos, dq, dk, 1e6, 1e-6, dqkv=d, **gains)
        with pytest.raises(RuntimeError, match="inplace"):
            y.backward()
        keep.backward()
    for y in inputs:
        y.backward()
