"""Refusals of the update operators (log-probs, q/k norm and rotation,
attention, AdamW) that need no GPU: every one is returned before any HIP call,
so the pointers here are never followed."""
import ctypes as C

import pytest
import torch

L = pytest.importorskip("paper_2606_28166_amd._lib", reason="libtandem.so not built")

from paper_2606_28166_amd import engine as E  # noqa: E402

P = 0x10000                      # an address that no call may reach
WS = 0x20000


def _status(fn, *args):
    st = fn(*args)
    assert st == L.OK or L.lib.tandem_last_error(None)
    return st


def _set(cfg, **kw):
    for k, v in kw.items():
        setattr(cfg, k, v)
    return cfg


def _logprob(**kw):
    return _set(L.LogprobCfg(4, 1000, L.F32, -1, 1000, 1000, 1000, 1.0, 0.0, 0.0), **kw)


def _logprob_call(cfg, z=P, zr=P, tok=P, logp=P, lse=P, kl=P, diff=P, ws=WS, wsb=1 << 20):
    return _status(L.lib.tandem_token_logprob, C.byref(cfg), z, zr, tok, logp, lse, kl, diff, ws, wsb, None)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), L.E_SHAPE), (dict(vocab=0), L.E_SHAPE), (dict(dtype=2), L.E_ARG),
    (dict(temperature=0.0), L.E_ARG), (dict(temperature=-1.0), L.E_ARG), (dict(temperature=float("nan")), L.E_ARG),
    (dict(temperature=float("inf")), L.E_ARG), (dict(temperature=1e-40), L.E_ARG), (dict(eos_id=1000), L.E_ARG),
    (dict(eos_bias=float("inf")), L.E_ARG), (dict(eos_bias_ref=float("nan")), L.E_ARG),
    (dict(logits_stride=999), L.E_SHAPE), (dict(ref_stride=999), L.E_SHAPE),
])
def test_logprob_refuses_settings(kw, code):
    assert _logprob_call(_logprob(**kw)) == code


def test_logprob_refuses_pointers():
    c = _logprob(rows=2, vocab=100000, logits_stride=100000, ref_stride=100000, grad_stride=100000)
    need = L.tandem_logprob_workspace_size(c)
    assert need > 0                                                  # few rows: cut into parts
    assert _logprob_call(c, z=None) == L.E_ARG
    assert _logprob_call(c, tok=None) == L.E_ARG
    assert _logprob_call(c, zr=None) == L.E_ARG                      # kl and lse_diff without a reference
    assert _logprob_call(c, kl=None) == L.E_ARG
    assert _logprob_call(c, z=P + 2) == L.E_ARG                      # float32 off its alignment
    assert _logprob_call(c, ws=None) == L.E_ARG
    assert _logprob_call(c, ws=WS + 16) == L.E_ARG
    assert _logprob_call(c, wsb=need - 1) == L.E_ARG
    assert L.lib.tandem_token_logprob(None, P, P, P, P, P, P, P, WS, 1, None) == L.E_ARG
    back = L.lib.tandem_token_logprob_backward
    assert _status(back, C.byref(c), P, P, P, P, P, P, None, None, P, None) == L.E_ARG      # no g_logp
    assert _status(back, C.byref(c), P, None, P, P, P, P, P, P, P, None) == L.E_ARG         # g_kl without reference
    assert _status(back, C.byref(c), P, P, P, P, None, P, P, P, P, None) == L.E_ARG         # g_kl without kl
    assert _status(back, C.byref(_set(_logprob(), grad_stride=999)), P, P, P, P, P, P, P, P, WS, None) == L.E_SHAPE
    # in place, but with another stride
    assert _status(back, C.byref(_set(_logprob(), grad_stride=1004)), P, P, P, P, P, P, P, P, P, None) == L.E_ARG
    # nothing to do
    assert _logprob_call(_logprob(rows=0), z=None, tok=None) == L.OK


def _qk(**kw):
    return _set(L.QkCfg(8, 4, 2, 64, L.BF16, 1e6, 1e-6, 512, 256, 128), **kw)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), L.E_SHAPE), (dict(n_q_heads=0), L.E_SHAPE), (dict(n_kv_heads=3), L.E_SHAPE),
    (dict(head_dim=96), L.E_UNSUPPORTED), (dict(head_dim=0), L.E_UNSUPPORTED), (dict(dtype=5), L.E_ARG),
    (dict(rope_theta=0.0), L.E_ARG), (dict(rms_eps=-1.0), L.E_ARG), (dict(rms_eps=float("nan")), L.E_ARG),
    (dict(qkv_stride=504), L.E_SHAPE), (dict(qkv_stride=516), L.E_ARG), (dict(q_stride=248), L.E_SHAPE),
    (dict(k_stride=132), L.E_ARG),
])
def test_qk_refuses_settings(kw, code):
    c = _qk(**kw)
    assert _status(L.lib.tandem_qk_norm_rope, C.byref(c), P, P, P, P, P, P, None) == code
    assert _status(L.lib.tandem_qk_norm_rope_backward, C.byref(c), P, P, P, P, P, P, P, P, P, WS, 1 << 20,
                   None) == code


def test_qk_refuses_pointers():
    c = _qk()
    fwd, bwd = L.lib.tandem_qk_norm_rope, L.lib.tandem_qk_norm_rope_backward
    assert _status(fwd, C.byref(c), P, P, None, P, P, P, None) == L.E_ARG        # one gain
    assert _status(fwd, C.byref(c), None, P, P, P, P, P, None) == L.E_ARG
    assert _status(fwd, C.byref(c), P + 8, P, P, P, P, P, None) == L.E_ARG       # off 16 bytes
    assert _status(fwd, C.byref(c), P, P, P, P, P + 2, P, None) == L.E_ARG
    assert _status(bwd, C.byref(c), P, P, P, P, P, P, P, None, P, WS, 1 << 20, None) == L.E_ARG   # gain without gradient
    assert _status(bwd, C.byref(c), P, P, P, P, P, P, P, P, P, None, 0, None) == L.E_ARG          # no workspace
    assert _status(bwd, C.byref(c), P, P, P, P, P, P, P, P, P, WS, 16, None) == L.E_ARG
    assert _status(fwd, C.byref(_qk(rows=0)), None, None, None, None, None, None, None) == L.OK


def _attn(**kw):
    return _set(L.AttentionCfg(64, 2, 4, 2, 64, L.BF16, 0.125, 256, 128, 128, 256, 256, 256, 128, 128), **kw)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), L.E_SHAPE), (dict(n_seqs=-1), L.E_SHAPE), (dict(n_kv_heads=3), L.E_SHAPE),
    (dict(n_kv_heads=0), L.E_SHAPE), (dict(head_dim=80), L.E_UNSUPPORTED), (dict(dtype=9), L.E_ARG),
    (dict(scale=0.0), L.E_ARG), (dict(scale=-1.0), L.E_ARG), (dict(scale=float("inf")), L.E_ARG),
    (dict(q_stride=248), L.E_SHAPE), (dict(k_stride=129), L.E_ARG), (dict(out_stride=8), L.E_SHAPE),
    (dict(v_stride=1 << 25), L.E_SHAPE), (dict(rows=2**31 - 1, n_q_heads=4096, n_kv_heads=4096, q_stride=1 << 18,
                                               k_stride=1 << 18, v_stride=1 << 18, out_stride=1 << 18,
                                               dout_stride=1 << 18, dq_stride=1 << 18, dk_stride=1 << 18,
                                               dv_stride=1 << 18), L.E_SHAPE),
])
def test_attention_refuses_settings(kw, code):
    c = _attn(**kw)
    assert _status(L.lib.tandem_attention, C.byref(c), P, P, P, P, P, P, None) == code
    assert _status(L.lib.tandem_attention_backward, C.byref(c), P, P, P, P, P, P, P, P, P, P, WS, 1 << 20,
                   None) == code


def test_attention_refuses_pointers():
    c = _attn()
    fwd, bwd = L.lib.tandem_attention, L.lib.tandem_attention_backward
    for i in range(6):
        args = [P] * 6
        args[i] = None
        assert _status(fwd, C.byref(c), *args, None) == L.E_ARG
    assert _status(fwd, C.byref(c), P, P + 4, P, P, P, P, None) == L.E_ARG
    for i in range(10):
        args = [P] * 10
        args[i] = None
        assert _status(bwd, C.byref(c), *args, WS, 1 << 20, None) == L.E_ARG
    assert _status(bwd, C.byref(c), *[P] * 10, None, 0, None) == L.E_ARG
    assert _status(bwd, C.byref(c), *[P] * 10, WS, L.tandem_attention_workspace_size(c) - 1, None) == L.E_ARG
    assert _status(bwd, C.byref(_attn(dq_stride=255)), *[P] * 10, WS, 1 << 20, None) == L.E_SHAPE
    assert _status(fwd, C.byref(_attn(rows=0)), None, None, None, None, None, None, None) == L.OK
    assert _status(fwd, C.byref(_attn(n_seqs=0)), None, None, None, None, None, None, None) == L.OK


def _adamw(n=100, cfg=None, **tensor):
    t = _set(L.AdamwTensor(P, P, n, 0, 0.0, L.F32, L.F32), **tensor)
    c = _set(L.AdamwCfg(1e-3, 0.9, 0.999, 1e-8, 1.0, 1, 128), **(cfg or {}))
    return c, (L.AdamwTensor * 1)(t)


@pytest.mark.parametrize("cfg,tensor,code", [
    (dict(lr=float("nan")), {}, L.E_ARG), (dict(beta1=1.0), {}, L.E_ARG), (dict(beta2=-0.1), {}, L.E_ARG),
    (dict(eps=0.0), {}, L.E_ARG), (dict(eps=1e-60), {}, L.E_ARG), (dict(max_norm=-1.0), {}, L.E_ARG),
    (dict(max_norm=float("inf")), {}, L.E_ARG), (dict(step=0), {}, L.E_ARG), (dict(arena_elems=-1), {}, L.E_SHAPE),
    (dict(arena_elems=99), {}, L.E_CAPACITY), ({}, dict(n=-1), L.E_SHAPE), ({}, dict(param=None), L.E_ARG),
    ({}, dict(grad=None), L.E_ARG), ({}, dict(param=P + 2), L.E_ARG), ({}, dict(grad_dtype=3), L.E_ARG),
    ({}, dict(weight_decay=-1.0), L.E_ARG), ({}, dict(state_offset=2), L.E_CAPACITY),
    ({}, dict(state_offset=32), L.E_CAPACITY), ({}, dict(state_offset=-4), L.E_CAPACITY),
])
def test_adamw_refuses_settings(cfg, tensor, code):
    c, t = _adamw(cfg=cfg, **tensor)
    assert _status(L.lib.tandem_adamw, C.byref(c), t, 1, P, P, None, P, WS, 1 << 20, None) == code


def test_adamw_refuses_pointers():
    c, t = _adamw()
    f = L.lib.tandem_adamw
    need = L.tandem_adamw_workspace_size(c, t, 1)
    assert need > 0
    assert _status(f, None, t, 1, P, P, None, P, WS, need, None) == L.E_ARG
    assert _status(f, C.byref(c), None, 1, P, P, None, P, WS, need, None) == L.E_ARG
    assert _status(f, C.byref(c), t, -1, P, P, None, P, WS, need, None) == L.E_ARG
    assert _status(f, C.byref(c), t, 1, None, P, None, P, WS, need, None) == L.E_ARG
    assert _status(f, C.byref(c), t, 1, P, P + 4, None, P, WS, need, None) == L.E_ARG
    assert _status(f, C.byref(c), t, 1, P, P, None, None, WS, need, None) == L.E_ARG      # clipping without norm
    assert _status(f, C.byref(c), t, 1, P, P, None, P, WS, need - 1, None) == L.E_ARG
    c.max_norm = 0.0
    assert L.tandem_adamw_workspace_size(c, t, 1) == 0
    assert _status(f, C.byref(c), None, 0, None, None, None, None, None, 0, None) == L.OK


def test_engine_refuses_cpu_tensors_and_shapes():
    z, tok = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        E.token_logprob(z, tok)
    with pytest.raises(ValueError):
        E.token_logprob(z.half(), tok)
    with pytest.raises(ValueError):
        E.qk_norm_rope(torch.zeros(2, 100), tok, 4, 2, 1e6, 1e-6)
    with pytest.raises(ValueError):
        E.qk_norm_rope(torch.zeros(2, 256), tok, 4, 2, 1e6, 1e-6)
    q = torch.zeros(2, 4, 32)
    with pytest.raises(ValueError):
        E.attention(q, q, q, torch.tensor([0, 2], dtype=torch.int32))
    with pytest.raises(ValueError):
        E.AdamW([])
    with pytest.raises(ValueError):
        E.AdamW([torch.zeros(4)])


def test_refuses_more_than_a_launch_covers():
    """A launch has fewer than 2^32 threads; indexes of rows stay in 31 bits."""
    big = 2**31 - 1
    for c in (_logprob(rows=big, vocab=1, logits_stride=1, ref_stride=1, grad_stride=1),
              _logprob(rows=1 << 24, vocab=5000, logits_stride=5000, ref_stride=5000, grad_stride=5000),
              _logprob(rows=1 << 20, vocab=200000, logits_stride=200000, ref_stride=200000, grad_stride=200000)):
        assert _logprob_call(c) == L.E_SHAPE
        assert _status(L.lib.tandem_token_logprob_backward, C.byref(c), P, P, P, P, P, P, P, P, P, None) == L.E_SHAPE
    for c in (_qk(rows=big), _qk(rows=(1 << 30) + 1), _qk(rows=1 << 30)):
        assert _status(L.lib.tandem_qk_norm_rope, C.byref(c), P, P, P, P, P, P, None) == L.E_SHAPE
        assert _status(L.lib.tandem_qk_norm_rope_backward, C.byref(c), P, P, P, P, P, P, P, P, P, WS, 1 << 20,
                       None) == L.E_SHAPE
    for c in (_attn(rows=big), _attn(rows=1 << 30), _attn(n_seqs=big), _attn(n_seqs=1 << 23)):
        assert _status(L.lib.tandem_attention, C.byref(c), P, P, P, P, P, P, None) == L.E_SHAPE
        assert _status(L.lib.tandem_attention_backward, C.byref(c), P, P, P, P, P, P, P, P, P, P, WS, 1 << 20,
                       None) == L.E_SHAPE


@pytest.mark.parametrize("clear", [-1, 32, 1 << 20])
def test_attention_refuses_outputs_to_clear_that_there_are_not(clear):
    c = _attn(clear=clear)
    assert _status(L.lib.tandem_attention, C.byref(c), P, P, P, P, P, P, None) == L.E_ARG
    assert _status(L.lib.tandem_attention_backward, C.byref(c), P, P, P, P, P, P, P, P, P, P, WS, 1 << 20, None) == L.E_ARG


def test_attention_takes_what_its_launches_cover():
    """The limit is that of the launches a call makes: 2^25 rows of 32 heads of 32 on 8 are 2^23 workgroups
    over the queries and 2^21 over the keys, whatever other shapes would take."""
    wide = dict(n_q_heads=32, n_kv_heads=8, head_dim=32, q_stride=1024, k_stride=256, v_stride=256, out_stride=1024,
                dout_stride=1024, dq_stride=1024, dk_stride=256, dv_stride=256)
    for rows in (1 << 25, (1 << 26) - 128):
        assert L.tandem_attention_workspace_size(_attn(rows=rows, **wide)) >= 2 * rows * 32 * 4
    c = _attn(rows=1 << 26, **wide)                               # 2^24 workgroups and two more for the sequences
    assert _status(L.lib.tandem_attention_workspace_size, C.byref(c), C.byref(C.c_size_t())) == L.E_SHAPE
    assert _status(L.lib.tandem_attention, C.byref(c), P, P, P, P, P, P, None) == L.E_SHAPE
    assert L.tandem_attention_workspace_size(_attn(n_seqs=0)) >= 0 and L.tandem_attention_workspace_size(_attn(rows=0)) >= 0
