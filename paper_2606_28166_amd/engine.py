"""Device-memory plumbing around the C ABI (PyTorch allocates, the library computes).

TandemEngine uploads two models' weights as torch tensors, allocates the KV
arena, the scratch buffer and the output arenas with the sizes the library
asks for, and forwards prefill/step calls to libtandem on the current torch
stream.  Nothing here computes any part of the rollout.
"""
from __future__ import annotations

import ctypes as C
from typing import Dict, List, Optional, Sequence

import numpy as np
import torch

from . import _lib as L

LAYER_KEYS = ("attn_norm", "w_qkv", "q_norm", "k_norm", "w_o", "ffn_norm", "w_gate_up", "w_down")


def _to_device(arr: np.ndarray, dev) -> torch.Tensor:
    if arr.dtype == np.uint16:          # bf16 bit patterns
        return torch.from_numpy(np.ascontiguousarray(arr).view(np.int16)).to(dev).view(torch.bfloat16)
    return torch.from_numpy(np.ascontiguousarray(arr)).to(dev)


def model_cfg(shape) -> L.ModelCfg:
    return L.ModelCfg(shape.n_layers, shape.d_model, shape.n_q_heads, shape.n_kv_heads, shape.head_dim,
                      shape.ffn_dim, shape.vocab, float(shape.rope_theta), float(shape.rms_eps),
                      1 if shape.qk_norm else 0, L.BF16 if shape.dtype == "bf16" else L.F32)


class DeviceModel:
    """One model's weights on the device plus its tandem_model descriptor."""

    def __init__(self, shape, weights: Dict[str, np.ndarray], dev):
        self.shape = shape
        self.t = {k: _to_device(v, dev) for k, v in weights.items()}
        ptrs = []
        for i in range(shape.n_layers):
            for k in LAYER_KEYS:
                t = self.t.get(f"layers.{i}.{k}")
                ptrs.append(t.data_ptr() if t is not None else 0)
        self.layer_ptrs = (C.c_void_p * len(ptrs))(*ptrs)
        self.desc = L.Model(model_cfg(shape), self.t["embed"].data_ptr(),
                            C.cast(self.layer_ptrs, C.POINTER(C.c_void_p)),
                            self.t["final_norm"].data_ptr(), self.t["lm_head"].data_ptr())


class TandemEngine:
    """junior_shape None (or models[1] None): the senior alone, through the
    same kernels (every token the senior's; switch is ignored)."""

    def __init__(self, senior_shape, senior_w, junior_shape, junior_w, switch, sample, seed: int,
                 max_seqs: int, max_ctx: int, max_prefill_tokens: int = 4096,
                 boundary_words: Optional[np.ndarray] = None, device: str = "cuda:0",
                 models: Optional[Sequence[Optional[DeviceModel]]] = None):
        if not torch.cuda.is_available():
            raise RuntimeError("TandemEngine needs a ROCm GPU (torch.cuda.is_available() is False)")
        self.dev = torch.device(device)
        torch.cuda.set_device(self.dev)
        if models is None:
            self.sen = DeviceModel(senior_shape, senior_w, self.dev)
            self.jun = DeviceModel(junior_shape, junior_w, self.dev) if junior_shape is not None else None
        else:
            self.sen, self.jun = models
        self.sample = sample
        self.max_seqs, self.max_new = max_seqs, sample.max_new
        self.V = self.sen.shape.vocab
        self.cap = L.Capacity(max_seqs, max_ctx, max_prefill_tokens)
        kvb, scb = L.tandem_workspace_size(self.sen.desc.cfg, self.jun.desc.cfg if self.jun else None, self.cap)
        self.kv_bytes, self.scratch_bytes = kvb, scb
        self.kv = torch.empty(kvb, dtype=torch.uint8, device=self.dev)
        self.scratch = torch.empty(scb, dtype=torch.uint8, device=self.dev)
        self.tokens = torch.full((max_seqs, self.max_new), -1, dtype=torch.int32, device=self.dev)
        self.owner = torch.zeros((max_seqs, self.max_new), dtype=torch.uint8, device=self.dev)
        self.logprob = torch.zeros((max_seqs, self.max_new), dtype=torch.float32, device=self.dev)
        self.length = torch.zeros(max_seqs, dtype=torch.int32, device=self.dev)
        self.bnd = None
        if boundary_words is not None:
            self.bnd = torch.from_numpy(np.ascontiguousarray(boundary_words).view(np.int32)).to(self.dev)
        self.sw = L.SwitchCfg(int(switch.mode), float(switch.p), int(switch.cap_k),
                              self.bnd.data_ptr() if self.bnd is not None else None, int(switch.first_owner))
        self.smp = L.SampleCfg(float(sample.temperature), int(sample.eos_id), float(sample.eos_bias_senior),
                               float(sample.eos_bias_junior), int(sample.max_new), int(seed))
        self.out = L.Outputs(self.tokens.data_ptr(), self.owner.data_ptr(), self.logprob.data_ptr(),
                             self.length.data_ptr())
        self.stream = torch.cuda.current_stream(self.dev)
        self.h = L.tandem_init(self.sen.desc, self.jun.desc if self.jun else None, self.sw, self.smp, self.cap,
                               self.kv.data_ptr(), kvb, self.scratch.data_ptr(), scb, self.out,
                               self.stream.cuda_stream)
        self.n_seq = 0
        self._forced = torch.full((max_seqs,), -1, dtype=torch.int32, device=self.dev)

    # ------------------------------------------------------------- calls
    def prefill(self, prompts: Sequence[np.ndarray], G: int) -> None:
        flat = np.concatenate([np.asarray(p, dtype=np.int32) for p in prompts])
        offs = np.concatenate([[0], np.cumsum([len(p) for p in prompts])]).astype(np.int64)
        self._prompt_dev = torch.from_numpy(flat).to(self.dev)
        L.tandem_prefill(self.h, self._prompt_dev.data_ptr(), offs.tolist(), len(prompts), G)
        self.n_seq = len(prompts) * G

    def step(self, want_active: bool = False):
        return L.tandem_step(self.h, want_active)

    def step_forced(self, forced, debug: bool = True, logits: bool = False, want_active: bool = False):
        """Append forced[s] (entries < 0: own sample); returns the debug tensors."""
        f = torch.as_tensor(np.asarray(forced, dtype=np.int32)).to(self.dev)
        self._forced[: len(f)].copy_(f)
        dbg = None
        res = {}
        if debug:
            res["sampled"] = torch.full((self.max_seqs,), -1, dtype=torch.int32, device=self.dev)
            res["margin"] = torch.zeros(self.max_seqs, dtype=torch.float32, device=self.dev)
            if logits:
                res["logits_senior"] = torch.zeros((self.max_seqs, self.V), dtype=torch.float32, device=self.dev)
                res["logits_junior"] = torch.zeros((self.max_seqs, self.V), dtype=torch.float32, device=self.dev)
            dbg = L.Debug(res["sampled"].data_ptr(), res["margin"].data_ptr(),
                          res["logits_senior"].data_ptr() if logits else None,
                          res["logits_junior"].data_ptr() if logits else None)
        n = L.tandem_step_forced(self.h, self._forced.data_ptr(), dbg, want_active)
        if want_active:
            res["n_active"] = n
        return res

    def timing(self, class_mask: int) -> None:
        """Time launches of the classes in class_mask (bit k = class k); 0 switches timing off."""
        L.tandem_timing_enable(self.h, class_mask)

    def timing_read(self):
        """{class name: (device ms, launches)} since the last timing() call."""
        names = {L.K_ATTENTION: "attention", L.K_GEMM: "gemm", L.K_SAMPLE: "sample", L.K_OTHER: "other"}
        return {v: L.tandem_timing_read(self.h, k) for k, v in names.items()}

    def score(self, out=None):
        """Dual-distribution scores of the step just taken: a device float32
        tensor [max_seqs][3] of (junior cross-entropy of the appended token,
        overlap, KL(senior || junior)) by sequence id; rows of sequences that
        were done before the step keep their previous contents."""
        if out is None:
            out = torch.full((self.max_seqs, 3), float("nan"), dtype=torch.float32, device=self.dev)
        L.tandem_score_step(self.h, out.data_ptr())
        return out

    def state(self):
        owner, c, t, pos, done = L.tandem_get_state(self.h, self.n_seq)
        return dict(owner=np.array(owner), c=np.array(c), t=np.array(t), pos=np.array(pos), done=np.array(done))

    def outputs(self):
        torch.cuda.synchronize(self.dev)
        n = self.n_seq
        return dict(tokens=self.tokens[:n].cpu().numpy(), owner=self.owner[:n].cpu().numpy(),
                    logprob=self.logprob[:n].cpu().numpy(), length=self.length[:n].cpu().numpy())

    def close(self) -> None:
        if getattr(self, "h", None):
            torch.cuda.synchronize(self.dev)
            L.tandem_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def grpo_loss(rewards: torch.Tensor, owner: torch.Tensor, length: torch.Tensor, logp_old: torch.Tensor,
              logp_new: Optional[torch.Tensor], G: int, clip_eps: float = 0.2, want_grad: bool = True,
              workspace: Optional[torch.Tensor] = None, noalloc: bool = False):
    """Senior-only GRPO loss pieces (tandem_grpo_loss) of S = len(rewards)
    rollouts in groups of G, on the current torch stream.  rewards float32
    [S]; owner uint8 [S][T]; length int32 [S]; logp_old / logp_new float32
    [S][T] (logp_new None: ratio 1).  Returns device tensors: advantages [S],
    loss [1], n_masked [1] and grad [S][T] (None unless want_grad).
    noalloc: call tandem_grpo_loss_noalloc (the library's own device
    workspace; the output tensors are still allocated here)."""
    S, T = owner.shape
    dev = owner.device
    for name, t, dt, shape in (("rewards", rewards, torch.float32, (S,)), ("owner", owner, torch.uint8, (S, T)),
                               ("length", length, torch.int32, (S,)), ("logp_old", logp_old, torch.float32, (S, T)),
                               ("logp_new", logp_new, torch.float32, (S, T))):
        if t is None:
            continue
        if t.dtype != dt or tuple(t.shape) != shape or t.device != dev or not t.is_contiguous():
            raise ValueError(f"grpo_loss: {name} must be a contiguous {dt} tensor of shape {shape} on {dev}")
    if S % G != 0:
        raise ValueError(f"grpo_loss: {S} rollouts do not form groups of {G}")
    cfg = L.GrpoCfg(S // G, G, T, float(clip_eps))
    adv = torch.empty(S, dtype=torch.float32, device=dev)
    loss = torch.empty(1, dtype=torch.float32, device=dev)
    n = torch.empty(1, dtype=torch.int32, device=dev)
    grad = torch.empty((S, T), dtype=torch.float32, device=dev) if want_grad else None
    if noalloc:
        L.tandem_grpo_loss_noalloc(cfg, rewards.data_ptr(), owner.data_ptr(), length.data_ptr(), logp_old.data_ptr(),
                                   logp_new.data_ptr() if logp_new is not None else None, adv.data_ptr(),
                                   grad.data_ptr() if grad is not None else None, loss.data_ptr(), n.data_ptr(),
                                   torch.cuda.current_stream(dev).cuda_stream)
        return dict(advantages=adv, loss=loss, n_masked=n, grad=grad)
    wsb = L.tandem_grpo_workspace_size(cfg)
    if workspace is None or workspace.numel() < wsb:
        workspace = torch.empty(wsb, dtype=torch.uint8, device=dev)
    L.tandem_grpo_loss(cfg, rewards.data_ptr(), owner.data_ptr(), length.data_ptr(), logp_old.data_ptr(),
                       logp_new.data_ptr() if logp_new is not None else None, adv.data_ptr(),
                       grad.data_ptr() if grad is not None else None, loss.data_ptr(), n.data_ptr(),
                       workspace.data_ptr(), wsb, torch.cuda.current_stream(dev).cuda_stream)
    return dict(advantages=adv, loss=loss, n_masked=n, grad=grad)


# ------------------------------------------------- the senior's update
#
# Each function below runs on the current torch stream of its tensors' device and
# returns device tensors; a forward function's dict is what its backward function
# takes.  Gradients are computed by explicit backward functions, there is no autograd
# graph.

_DT = {torch.bfloat16: L.BF16, torch.float32: L.F32}


def _same(who: str, name: str, t: torch.Tensor, dtype, shape, dev) -> None:
    """A contiguous tensor of this dtype, shape and device."""
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or t.device != dev or not t.is_contiguous():
        raise ValueError(f"{who}: {name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {dev}")


def _rows(who: str, name: str, t: torch.Tensor, dtype, shape, dev) -> int:
    """The row stride of a tensor whose rows are contiguous ([rows, ...])."""
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or t.device != dev:
        raise ValueError(f"{who}: {name} must be a {dtype} tensor of shape {tuple(shape)} on {dev}")
    width = 1
    for size, stride in zip(reversed(t.shape[1:]), reversed(t.stride()[1:])):
        if size != 1 and stride != width:
            raise ValueError(f"{who}: the rows of {name} must be contiguous")
        width *= size
    # one row: any stride does
    return t.stride(0) if t.shape[0] > 1 else width


def _on(dev):
    """The current stream of dev; a CPU device is refused here, before its memory reaches a kernel."""
    if dev.type != "cuda":
        raise ValueError(f"tensors must be on a GPU, got {dev}")
    return torch.cuda.current_stream(dev).cuda_stream


def _ptr(t: Optional[torch.Tensor]):
    return t.data_ptr() if t is not None else None


def _workspace(t: Optional[torch.Tensor], need: int, dev) -> Optional[torch.Tensor]:
    """t if it is large enough, a new one otherwise; None when nothing is needed."""
    if need == 0:
        return None
    if t is None or t.numel() * t.element_size() < need or t.device != dev:
        return torch.empty(need, dtype=torch.uint8, device=dev)
    return t


def _logprob_cfg(who, logits, tokens, ref, temperature, eos_id, eos_bias, eos_bias_ref):
    if logits.dim() != 2 or logits.dtype not in _DT:
        raise ValueError(f"{who}: logits must be a bfloat16 or float32 tensor [rows][vocab]")
    R, V = logits.shape
    _on(logits.device)
    ld = _rows(who, "logits", logits, logits.dtype, (R, V), logits.device)
    ldr = _rows(who, "ref", ref, logits.dtype, (R, V), logits.device) if ref is not None else V
    _same(who, "tokens", tokens, torch.int32, (R,), logits.device)
    return L.LogprobCfg(R, V, _DT[logits.dtype], int(eos_id), ld, ldr, V, float(temperature), float(eos_bias),
                        float(eos_bias_ref))


def token_logprob(logits: torch.Tensor, tokens: torch.Tensor, ref: Optional[torch.Tensor] = None,
                  temperature: float = 1.0, eos_id: int = -1, eos_bias: float = 0.0, eos_bias_ref: float = 0.0,
                  workspace: Optional[torch.Tensor] = None):
    """Log-probs of tokens int32 [R] under logits [R][V] (bfloat16 or float32,
    rows contiguous), and with ref (a frozen model's logits) the KL divergence
    from it (tandem_token_logprob).  The scores are those the rollout samples
    from, (z + eos_bias e_eos) / temperature.  Tokens outside the vocabulary
    (-1: padding) leave their row out.  Returns logp, lse, kl, lse_diff, each
    float32 [R] (the last two None without ref)."""
    cfg = _logprob_cfg("token_logprob", logits, tokens, ref, temperature, eos_id, eos_bias, eos_bias_ref)
    dev, R = logits.device, logits.shape[0]
    need = L.tandem_logprob_workspace_size(cfg)
    workspace = _workspace(workspace, need, dev)
    out = torch.empty((4 if ref is not None else 2, R), dtype=torch.float32, device=dev)
    kl, diff = (out[2], out[3]) if ref is not None else (None, None)
    with torch.cuda.device(dev):
        L.tandem_token_logprob(cfg, logits.data_ptr(), _ptr(ref), tokens.data_ptr(), out[0].data_ptr(),
                               out[1].data_ptr(), _ptr(kl), _ptr(diff), _ptr(workspace), need, _on(dev))
    return dict(logp=out[0], lse=out[1], kl=kl, lse_diff=diff)


def token_logprob_backward(logits: torch.Tensor, tokens: torch.Tensor, fwd, g_logp: torch.Tensor,
                           g_kl: Optional[torch.Tensor] = None, ref: Optional[torch.Tensor] = None,
                           temperature: float = 1.0, eos_id: int = -1, eos_bias: float = 0.0,
                           eos_bias_ref: float = 0.0, out: Optional[torch.Tensor] = None):
    """Gradient with respect to logits of sum(g_logp logp + g_kl kl), in the
    logits' dtype; fwd is what token_logprob returned for the same arguments.
    out may be logits itself: the gradient then takes its place."""
    who = "token_logprob_backward"
    cfg = _logprob_cfg(who, logits, tokens, ref, temperature, eos_id, eos_bias, eos_bias_ref)
    dev, (R, V) = logits.device, logits.shape
    if g_kl is not None and (ref is None or fwd["kl"] is None):
        raise ValueError(f"{who}: g_kl needs ref, in the forward pass too")
    for name, t in (("g_logp", g_logp), ("g_kl", g_kl), ("fwd['lse']", fwd["lse"]),
                    ("fwd['kl']", fwd["kl"] if g_kl is not None else None),
                    ("fwd['lse_diff']", fwd["lse_diff"] if g_kl is not None else None)):
        if t is not None:
            _same(who, name, t, torch.float32, (R,), dev)
    if out is None:
        out = torch.empty((R, V), dtype=logits.dtype, device=dev)
    cfg.grad_stride = _rows(who, "out", out, logits.dtype, (R, V), dev)
    kl, diff = (fwd["kl"], fwd["lse_diff"]) if g_kl is not None else (None, None)
    with torch.cuda.device(dev):
        L.tandem_token_logprob_backward(cfg, logits.data_ptr(), _ptr(ref if g_kl is not None else None),
                                        tokens.data_ptr(), fwd["lse"].data_ptr(), _ptr(kl), _ptr(diff),
                                        g_logp.data_ptr(), _ptr(g_kl), out.data_ptr(), _on(dev))
    return out


def _qk_cfg(who, qkv, positions, n_q, n_kv, theta, eps, q_gain, k_gain):
    if qkv.dim() != 2 or qkv.dtype not in _DT or qkv.shape[1] % (n_q + 2 * n_kv) != 0:
        raise ValueError(f"{who}: qkv must be a bfloat16 or float32 tensor [rows][(n_q + 2 n_kv) * head_dim]")
    N, hd = qkv.shape[0], qkv.shape[1] // (n_q + 2 * n_kv)
    _on(qkv.device)
    ld = _rows(who, "qkv", qkv, qkv.dtype, qkv.shape, qkv.device)
    _same(who, "positions", positions, torch.int32, (N,), qkv.device)
    for name, t in (("q_gain", q_gain), ("k_gain", k_gain)):
        if t is not None:
            _same(who, name, t, torch.float32, (hd,), qkv.device)
    return L.QkCfg(N, n_q, n_kv, hd, _DT[qkv.dtype], float(theta), float(eps), ld, n_q * hd, n_kv * hd)


def qk_norm_rope(qkv: torch.Tensor, positions: torch.Tensor, n_q: int, n_kv: int, theta: float, eps: float,
                 q_gain: Optional[torch.Tensor] = None, k_gain: Optional[torch.Tensor] = None):
    """Per-head RMSNorm (with gains) and rotary embedding of the query and key
    heads of a packed QKV projection [N][(n_q + 2 n_kv) * head_dim] at
    positions int32 [N] (tandem_qk_norm_rope).  Returns q [N][n_q][head_dim],
    k [N][n_kv][head_dim] and v, a view of the value columns."""
    who = "qk_norm_rope"
    cfg = _qk_cfg(who, qkv, positions, n_q, n_kv, theta, eps, q_gain, k_gain)
    N, hd, dev = cfg.rows, cfg.head_dim, qkv.device
    q = torch.empty((N, n_q, hd), dtype=qkv.dtype, device=dev)
    k = torch.empty((N, n_kv, hd), dtype=qkv.dtype, device=dev)
    with torch.cuda.device(dev):
        L.tandem_qk_norm_rope(cfg, qkv.data_ptr(), _ptr(q_gain), _ptr(k_gain), positions.data_ptr(), q.data_ptr(),
                              k.data_ptr(), _on(dev))
    return dict(q=q, k=k, v=qkv[:, (n_q + n_kv) * hd:].unflatten(1, (n_kv, hd)))


def qk_norm_rope_backward(qkv: torch.Tensor, positions: torch.Tensor, dq: torch.Tensor, dk: torch.Tensor,
                          theta: float, eps: float, q_gain: Optional[torch.Tensor] = None,
                          k_gain: Optional[torch.Tensor] = None, dqkv: Optional[torch.Tensor] = None,
                          workspace: Optional[torch.Tensor] = None):
    """Gradients of qk_norm_rope's inputs from those of its outputs, dq
    [N][n_q][head_dim] and dk [N][n_kv][head_dim].  dqkv (same layout as qkv)
    receives the query and key columns; its value columns are left as they are
    (attention_backward writes them through a view), or are zero in a tensor
    allocated here.  Returns dqkv, dq_gain, dk_gain (None without gains)."""
    who = "qk_norm_rope_backward"
    if dq.dim() != 3 or dk.dim() != 3:
        raise ValueError(f"{who}: dq and dk must be [rows][heads][head_dim]")
    n_q, n_kv = dq.shape[1], dk.shape[1]
    cfg = _qk_cfg(who, qkv, positions, n_q, n_kv, theta, eps, q_gain, k_gain)
    N, hd, dev = cfg.rows, cfg.head_dim, qkv.device
    cfg.q_stride = _rows(who, "dq", dq, qkv.dtype, (N, n_q, hd), dev)
    cfg.k_stride = _rows(who, "dk", dk, qkv.dtype, (N, n_kv, hd), dev)
    if dqkv is None:
        dqkv = torch.empty_strided(qkv.shape, (cfg.qkv_stride, 1), dtype=qkv.dtype, device=dev)
        dqkv[:, (n_q + n_kv) * hd:].zero_()
    elif _rows(who, "dqkv", dqkv, qkv.dtype, qkv.shape, dev) != cfg.qkv_stride:
        raise ValueError(f"{who}: dqkv must have the strides of qkv")
    if (q_gain is None) != (k_gain is None):
        raise ValueError(f"{who}: q_gain and k_gain go together")
    gain = torch.empty((2, hd), dtype=torch.float32, device=dev) if q_gain is not None else None
    need = L.tandem_qk_workspace_size(cfg) if q_gain is not None else 0
    workspace = _workspace(workspace, need, dev)
    dgq, dgk = (gain[0], gain[1]) if gain is not None else (None, None)
    with torch.cuda.device(dev):
        L.tandem_qk_norm_rope_backward(cfg, qkv.data_ptr(), _ptr(q_gain), _ptr(k_gain), positions.data_ptr(),
                                       dq.data_ptr(), dk.data_ptr(), dqkv.data_ptr(), _ptr(dgq), _ptr(dgk),
                                       _ptr(workspace), need, _on(dev))
    return dict(dqkv=dqkv, dq_gain=dgq, dk_gain=dgk)


def _attention_cfg(who, q, k, v, offsets, scale):
    if q.dim() != 3 or k.dim() != 3 or q.dtype not in _DT:
        raise ValueError(f"{who}: q and k must be bfloat16 or float32 tensors [rows][heads][head_dim]")
    (N, nq, hd), nkv, dev = q.shape, k.shape[1], q.device
    _on(dev)
    if offsets.dim() != 1 or offsets.numel() < 1:
        raise ValueError(f"{who}: offsets must hold at least one entry")
    _same(who, "offsets", offsets, torch.int32, offsets.shape, dev)
    return L.AttentionCfg(N, offsets.numel() - 1, nq, nkv, hd, _DT[q.dtype],
                          float(scale) if scale is not None else hd ** -0.5,
                          _rows(who, "q", q, q.dtype, q.shape, dev), _rows(who, "k", k, q.dtype, (N, nkv, hd), dev),
                          _rows(who, "v", v, q.dtype, (N, nkv, hd), dev), nq * hd, nq * hd, nq * hd, nkv * hd,
                          nkv * hd)


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, offsets: torch.Tensor,
              scale: Optional[float] = None, out: Optional[torch.Tensor] = None):
    """Causal grouped-query attention over packed sequences (tandem_attention):
    rows offsets[s] .. offsets[s + 1] - 1 (int32 on the device) of q
    [N][n_q][head_dim], k and v [N][n_kv][head_dim] are sequence s.  scale:
    1 / sqrt(head_dim) by default.  Returns out [N][n_q][head_dim] and lse
    float32 [n_q][N]; rows that belong to no sequence are not written."""
    who = "attention"
    cfg = _attention_cfg(who, q, k, v, offsets, scale)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    cfg.out_stride = _rows(who, "out", out, q.dtype, q.shape, q.device)
    lse = torch.empty((cfg.n_q_heads, cfg.rows), dtype=torch.float32, device=q.device)
    with torch.cuda.device(q.device):
        L.tandem_attention(cfg, q.data_ptr(), k.data_ptr(), v.data_ptr(), offsets.data_ptr(), out.data_ptr(),
                           lse.data_ptr(), _on(q.device))
    return dict(out=out, lse=lse)


def attention_backward(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                       lse: torch.Tensor, offsets: torch.Tensor, scale: Optional[float] = None,
                       dq: Optional[torch.Tensor] = None, dk: Optional[torch.Tensor] = None,
                       dv: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Gradients of attention's q, k and v for the gradient dout of its out
    (tandem_attention_backward).  dq, dk, dv may be given, also as views (the
    value columns of qk_norm_rope_backward's dqkv).  Returns dq, dk, dv."""
    who = "attention_backward"
    cfg = _attention_cfg(who, q, k, v, offsets, scale)
    dev = q.device
    cfg.out_stride = _rows(who, "out", out, q.dtype, q.shape, dev)
    cfg.dout_stride = _rows(who, "dout", dout, q.dtype, q.shape, dev)
    _same(who, "lse", lse, torch.float32, (cfg.n_q_heads, cfg.rows), dev)
    dq = torch.empty(q.shape, dtype=q.dtype, device=dev) if dq is None else dq
    dk = torch.empty(k.shape, dtype=q.dtype, device=dev) if dk is None else dk
    dv = torch.empty(k.shape, dtype=q.dtype, device=dev) if dv is None else dv
    cfg.dq_stride = _rows(who, "dq", dq, q.dtype, q.shape, dev)
    cfg.dk_stride = _rows(who, "dk", dk, q.dtype, k.shape, dev)
    cfg.dv_stride = _rows(who, "dv", dv, q.dtype, k.shape, dev)
    need = L.tandem_attention_workspace_size(cfg)
    workspace = _workspace(workspace, need, dev)
    with torch.cuda.device(dev):
        L.tandem_attention_backward(cfg, dout.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                                    lse.data_ptr(), offsets.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
                                    _ptr(workspace), need, _on(dev))
    return dict(dq=dq, dk=dk, dv=dv)


class AdamW:
    """AdamW over a list of weight tensors (tandem_adamw): float32 states in
    two arenas, and with master a float32 copy of every weight in a third, which
    is what the update is applied to (a bfloat16 weight is its rounding; at
    learning rates of 1e-6 it would otherwise not move).

    params: contiguous bfloat16 or float32 tensors on one GPU, updated in place.
    weight_decay: one number, or one per tensor.  max_norm > 0 clips by the
    global norm of the gradients.  master None: where any weight is bfloat16.
    state: what state() returned, to resume (its tensors are used, not copied)."""

    ALIGN = 64      # a tensor's state begins at a multiple of this many elements

    def __init__(self, params: Sequence[torch.Tensor], betas=(0.9, 0.999), eps: float = 1e-8, weight_decay=0.0,
                 max_norm: float = 0.0, master: Optional[bool] = None, state: Optional[dict] = None):
        self.params = list(params)
        if not self.params:
            raise ValueError("AdamW: no tensors")
        self.dev = self.params[0].device
        _on(self.dev)
        for p in self.params:
            if p.dtype not in _DT or p.device != self.dev or not p.is_contiguous():
                raise ValueError(f"AdamW: weights must be contiguous bfloat16 or float32 tensors on {self.dev}")
        n = len(self.params)
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * n
        if len(decay) != n:
            raise ValueError(f"AdamW: {len(decay)} weight decays for {n} tensors")
        self.betas, self.eps, self.max_norm = betas, float(eps), float(max_norm)
        self.offsets, total = [], 0
        for p in self.params:
            self.offsets.append(total)
            total += -(-p.numel() // self.ALIGN) * self.ALIGN
        self.elems = total
        if state is not None:
            self.steps, self.m, self.v, self.master = int(state["step"]), state["m"], state["v"], state["master"]
            for name in ("m", "v", "master"):
                if state[name] is not None:
                    _same("AdamW", name, state[name], torch.float32, (total,), self.dev)
        else:
            if master is None:
                master = any(p.dtype == torch.bfloat16 for p in self.params)
            self.steps = 0
            self.m = torch.zeros(total, dtype=torch.float32, device=self.dev)
            self.v = torch.zeros(total, dtype=torch.float32, device=self.dev)
            self.master = torch.zeros(total, dtype=torch.float32, device=self.dev) if master else None
            if master:
                for p, o in zip(self.params, self.offsets):
                    self.master[o:o + p.numel()].copy_(p.reshape(-1))
        self._table = (L.AdamwTensor * n)(*[
            L.AdamwTensor(p.data_ptr(), None, p.numel(), o, float(w), _DT[p.dtype], _DT[p.dtype])
            for p, o, w in zip(self.params, self.offsets, decay)])

    def state(self) -> dict:
        """The optimizer's state, to be saved and given to another AdamW."""
        return dict(step=self.steps, m=self.m, v=self.v, master=self.master)

    def step(self, grads: Sequence[torch.Tensor], lr: float) -> Optional[torch.Tensor]:
        """One step with grads (one per weight, of its shape, bfloat16 or
        float32).  Returns the gradients' norm before clipping, a float32 scalar on
        the device (None without clipping).  A step captured into a graph
        repeats that step's number when it is replayed."""
        if len(grads) != len(self.params):
            raise ValueError(f"AdamW: {len(grads)} gradients for {len(self.params)} tensors")
        for d, g, p in zip(self._table, grads, self.params):
            if g.shape != p.shape or g.dtype not in _DT or g.device != self.dev or not g.is_contiguous():
                raise ValueError(f"AdamW: a gradient must be a contiguous bfloat16 or float32 tensor of shape "
                                 f"{tuple(p.shape)} on {self.dev}")
            # a weight whose storage was replaced since the last step is followed
            d.param, d.grad, d.grad_dtype = p.data_ptr(), g.data_ptr(), _DT[g.dtype]
        cfg = L.AdamwCfg(float(lr), float(self.betas[0]), float(self.betas[1]), self.eps, self.max_norm,
                         self.steps + 1, self.elems)
        need = L.tandem_adamw_workspace_size(cfg, self._table, len(self.params))
        norm = torch.empty((), dtype=torch.float32, device=self.dev) if self.max_norm > 0 else None
        workspace = _workspace(None, need, self.dev)
        with torch.cuda.device(self.dev):
            L.tandem_adamw(cfg, self._table, len(self.params), self.m.data_ptr(), self.v.data_ptr(),
                           _ptr(self.master), _ptr(norm), _ptr(workspace), need, _on(self.dev))
        self.steps += 1
        return norm
