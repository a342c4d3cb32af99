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
# graph.  A small call is bound by the host, so the checks are few comparisons per tensor
# and outputs of one kind share an allocation.

_DT = {torch.bfloat16: L.BF16, torch.float32: L.F32}
_lib = L.lib


_MOST = 0x7FFFFFFF      # the library counts rows in 32 bits


def _count(who: str, n: int) -> None:
    if n > _MOST:
        raise ValueError(f"{who}: {n} rows are too many")


def _same(who: str, name: str, t: torch.Tensor, dtype, shape, dev) -> None:
    """A contiguous tensor of this dtype, shape and device."""
    if t.dtype is not dtype or t.shape != shape or t.device != dev or not t.is_contiguous():
        raise ValueError(f"{who}: {name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {dev}")


def _rows(who: str, name: str, t: torch.Tensor, dtype, shape, dev) -> int:
    """The row stride of a tensor whose rows are contiguous ([rows, ...])."""
    if t.dtype is not dtype or t.shape != shape or t.device != dev:
        raise ValueError(f"{who}: {name} must be a {dtype} tensor of shape {tuple(shape)} on {dev}")
    stride = t.stride()
    width = 1
    for i in range(len(stride) - 1, 0, -1):
        size = shape[i]
        if stride[i] != width and size != 1:
            raise ValueError(f"{who}: the rows of {name} must be contiguous")
        width *= size
    # one row: any stride does
    return stride[0] if shape[0] > 1 else width


def _gpu(dev) -> None:
    """Refuses a CPU device before its memory reaches a kernel."""
    if dev.type != "cuda":
        raise ValueError(f"tensors must be on a GPU, got {dev}")


def _run(dev, fn, *args) -> None:
    """fn(*args, the current stream of dev), with dev current."""
    index = dev.index
    if torch._C._cuda_getDevice() != index:
        with torch.cuda.device(dev):
            L.check(fn(*args, torch._C._cuda_getCurrentRawStream(index)))
        return
    status = fn(*args, torch._C._cuda_getCurrentRawStream(index))
    if status != L.OK:
        L.check(status)


def _written(*tensors: Optional[torch.Tensor]) -> None:
    """Tells autograd that these tensors of the caller's (None: not given) hold other values
    now: a graph that saved one of them refuses its backward pass instead of using the new values."""
    for t in tensors:
        if t is not None:
            torch._C._increment_version([t])


def _need(fn, *args) -> int:
    """The workspace that a *_workspace_size call asks for."""
    n = C.c_size_t()
    status = fn(*args, n)
    if status != L.OK:
        L.check(status)
    return n.value


def _ptr(t: Optional[torch.Tensor]):
    return t.data_ptr() if t is not None else None


def _workspace(t: Optional[torch.Tensor], need: int, dev) -> Optional[torch.Tensor]:
    """t if it is large enough and contiguous, a new one otherwise; None when nothing is needed."""
    if need == 0:
        return None
    if t is None or t.numel() * t.element_size() < need or t.device != dev or not t.is_contiguous():
        return torch.empty(need, dtype=torch.uint8, device=dev)
    return t


def _logprob_cfg(who, logits, tokens, ref, temperature, eos_id, eos_bias, eos_bias_ref):
    dt = logits.dtype
    if logits.dim() != 2 or dt not in _DT:
        raise ValueError(f"{who}: logits must be a bfloat16 or float32 tensor [rows][vocab]")
    shape, dev = logits.shape, logits.device
    R, V = shape
    _count(who, max(R, V))
    _gpu(dev)
    ld = _rows(who, "logits", logits, dt, shape, dev)
    ldr = _rows(who, "ref", ref, dt, shape, dev) if ref is not None else V
    _same(who, "tokens", tokens, torch.int32, (R,), dev)
    return L.LogprobCfg(R, V, _DT[dt], eos_id, ld, ldr, V, temperature, eos_bias, eos_bias_ref), dev


def token_logprob(logits: torch.Tensor, tokens: torch.Tensor, ref: Optional[torch.Tensor] = None,
                  temperature: float = 1.0, eos_id: int = -1, eos_bias: float = 0.0, eos_bias_ref: float = 0.0,
                  workspace: Optional[torch.Tensor] = None):
    """Log-probs of tokens int32 [R] under logits [R][V] (bfloat16 or float32,
    rows contiguous), and with ref (a frozen model's logits) the KL divergence
    from it (tandem_token_logprob).  The scores are those the rollout samples
    from, (z + eos_bias e_eos) / temperature.  Tokens outside the vocabulary
    (-1: padding) leave their row out.  Returns logp, lse, kl, lse_diff, each
    float32 [R] (the last two None without ref)."""
    cfg, dev = _logprob_cfg("token_logprob", logits, tokens, ref, temperature, eos_id, eos_bias, eos_bias_ref)
    R = cfg.rows
    need = _need(_lib.tandem_logprob_workspace_size, cfg)
    workspace = _workspace(workspace, need, dev)
    out = torch.empty((4 if ref is not None else 2, R), dtype=torch.float32, device=dev)
    p = out.data_ptr()
    if ref is not None:
        _run(dev, _lib.tandem_token_logprob, cfg, logits.data_ptr(), ref.data_ptr(), tokens.data_ptr(), p, p + 4 * R,
             p + 8 * R, p + 12 * R, _ptr(workspace), need)
        logp, lse, kl, diff = out.unbind(0)
        return dict(logp=logp, lse=lse, kl=kl, lse_diff=diff)
    _run(dev, _lib.tandem_token_logprob, cfg, logits.data_ptr(), None, tokens.data_ptr(), p, p + 4 * R, None, None,
         _ptr(workspace), need)
    logp, lse = out.unbind(0)
    return dict(logp=logp, lse=lse, kl=None, lse_diff=None)


def token_logprob_backward(logits: torch.Tensor, tokens: torch.Tensor, fwd, g_logp: torch.Tensor,
                           g_kl: Optional[torch.Tensor] = None, ref: Optional[torch.Tensor] = None,
                           temperature: float = 1.0, eos_id: int = -1, eos_bias: float = 0.0,
                           eos_bias_ref: float = 0.0, out: Optional[torch.Tensor] = None):
    """Gradient with respect to logits of sum(g_logp logp + g_kl kl), in the
    logits' dtype; fwd is what token_logprob returned for the same arguments.
    out may be logits itself: the gradient then takes its place."""
    who = "token_logprob_backward"
    cfg, dev = _logprob_cfg(who, logits, tokens, ref, temperature, eos_id, eos_bias, eos_bias_ref)
    row = (cfg.rows,)
    lse, kl, diff = fwd["lse"], None, None
    _same(who, "g_logp", g_logp, torch.float32, row, dev)
    _same(who, "fwd['lse']", lse, torch.float32, row, dev)
    if g_kl is not None:
        kl, diff = fwd["kl"], fwd["lse_diff"]
        if ref is None or kl is None:
            raise ValueError(f"{who}: g_kl needs ref, in the forward pass too")
        _same(who, "g_kl", g_kl, torch.float32, row, dev)
        _same(who, "fwd['kl']", kl, torch.float32, row, dev)
        _same(who, "fwd['lse_diff']", diff, torch.float32, row, dev)
    else:
        ref = None
    given = out
    if out is None:
        out = torch.empty(logits.shape, dtype=logits.dtype, device=dev)
    else:
        cfg.grad_stride = _rows(who, "out", out, logits.dtype, logits.shape, dev)
    _run(dev, _lib.tandem_token_logprob_backward, cfg, logits.data_ptr(), _ptr(ref), tokens.data_ptr(),
         lse.data_ptr(), _ptr(kl), _ptr(diff), g_logp.data_ptr(), _ptr(g_kl), out.data_ptr())
    _written(given)
    return out


def _qk_cfg(who, qkv, positions, n_q, n_kv, theta, eps, q_gain, k_gain):
    dt, dev = qkv.dtype, qkv.device
    if qkv.dim() != 2 or dt not in _DT or n_q < 1 or n_kv < 1 or qkv.shape[1] % (n_q + 2 * n_kv) != 0:
        raise ValueError(f"{who}: qkv must be a bfloat16 or float32 tensor [rows][(n_q + 2 n_kv) * head_dim]")
    N, cols = qkv.shape
    _count(who, N)
    hd = cols // (n_q + 2 * n_kv)
    _gpu(dev)
    ld = _rows(who, "qkv", qkv, dt, qkv.shape, dev)
    _same(who, "positions", positions, torch.int32, (N,), dev)
    if (q_gain is None) != (k_gain is None):
        raise ValueError(f"{who}: q_gain and k_gain go together")
    if q_gain is not None:
        _same(who, "q_gain", q_gain, torch.float32, (hd,), dev)
        _same(who, "k_gain", k_gain, torch.float32, (hd,), dev)
    return L.QkCfg(N, n_q, n_kv, hd, _DT[dt], theta, eps, ld, n_q * hd, n_kv * hd), dev


def qk_norm_rope(qkv: torch.Tensor, positions: torch.Tensor, n_q: int, n_kv: int, theta: float, eps: float,
                 q_gain: Optional[torch.Tensor] = None, k_gain: Optional[torch.Tensor] = None):
    """Per-head RMSNorm (with gains) and rotary embedding of the query and key
    heads of a packed QKV projection [N][(n_q + 2 n_kv) * head_dim] at
    positions int32 [N] (tandem_qk_norm_rope).  Returns q [N][n_q][head_dim],
    k [N][n_kv][head_dim] and v, a view of the value columns."""
    cfg, dev = _qk_cfg("qk_norm_rope", qkv, positions, n_q, n_kv, theta, eps, q_gain, k_gain)
    N, hd = cfg.rows, cfg.head_dim
    q = torch.empty((N, n_q, hd), dtype=qkv.dtype, device=dev)
    k = torch.empty((N, n_kv, hd), dtype=qkv.dtype, device=dev)
    _run(dev, _lib.tandem_qk_norm_rope, cfg, qkv.data_ptr(), _ptr(q_gain), _ptr(k_gain), positions.data_ptr(),
         q.data_ptr(), k.data_ptr())
    v = qkv.as_strided((N, n_kv, hd), (qkv.stride(0), hd, 1), qkv.storage_offset() + (n_q + n_kv) * hd)
    return dict(q=q, k=k, v=v)


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
    cfg, dev = _qk_cfg(who, qkv, positions, n_q, n_kv, theta, eps, q_gain, k_gain)
    N, hd, dt = cfg.rows, cfg.head_dim, qkv.dtype
    cfg.q_stride = _rows(who, "dq", dq, dt, (N, n_q, hd), dev)
    cfg.k_stride = _rows(who, "dk", dk, dt, (N, n_kv, hd), dev)
    given = dqkv
    if dqkv is None:
        dqkv = torch.empty_strided(qkv.shape, (cfg.qkv_stride, 1), dtype=dt, device=dev)
        dqkv[:, (n_q + n_kv) * hd:].zero_()
    elif _rows(who, "dqkv", dqkv, dt, qkv.shape, dev) != cfg.qkv_stride:
        raise ValueError(f"{who}: dqkv must have the strides of qkv")
    if q_gain is None:
        _run(dev, _lib.tandem_qk_norm_rope_backward, cfg, qkv.data_ptr(), None, None, positions.data_ptr(),
             dq.data_ptr(), dk.data_ptr(), dqkv.data_ptr(), None, None, None, 0)
        _written(given)
        return dict(dqkv=dqkv, dq_gain=None, dk_gain=None)
    gain = torch.empty((2, hd), dtype=torch.float32, device=dev)
    p = gain.data_ptr()
    need = _need(_lib.tandem_qk_workspace_size, cfg)
    workspace = _workspace(workspace, need, dev)
    _run(dev, _lib.tandem_qk_norm_rope_backward, cfg, qkv.data_ptr(), q_gain.data_ptr(), k_gain.data_ptr(),
         positions.data_ptr(), dq.data_ptr(), dk.data_ptr(), dqkv.data_ptr(), p, p + 4 * hd, workspace.data_ptr(), need)
    _written(given)
    dgq, dgk = gain.unbind(0)
    return dict(dqkv=dqkv, dq_gain=dgq, dk_gain=dgk)


def _attention_cfg(who, q, k, v, offsets, scale):
    dt, dev = q.dtype, q.device
    if q.dim() != 3 or k.dim() != 3 or dt not in _DT:
        raise ValueError(f"{who}: q and k must be bfloat16 or float32 tensors [rows][heads][head_dim]")
    _gpu(dev)
    N, nq, hd = q.shape
    nkv = k.shape[1]
    _count(who, max(N, offsets.numel()))
    heads = (N, nkv, hd)
    if offsets.dim() != 1 or offsets.numel() < 1:
        raise ValueError(f"{who}: offsets must hold at least one entry")
    _same(who, "offsets", offsets, torch.int32, offsets.shape, dev)
    qs, ks = nq * hd, nkv * hd
    return L.AttentionCfg(N, offsets.numel() - 1, nq, nkv, hd, _DT[dt],
                          scale if scale is not None else hd ** -0.5 if hd > 0 else 0.0,
                          _rows(who, "q", q, dt, q.shape, dev), _rows(who, "k", k, dt, heads, dev),
                          _rows(who, "v", v, dt, heads, dev), qs, qs, qs, ks, ks), dt, dev


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, offsets: torch.Tensor,
              scale: Optional[float] = None, out: Optional[torch.Tensor] = None):
    """Causal grouped-query attention over packed sequences (tandem_attention):
    rows offsets[s] .. offsets[s + 1] - 1 (int32 on the device) of q
    [N][n_q][head_dim], k and v [N][n_kv][head_dim] are sequence s.  scale:
    1 / sqrt(head_dim) by default.  Returns out [N][n_q][head_dim] and lse
    float32 [n_q][N]; rows that belong to no sequence are 0 in them, but left as
    they are in an out that is given."""
    cfg, dt, dev = _attention_cfg("attention", q, k, v, offsets, scale)
    new = torch.empty if cfg.n_seqs > 0 else torch.zeros          # the library clears beside sequences only
    cfg.clear = L.CLEAR_LSE
    given = out
    if out is None:
        out = new(q.shape, dtype=dt, device=dev)
        cfg.clear |= L.CLEAR_OUT
    else:
        cfg.out_stride = _rows("attention", "out", out, dt, q.shape, dev)
    lse = new((cfg.n_q_heads, cfg.rows), dtype=torch.float32, device=dev)
    _run(dev, _lib.tandem_attention, cfg, q.data_ptr(), k.data_ptr(), v.data_ptr(), offsets.data_ptr(), out.data_ptr(),
         lse.data_ptr())
    _written(given)
    return dict(out=out, lse=lse)


def attention_backward(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                       lse: torch.Tensor, offsets: torch.Tensor, scale: Optional[float] = None,
                       dq: Optional[torch.Tensor] = None, dk: Optional[torch.Tensor] = None,
                       dv: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Gradients of attention's q, k and v for the gradient dout of its out
    (tandem_attention_backward).  dq, dk, dv may be given, also as views (the
    value columns of qk_norm_rope_backward's dqkv).  Returns dq, dk, dv; rows that
    belong to no sequence are 0 in those allocated here, and left as they are in given
    ones."""
    who = "attention_backward"
    cfg, dt, dev = _attention_cfg(who, q, k, v, offsets, scale)
    qs, ks = q.shape, k.shape
    cfg.out_stride = _rows(who, "out", out, dt, qs, dev)
    cfg.dout_stride = _rows(who, "dout", dout, dt, qs, dev)
    _same(who, "lse", lse, torch.float32, (cfg.n_q_heads, cfg.rows), dev)
    new = torch.empty if cfg.n_seqs > 0 else torch.zeros
    given = (dq, dk, dv)
    if dq is None:
        dq = new(qs, dtype=dt, device=dev)
        cfg.clear |= L.CLEAR_DQ
    else:
        cfg.dq_stride = _rows(who, "dq", dq, dt, qs, dev)
    if dk is None:
        dk = new(ks, dtype=dt, device=dev)
        cfg.clear |= L.CLEAR_DK
    else:
        cfg.dk_stride = _rows(who, "dk", dk, dt, ks, dev)
    if dv is None:
        dv = new(ks, dtype=dt, device=dev)
        cfg.clear |= L.CLEAR_DV
    else:
        cfg.dv_stride = _rows(who, "dv", dv, dt, ks, dev)
    need = _need(_lib.tandem_attention_workspace_size, cfg)
    workspace = _workspace(workspace, need, dev)
    _run(dev, _lib.tandem_attention_backward, cfg, dout.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(),
         out.data_ptr(), lse.data_ptr(), offsets.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
         _ptr(workspace), need)
    _written(*given)
    return dict(dq=dq, dk=dk, dv=dv)


class AdamW:
    """AdamW over a list of weight tensors (tandem_adamw): float32 states in
    two arenas, and with master a float32 copy of every weight in a third, which
    is what the update is applied to (a bfloat16 weight is its rounding; at
    learning rates of 1e-6 it would otherwise not move).

    params: contiguous bfloat16 or float32 tensors on one GPU that share no
    memory, updated in place (as autograd knows: a graph that saved a weight before a
    step does not run backward after it).
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
        _gpu(self.dev)
        self._shapes = [p.shape for p in self.params]
        self._types = [p.dtype for p in self.params]
        self._places = self._check_params()
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
                if state[name] is None and name != "master":
                    raise ValueError(f"AdamW: the state has no {name}")
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
                    self.master[o:o + p.numel()].copy_(p.detach().reshape(-1))
        # the tensors' table as the library reads it, and a view of it by columns
        self._table = (L.AdamwTensor * n)(*[
            L.AdamwTensor(p.data_ptr(), None, p.numel(), o, float(w), _DT[p.dtype], _DT[p.dtype])
            for p, o, w in zip(self.params, self.offsets, decay)])
        self._columns = np.frombuffer(self._table, dtype=np.dtype(
            [(name, {C.c_void_p: np.uint64, C.c_int64: np.int64, C.c_double: np.float64, C.c_int32: np.int32}[t])
             for name, t in L.AdamwTensor._fields_]))
        self._grad_types = self._types
        self._workspace_bytes = None

    def _check_params(self) -> list:
        """The weights' addresses; refuses weights that a step cannot write."""
        spans = []
        for p, t, s in zip(self.params, self._types, self._shapes):
            if p.dtype not in _DT or p.device != self.dev or not p.is_contiguous():
                raise ValueError(f"AdamW: weights must be contiguous bfloat16 or float32 tensors on {self.dev}")
            if p.dtype != t or p.shape != s:
                raise ValueError("AdamW: a weight's type or shape has changed")
            if p.numel() > 0:
                spans.append((p.data_ptr(), p.data_ptr() + p.numel() * p.element_size()))
        spans.sort()
        if any(a[1] > b[0] for a, b in zip(spans, spans[1:])):
            raise ValueError("AdamW: weights share memory")
        return [p.data_ptr() for p in self.params]

    def state(self) -> dict:
        """The optimizer's state, to be saved and given to another AdamW."""
        return dict(step=self.steps, m=self.m, v=self.v, master=self.master)

    def step(self, grads: Sequence[torch.Tensor], lr: float) -> Optional[torch.Tensor]:
        """One step with grads (one per weight, of its shape, bfloat16 or
        float32).  Returns the gradients' norm before clipping, a float32 scalar on
        the device (None without clipping).  A step captured into a graph
        repeats that step's number when it is replayed."""
        index = self.dev.index
        types = [g.dtype for g in grads]
        if ([g.shape for g in grads] != self._shapes or not all([g.is_contiguous() for g in grads])
                or [g.get_device() for g in grads] != [index] * len(self._shapes)):
            raise ValueError(f"AdamW: the gradients must be contiguous tensors of the {len(self.params)} weights' shapes "
                             f"on {self.dev}")
        if types != self._grad_types:
            if not all(t in _DT for t in types):
                raise ValueError("AdamW: gradients must be bfloat16 or float32")
            self._columns["grad_dtype"] = [_DT[t] for t in types]
            self._grad_types = types
        # a weight whose storage was replaced since the last step is followed
        if ([p.data_ptr() for p in self.params] != self._places or not all([p.is_contiguous() for p in self.params])
                or [p.dtype for p in self.params] != self._types or [p.shape for p in self.params] != self._shapes):
            self._places = self._check_params()
            self._columns["param"] = self._places
        self._columns["grad"] = [g.data_ptr() for g in grads]
        b1, b2 = self.betas
        cfg = L.AdamwCfg(lr, b1, b2, self.eps, self.max_norm, self.steps + 1, self.elems)
        need, norm = 0, None
        if self.max_norm > 0:
            if self._workspace_bytes is None:          # a matter of the weights' sizes
                self._workspace_bytes = _need(_lib.tandem_adamw_workspace_size, cfg, self._table, len(types))
            need = self._workspace_bytes
            norm = torch.empty((), dtype=torch.float32, device=self.dev)
        workspace = _workspace(None, need, self.dev)
        _run(self.dev, _lib.tandem_adamw, cfg, self._table, len(types), self.m.data_ptr(), self.v.data_ptr(),
             _ptr(self.master), _ptr(norm), _ptr(workspace), need)
        torch._C._increment_version(self.params)       # for graphs that saved a weight
        self.steps += 1
        return norm
