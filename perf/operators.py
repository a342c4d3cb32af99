"""The operators of the senior's update, from logits to weights, as cases whose time is measured.

A rollout leaves tokens, authorship and log-probs; the senior-only GRPO loss leaves a gradient with respect to
log-probs.  The operators here lead from there to the next rollout's weights:

    logp_fwd, logp_bwd   log-probs of the emitted tokens from the logits (and the KL to the frozen junior), and
                         the gradient with respect to the logits
    qk_fwd, qk_bwd       per-head norms of q and k with the rotary embedding, out of the packed QKV projection
    attn_fwd, attn_bwd   causal grouped-query attention over packed rollouts
    adamw                one optimizer step over all tensors of a model, gradient clipping included

The model pairs are the repository's workloads: "tiny" (float32, head size 32), "small" (bf16, 64) and "qwen"
(bf16, 128, q/k norms), senior or junior.  Values are drawn at the scale that the path meets: unit-RMS heads,
logits of a peaked next-token distribution and a junior close to the senior, gradients of a token-mean loss.
"""
import math

import torch

own = False

DEV = "cuda:0"

# n_q, n_kv, head_dim, d_model, ffn (of those that are trained), vocab, q/k norm, dtype
MODELS = {
    "tiny": (4, 2, 32, 128, 512, 512, False, "f32"),
    "tiny_junior": (2, 1, 32, 64, None, 512, False, "f32"),
    "small": (16, 4, 64, 1024, 4096, 32000, False, "bf16"),
    "small_junior": (8, 2, 64, 512, None, 32000, False, "bf16"),
    "qwen": (32, 8, 128, 2560, 9728, 151936, True, "bf16"),
    "qwen_junior": (16, 8, 128, 1024, None, 151936, True, "bf16"),
}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
THETA, EPS = 1.0e6, 1.0e-6


def listed():
    return [
        # scoring one step of a tandem batch of four sequences under both models: latency, rows far fewer than the
        # device's compute units, logits as the framework's float32 dumps hold them
        dict(name="logp_fwd_step", kind="logp_fwd", rows=4, vocab=151936, dtype="f32", ref=True, temperature=1.0,
             eos=-1),
        # one micro-batch of rollout positions at the large vocabulary, with the KL to the junior
        dict(name="logp_fwd_kl", kind="logp_fwd", rows=2048, vocab=151936, dtype="bf16", ref=True, temperature=1.0,
             eos=-1),
        # the way back of such a micro-batch
        dict(name="logp_bwd_kl", kind="logp_bwd", rows=1024, vocab=151936, dtype="bf16", ref=True, temperature=1.0,
             eos=-1),
        # a padded vocabulary that is not a multiple of 4, rollout temperature 0.6, EOS bias, no KL
        dict(name="logp_bwd_odd", kind="logp_bwd", rows=509, vocab=32001, dtype="f32", ref=False, temperature=0.6,
             eos=31999),
        # sixteen rollouts' q and k of one senior layer
        dict(name="qk_fwd_rollouts", kind="qk_fwd", model="qwen", tokens=18432, max_pos=2303),
        # an odd number of positions of the junior's shape, backward, long contexts
        dict(name="qk_bwd_odd", kind="qk_bwd", model="qwen_junior", tokens=4097, max_pos=8703),
        # the smallest call: a few sequences of a float32 model of one to 48 tokens
        dict(name="attn_fwd_tiny", kind="attn_fwd", model="tiny", seqs=4, max_len=48, zero=False),
        # sixteen ragged rollouts (prompt and up to 2048 new tokens) through one senior layer
        dict(name="attn_fwd_rollouts", kind="attn_fwd", model="qwen", seqs=16, max_len=2303, zero=False),
        # the same batch's backward pass
        dict(name="attn_bwd_rollouts", kind="attn_bwd", model="qwen", seqs=16, max_len=2303, zero=False),
        # one long chain of thought, backward: few heads, a long axis
        dict(name="attn_bwd_long", kind="attn_bwd", model="small", seqs=1, max_len=8703, zero=False),
        # a tiny float32 model's optimizer step: latency, many small tensors
        dict(name="adamw_tiny", kind="adamw", model="tiny", layers=2, heads=True, master=False, max_norm=1.0),
        # two layers of the large senior: bandwidth
        dict(name="adamw_layers", kind="adamw", model="qwen", layers=2, heads=False, master=True, max_norm=1.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["logp_fwd", "logp_bwd", "qk_fwd", "qk_bwd", "attn_fwd", "attn_bwd", "adamw"])
    if kind in ("logp_fwd", "logp_bwd"):
        vocab = rng.choice([512, 32000, 32001, 151936, _log_int(rng, 2, 200000)])
        ref, dtype = rng.random() < 0.5, rng.choice(["bf16", "f32"])
        most = 2048 * 151936 // (2 if kind == "logp_bwd" else 1) // (2 if dtype == "f32" else 1)
        rows = _log_int(rng, 1, max(1, min(65536, most // vocab)))
        return dict(kind=kind, rows=rows, vocab=vocab, dtype=dtype, ref=ref,
                    temperature=rng.choice([1.0, 0.6, 1.3]), eos=rng.choice([-1, vocab - 1]))
    model = rng.choice(list(MODELS))
    nq, nkv, hd = MODELS[model][:3]
    if kind in ("qk_fwd", "qk_bwd"):
        most = 18432 * 40 * 128 // ((nq + nkv) * hd) // (2 if MODELS[model][7] == "f32" else 1)
        return dict(kind=kind, model=model, tokens=_log_int(rng, 1, most), max_pos=_log_int(rng, 1, 100000))
    if kind in ("attn_fwd", "attn_bwd"):
        # lengths of one token up to the long chains, as many sequences as the largest listed work allows
        max_len = _log_int(rng, 1, 8703)
        most = 16 * 2303 * 2303 * 32 * 128 // (nq * hd * max_len * max_len)
        if MODELS[model][7] == "f32":
            most //= 2
        seqs = _log_int(rng, 1, max(1, min(256, most)))
        return dict(kind=kind, model=model, seqs=seqs, max_len=max_len, zero=rng.random() < 0.3)
    model = rng.choice(["tiny", "small", "qwen"])       # the juniors are frozen
    layers = rng.randint(1, 2 if model == "qwen" else 4)
    return dict(kind=kind, model=model, layers=layers, heads=rng.random() < 0.5 and model != "qwen",
                master=rng.random() < 0.7 and model != "tiny", max_norm=rng.choice([0.0, 1.0]))


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _lengths(case, seed):
    """Sequence lengths in the order of the seed: one is the longest, the others uniform in [1, max_len], one of
    them empty with `zero`.  A case's total length is its own, not the seed's."""
    g = torch.Generator()
    g.manual_seed(100003 * case["seqs"] + case["max_len"])
    n = torch.randint(1, case["max_len"] + 1, (case["seqs"],), generator=g)
    n[0] = case["max_len"]
    if case["zero"] and case["seqs"] > 1:
        n[1] = 0
    g.manual_seed(int(seed) + 17)
    return n[torch.randperm(case["seqs"], generator=g)]


def _live_rows(case):
    """Rows of a log-prob case that hold a token; the others (padding) are left out."""
    return case["rows"] - case["rows"] // 5


def _prepare_logp(case, seed):
    g = _gen(seed)
    R, V, dt = case["rows"], case["vocab"], DT[case["dtype"]]
    z = torch.randn((R, V), generator=g, device=DEV).mul_(2.5)
    # the emitted token: sampled from the distribution itself
    u = torch.rand((R, V), generator=g, device=DEV).clamp_(1e-7, 1 - 1e-7)
    tok = (z - torch.log(-torch.log(u))).argmax(dim=1).to(torch.int32)
    del u
    dead = torch.randperm(R, generator=g, device=DEV)[_live_rows(case):]
    tok[dead] = -1
    zr = (z + 0.3 * torch.randn((R, V), generator=g, device=DEV)).to(dt) if case["ref"] else None
    s = dict(case=case, z=z.to(dt), ref=zr, tok=tok, opts=_logp_opts(case))
    if case["kind"] == "logp_bwd":
        s["fwd"] = _plain_logp(s)
        n = max(1, _live_rows(case))
        s["g_logp"] = torch.randn((R,), generator=g, device=DEV) / n
        s["g_kl"] = torch.full((R,), 0.05 / n, device=DEV) if case["ref"] else None
    return s


def _logp_opts(case):
    eos = case["eos"]
    return dict(temperature=case["temperature"], eos_id=eos, eos_bias=2.2608 if eos >= 0 else 0.0,
                eos_bias_ref=2.0414 if eos >= 0 else 0.0)


def _prepare_qk(case, seed):
    g = _gen(seed)
    nq, nkv, hd, _, _, _, norm, dtype = MODELS[case["model"]]
    N, dt = case["tokens"], DT[dtype]
    qkv = torch.randn((N, (nq + 2 * nkv) * hd), generator=g, device=DEV).to(dt)
    pos = torch.randint(0, case["max_pos"] + 1, (N,), generator=g, device=DEV, dtype=torch.int32)
    gain = [1.0 + 0.1 * torch.randn((hd,), generator=g, device=DEV) for _ in range(2)] if norm else [None, None]
    s = dict(case=case, qkv=qkv, pos=pos, nq=nq, nkv=nkv, hd=hd, gq=gain[0], gk=gain[1])
    if case["kind"] == "qk_bwd":
        s["dq"] = (1e-3 * torch.randn((N, nq, hd), generator=g, device=DEV)).to(dt)
        s["dk"] = (1e-3 * torch.randn((N, nkv, hd), generator=g, device=DEV)).to(dt)
        # the attention's backward pass has written the value columns
        s["dqkv"] = torch.zeros((N, (nq + 2 * nkv) * hd), device=DEV, dtype=dt)
        s["dqkv"][:, (nq + nkv) * hd:] = (1e-3 * torch.randn((N, nkv * hd), generator=g, device=DEV)).to(dt)
    return s


def _prepare_attn(case, seed):
    g = _gen(seed)
    nq, nkv, hd, _, _, _, _, dtype = MODELS[case["model"]]
    dt = DT[dtype]
    lens = _lengths(case, seed)
    N = int(lens.sum())
    q = (1.5 * torch.randn((N, nq, hd), generator=g, device=DEV)).to(dt)
    k = (1.5 * torch.randn((N, nkv, hd), generator=g, device=DEV)).to(dt)
    # the values stay where the QKV projection left them
    qkv = torch.randn((N, (nq + 2 * nkv) * hd), generator=g, device=DEV).to(dt)
    v = qkv[:, (nq + nkv) * hd:].view(N, nkv, hd)
    offs = torch.cat([torch.zeros(1, dtype=torch.int64), lens.cumsum(0)]).to(torch.int32).to(DEV)
    s = dict(case=case, q=q, k=k, v=v, qkv=qkv, offs=offs, seqs=case["seqs"], max_len=case["max_len"])
    if case["kind"] == "attn_bwd":
        s["dout"] = (1e-3 * torch.randn((N, nq, hd), generator=g, device=DEV)).to(dt)
        s["out"], s["lse"] = _plain_attn(s)
    return s


def _adamw_shapes(case):
    nq, nkv, hd, d, ffn, vocab, norm, dtype = MODELS[case["model"]]
    mats, gains = DT[dtype], torch.float32
    out = []
    for _ in range(case["layers"]):
        out += [((d,), gains), (((nq + 2 * nkv) * hd, d), mats)]
        out += [((hd,), gains), ((hd,), gains)] if norm else []
        out += [((d, nq * hd), mats), ((d,), gains), ((2 * ffn, d), mats), ((d, ffn), mats)]
    if case["heads"]:
        out += [((vocab, d), mats), ((d,), gains), ((vocab, d), mats)]
    return out


ARENA = 64      # a tensor's optimizer state begins at a multiple of 64 elements


def _flat(xs):
    """Tensors as one float32 arena."""
    return torch.cat([torch.nn.functional.pad(x.reshape(-1).float(), (0, -x.numel() % ARENA)) for x in xs])


def _prepare_adamw(case, seed):
    g = _gen(seed)
    shapes = _adamw_shapes(case)
    start = [torch.randn(s, generator=g, device=DEV).mul_(0.02).add_(1.0 if len(s) == 1 else 0.0) for s, _ in shapes]
    params = [p.to(dt) for p, (_, dt) in zip(start, shapes)]
    grads = [torch.randn(s, generator=g, device=DEV).mul_(1e-3).to(dt) for s, dt in shapes]
    master = _flat(start) if case["master"] else None
    del start
    inside = _flat([torch.ones(s, device=DEV) for s, _ in shapes])
    m = torch.randn(inside.shape, generator=g, device=DEV).mul_(3e-4).mul_(inside)
    v = torch.rand(inside.shape, generator=g, device=DEV).mul_(2e-6).mul_(inside)
    del inside
    s = dict(case=case, params=params, grads=grads, m=m, v=v, master=master, step=100, lr=1e-6, betas=(0.9, 0.999),
             eps=1e-8, decay=[0.01 if len(sh) > 1 else 0.0 for sh, _ in shapes])
    if own:
        from paper_2606_28166_amd import engine as E
        s["opt"] = E.AdamW(params, betas=s["betas"], eps=s["eps"], weight_decay=s["decay"],
                           max_norm=case["max_norm"], state=dict(step=s["step"], m=m, v=v, master=master))
    else:
        s["decay_flat"] = _flat([torch.full(sh, w, device=DEV) for (sh, _), w in zip(shapes, s["decay"])])
    return s


def prepare(case, seed):
    kind = case["kind"]
    make = _prepare_logp if kind.startswith("logp") else _prepare_qk if kind.startswith("qk") else \
        _prepare_attn if kind.startswith("attn") else _prepare_adamw
    return make(case, seed)


# ------------------------------------------------------------------ the plain forms

def _scores(z, bias, s):
    o = s["opts"]
    if o["eos_id"] < 0:
        return z.float() / o["temperature"]
    z = z.to(torch.float32, copy=True)
    z[:, o["eos_id"]] += bias
    return z.div_(o["temperature"])


def _plain_logp(s):
    x = _scores(s["z"], s["opts"]["eos_bias"], s)
    live = s["tok"] >= 0
    top = x.amax(dim=1, keepdim=True)
    e = torch.exp(x - top)
    l = e.sum(dim=1)
    lse = top[:, 0] + torch.log(l)
    at = x.gather(1, s["tok"].clamp(min=0).long()[:, None])[:, 0]
    zero = torch.zeros_like(lse)
    r = dict(logp=torch.where(live, (at - top[:, 0]) - torch.log(l), zero), lse=torch.where(live, lse, zero))
    if s["ref"] is not None:
        y = _scores(s["ref"], s["opts"]["eos_bias_ref"], s)
        topr = y.amax(dim=1, keepdim=True)
        lr = torch.exp(y - topr).double().sum(dim=1)
        # the two log-sum-exps are close: their difference, and the mean of the scores' difference, in 64 bits
        diff = (top[:, 0].double() - topr[:, 0].double()) + torch.log(e.double().sum(dim=1)) - torch.log(lr)
        mean = (e * (x - y)).double().sum(dim=1) / e.double().sum(dim=1)
        r["kl"] = torch.where(live, (mean - diff).float(), zero)
        r["lse_diff"] = torch.where(live, diff.float(), zero)
    return r


def _plain_logp_backward(s):
    x = _scores(s["z"], s["opts"]["eos_bias"], s)
    live = s["tok"] >= 0
    f = s["fwd"]
    p = torch.exp(x - f["lse"][:, None])
    grad = -s["g_logp"][:, None] * p
    if s["ref"] is not None:
        y = _scores(s["ref"], s["opts"]["eos_bias_ref"], s)
        grad += s["g_kl"][:, None] * p * (x - y - (f["lse_diff"] + f["kl"])[:, None])
    grad.scatter_add_(1, s["tok"].clamp(min=0).long()[:, None], s["g_logp"][:, None])
    grad = grad / s["opts"]["temperature"]
    return torch.where(live[:, None], grad, torch.zeros_like(grad)).to(s["z"].dtype)


def _angles(s):
    i = torch.arange(s["hd"] // 2, device=DEV, dtype=torch.float64)
    a = s["pos"].double()[:, None] * torch.pow(torch.tensor(THETA, dtype=torch.float64, device=DEV),
                                               -2.0 * i / s["hd"])
    return torch.cos(a).float()[:, None, :], torch.sin(a).float()[:, None, :]


def _heads(s):
    nq, nkv, hd = s["nq"], s["nkv"], s["hd"]
    x = s["qkv"].view(-1, nq + 2 * nkv, hd)
    return x[:, :nq].float(), x[:, nq:nq + nkv].float()


def _plain_qk(s):
    c, n = _angles(s)
    h = s["hd"] // 2

    def one(x, gain):
        if gain is not None:
            x = x * torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + EPS) * gain
        a, b = x[..., :h], x[..., h:]
        return torch.cat([a * c - b * n, b * c + a * n], dim=-1).to(s["qkv"].dtype)

    q, k = _heads(s)
    return dict(q=one(q, s["gq"]), k=one(k, s["gk"]))


def _plain_qk_backward(s):
    c, n = _angles(s)
    nq, nkv, hd = s["nq"], s["nkv"], s["hd"]
    h = hd // 2

    def one(x, dy, gain):
        a, b = dy[..., :h].float(), dy[..., h:].float()
        dn = torch.cat([a * c + b * n, b * c - a * n], dim=-1)
        if gain is None:
            return dn, None
        r = torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + EPS)
        dg = (dn * (x * r)).double().sum(dim=(0, 1)).float()
        t = dn * gain
        return r * (t - x * (r * r) * (t * x).mean(dim=-1, keepdim=True)), dg

    q, k = _heads(s)
    dq, dgq = one(q, s["dq"], s["gq"])
    dk, dgk = one(k, s["dk"], s["gk"])
    out = s["dqkv"].view(-1, nq + 2 * nkv, hd)
    out[:, :nq] = dq.to(out.dtype)
    out[:, nq:nq + nkv] = dk.to(out.dtype)
    r = dict(dqkv=s["dqkv"])
    if dgq is not None:
        r.update(dq_gain=dgq, dk_gain=dgk)
    return r


def _padded(s):
    """Index of every (sequence, position) into the packed rows, and which of them exist."""
    o = s["offs"].long()
    at = o[:-1, None] + torch.arange(s["max_len"], device=DEV)[None, :]
    live = at < o[1:, None]
    return torch.where(live, at, torch.zeros_like(at)), live


def _batched(x, at, live, group):
    """[N][heads][hd] as float32 [sequence][head * group][position][hd], zero where there is no token."""
    y = x.float()[at] * live[:, :, None, None]
    return y.permute(0, 2, 1, 3).repeat_interleave(group, dim=1).contiguous()


def _probabilities(q, k, live, scale):
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(scale)
    L = s.shape[-1]
    see = torch.ones((L, L), dtype=torch.bool, device=DEV).tril_()
    s.masked_fill_(~(see[None, None] & live[:, None, None, :]), -math.inf)
    top = s.amax(dim=-1, keepdim=True)
    top = torch.where(live[:, None, :, None], top, torch.zeros_like(top))
    p = s.sub_(top).exp_()
    l = p.sum(dim=-1, keepdim=True)
    lse = (top + torch.log(l))[..., 0]
    return p.div_(torch.where(l > 0, l, torch.ones_like(l))), lse


def _packed(x, live, heads, group, dtype):
    """[sequence][head][position][hd] back as packed rows; heads that share a key head are added."""
    n, _, L, hd = x.shape
    if group > 1:
        x = x.view(n, heads, group, L, hd).sum(dim=2)
    return x.permute(0, 2, 1, 3)[live].to(dtype)


def _plain_attn(s):
    q, k, v = s["q"], s["k"], s["v"]
    nq, nkv, hd = q.shape[1], k.shape[1], q.shape[2]
    at, live = _padded(s)
    p, lse = _probabilities(_batched(q, at, live, 1), _batched(k, at, live, nq // nkv), live, hd ** -0.5)
    o = torch.matmul(p, _batched(v, at, live, nq // nkv))
    return _packed(o, live, nq, 1, q.dtype), lse.permute(0, 2, 1)[live].t().contiguous()


def _plain_attn_backward(s):
    q, k, v = s["q"], s["k"], s["v"]
    nq, nkv, hd = q.shape[1], k.shape[1], q.shape[2]
    group, scale = nq // nkv, hd ** -0.5
    at, live = _padded(s)
    qb, kb, vb = _batched(q, at, live, 1), _batched(k, at, live, group), _batched(v, at, live, group)
    do = _batched(s["dout"], at, live, 1)
    p, _ = _probabilities(qb, kb, live, scale)
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    dp = torch.matmul(do, vb.transpose(2, 3).contiguous())
    dp.sub_((p * dp).sum(dim=-1, keepdim=True)).mul_(p).mul_(scale)
    del p
    dq = torch.matmul(dp, kb)
    dk = torch.matmul(dp.transpose(2, 3).contiguous(), qb)
    return dict(dq=_packed(dq, live, nq, 1, q.dtype), dk=_packed(dk, live, nkv, group, q.dtype),
                dv=_packed(dv, live, nkv, group, q.dtype))


def _split(flat, like):
    sizes = [x.numel() + -x.numel() % ARENA for x in like]
    return [f[:x.numel()].view(x.shape) for f, x in zip(flat.split(sizes), like)]


def _plain_adamw(s):
    s["step"] += 1
    b1, b2 = s["betas"]
    g = _flat(s["grads"])
    norm, most = None, s["case"]["max_norm"]
    if most > 0:
        norm = torch.sqrt(g.double().square().sum()).float()
        g = g * torch.clamp(most / (norm + 1e-6), max=1.0)
    s["m"].mul_(b1).add_(g * (1.0 - b1))
    s["v"].mul_(b2).add_(g * g * (1.0 - b2))
    step = (s["m"] / (1.0 - b1 ** s["step"])) / (torch.sqrt(s["v"] / (1.0 - b2 ** s["step"])) + s["eps"])
    w = s["master"] if s["master"] is not None else _flat(s["params"])
    w.sub_(w * s["decay_flat"] * s["lr"]).sub_(step * s["lr"])
    [p.copy_(x) for p, x in zip(s["params"], _split(w, s["params"]))]
    return norm


def _adamw_outputs(s, norm):
    r = dict(params=s["params"], m=s["m"], v=s["v"], master=s["master"], norm=norm)
    return {k: v for k, v in r.items() if v is not None}


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind == "logp_fwd":
        return _plain_logp(s)
    if kind == "logp_bwd":
        return dict(grad=_plain_logp_backward(s))
    if kind == "qk_fwd":
        return _plain_qk(s)
    if kind == "qk_bwd":
        return _plain_qk_backward(s)
    if kind == "attn_fwd":
        return dict(zip(("out", "lse"), _plain_attn(s)))
    if kind == "attn_bwd":
        return _plain_attn_backward(s)
    return _adamw_outputs(s, _plain_adamw(s))


# ------------------------------------------------------------------ one pass

def _run_own(s):
    from paper_2606_28166_amd import engine as E
    kind = s["case"]["kind"]
    if kind == "logp_fwd":
        r = E.token_logprob(s["z"], s["tok"], ref=s["ref"], **s["opts"])
        return {k: v for k, v in r.items() if v is not None}
    if kind == "logp_bwd":
        return dict(grad=E.token_logprob_backward(s["z"], s["tok"], s["fwd"], s["g_logp"], g_kl=s["g_kl"],
                                                  ref=s["ref"], **s["opts"]))
    if kind == "qk_fwd":
        r = E.qk_norm_rope(s["qkv"], s["pos"], s["nq"], s["nkv"], THETA, EPS, q_gain=s["gq"], k_gain=s["gk"])
        return dict(q=r["q"], k=r["k"])
    if kind == "qk_bwd":
        r = E.qk_norm_rope_backward(s["qkv"], s["pos"], s["dq"], s["dk"], THETA, EPS, q_gain=s["gq"], k_gain=s["gk"],
                                    dqkv=s["dqkv"])
        return {k: v for k, v in r.items() if v is not None}
    if kind == "attn_fwd":
        r = E.attention(s["q"], s["k"], s["v"], s["offs"])
        return dict(out=r["out"], lse=r["lse"])
    if kind == "attn_bwd":
        r = E.attention_backward(s["dout"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["offs"])
        return dict(dq=r["dq"], dk=r["dk"], dv=r["dv"])
    return _adamw_outputs(s, s["opt"].step(s["grads"], s["lr"]))


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    kind = case["kind"]
    if kind.startswith("logp"):
        e = 2 if case["dtype"] == "bf16" else 4
        arrays = (2 if case["ref"] else 1) * _live_rows(case)
        cells = arrays * case["vocab"]
        if kind == "logp_bwd":
            return dict(bytes=e * (cells + case["rows"] * case["vocab"]), flops=8.0 * cells)
        return dict(bytes=e * cells, flops=4.0 * cells)
    nq, nkv, hd, _, _, _, _, dtype = MODELS[case["model"]]
    e = 2 if dtype == "bf16" else 4
    if kind.startswith("qk"):
        cells = case["tokens"] * (nq + nkv) * hd
        return dict(bytes=(2 if kind == "qk_fwd" else 3) * e * cells, flops=(12.0 if kind == "qk_fwd" else 24.0) * cells)
    if kind.startswith("attn"):
        n = _lengths(case, 0).double()
        tokens, pairs = float(n.sum()), float((n * (n + 1) / 2).sum())
        if kind == "attn_fwd":
            return dict(bytes=tokens * (e * (2 * nq + 2 * nkv) * hd + 4 * nq), flops=4.0 * pairs * nq * hd)
        return dict(bytes=tokens * (e * (4 * nq + 4 * nkv) * hd + 4 * nq), flops=10.0 * pairs * nq * hd)
    n = bytes_ = 0
    for sh, dt in _adamw_shapes(case):
        k = math.prod(sh)
        n += k
        # m and v both ways, the gradient in, the weight out, and the weights in: the master copy both ways or itself
        e = 2 if dt == torch.bfloat16 else 4
        bytes_ += k * (16 + 2 * e + (8 if case["master"] else e))
    return dict(bytes=bytes_, flops=16.0 * n)


# ------------------------------------------------------------------ the definitions in 64 bits

def _exact_logp(case, s):
    o, d = s["opts"], torch.float64
    R, V = case["rows"], case["vocab"]
    outs = []
    for a in range(0, R, 256):
        z = s["z"][a:a + 256].to(d)
        tok = s["tok"][a:a + 256].long()
        live = tok >= 0
        hot = torch.nn.functional.one_hot(tok.clamp(min=0), V).to(d) if case["kind"] == "logp_bwd" else None
        e = torch.zeros(V, dtype=d, device=DEV)
        if o["eos_id"] >= 0:
            e[o["eos_id"]] = 1.0
        lp = torch.log_softmax((z + o["eos_bias"] * e) / o["temperature"], dim=1)
        lse = torch.logsumexp((z + o["eos_bias"] * e) / o["temperature"], dim=1)
        r = dict(logp=lp.gather(1, tok.clamp(min=0)[:, None])[:, 0], lse=lse)
        if case["ref"]:
            y = (s["ref"][a:a + 256].to(d) + o["eos_bias_ref"] * e) / o["temperature"]
            lq = torch.log_softmax(y, dim=1)
            r["kl"] = (lp.exp() * (lp - lq)).sum(dim=1)
            r["lse_diff"] = lse - torch.logsumexp(y, dim=1)
        if case["kind"] == "logp_bwd":
            p = lp.exp()
            g = s["g_logp"][a:a + 256].to(d)[:, None] * (hot - p)
            if case["ref"]:
                g = g + s["g_kl"][a:a + 256].to(d)[:, None] * p * (lp - lq - r["kl"][:, None])
            r = dict(grad=(g / o["temperature"]))
        outs.append({k: torch.where(live[:, None] if v.dim() == 2 else live, v, torch.zeros_like(v))
                     for k, v in r.items()})
    return {k: torch.cat([x[k] for x in outs]) for k in outs[0]}


def _exact_qk(case, s):
    d = torch.float64
    nq, nkv, hd = s["nq"], s["nkv"], s["hd"]
    h = hd // 2
    freq = torch.tensor([THETA ** (-2.0 * i / hd) for i in range(h)], dtype=d, device=DEV)
    turn = torch.polar(torch.ones((), dtype=d, device=DEV), s["pos"].to(d)[:, None] * freq)[:, None, :]

    def forward(x, gain):
        if gain is not None:
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / hd + EPS) * gain
        c = torch.complex(x[..., :h].contiguous(), x[..., h:].contiguous()) * turn
        return torch.cat([c.real, c.imag], dim=-1)

    x = s["qkv"].to(d).view(-1, nq + 2 * nkv, hd)
    parts = [(x[:, :nq], s["gq"]), (x[:, nq:nq + nkv], s["gk"])]
    if case["kind"] == "qk_fwd":
        return dict(zip(("q", "k"), [forward(a, None if g is None else g.to(d)) for a, g in parts]))
    got, gains = [], []
    for (a, g), dy in zip(parts, (s["dq"], s["dk"])):
        a = a.clone().requires_grad_(True)
        g = None if g is None else g.to(d).requires_grad_(True)
        forward(a, g).backward(dy.to(d))
        got.append(a.grad)
        gains.append(None if g is None else g.grad)
    v = s["dqkv"].to(d).view(-1, nq + 2 * nkv, hd)[:, nq + nkv:]
    r = dict(dqkv=torch.cat(got + [v], dim=1).reshape(x.shape[0], -1))
    if gains[0] is not None:
        r.update(dq_gain=gains[0], dk_gain=gains[1])
    return r


def _exact_attn(case, s):
    d = torch.float64
    q, k, v = s["q"], s["k"], s["v"]
    nq, nkv, hd = q.shape[1], k.shape[1], q.shape[2]
    group = nq // nkv
    out = {n: torch.zeros(x.shape, dtype=d, device=DEV)
           for n, x in (("out", q), ("dq", q), ("dk", k), ("dv", k))}
    lse = torch.zeros((nq, q.shape[0]), dtype=d, device=DEV)
    ends = s["offs"].tolist()
    for a, b in zip(ends[:-1], ends[1:]):
        if a == b:
            continue
        see = torch.arange(b - a, device=DEV)
        see = see[:, None] >= see[None, :]
        for j in range(nkv):
            kk, vv = k[a:b, j].to(d), v[a:b, j].to(d)
            for i in range(j * group, (j + 1) * group):
                qq = q[a:b, i].to(d)
                w = (qq @ kk.t().contiguous()) / math.sqrt(hd)
                w = torch.where(see, w, torch.full_like(w, -math.inf))
                lse[i, a:b] = torch.logsumexp(w, dim=1)
                w = torch.softmax(w, dim=1)
                o = w @ vv
                out["out"][a:b, i] = o
                if case["kind"] == "attn_bwd":
                    do = s["dout"][a:b, i].to(d)
                    ds = w * (do @ vv.t().contiguous() - (do * o).sum(1, keepdim=True)) / math.sqrt(hd)
                    out["dq"][a:b, i] = ds @ kk
                    out["dk"][a:b, j] += ds.t().contiguous() @ qq
                    out["dv"][a:b, j] += w.t().contiguous() @ do
    if case["kind"] == "attn_fwd":
        return dict(out=out["out"], lse=lse)
    return dict(dq=out["dq"], dk=out["dk"], dv=out["dv"])


def _exact_adamw(case, s):
    d = torch.float64
    t = s["step"] + 1
    b1, b2 = s["betas"]
    grads = [g.to(d) for g in s["grads"]]
    norm = torch.sqrt(sum((g * g).sum() for g in grads))
    c = torch.clamp(case["max_norm"] / (norm + 1e-6), max=1.0) if case["max_norm"] > 0 else 1.0
    m, v = s["m"].to(d), s["v"].to(d)
    w = s["master"].to(d) if case["master"] else _flat(s["params"]).to(d)
    params, at = [], 0
    for g, decay in zip(grads, s["decay"]):
        part = slice(at, at + g.numel())
        x = c * g.reshape(-1)
        m[part] = b1 * m[part] + (1 - b1) * x
        v[part] = b2 * v[part] + (1 - b2) * x * x
        move = (m[part] / (1 - b1 ** t)) / (torch.sqrt(v[part] / (1 - b2 ** t)) + s["eps"])
        w[part] = w[part] * (1 - s["lr"] * decay) - s["lr"] * move
        params.append(w[part].view(g.shape))
        at += g.numel() + -g.numel() % ARENA
    r = dict(params=params, m=m, v=v)
    if case["master"]:
        r["master"] = w
    if case["max_norm"] > 0:
        r["norm"] = norm
    return r


def exact(case, seed):
    kind = case["kind"]
    s = prepare(case, seed)
    if kind.startswith("logp"):
        return _exact_logp(case, s)
    if kind.startswith("qk"):
        return _exact_qk(case, s)
    if kind.startswith("attn"):
        return _exact_attn(case, s)
    return _exact_adamw(case, s)
