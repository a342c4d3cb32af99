// The C entry points of the senior's update (handle-free): argument checks,
// workspace layout and launches.  No call allocates, synchronises or throws.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "status.h"
#include "tandem.h"
#include "update.h"
#include "update_plan.h"

using namespace tandem;

namespace {

constexpr int64_t kMaxGrid = 0xFFFFFFFFll / 256;   // workgroups of a launch: fewer than 2^32 threads, up to 256 each
constexpr int32_t kMaxRows = 1 << 30;              // indexes of rows past the last of a workgroup stay in 31 bits

__attribute__((format(printf, 2, 3))) tandem_status refuse(tandem_status s, const char* fmt, ...) {
  char b[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(b, sizeof b, fmt, ap);
  va_end(ap);
  return report(s, b);
}

tandem_status hip_failed(const char* who, hipError_t e) {
  return refuse(TANDEM_E_HIP, "%s: %s", who, hipGetErrorString(e));
}

// Makes the stream's device current for the launches of one call.
class DeviceOf {
 public:
  explicit DeviceOf(hipStream_t st) {
    if (!st) return;                          // the null stream belongs to the current device
    hipDevice_t dev = 0;
    int now = 0;
    err_ = hipStreamGetDevice(st, &dev);
    if (err_ == hipSuccess) err_ = hipGetDevice(&now);
    if (err_ != hipSuccess || dev == now) return;
    err_ = hipSetDevice(dev);
    if (err_ == hipSuccess) back_ = now;
  }
  ~DeviceOf() {
    if (back_ >= 0) (void)hipSetDevice(back_);
  }
  DeviceOf(const DeviceOf&) = delete;
  DeviceOf& operator=(const DeviceOf&) = delete;
  hipError_t error() const { return err_; }

 private:
  hipError_t err_ = hipSuccess;
  int back_ = -1;
};

// Runs launch() on the stream's device and turns its result into a status.
template <typename F>
tandem_status enqueue(const char* who, void* stream, F&& launch) {
  DeviceOf dev(static_cast<hipStream_t>(stream));
  hipError_t e = dev.error();
  if (e == hipSuccess) e = launch(static_cast<hipStream_t>(stream));
  return e == hipSuccess ? TANDEM_OK : hip_failed(who, e);
}

bool dtype_ok(int32_t dt) { return dt == TANDEM_BF16 || dt == TANDEM_F32; }
int elem(int32_t dt) { return dt == TANDEM_BF16 ? 2 : 4; }
bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
size_t up256(size_t n) { return (n + 255) / 256 * 256; }

tandem_status check_workspace(const char* who, const void* ws, size_t have, size_t need) {
  if (need == 0) return TANDEM_OK;
  if (!ws) return refuse(TANDEM_E_ARG, "%s: workspace is NULL", who);
  if (!aligned(ws, 256)) return refuse(TANDEM_E_ARG, "%s: workspace must be 256-byte aligned", who);
  if (have < need) return refuse(TANDEM_E_ARG, "%s: workspace is smaller than its workspace_size", who);
  return TANDEM_OK;
}

// ---------------------------------------------------------------- log-probs

tandem_status logprob_check(const char* who, const tandem_logprob_cfg* c, LogprobArgs* a, size_t* bytes) {
  if (!c) return refuse(TANDEM_E_ARG, "%s: cfg is NULL", who);
  if (c->rows < 0 || c->vocab < 1) return refuse(TANDEM_E_SHAPE, "%s: rows must be >= 0 and vocab >= 1", who);
  if (c->vocab > (1 << 30)) return refuse(TANDEM_E_SHAPE, "%s: vocab must be at most 2^30", who);
  if (logprob_blocks(c->rows, c->vocab) > kMaxGrid)
    return refuse(TANDEM_E_SHAPE, "%s: rows * vocab exceeds what one launch covers", who);
  if (!dtype_ok(c->dtype)) return refuse(TANDEM_E_ARG, "%s: dtype must be TANDEM_BF16 or TANDEM_F32", who);
  if (!(c->temperature > 0.f) || !std::isfinite(c->temperature) || !std::isfinite(1.f / c->temperature))
    return refuse(TANDEM_E_ARG, "%s: temperature must be positive, with a finite reciprocal", who);
  if (c->eos_id >= c->vocab) return refuse(TANDEM_E_ARG, "%s: eos_id lies outside the vocabulary", who);
  if (!std::isfinite(c->eos_bias) || !std::isfinite(c->eos_bias_ref))
    return refuse(TANDEM_E_ARG, "%s: the EOS biases must be finite", who);
  if (c->logits_stride < c->vocab) return refuse(TANDEM_E_SHAPE, "%s: logits_stride is below vocab", who);
  *a = LogprobArgs{};
  a->R = c->rows; a->V = c->vocab;
  a->ldz = c->logits_stride; a->ldr = c->ref_stride; a->ldg = c->grad_stride;
  a->inv_t = 1.f / c->temperature;
  a->eos = c->eos_id < 0 ? -1 : c->eos_id; a->bias = c->eos_bias; a->bias_r = c->eos_bias_ref;
  a->splits = logprob_splits(a->R, a->V, &a->chunk);
  *bytes = a->splits > 1 ? up256((size_t)a->R * a->splits * kLogprobPart * sizeof(float)) : 0;
  return TANDEM_OK;
}

// ---------------------------------------------------------------- q/k norm and rotation

tandem_status heads_check(const char* who, int32_t rows, int32_t nq, int32_t nkv, int32_t hd, int32_t dtype) {
  if (rows < 0 || nq < 1 || nkv < 1) return refuse(TANDEM_E_SHAPE, "%s: rows must be >= 0 and heads >= 1", who);
  if (rows > kMaxRows) return refuse(TANDEM_E_SHAPE, "%s: rows must be at most 2^30", who);
  if (nq % nkv != 0) return refuse(TANDEM_E_SHAPE, "%s: n_q_heads must be a multiple of n_kv_heads", who);
  if (hd != 32 && hd != 64 && hd != 128)
    return refuse(TANDEM_E_UNSUPPORTED, "%s: head_dim %d unsupported (32, 64 or 128)", who, hd);
  if (nq > 4096) return refuse(TANDEM_E_UNSUPPORTED, "%s: at most 4096 query heads", who);
  if (!dtype_ok(dtype)) return refuse(TANDEM_E_ARG, "%s: dtype must be TANDEM_BF16 or TANDEM_F32", who);
  return TANDEM_OK;
}

tandem_status stride_check(const char* who, const char* what, int64_t stride, int64_t least, int32_t dtype) {
  if (stride < least) return refuse(TANDEM_E_SHAPE, "%s: %s is below a row's length", who, what);
  if (stride * elem(dtype) % 16 != 0) return refuse(TANDEM_E_ARG, "%s: %s must be a multiple of 16 bytes", who, what);
  // 64 rows are addressed in 31 bits from the first
  if (stride > (int64_t)1 << 22) return refuse(TANDEM_E_SHAPE, "%s: %s must be at most 2^22", who, what);
  return TANDEM_OK;
}

tandem_status qk_check(const char* who, const tandem_qk_cfg* c, QkArgs* a) {
  if (!c) return refuse(TANDEM_E_ARG, "%s: cfg is NULL", who);
  tandem_status s = heads_check(who, c->rows, c->n_q_heads, c->n_kv_heads, c->head_dim, c->dtype);
  if (s != TANDEM_OK) return s;
  if (!(c->rms_eps >= 0.f) || !std::isfinite(c->rms_eps) || !(c->rope_theta > 0.f) || !std::isfinite(c->rope_theta))
    return refuse(TANDEM_E_ARG, "%s: rms_eps must be finite and >= 0, rope_theta finite and > 0", who);
  const int64_t hd = c->head_dim;
  if ((s = stride_check(who, "qkv_stride", c->qkv_stride, (c->n_q_heads + 2LL * c->n_kv_heads) * hd, c->dtype)) !=
      TANDEM_OK)
    return s;
  if ((s = stride_check(who, "q_stride", c->q_stride, c->n_q_heads * hd, c->dtype)) != TANDEM_OK) return s;
  if ((s = stride_check(who, "k_stride", c->k_stride, c->n_kv_heads * hd, c->dtype)) != TANDEM_OK) return s;
  if (qk_blocks(c->rows, c->n_q_heads, c->n_kv_heads, c->head_dim) > kMaxGrid)
    return refuse(TANDEM_E_SHAPE, "%s: rows exceed what one launch covers", who);
  *a = QkArgs{};
  a->N = c->rows; a->nq = c->n_q_heads; a->nkv = c->n_kv_heads; a->hd = c->head_dim;
  a->ld = c->qkv_stride; a->ldq = c->q_stride; a->ldk = c->k_stride;
  a->eps = c->rms_eps;
  for (int i = 0; i < a->hd / 2; ++i)
    a->turns[i] = std::pow((double)c->rope_theta, -2.0 * i / a->hd) / 6.283185307179586476925286766559;
  return TANDEM_OK;
}

// ---------------------------------------------------------------- attention

tandem_status attention_check(const char* who, const tandem_attention_cfg* c, bool backward, FlashArgs* a) {
  if (!c) return refuse(TANDEM_E_ARG, "%s: cfg is NULL", who);
  tandem_status s = heads_check(who, c->rows, c->n_q_heads, c->n_kv_heads, c->head_dim, c->dtype);
  if (s != TANDEM_OK) return s;
  if (c->n_seqs < 0) return refuse(TANDEM_E_SHAPE, "%s: n_seqs must be >= 0", who);
  if (!(c->scale > 0.f) || !std::isfinite(c->scale))
    return refuse(TANDEM_E_ARG, "%s: scale must be finite and > 0", who);
  if ((uint32_t)c->clear > (TANDEM_CLEAR_OUT | TANDEM_CLEAR_LSE | TANDEM_CLEAR_DQ | TANDEM_CLEAR_DK | TANDEM_CLEAR_DV))
    return refuse(TANDEM_E_ARG, "%s: clear names outputs that there are not", who);
  const int64_t q = (int64_t)c->n_q_heads * c->head_dim, kv = (int64_t)c->n_kv_heads * c->head_dim;
  const struct { const char* what; int64_t stride, least; } st[] = {
      {"q_stride", c->q_stride, q},       {"k_stride", c->k_stride, kv},   {"v_stride", c->v_stride, kv},
      {"out_stride", c->out_stride, q},   {"dout_stride", c->dout_stride, q}, {"dq_stride", c->dq_stride, q},
      {"dk_stride", c->dk_stride, kv},    {"dv_stride", c->dv_stride, kv}};
  for (int i = 0; i < (backward ? 8 : 4); ++i)
    if ((s = stride_check(who, st[i].what, st[i].stride, st[i].least, c->dtype)) != TANDEM_OK) return s;
  *a = FlashArgs{};
  a->N = c->rows; a->n_seqs = c->n_seqs; a->nq = c->n_q_heads; a->nkv = c->n_kv_heads;
  if (flash_blocks(*a, c->head_dim, c->dtype, backward) > kMaxGrid)
    return refuse(TANDEM_E_SHAPE, "%s: rows and sequences times heads exceed what one launch covers", who);
  a->scale = c->scale;
  a->ldq = c->q_stride; a->ldk = c->k_stride; a->ldv = c->v_stride; a->ldo = c->out_stride;
  a->lddo = c->dout_stride; a->lddq = c->dq_stride; a->lddk = c->dk_stride; a->lddv = c->dv_stride;
  a->clear = c->clear;
  return TANDEM_OK;
}

// The backward pass's workspace: two statistics per row and head, and the sums of the parts.
size_t attention_stat_bytes(const FlashArgs& a) { return up256((size_t)a.N * a.nq * sizeof(float)); }
size_t attention_bytes(const FlashArgs& a, int hd, int dtype) {
  const int parts = flash_parts(a.N, a.n_seqs, a.nq, a.nkv, hd, dtype == TANDEM_BF16);
  return 2 * attention_stat_bytes(a) + (parts > 1 ? (size_t)2 * parts * a.N * a.nkv * hd * sizeof(float) : 0);
}

// ---------------------------------------------------------------- AdamW

tandem_status adamw_check(const char* who, const tandem_adamw_cfg* c, const tandem_adamw_tensor* t, int32_t n,
                          int64_t* chunks) {
  if (!c) return refuse(TANDEM_E_ARG, "%s: cfg is NULL", who);
  if (n < 0 || (n > 0 && !t)) return refuse(TANDEM_E_ARG, "%s: tensors is NULL or n_tensors negative", who);
  if (!std::isfinite(c->lr)) return refuse(TANDEM_E_ARG, "%s: lr must be finite", who);
  if (!(c->beta1 >= 0.0 && c->beta1 < 1.0) || !(c->beta2 >= 0.0 && c->beta2 < 1.0))
    return refuse(TANDEM_E_ARG, "%s: the betas must lie in [0, 1)", who);
  if (!((float)c->eps > 0.f) || !std::isfinite((float)c->eps))
    return refuse(TANDEM_E_ARG, "%s: eps must be finite and > 0 as a float", who);
  if (!(c->max_norm >= 0.0) || !std::isfinite(c->max_norm))
    return refuse(TANDEM_E_ARG, "%s: max_norm must be finite and >= 0", who);
  if (c->step < 1) return refuse(TANDEM_E_ARG, "%s: step must be >= 1", who);
  if (c->arena_elems < 0) return refuse(TANDEM_E_SHAPE, "%s: arena_elems must be >= 0", who);
  int64_t total = 0;
  for (int i = 0; i < n; ++i) {
    if (t[i].n < 0) return refuse(TANDEM_E_SHAPE, "%s: tensor %d has a negative size", who, i);
    if (t[i].n > 0 && (!t[i].param || !t[i].grad)) return refuse(TANDEM_E_ARG, "%s: tensor %d has a NULL pointer", who, i);
    if (!dtype_ok(t[i].param_dtype) || !dtype_ok(t[i].grad_dtype))
      return refuse(TANDEM_E_ARG, "%s: tensor %d: dtypes must be TANDEM_BF16 or TANDEM_F32", who, i);
    if (!aligned(t[i].param, elem(t[i].param_dtype)) || !aligned(t[i].grad, elem(t[i].grad_dtype)))
      return refuse(TANDEM_E_ARG, "%s: tensor %d is not aligned to its elements", who, i);
    if (!(t[i].weight_decay >= 0.0) || !std::isfinite(t[i].weight_decay))
      return refuse(TANDEM_E_ARG, "%s: tensor %d: weight_decay must be finite and >= 0", who, i);
    if (t[i].state_offset < 0 || t[i].state_offset % 4 != 0 || t[i].state_offset > c->arena_elems ||
        t[i].n > c->arena_elems - t[i].state_offset)
      return refuse(TANDEM_E_CAPACITY, "%s: tensor %d's state lies outside the arenas or off a multiple of 4", who, i);
    total += (t[i].n + kAdamwChunk - 1) / kAdamwChunk;
    if (total > kMaxGrid) return refuse(TANDEM_E_SHAPE, "%s: too many elements", who);
  }
  *chunks = total;
  return TANDEM_OK;
}

// The workspace with clipping: the factor, then the chunks' sums of squares.
size_t adamw_bytes(const tandem_adamw_cfg* c, int64_t chunks) {
  return c->max_norm > 0.0 ? 256 + up256((size_t)chunks * sizeof(double)) : 0;
}

}  // namespace

extern "C" {

tandem_status tandem_logprob_workspace_size(const tandem_logprob_cfg* cfg, size_t* bytes) {
  const char* who = "tandem_logprob_workspace_size";
  if (!bytes) return refuse(TANDEM_E_ARG, "%s: bytes is NULL", who);
  LogprobArgs a;
  return logprob_check(who, cfg, &a, bytes);
}

tandem_status tandem_token_logprob(const tandem_logprob_cfg* cfg, const void* logits, const void* logits_ref,
                                   const int32_t* tokens, float* logp, float* lse, float* kl, float* lse_diff,
                                   void* workspace, size_t workspace_bytes, void* stream) {
  const char* who = "tandem_token_logprob";
  LogprobArgs a;
  size_t need = 0;
  tandem_status s = logprob_check(who, cfg, &a, &need);
  if (s != TANDEM_OK) return s;
  if (!logits_ref != !kl || !logits_ref != !lse_diff)
    return refuse(TANDEM_E_ARG, "%s: logits_ref, kl and lse_diff go together", who);
  if (logits_ref && cfg->ref_stride < cfg->vocab) return refuse(TANDEM_E_SHAPE, "%s: ref_stride is below vocab", who);
  if (a.R == 0) return TANDEM_OK;
  if (!logits || !tokens || !logp || !lse) return refuse(TANDEM_E_ARG, "%s: a required pointer is NULL", who);
  if (!aligned(logits, elem(cfg->dtype)) || !aligned(logits_ref, elem(cfg->dtype)))
    return refuse(TANDEM_E_ARG, "%s: logits are not aligned to their elements", who);
  if ((s = check_workspace(who, workspace, workspace_bytes, need)) != TANDEM_OK) return s;
  a.z = logits; a.zr = logits_ref; a.tok = tokens;
  a.logp = logp; a.lse = lse; a.kl = kl; a.diff = lse_diff;
  a.part = static_cast<float*>(workspace);
  return enqueue(who, stream, [&](hipStream_t st) { return launch_logprob(a, cfg->dtype, st); });
}

tandem_status tandem_token_logprob_backward(const tandem_logprob_cfg* cfg, const void* logits,
                                            const void* logits_ref, const int32_t* tokens, const float* lse,
                                            const float* kl, const float* lse_diff, const float* g_logp,
                                            const float* g_kl, void* grad, void* stream) {
  const char* who = "tandem_token_logprob_backward";
  LogprobArgs a;
  size_t need = 0;
  const tandem_status s = logprob_check(who, cfg, &a, &need);
  if (s != TANDEM_OK) return s;
  if (cfg->grad_stride < cfg->vocab) return refuse(TANDEM_E_SHAPE, "%s: grad_stride is below vocab", who);
  if (g_kl && cfg->ref_stride < cfg->vocab) return refuse(TANDEM_E_SHAPE, "%s: ref_stride is below vocab", who);
  if (a.R == 0) return TANDEM_OK;
  if (!logits || !tokens || !lse || !g_logp || !grad || (g_kl && (!logits_ref || !kl || !lse_diff)))
    return refuse(TANDEM_E_ARG, "%s: a required pointer is NULL", who);
  if (!aligned(logits, elem(cfg->dtype)) || !aligned(logits_ref, elem(cfg->dtype)) || !aligned(grad, elem(cfg->dtype)))
    return refuse(TANDEM_E_ARG, "%s: logits or grad are not aligned to their elements", who);
  if (grad == logits && cfg->grad_stride != cfg->logits_stride)
    return refuse(TANDEM_E_ARG, "%s: a gradient in place of the logits needs their stride", who);
  a.z = logits; a.zr = g_kl ? logits_ref : nullptr; a.tok = tokens;
  // read only; the launcher's arguments are shared with the forward pass
  a.lse = const_cast<float*>(lse); a.kl = const_cast<float*>(kl); a.diff = const_cast<float*>(lse_diff);
  a.g_logp = g_logp; a.g_kl = g_kl; a.grad = grad;
  return enqueue(who, stream, [&](hipStream_t st) { return launch_logprob_backward(a, cfg->dtype, st); });
}

tandem_status tandem_qk_workspace_size(const tandem_qk_cfg* cfg, size_t* bytes) {
  const char* who = "tandem_qk_workspace_size";
  if (!bytes) return refuse(TANDEM_E_ARG, "%s: bytes is NULL", who);
  QkArgs a;
  const tandem_status s = qk_check(who, cfg, &a);
  if (s != TANDEM_OK) return s;
  *bytes = up256((size_t)qk_backward_blocks(a.N, a.nq, a.nkv, a.hd) * 2 * a.hd * sizeof(float));
  return TANDEM_OK;
}

tandem_status tandem_qk_norm_rope(const tandem_qk_cfg* cfg, const void* qkv, const float* q_gain,
                                  const float* k_gain, const int32_t* positions, void* q, void* k, void* stream) {
  const char* who = "tandem_qk_norm_rope";
  QkArgs a;
  const tandem_status s = qk_check(who, cfg, &a);
  if (s != TANDEM_OK) return s;
  if (!q_gain != !k_gain) return refuse(TANDEM_E_ARG, "%s: q_gain and k_gain go together", who);
  if (a.N == 0) return TANDEM_OK;
  if (!qkv || !positions || !q || !k) return refuse(TANDEM_E_ARG, "%s: a required pointer is NULL", who);
  if (!aligned(qkv, 16) || !aligned(q, 16) || !aligned(k, 16))
    return refuse(TANDEM_E_ARG, "%s: qkv, q and k must be 16-byte aligned", who);
  a.qkv = qkv; a.gq = q_gain; a.gk = k_gain; a.pos = positions; a.q = q; a.k = k;
  return enqueue(who, stream, [&](hipStream_t st) { return launch_qk(a, cfg->dtype, st); });
}

tandem_status tandem_qk_norm_rope_backward(const tandem_qk_cfg* cfg, const void* qkv, const float* q_gain,
                                           const float* k_gain, const int32_t* positions, const void* dq,
                                           const void* dk, void* dqkv, float* dq_gain, float* dk_gain,
                                           void* workspace, size_t workspace_bytes, void* stream) {
  const char* who = "tandem_qk_norm_rope_backward";
  QkArgs a;
  tandem_status s = qk_check(who, cfg, &a);
  if (s != TANDEM_OK) return s;
  if (!q_gain != !k_gain || !q_gain != !dq_gain || !q_gain != !dk_gain)
    return refuse(TANDEM_E_ARG, "%s: the gains and their gradients go together", who);
  if (a.N > 0 && (!qkv || !positions || !dq || !dk || !dqkv))
    return refuse(TANDEM_E_ARG, "%s: a required pointer is NULL", who);
  if (!aligned(qkv, 16) || !aligned(dq, 16) || !aligned(dk, 16) || !aligned(dqkv, 16))
    return refuse(TANDEM_E_ARG, "%s: qkv, dq, dk and dqkv must be 16-byte aligned", who);
  const size_t need = up256((size_t)qk_backward_blocks(a.N, a.nq, a.nkv, a.hd) * 2 * a.hd * sizeof(float));
  if (q_gain && (s = check_workspace(who, workspace, workspace_bytes, need)) != TANDEM_OK) return s;
  if (a.N == 0 && !q_gain) return TANDEM_OK;
  a.qkv = qkv; a.gq = q_gain; a.gk = k_gain; a.pos = positions; a.dq = dq; a.dk = dk; a.dqkv = dqkv;
  a.dgq = dq_gain; a.dgk = dk_gain; a.part = static_cast<float*>(workspace);
  return enqueue(who, stream, [&](hipStream_t st) { return launch_qk_backward(a, cfg->dtype, st); });
}

tandem_status tandem_attention_workspace_size(const tandem_attention_cfg* cfg, size_t* bytes) {
  const char* who = "tandem_attention_workspace_size";
  if (!bytes) return refuse(TANDEM_E_ARG, "%s: bytes is NULL", who);
  FlashArgs a;
  const tandem_status s = attention_check(who, cfg, true, &a);
  if (s != TANDEM_OK) return s;
  *bytes = attention_bytes(a, cfg->head_dim, cfg->dtype);
  return TANDEM_OK;
}

tandem_status tandem_attention(const tandem_attention_cfg* cfg, const void* q, const void* k, const void* v,
                               const int32_t* offsets, void* out, float* lse, void* stream) {
  const char* who = "tandem_attention";
  FlashArgs a;
  const tandem_status s = attention_check(who, cfg, false, &a);
  if (s != TANDEM_OK) return s;
  if (a.N == 0 || a.n_seqs == 0) return TANDEM_OK;
  if (!q || !k || !v || !offsets || !out || !lse) return refuse(TANDEM_E_ARG, "%s: a required pointer is NULL", who);
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16))
    return refuse(TANDEM_E_ARG, "%s: q, k, v and out must be 16-byte aligned", who);
  a.q = q; a.k = k; a.v = v; a.offs = offsets; a.out = out; a.lse = lse;
  return enqueue(who, stream, [&](hipStream_t st) { return launch_flash(a, cfg->head_dim, cfg->dtype, st); });
}

tandem_status tandem_attention_backward(const tandem_attention_cfg* cfg, const void* dout, const void* q,
                                        const void* k, const void* v, const void* out, const float* lse,
                                        const int32_t* offsets, void* dq, void* dk, void* dv, void* workspace,
                                        size_t workspace_bytes, void* stream) {
  const char* who = "tandem_attention_backward";
  FlashArgs a;
  tandem_status s = attention_check(who, cfg, true, &a);
  if (s != TANDEM_OK) return s;
  if (a.N == 0 || a.n_seqs == 0) return TANDEM_OK;
  if (!dout || !q || !k || !v || !out || !lse || !offsets || !dq || !dk || !dv)
    return refuse(TANDEM_E_ARG, "%s: a required pointer is NULL", who);
  for (const void* p : {dout, q, k, v, out, (const void*)dq, (const void*)dk, (const void*)dv})
    if (!aligned(p, 16)) return refuse(TANDEM_E_ARG, "%s: every array must be 16-byte aligned", who);
  const size_t need = attention_bytes(a, cfg->head_dim, cfg->dtype);
  if ((s = check_workspace(who, workspace, workspace_bytes, need)) != TANDEM_OK) return s;
  a.q = q; a.k = k; a.v = v; a.offs = offsets;
  a.out = const_cast<void*>(out); a.lse = const_cast<float*>(lse);      // read only here
  a.dout = dout; a.dq = dq; a.dk = dk; a.dv = dv;
  a.ndelta = static_cast<float*>(workspace);
  a.lse2 = reinterpret_cast<float*>(static_cast<char*>(workspace) + attention_stat_bytes(a));
  a.sums = reinterpret_cast<float*>(static_cast<char*>(workspace) + 2 * attention_stat_bytes(a));
  return enqueue(who, stream, [&](hipStream_t st) { return launch_flash_backward(a, cfg->head_dim, cfg->dtype, st); });
}

tandem_status tandem_adamw_workspace_size(const tandem_adamw_cfg* cfg, const tandem_adamw_tensor* tensors,
                                          int32_t n_tensors, size_t* bytes) {
  const char* who = "tandem_adamw_workspace_size";
  if (!bytes) return refuse(TANDEM_E_ARG, "%s: bytes is NULL", who);
  int64_t chunks = 0;
  const tandem_status s = adamw_check(who, cfg, tensors, n_tensors, &chunks);
  if (s != TANDEM_OK) return s;
  *bytes = adamw_bytes(cfg, chunks);
  return TANDEM_OK;
}

tandem_status tandem_adamw(const tandem_adamw_cfg* cfg, const tandem_adamw_tensor* tensors, int32_t n_tensors,
                           float* m, float* v, float* master, float* norm, void* workspace, size_t workspace_bytes,
                           void* stream) {
  const char* who = "tandem_adamw";
  int64_t chunks = 0;
  tandem_status s = adamw_check(who, cfg, tensors, n_tensors, &chunks);
  if (s != TANDEM_OK) return s;
  const bool clipped = cfg->max_norm > 0.0;
  if (clipped && !norm) return refuse(TANDEM_E_ARG, "%s: clipping needs norm", who);
  if ((s = check_workspace(who, workspace, workspace_bytes, adamw_bytes(cfg, chunks))) != TANDEM_OK) return s;
  if (chunks > 0 && (!m || !v)) return refuse(TANDEM_E_ARG, "%s: m or v is NULL", who);
  if (!aligned(m, 16) || !aligned(v, 16) || !aligned(master, 16))
    return refuse(TANDEM_E_ARG, "%s: the arenas must be 16-byte aligned", who);

  float* clip = static_cast<float*>(workspace);
  double* part = reinterpret_cast<double*>(static_cast<char*>(workspace) + 256);
  return enqueue(who, stream, [&](hipStream_t st) {
    AdamwArgs a{};
    a.m = m; a.v = v; a.master = master;
    a.b1 = (float)cfg->beta1; a.c1 = (float)(1.0 - cfg->beta1);
    a.b2 = (float)cfg->beta2; a.c2 = (float)(1.0 - cfg->beta2);
    a.lr = (float)cfg->lr; a.eps = (float)cfg->eps;
    a.inv_bc1 = (float)(1.0 / (1.0 - std::pow(cfg->beta1, cfg->step)));
    a.inv_bc2 = (float)(1.0 / (1.0 - std::pow(cfg->beta2, cfg->step)));
    a.few = clipped && chunks <= kAdamwFew ? (int)chunks : 0;
    a.clip = clipped && !a.few ? clip : nullptr;
    a.max_norm = cfg->max_norm;
    // pass 0 (with clipping): the sums of squares; pass 1: the update
    for (int pass = clipped ? 0 : 1; pass < 2; ++pass) {
      int64_t before = 0;                     // chunks of earlier launches
      for (int i = 0; i < n_tensors;) {
        a.n = 0;
        a.p16[0] = a.p16[1] = a.g16[0] = a.g16[1] = 0;
        int64_t grid = 0;
        for (; i < n_tensors && a.n < kAdamwTensors; ++i) {
          const tandem_adamw_tensor& t = tensors[i];
          if (t.n == 0) continue;
          AdamwTensor& d = a.t[a.n];
          d.p = t.param; d.g = t.grad; d.n = t.n; d.off = t.state_offset;
          d.lr_decay = (float)(cfg->lr * t.weight_decay);
          d.first = (int)grid;
          if (t.param_dtype == TANDEM_BF16) a.p16[a.n >> 6] |= 1ull << (a.n & 63);
          if (t.grad_dtype == TANDEM_BF16) a.g16[a.n >> 6] |= 1ull << (a.n & 63);
          grid += (t.n + kAdamwChunk - 1) / kAdamwChunk;
          ++a.n;
        }
        if (grid == 0) continue;
        // the update's launches all read the sums from the first on, and one of them reports the norm
        a.part = pass == 0 ? part + before : part;
        a.norm = a.few && before == 0 ? norm : nullptr;
        before += grid;
        const hipError_t e = pass == 0 ? launch_adamw_norm(a, (int)grid, st) : launch_adamw(a, (int)grid, st);
        if (e != hipSuccess) return e;
      }
      if (pass == 0 && (!a.few || before == 0)) {
        const hipError_t e = launch_adamw_clip(part, (int)before, cfg->max_norm, norm, clip, st);
        if (e != hipSuccess) return e;
      }
    }
    return hipSuccess;
  });
}

}  // extern "C"
