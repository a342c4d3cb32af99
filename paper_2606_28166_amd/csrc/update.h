// Launchers of the update operators' kernels (internal to libtandem): checked
// arguments in, hipError_t out.  The mathematics stands in tandem.h.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"
#include "tandem.h"

namespace tandem {

// ------------------------------------------------ log-probs from logits
struct LogprobArgs {
  int R, V;
  const void* z; const void* zr;           // logits, reference logits (NULL: none)
  int64_t ldz, ldr, ldg;                   // row strides, elements
  const int32_t* tok;
  float inv_t;                             // 1 / temperature
  int eos; float bias, bias_r;             // eos < 0: no bias
  float* logp; float* lse; float* kl; float* diff;                     // outputs, of the backward pass inputs
  const float* g_logp; const float* g_kl;
  void* grad;
  float* part;                             // [R][splits][kLogprobPart]: partials of a row cut into splits
  int splits, chunk;                       // forward: a row's parts, and their length in entries
};
constexpr int kLogprobPart = 8;            // floats: a part's two maxima and three sums of 64 bits
// How the forward pass cuts a row: the number of parts (1: no workspace).
int logprob_splits(int R, int V, int* chunk);
int64_t logprob_blocks(int R, int V);      // workgroups of the largest launch
hipError_t launch_logprob(const LogprobArgs& a, int dtype, hipStream_t st);
hipError_t launch_logprob_backward(const LogprobArgs& a, int dtype, hipStream_t st);

// ------------------------------------------------ q/k norm and rotation
struct QkArgs {
  int N, nq, nkv, hd;
  const void* qkv; int64_t ld, ldq, ldk;
  const float* gq; const float* gk;        // NULL: no norm
  const int32_t* pos;
  float eps;
  double turns[64];                        // theta^(-2i/hd) / 2 pi: turns per position of frequency i
  void* q; void* k;                        // forward outputs
  const void* dq; const void* dk;          // backward inputs
  void* dqkv;
  float* dgq; float* dgk;
  float* part;                             // [blocks][2][hd]: the gains' gradients by workgroup
};
int64_t qk_blocks(int N, int nq, int nkv, int hd);         // workgroups of the forward pass
int qk_backward_blocks(int N, int nq, int nkv, int hd);   // workgroups of the backward pass
hipError_t launch_qk(const QkArgs& a, int dtype, hipStream_t st);
hipError_t launch_qk_backward(const QkArgs& a, int dtype, hipStream_t st);

// ------------------------------------------------ attention over packed sequences
struct FlashArgs {
  int N, n_seqs, nq, nkv;
  float scale;
  const void* q; const void* k; const void* v; const int32_t* offs;
  int64_t ldq, ldk, ldv, ldo;
  void* out; float* lse;                   // outputs of the forward pass, inputs of the backward
  const void* dout; void* dq; void* dk; void* dv;
  int64_t lddo, lddq, lddk, lddv;
  float* ndelta; float* lse2;              // workspace of the backward pass, [nq][N] each
  int clear;                               // TANDEM_CLEAR_*
  float* sums;                             // and [dV, dK][parts][N][nkv][hd], where the work on a tile is cut into parts
};
// workgroups of the largest launch (a.N, n_seqs, nq, nkv)
int64_t flash_blocks(const FlashArgs& a, int hd, int dtype, bool backward);
hipError_t launch_flash(const FlashArgs& a, int hd, int dtype, hipStream_t st);
hipError_t launch_flash_backward(const FlashArgs& a, int hd, int dtype, hipStream_t st);

// ------------------------------------------------ AdamW over many tensors
struct AdamwTensor {
  void* p; const void* g;
  int64_t n, off;
  float lr_decay;                          // lr * weight_decay
  int first;                               // the tensor's first chunk of this launch
};
// A launch takes up to kAdamwTensors tensors by value: the argument block is at
// most 4 KB, and nothing has to be uploaded.
constexpr int kAdamwTensors = 96;
constexpr int kAdamwChunk = 8192;          // elements per workgroup
constexpr int kAdamwFew = 512;             // chunks whose sums every workgroup of the update can add up
struct AdamwArgs {
  float* m; float* v; float* master;
  float b1, c1, b2, c2;                    // betas and 1 - beta
  float lr, inv_bc1, inv_bc2, eps;         // 1 / (1 - beta^t)
  const float* clip;                       // device scalar c, or NULL (c = 1, or from few chunks' sums)
  double* part;                            // sums of squares by chunk
  int few;                                 // > 0: the update adds up that many chunks' sums itself
  float* norm; double max_norm;            // of the update then: norm NULL in all launches but the first
  int n;                                   // tensors of this launch
  uint64_t p16[2], g16[2];                 // bit i: tensor i's weights / gradient are bf16
  AdamwTensor t[kAdamwTensors];
};
static_assert(sizeof(AdamwArgs) <= 4096, "kernel argument block");
hipError_t launch_adamw_norm(const AdamwArgs& a, int chunks, hipStream_t st);
hipError_t launch_adamw_clip(const double* part, int chunks, double max_norm, float* norm, float* clip,
                             hipStream_t st);
hipError_t launch_adamw(const AdamwArgs& a, int chunks, hipStream_t st);

}  // namespace tandem
