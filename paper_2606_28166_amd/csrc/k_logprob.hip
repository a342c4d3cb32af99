// k_logprob.hip — log-probs of given tokens from logits, the divergence from a
// reference model's logits, and the gradient of both with respect to the logits.
//
// Forward: one pass over a row with the running maximum m and the sums taken
// against it, l = sum e^(s - m) and (with a reference) w = sum e^(s - m) (s - s'),
// beside the reference's own m', l'.  Then lse = m + log l, logp = (s_y - m) - log l,
// lse - lse' = (m - m') + log(l / l') and KL = w / l - (lse - lse'): each difference
// is formed before it is added to something large, so a small KL keeps its digits.
// Backward: p = e^(s - lse) again, elementwise.
// All sums are float32, logits are converted as they are read.
#include "common.h"
#include "update.h"

namespace tandem {
namespace {

// 8 entries per load: rows start at any multiple of an element's size
typedef uint32_t u32x4_e2 __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_e4 __attribute__((ext_vector_type(4), aligned(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// bf16 pair: element 0 in the low half
__device__ __forceinline__ float lo16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi16(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

template <typename T> struct Row8;
template <> struct Row8<bf16_t> {
  u32x4_e2 r;
  __device__ __forceinline__ void load(const bf16_t* p) { r = *reinterpret_cast<const u32x4_e2*>(p); }
  __device__ __forceinline__ float get(int e) const { return (e & 1) ? hi16(r[e >> 1]) : lo16(r[e >> 1]); }
};
template <> struct Row8<float> {
  f32x4_e4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = *reinterpret_cast<const f32x4_e4*>(p);
    b = *reinterpret_cast<const f32x4_e4*>(p + 4);
  }
  __device__ __forceinline__ float get(int e) const { return e < 4 ? a[e & 3] : b[e & 3]; }
};

// bf16 with round to nearest even; a NaN stays one
__device__ __forceinline__ uint32_t bf16_any(float f) {
  return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)f);
}
__device__ __forceinline__ void store8(bf16_t* p, const float* v) {
  u32x4_e2 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = bf16_any(v[2 * i]) | (bf16_any(v[2 * i + 1]) << 16);
  *reinterpret_cast<u32x4_e2*>(p) = r;
}
__device__ __forceinline__ void store8(float* p, const float* v) {
  *reinterpret_cast<f32x4_e4*>(p) = f32x4_e4{v[0], v[1], v[2], v[3]};
  *reinterpret_cast<f32x4_e4*>(p + 4) = f32x4_e4{v[4], v[5], v[6], v[7]};
}
__device__ __forceinline__ void store1(bf16_t* p, float v) { *p = (bf16_t)bf16_any(v); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }

// Statistics of a part of a row; m is in units of the (biased) logits.
struct Stats {
  float m, l, w, mr, lr;
};

// What e^((z - m) / T) is taken against: a part with nothing above -inf has m =
// -inf, and its differences must still be -inf and not NaN.
__device__ __forceinline__ float against(float m) { return m == -INFINITY ? 0.f : m; }

template <bool REF>
__device__ __forceinline__ Stats merge(const Stats& a, const Stats& b, float c2) {
  Stats r;
  r.m = fmaxf(a.m, b.m);
  const float m = against(r.m);
  const float fa = __builtin_amdgcn_exp2f((a.m - m) * c2), fb = __builtin_amdgcn_exp2f((b.m - m) * c2);
  r.l = a.l * fa + b.l * fb;
  r.w = r.mr = r.lr = 0.f;
  if (REF) {
    r.w = a.w * fa + b.w * fb;
    r.mr = fmaxf(a.mr, b.mr);
    const float n = against(r.mr);
    r.lr = a.lr * __builtin_amdgcn_exp2f((a.mr - n) * c2) + b.lr * __builtin_amdgcn_exp2f((b.mr - n) * c2);
  }
  return r;
}

template <bool REF>
__device__ __forceinline__ Stats shuffle_merge(Stats s, int lanes, float c2) {
  for (int o = lanes / 2; o > 0; o >>= 1) {
    Stats t;
    t.m = __shfl_xor(s.m, o, kWave);
    t.l = __shfl_xor(s.l, o, kWave);
    t.w = REF ? __shfl_xor(s.w, o, kWave) : 0.f;
    t.mr = REF ? __shfl_xor(s.mr, o, kWave) : -INFINITY;
    t.lr = REF ? __shfl_xor(s.lr, o, kWave) : 0.f;
    s = merge<REF>(s, t, c2);
  }
  return s;
}

// Folds 8 entries (those past the row's end are -inf) into the running statistics.
template <bool REF>
__device__ __forceinline__ void fold8(Stats& s, const float* x, const float* y, float c2) {
  float mx = s.m, my = s.mr;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    mx = fmaxf(mx, x[e]);
    if (REF) my = fmaxf(my, y[e]);
  }
  const float m = against(mx), n = against(my);
  const float f = __builtin_amdgcn_exp2f((s.m - m) * c2);
  float l = 0.f, w = 0.f, lr = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float p = __builtin_amdgcn_exp2f((x[e] - m) * c2);
    l += p;
    if (REF) {
      w += p * (p > 0.f ? x[e] - y[e] : 0.f);
      lr += __builtin_amdgcn_exp2f((y[e] - n) * c2);
    }
  }
  s.l = s.l * f + l;
  s.m = mx;
  if (REF) {
    s.w = s.w * f + w;
    s.lr = s.lr * __builtin_amdgcn_exp2f((s.mr - n) * c2) + lr;
    s.mr = my;
  }
}

// A row's outputs from its statistics.
template <typename T, bool REF>
__device__ __forceinline__ void finish(const LogprobArgs& a, int r, const Stats& s) {
  const int y = a.tok[r];
  const float zy = ld(reinterpret_cast<const T*>(a.z) + (size_t)r * a.ldz + y) + (y == a.eos ? a.bias : 0.f);
  const float ll = logf(s.l);
  a.logp[r] = (zy - s.m) * a.inv_t - ll;
  a.lse[r] = s.m * a.inv_t + ll;
  if (REF) {
    const float diff = (s.m - s.mr) * a.inv_t + logf(s.l / s.lr);
    a.diff[r] = diff;
    a.kl[r] = s.w * a.inv_t / s.l - diff;
  }
}

__device__ __forceinline__ void left_out(const LogprobArgs& a, int r, bool ref) {
  a.logp[r] = 0.f;
  a.lse[r] = 0.f;
  if (ref) a.kl[r] = a.diff[r] = 0.f;
}

// NT threads per row part, 256 threads per workgroup.  gridDim.x covers the rows
// (256 / NT per workgroup), gridDim.y the parts of a row.
template <typename T, bool REF, int NT>
__global__ __launch_bounds__(256) void logprob_kernel(LogprobArgs a) {
  constexpr int RPB = 256 / NT;
  __shared__ Stats red[4];
  const int tid = threadIdx.x % NT, r = blockIdx.x * RPB + threadIdx.x / NT;
  const int part = blockIdx.y;
  // a row that is left out is uniform over its NT threads
  const int y = r < a.R ? a.tok[r] : -1;
  const bool live = y >= 0 && y < a.V;
  if (NT == 256 && !live) {
    if (part == 0 && tid == 0) left_out(a, r, REF);
    return;
  }
  const float c2 = a.inv_t * kLog2e;
  Stats s = {-INFINITY, 0.f, 0.f, -INFINITY, 0.f};
  if (live) {
    const int v0 = part * a.chunk, v1 = min(a.V, v0 + a.chunk);
    const T* z = reinterpret_cast<const T*>(a.z) + (size_t)r * a.ldz;
    const T* zr = REF ? reinterpret_cast<const T*>(a.zr) + (size_t)r * a.ldr : nullptr;
    auto biased = [&](float* x, float* q, int v) {
      const int e0 = a.eos - v;
      if (a.eos >= 0 && e0 >= 0 && e0 < 8) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e == e0) {
            x[e] += a.bias;
            if (REF) q[e] += a.bias_r;
          }
      }
    };
    int v = v0 + 8 * tid;
    for (; v + 8 <= v1; v += 8 * NT) {
      Row8<T> c, d;
      c.load(z + v);
      if (REF) d.load(zr + v);
      float x[8], q[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] = c.get(e);
        q[e] = REF ? d.get(e) : 0.f;
      }
      biased(x, q, v);
      fold8<REF>(s, x, q, c2);
    }
    if (v < v1) {
      float x[8], q[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] = v + e < v1 ? ld(z + v + e) : -INFINITY;
        q[e] = REF && v + e < v1 ? ld(zr + v + e) : -INFINITY;
      }
      biased(x, q, v);
      fold8<REF>(s, x, q, c2);
    }
  }
  s = shuffle_merge<REF>(s, NT < kWave ? NT : kWave, c2);
  if (NT > kWave) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x / kWave] = s;
    __syncthreads();
    s = red[0];
#pragma unroll
    for (int i = 1; i < NT / kWave; ++i) s = merge<REF>(s, red[i], c2);
  }
  if (tid != 0 || r >= a.R) return;
  if (!live) {
    left_out(a, r, REF);
  } else if (a.splits > 1) {
    float* p = a.part + ((size_t)r * a.splits + part) * kLogprobPart;
    p[0] = s.m; p[1] = s.l; p[2] = s.w; p[3] = s.mr; p[4] = s.lr;
  } else {
    finish<T, REF>(a, r, s);
  }
}

// Joins a row's parts: a wave per row.
template <typename T, bool REF>
__global__ __launch_bounds__(64) void logprob_join_kernel(LogprobArgs a) {
  const int r = blockIdx.x, lane = threadIdx.x;
  const int y = a.tok[r];
  if (y < 0 || y >= a.V) return;             // written by the first launch
  const float c2 = a.inv_t * kLog2e;
  Stats s = {-INFINITY, 0.f, 0.f, -INFINITY, 0.f};
  for (int i = lane; i < a.splits; i += kWave) {
    const float* p = a.part + ((size_t)r * a.splits + i) * kLogprobPart;
    s = merge<REF>(s, Stats{p[0], p[1], p[2], p[3], p[4]}, c2);
  }
  s = shuffle_merge<REF>(s, kWave, c2);
  if (lane == 0) finish<T, REF>(a, r, s);
}

// Elementwise over a part of a row: gridDim.x parts of kGradChunk entries, gridDim.y rows.
constexpr int kGradChunk = 8192;

template <typename T, bool REF>
__global__ __launch_bounds__(256) void logprob_grad_kernel(LogprobArgs a, int parts) {
  const int r = blockIdx.x / parts, part = blockIdx.x % parts;
  const int y = a.tok[r];
  const bool in = y >= 0 && y < a.V;
  const float g = in ? a.g_logp[r] : 0.f, k = REF && in ? a.g_kl[r] : 0.f;
  const int v0 = part * kGradChunk, v1 = min(a.V, v0 + kGradChunk);
  T* out = reinterpret_cast<T*>(a.grad) + (size_t)r * a.ldg;
  if (g == 0.f && k == 0.f) {
    const float zero[8] = {};
    int v = v0 + 8 * (int)threadIdx.x;
    for (; v + 8 <= v1; v += 2048) store8(out + v, zero);
    for (; v < v1; ++v) store1(out + v, 0.f);
    return;
  }
  const T* z = reinterpret_cast<const T*>(a.z) + (size_t)r * a.ldz;
  const bool kl = REF && k != 0.f;           // uniform over the row
  const T* zr = REF ? reinterpret_cast<const T*>(a.zr) + (size_t)r * a.ldr : nullptr;
  const float lse = a.lse[r];
  // dz_v = p (A + B (z_v - z'_v)), and g / T more at the token
  const float A = a.inv_t * (kl ? -g - k * (a.diff[r] + a.kl[r]) : -g);
  const float B = kl ? a.inv_t * k * a.inv_t : 0.f;
  const float at = g * a.inv_t;
  auto one = [&](float x, float q) {
    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x, a.inv_t, -lse) * kLog2e);
    return REF ? p * (A + B * (kl && p > 0.f ? x - q : 0.f)) : p * A;
  };
  auto marked = [&](float* x, float* q, int v, int id, float b, float br) {
    const int e0 = id - v;
    if (e0 >= 0 && e0 < 8) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e == e0) {
          x[e] += b;
          if (REF) q[e] += br;
        }
    }
  };
  int v = v0 + 8 * (int)threadIdx.x;
  for (; v + 8 <= v1; v += 2048) {
    Row8<T> c, d;
    c.load(z + v);
    if (kl) d.load(zr + v);
    float x[8], q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = c.get(e);
      q[e] = kl ? d.get(e) : 0.f;
    }
    if (a.eos >= 0) marked(x, q, v, a.eos, a.bias, a.bias_r);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = one(x[e], q[e]);
    marked(x, q, v, y, at, 0.f);
    store8(out + v, x);
  }
  for (; v < v1; ++v) {
    const float b = v == a.eos ? a.bias : 0.f, br = v == a.eos ? a.bias_r : 0.f;
    const float x = ld(z + v) + b, q = kl ? ld(zr + v) + br : 0.f;
    store1(out + v, one(x, q) + (v == y ? at : 0.f));
  }
}

template <typename T, bool REF>
hipError_t run(const LogprobArgs& a, hipStream_t st) {
  if (a.splits > 1) {
    logprob_kernel<T, REF, 256><<<dim3(a.R, a.splits), 256, 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    logprob_join_kernel<T, REF><<<a.R, 64, 0, st>>>(a);
  } else if (a.V <= 2048) {
    logprob_kernel<T, REF, 64><<<(a.R + 3) / 4, 256, 0, st>>>(a);
  } else {
    logprob_kernel<T, REF, 256><<<a.R, 256, 0, st>>>(a);
  }
  return hipGetLastError();
}

template <typename T, bool REF>
hipError_t run_grad(const LogprobArgs& a, hipStream_t st) {
  const int parts = (a.V + kGradChunk - 1) / kGradChunk;
  logprob_grad_kernel<T, REF><<<(unsigned)(a.R * (size_t)parts), 256, 0, st>>>(a, parts);
  return hipGetLastError();
}

}  // namespace

int logprob_splits(int R, int V, int* chunk) {
  // Enough workgroups to fill the device (1024 of 256 threads), in parts of at
  // least 4096 entries.
  const int most = (V + 4095) / 4096;
  int want = (1024 + R - 1) / (R > 0 ? R : 1);
  if (want > most) want = most;
  if (want < 1) want = 1;
  int c = (V + want - 1) / want;
  c = (c + 2047) / 2048 * 2048;              // whole passes of 256 threads by 8 entries
  *chunk = c;
  return (V + c - 1) / c;
}

hipError_t launch_logprob(const LogprobArgs& a, int dtype, hipStream_t st) {
  if (dtype == DT_BF16) return a.zr ? run<bf16_t, true>(a, st) : run<bf16_t, false>(a, st);
  return a.zr ? run<float, true>(a, st) : run<float, false>(a, st);
}

hipError_t launch_logprob_backward(const LogprobArgs& a, int dtype, hipStream_t st) {
  if (dtype == DT_BF16) return a.g_kl ? run_grad<bf16_t, true>(a, st) : run_grad<bf16_t, false>(a, st);
  return a.g_kl ? run_grad<float, true>(a, st) : run_grad<float, false>(a, st);
}

}  // namespace tandem
