// k_logprob.hip — log-probs of given tokens from logits, the divergence from a
// reference model's logits, and the gradient of both with respect to the logits.
//
// Forward: one pass over a row with the running maximum m and the sums taken against
// it, l = sum e^(s - m) and (with a reference) w = sum e^(s - m) (s - s'), beside the
// reference's own m', l'.  Then lse = m + log l, logp = (s_y - m) - log l,
// lse - lse' = (m - m') + log l - log l' and KL = w / l - (lse - lse').  The maxima are kept
// in powers of two, rounded once, and everything is taken against the rounded numbers; the
// differences are formed in 64 bits, once a row, so that a small KL keeps its digits.
// Backward: p = e^(s - lse) again, elementwise; rows whose lse is so large that its own rounding
// counts are summed anew.
// Logits are converted to float32 as they are read.
#include "common.h"
#include "update.h"

namespace tandem {
namespace {

// 8 entries per load: rows start at any multiple of an element's size
typedef uint32_t u32x4_e2 __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_e4 __attribute__((ext_vector_type(4), aligned(4)));

constexpr float kLog2e = 1.4426950408889634f;

// What the powers of two bear, in them.  A row's maximum is rounded by half a step: up to kMost
// that changes the sums by a factor of 2 at most, which their logarithm takes back; from 2^30 on
// it takes them out of float32's range.  Rows beyond, and those with nothing above -inf, are
// taken in units of the logits (logit_row).  From kFar on the differences of the two models'
// logits and their weights are summed in 64 bits alone, since a KL is what is left of their mean
// after the models' offsets.
constexpr float kMost = 0x1p24f, kFar = 0x1p10f;

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

// Statistics of a part of a row; the maxima in powers of two.  The sums are of 64 bits, what
// is added to them the float32 sum of 8 entries: a KL divergence is the small difference of
// what they hold (of 151936 logits and a reference near by it was off by 1.5e-6 of itself
// with float32 sums, 3.8e-7 with these).
struct Stats {
  float m, mr;
  double l, w, lr;
};
static_assert(sizeof(Stats) == kLogprobPart * sizeof(float), "a part in the workspace");
__device__ __forceinline__ Stats no_stats() { return Stats{-INFINITY, -INFINITY, 0.0, 0.0, 0.0}; }

// What a score is taken against: a part with nothing above -inf has m = -inf, and its
// differences must still be -inf and not NaN.
__device__ __forceinline__ float against(float m) { return m == -INFINITY ? 0.f : m; }

// The sums taken against higher maxima.  A weighted difference may be infinite (the reference
// excludes an entry) where what it is weighted with vanishes.
template <bool REF>
__device__ __forceinline__ void raise(Stats& s, float m, float mr) {
  const float f = __builtin_amdgcn_exp2f(s.m - against(m));
  s.l *= (double)f;
  s.m = m;
  if (REF) {
    s.w = f > 0.f ? s.w * (double)f : 0.0;
    s.lr *= (double)__builtin_amdgcn_exp2f(s.mr - against(mr));
    s.mr = mr;
  }
}

template <bool REF>
__device__ __forceinline__ Stats wave_merge(Stats s) {
  raise<REF>(s, wave_max(s.m), REF ? wave_max(s.mr) : 0.f);
#pragma unroll
  for (int o = kWave / 2; o > 0; o >>= 1) {
    s.l += __shfl_xor(s.l, o, kWave);
    if (REF) {
      s.w += __shfl_xor(s.w, o, kWave);
      s.lr += __shfl_xor(s.lr, o, kWave);
    }
  }
  return s;
}

// 8 entries of a row and of the reference's.
template <bool REF> struct Eight {
  float x[8], y[8];

  template <typename T> __device__ __forceinline__ void take(const Row8<T>& c, const Row8<T>& d) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = c.get(e);
      y[e] = REF ? d.get(e) : 0.f;
    }
  }
  // entries v .. v1 - 1 of fewer than 8; -inf for the others
  template <typename T> __device__ __forceinline__ void some(const T* z, const T* zr, int v, int v1) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = v + e < v1 ? ld(z + v + e) : -INFINITY;
      y[e] = REF && v + e < v1 ? ld(zr + v + e) : -INFINITY;
    }
  }
  // a, b added to entry i where it is one of these
  __device__ __forceinline__ void add(int i, float a, float b) {
    if ((unsigned)i >= 8u) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] += e == i ? a : 0.f;
      if (REF) y[e] += e == i ? b : 0.f;
    }
  }
};

// Folds 8 entries into the running statistics: some 13 vector operations per logit and its
// reference, an exponential counting two.  `far` is whether a maximum of this wave passes kFar.
template <bool REF>
__device__ __forceinline__ void fold(Stats& s, bool& far, const Eight<REF>& a, float c2) {
  float mx = a.x[0], my = a.y[0], lo = fminf(a.x[0], a.y[0]);
#pragma unroll
  for (int e = 1; e < 8; ++e) {
    mx = fmaxf(mx, a.x[e]);
    if (REF) {
      my = fmaxf(my, a.y[e]);
      lo = fminf(lo, fminf(a.x[e], a.y[e]));
    }
  }
  mx *= c2;
  my *= c2;
  if (__any(mx > s.m || (REF && my > s.mr))) {             // seldom, but at a row's beginning
    raise<REF>(s, fmaxf(s.m, mx), REF ? fmaxf(s.mr, my) : 0.f);
    if (REF) far = __any(fmaxf(fabsf(against(s.m)), fabsf(against(s.mr))) > kFar);
  }
  const float m = -against(s.m), n = -against(s.mr);
  float p[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(a.x[e], c2, m));
  if (REF) {
    float lr = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) lr += __builtin_amdgcn_exp2f(__builtin_fmaf(a.y[e], c2, n));
    s.lr += (double)lr;
    // scores of -inf on either side: an entry of probability 0 adds nothing, whatever they differ by
    if (__any(far || lo == -INFINITY)) {
      if (__any(far)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          s.l += (double)p[e];
          s.w += p[e] > 0.f ? (double)p[e] * ((double)a.x[e] - (double)a.y[e]) : (double)p[e];
        }
        return;
      }
      float l = 0.f, w = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        l += p[e];
        w += p[e] > 0.f ? p[e] * (a.x[e] - a.y[e]) : p[e];
      }
      s.l += (double)l;
      s.w += (double)w;
      return;
    }
  }
  float l = 0.f, w = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    l += p[e];
    if (REF) w += p[e] * (a.x[e] - a.y[e]);
  }
  s.l += (double)l;
  if (REF) s.w += (double)w;
}

// A row (or its reference's) whose largest score the powers of two do not bear, or that has none
// above -inf: in units of the logits, by one wave.  1024 rows of 151936 bf16 logits at T = 1e-7, all of them such,
// 443 us and with a reference 676, where T = 1 takes 60 and 118.
template <typename T, bool REF>
__device__ __forceinline__ void logit_row(const LogprobArgs& a, int r, int lane) {
  const T* z = reinterpret_cast<const T*>(a.z) + (size_t)r * a.ldz;
  const T* zr = REF ? reinterpret_cast<const T*>(a.zr) + (size_t)r * a.ldr : nullptr;
  // use() of the row's entries, 8 at a time
  auto each = [&](auto&& use) {
    for (int v = 8 * lane; v < a.V; v += 8 * kWave) {
      Eight<REF> e;
      if (v + 8 <= a.V) {
        Row8<T> c, d;
        c.load(z + v);
        if (REF) d.load(zr + v);
        e.take(c, d);
      } else {
        e.some(z, zr, v, a.V);
      }
      if (a.eos >= 0) e.add(a.eos - v, a.bias, a.bias_r);
      use(e);
    }
  };
  float m = -INFINITY, n = -INFINITY;
  each([&](const Eight<REF>& e) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      m = fmaxf(m, e.x[i]);
      if (REF) n = fmaxf(n, e.y[i]);
    }
  });
  m = wave_max(m);
  n = wave_max(n);
  // the differences against the maxima's: their common part would leave 64 bits few digits of the KL
  const double m0 = (double)against(m), n0 = (double)against(n);
  double l = 0.0, w = 0.0, lr = 0.0;
  each([&](const Eight<REF>& e) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float p = expf((e.x[i] - against(m)) * a.inv_t);
      l += (double)p;
      if (REF) {
        w += p > 0.f ? (double)p * (((double)e.x[i] - m0) - ((double)e.y[i] - n0)) : (double)p;
        lr += (double)expf((e.y[i] - against(n)) * a.inv_t);
      }
    }
  });
#pragma unroll
  for (int o = kWave / 2; o > 0; o >>= 1) {
    l += __shfl_xor(l, o, kWave);
    w += __shfl_xor(w, o, kWave);
    lr += __shfl_xor(lr, o, kWave);
  }
  if (lane != 0) return;
  const int y = a.tok[r];
  const float zy = ld(z + y) + (y == a.eos ? a.bias : 0.f);
  const double t = (double)a.inv_t, ll = log(l);
  a.logp[r] = (float)(((double)zy - (double)m) * t - ll);
  a.lse[r] = (float)((double)m * t + ll);
  if (REF) {
    const double sums = ll - log(lr);
    a.diff[r] = (float)(((double)m - (double)n) * t + sums);
    a.kl[r] = (float)(w * t / l - sums);
  }
}

// A row's outputs from its statistics, by one wave.
template <typename T, bool REF>
__device__ __forceinline__ void finish(const LogprobArgs& a, int r, const Stats& s, int lane) {
  if (!(fabsf(s.m) <= kMost) || (REF && !(fabsf(s.mr) <= kMost))) {
    logit_row<T, REF>(a, r, lane);
    return;
  }
  if (lane != 0) return;
  const int y = a.tok[r];
  const float zy = ld(reinterpret_cast<const T*>(a.z) + (size_t)r * a.ldz + y) + (y == a.eos ? a.bias : 0.f);
  // the maxima back into nats by the factor that took them out of them, as it was rounded
  const float c2 = a.inv_t * kLog2e;
  const double nats = (double)a.inv_t / (double)c2, ll = log(s.l);
  a.logp[r] = (float)(((double)zy * (double)c2 - (double)s.m) * nats - ll);
  a.lse[r] = (float)((double)s.m * nats + ll);
  if (REF) {
    const double diff = ((double)s.m - (double)s.mr) * nats + (ll - log(s.lr));
    a.diff[r] = (float)diff;
    a.kl[r] = (float)(s.w * (double)a.inv_t / s.l - diff);
  }
}

__device__ __forceinline__ void left_out(const LogprobArgs& a, int r, bool ref) {
  a.logp[r] = 0.f;
  a.lse[r] = 0.f;
  if (ref) a.kl[r] = a.diff[r] = 0.f;
}

// NT threads per row: a wave, four rows to a workgroup, or a workgroup.  gridDim.x covers the
// rows, gridDim.y the parts of a row.  A thread's next 8 entries are on their way while it
// folds the last ones.
//
// Bound by HBM, with the vector unit close behind (13 operations for the 4
// bytes of a bf16 logit and its reference): 2048 rows of 151936, a fifth left out, 201 us, 5.0 TB/s.
template <typename T, bool REF, int NT>
__global__ __launch_bounds__(256) void logprob_kernel(LogprobArgs a) {
  constexpr int RPB = 256 / NT;
  __shared__ Stats red[4];
  const int tid = threadIdx.x % NT, lane = threadIdx.x & 63, r = blockIdx.x * RPB + threadIdx.x / NT;
  // a row that is left out is uniform over its NT threads
  const int y = r < a.R ? a.tok[r] : -1;
  const bool live = y >= 0 && y < a.V;
  if (!live) {
    if (blockIdx.y == 0 && tid == 0 && r < a.R) left_out(a, r, REF);
    return;
  }
  const float c2 = a.inv_t * kLog2e;
  Stats s = no_stats();
  bool far = false;
  const int v0 = blockIdx.y * a.chunk, v1 = min(a.V, v0 + a.chunk);
  const T* z = reinterpret_cast<const T*>(a.z) + (size_t)r * a.ldz;
  const T* zr = REF ? reinterpret_cast<const T*>(a.zr) + (size_t)r * a.ldr : nullptr;
  int v = v0 + 8 * tid;
  Row8<T> c, d;
  if (v + 8 <= v1) {
    c.load(z + v);
    if (REF) d.load(zr + v);
  }
  for (; v + 8 <= v1; v += 8 * NT) {
    Eight<REF> e;
    e.take(c, d);
    if (v + 8 * NT + 8 <= v1) {
      c.load(z + v + 8 * NT);
      if (REF) d.load(zr + v + 8 * NT);
    }
    if (a.eos >= 0) e.add(a.eos - v, a.bias, a.bias_r);
    fold<REF>(s, far, e, c2);
  }
  if (v < v1) {
    Eight<REF> e;
    e.some(z, zr, v, v1);
    if (a.eos >= 0) e.add(a.eos - v, a.bias, a.bias_r);
    fold<REF>(s, far, e, c2);
  }
  s = wave_merge<REF>(s);
  if (NT > kWave) {
    if (lane == 0) red[threadIdx.x / kWave] = s;
    __syncthreads();
    if (threadIdx.x >= kWave) return;
    s = wave_merge<REF>(lane < NT / kWave ? red[lane] : no_stats());
  }
  if (a.splits > 1) {
    if (lane == 0) {
      reinterpret_cast<Stats*>(a.part)[(size_t)r * a.splits + blockIdx.y] = s;
    }
  } else {
    finish<T, REF>(a, r, s, lane);
  }
}

// Joins a row's parts: a wave per row.
template <typename T, bool REF>
__global__ __launch_bounds__(64) void logprob_join_kernel(LogprobArgs a) {
  const int r = blockIdx.x, lane = threadIdx.x;
  const int y = a.tok[r];
  if (y < 0 || y >= a.V) return;             // written by the first launch
  Stats s = no_stats();
  for (int i = lane; i < a.splits; i += kWave) {
    Stats t = reinterpret_cast<const Stats*>(a.part)[(size_t)r * a.splits + i];
    const float m = fmaxf(s.m, t.m), mr = fmaxf(s.mr, t.mr);
    raise<REF>(s, m, mr);
    raise<REF>(t, m, mr);
    s.l += t.l;
    s.w += t.w;
    s.lr += t.lr;
  }
  finish<T, REF>(a, r, wave_merge<REF>(s), lane);
}

// Elementwise over kGradChunk entries of a row, bound by HBM: 1024 rows of 151936 bf16 logits
// and their reference, a fifth left out, 151 us, 5.4 TB/s; 509 rows of 32001 float32 logits without
// one 25 us, 4.6 TB/s.
constexpr int kGradChunk = 8192;

// Up to what log-sum-exp, and mean difference of the two models' scores, a row's gradient takes
// them as they were rounded: half a step of lse is an error of p, in bf16 2^-13, a 32nd of the
// result's own rounding, in float32 2^-17.
template <typename T> constexpr float kGradMost = sizeof(T) == 2 ? 4096.f : 256.f;

// What a row's gradient is made of: dz_v = p (A + B (z_v - z'_v)), and `at` more at the token.
struct RowGrad {
  float A, B, at, lse, inv_t;
};
template <bool KL>
__device__ __forceinline__ float grad_of(const RowGrad& g, float x, float y) {
  // the difference first: what is rounded after it is of its size, not of the log-sum-exp's
  const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x, g.inv_t, -g.lse) * kLog2e);
  // an entry of probability 0 has no gradient, whatever the scores differ by
  return KL ? (p > 0.f ? p * __builtin_fmaf(g.B, x - y, g.A) : p) : p * g.A;
}

template <typename T, bool KL>
__device__ __forceinline__ void grad_chunk(const LogprobArgs& a, const RowGrad& g, const T* z, const T* zr, T* out,
                                           int y, int v0, int v1) {
  int v = v0 + 8 * (int)threadIdx.x;
  constexpr int STEP = 8 * 256;
  // two vectors of 8 at a time: both are on their way before the first is needed
  for (; v + STEP + 8 <= v1; v += 2 * STEP) {
    Row8<T> c[2], d[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      c[i].load(z + v + i * STEP);
      if (KL) d[i].load(zr + v + i * STEP);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int u = v + i * STEP;
      Eight<KL> e;
      e.take(c[i], d[i]);
      if (a.eos >= 0) e.add(a.eos - u, a.bias, a.bias_r);
#pragma unroll
      for (int k = 0; k < 8; ++k) e.x[k] = grad_of<KL>(g, e.x[k], e.y[k]);
      e.add(y - u, g.at, 0.f);
      store8(out + u, e.x);
    }
  }
  for (; v + 8 <= v1; v += STEP) {
    Row8<T> c, d;
    c.load(z + v);
    if (KL) d.load(zr + v);
    Eight<KL> e;
    e.take(c, d);
    if (a.eos >= 0) e.add(a.eos - v, a.bias, a.bias_r);
#pragma unroll
    for (int k = 0; k < 8; ++k) e.x[k] = grad_of<KL>(g, e.x[k], e.y[k]);
    e.add(y - v, g.at, 0.f);
    store8(out + v, e.x);
  }
  for (; v < v1; ++v) {
    const bool eos = v == a.eos;
    const float x = ld(z + v) + (eos ? a.bias : 0.f), q = KL ? ld(zr + v) + (eos ? a.bias_r : 0.f) : 0.f;
    store1(out + v, grad_of<KL>(g, x, q) + (v == y ? g.at : 0.f));
  }
}

__device__ __forceinline__ double workgroup_sum(double v, double* room) {
#pragma unroll
  for (int o = kWave / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  if ((threadIdx.x & 63) == 0) room[threadIdx.x / kWave] = v;
  __syncthreads();
  return (room[0] + room[1]) + (room[2] + room[3]);
}

// The same of other rows, and of those without a distribution: maximum, sum and mean difference
// anew, in units of the logits, and from them dz_v = (g ([v = y] - p) + k p ((s_v - s'_v) - mean)) / T.
// One workgroup takes the whole row: the gradient may take the logits' place.  1024 rows of 151936
// bf16 logits at T = 1e-3, all of them such, 539 us and with a reference 763, where T = 1 takes 115 and 177.
template <typename T, bool KL>
__device__ __forceinline__ void logit_grad(const LogprobArgs& a, float g, float k, const T* z, const T* zr, T* out,
                                           int y) {
  __shared__ float red[2][4];
  __shared__ double sums[2][4];
  // use(first entry, entries) of the row, 8 at a time
  auto each = [&](auto&& use) {
    for (int v = 8 * (int)threadIdx.x; v < a.V; v += 8 * 256) {
      Eight<KL> e;
      if (v + 8 <= a.V) {
        Row8<T> c, d;
        c.load(z + v);
        if (KL) d.load(zr + v);
        e.take(c, d);
      } else {
        e.some(z, zr, v, a.V);
      }
      if (a.eos >= 0) e.add(a.eos - v, a.bias, a.bias_r);
      use(v, e);
    }
  };
  float m = -INFINITY, n = -INFINITY;
  each([&](int, const Eight<KL>& e) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      m = fmaxf(m, e.x[i]);
      if (KL) n = fmaxf(n, e.y[i]);
    }
  });
  m = wave_max(m);
  n = wave_max(n);
  if ((threadIdx.x & 63) == 0) {
    red[0][threadIdx.x / kWave] = m;
    red[1][threadIdx.x / kWave] = n;
  }
  __syncthreads();
  m = against(fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3])));
  n = against(fmaxf(fmaxf(red[1][0], red[1][1]), fmaxf(red[1][2], red[1][3])));
  // a difference of the models' logits against that of their maxima, which may be far larger
  auto apart = [&](float x, float y) { return ((double)x - (double)m) - ((double)y - (double)n); };
  double l = 0.0, w = 0.0;
  each([&](int, const Eight<KL>& e) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float p = expf((e.x[i] - m) * a.inv_t);
      l += (double)p;
      // an entry of probability 0 adds nothing, whatever the scores differ by; nor has it a gradient
      if (KL) w += p > 0.f ? (double)p * apart(e.x[i], e.y[i]) : (double)p;
    }
  });
  l = workgroup_sum(l, sums[0]);
  const double mean = KL ? workgroup_sum(w, sums[1]) / l : 0.0, t = (double)a.inv_t;
  each([&](int v, const Eight<KL>& e) {
    float r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const double p = (double)expf((e.x[i] - m) * a.inv_t) / l;
      double d = (double)g * ((v + i == y ? 1.0 : 0.0) - p);
      if (KL && !(p == 0.0)) d += (double)k * p * (t * (apart(e.x[i], e.y[i]) - mean));
      r[i] = (float)(d * t);
    }
    if (v + 8 <= a.V) {
      store8(out + v, r);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (v + i < a.V) store1(out + v + i, r[i]);
    }
  });
}

template <typename T, bool REF>
__global__ __launch_bounds__(256) void logprob_grad_kernel(LogprobArgs a, int parts) {
  const int r = blockIdx.x / parts, part = blockIdx.x % parts;
  const int y = a.tok[r];
  const bool in = y >= 0 && y < a.V;
  const float g = in ? a.g_logp[r] : 0.f, k = REF && in ? a.g_kl[r] : 0.f;
  const int v0 = part * kGradChunk, v1 = min(a.V, v0 + kGradChunk);
  T* out = reinterpret_cast<T*>(a.grad) + (size_t)r * a.ldg;
  if (g == 0.f && k == 0.f) {
    float zero[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) zero[e] = 0.f;
    int v = v0 + 8 * (int)threadIdx.x;
    for (; v + 8 <= v1; v += 2048) store8(out + v, zero);
    for (; v < v1; ++v) store1(out + v, 0.f);
    return;
  }
  const T* z = reinterpret_cast<const T*>(a.z) + (size_t)r * a.ldz;
  const T* zr = REF ? reinterpret_cast<const T*>(a.zr) + (size_t)r * a.ldr : nullptr;
  const float at = g * a.inv_t, lse = a.lse[r];
  const bool near = fabsf(lse) < kGradMost<T>;             // false of a NaN
  if (REF && k != 0.f) {
    const float mean = a.diff[r] + a.kl[r], B = a.inv_t * k * a.inv_t;
    // B of a temperature below 1e-19 may be infinite, and what it is times 0
    if (near && fabsf(mean) < kGradMost<T> && fabsf(B) < INFINITY) {
      const RowGrad q = {a.inv_t * (-g - k * mean), B, at, lse, a.inv_t};
      grad_chunk<T, true>(a, q, z, zr, out, y, v0, v1);
    } else if (part == 0) {
      logit_grad<T, true>(a, g, k, z, zr, out, y);
    }
  } else if (near) {
    const RowGrad q = {-at, 0.f, at, lse, a.inv_t};
    grad_chunk<T, false>(a, q, z, nullptr, out, y, v0, v1);
  } else if (part == 0) {
    logit_grad<T, false>(a, g, 0.f, z, nullptr, out, y);
  }
}

template <typename T, bool REF>
hipError_t run(const LogprobArgs& a, hipStream_t st) {
  if (a.splits > 1) {
    logprob_kernel<T, REF, 256><<<dim3(a.R, a.splits), 256, 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    logprob_join_kernel<T, REF><<<a.R, 64, 0, st>>>(a);
  } else if (a.V <= 2048) {                  // a short row is a wave's
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
  // Few rows are cut into parts of at least a pass of 256 threads by 8 entries, about 1024
  // workgroups together: one compute unit alone reads at some 46 GB/s.  Four rows of 151936
  // float32 logits and their reference, replayed from a graph: 7.8 us with the join (9.6 in parts
  // of 8192; whole 26 by 1024 threads each).  A row of fewer than two parts of 8192 stays whole,
  // which spares the second launch: eight of 8192 6.6 us, in parts 7.1, and 11.3 and 15.6 where
  // each call is the host's.
  int want = (1024 + R - 1) / (R > 0 ? R : 1);
  if (want < 2 || V < 2 * 8192) {
    *chunk = V;
    return 1;
  }
  if (want > V / 2048) want = V / 2048;
  int c = (V + want - 1) / want;
  c = (c + 2047) / 2048 * 2048;              // whole passes
  *chunk = c;
  return (V + c - 1) / c;
}

int64_t logprob_blocks(int R, int V) {
  int chunk = 0;
  const int splits = logprob_splits(R, V, &chunk);
  const int64_t forward = splits > 1 ? (int64_t)R * splits : V <= 2048 ? ((int64_t)R + 3) / 4 : R;
  const int64_t backward = (int64_t)R * ((V + kGradChunk - 1) / kGradChunk);
  return forward > backward ? forward : backward;
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
