// k_qk.hip — per-head RMSNorm of q and k with the rotary embedding in the same
// pass, and its gradient.
//
// A lane holds 8 elements i .. i+7 of a head's first half and the 8 rotated with
// them, i + h .. i + h + 7 (h = hd / 2): two 16-byte loads of bf16, no exchange for
// the rotation, and the sums of a head run over its hd / 16 lanes.  The 8 angles of
// a lane belong to its position, so a lane keeps them over all the heads it takes
// of one row.  An angle is turns = position * theta^(-2i/hd) / 2 pi in 64 bits, of
// which the fraction is left: a far position loses nothing.  Memory bound: each
// element once in, once out (backward: two in).  18432 rows of 40 heads of 128 take 71 us, 5.3 TB/s;
// backward 4097 rows of 24 heads 21 us, 3.5 TB/s, and 4 for the gains' sums.
//
// The gains' gradients are summed in a lane over its rows, then over the
// workgroup's lanes in LDS, then over workgroups in a second launch, each in a fixed
// order.
#include "common.h"
#include "update.h"

namespace tandem {
namespace {

template <typename T> struct Vec8;
template <> struct Vec8<bf16_t> {
  u32x4_t r;
  __device__ __forceinline__ void load(const bf16_t* p) { r = *reinterpret_cast<const u32x4_t*>(p); }
  __device__ __forceinline__ float get(int e) const {
    return (e & 1) ? __uint_as_float(r[e >> 1] & 0xFFFF0000u) : __uint_as_float(r[e >> 1] << 16);
  }
  __device__ __forceinline__ static void store(bf16_t* p, const float* v) {
    u32x4_t r;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      r[i] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * i]) |
             ((uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * i + 1]) << 16);
    *reinterpret_cast<u32x4_t*>(p) = r;
  }
};
template <> struct Vec8<float> {
  f32x4_t a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = *reinterpret_cast<const f32x4_t*>(p);
    b = *reinterpret_cast<const f32x4_t*>(p + 4);
  }
  __device__ __forceinline__ float get(int e) const { return e < 4 ? a[e & 3] : b[e & 3]; }
  __device__ __forceinline__ static void store(float* p, const float* v) {
    *reinterpret_cast<f32x4_t*>(p) = f32x4_t{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4_t*>(p + 4) = f32x4_t{v[4], v[5], v[6], v[7]};
  }
};

// cos and sin of 2 pi turns
__device__ __forceinline__ void turn(double turns, float* c, float* s) {
  const float f = (float)(turns - rint(turns));      // [-1/2, 1/2]
  sincospif(2.f * f, s, c);
}

template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}

// How a workgroup's 256 threads lie on rows: LANES = hd / 16 lanes per head, `phases`
// heads of a row side by side, the rest of the heads one after another.
struct Place {
  int row, head, step, lane;      // head: the first of this thread, then every step-th
};
template <int HD>
__device__ __forceinline__ Place place(int phases, int block) {
  constexpr int LANES = HD / 16;
  const int t = threadIdx.x / LANES;
  return Place{block * (256 / LANES / phases) + t / phases, t % phases, phases, (int)threadIdx.x % LANES};
}

template <typename T, int HD>
__global__ __launch_bounds__(256) void qk_kernel(QkArgs a, int phases) {
  constexpr int H = HD / 2, LANES = HD / 16;
  const Place w = place<HD>(phases, blockIdx.x);
  if (w.row >= a.N) return;                  // LANES lanes of a head stay together
  const int i0 = 8 * w.lane;
  const T* src = reinterpret_cast<const T*>(a.qkv) + (size_t)w.row * a.ld;
  Vec8<T> u, v;
  if (w.head < a.nq + a.nkv) {
    u.load(src + w.head * HD + i0);
    v.load(src + w.head * HD + H + i0);
  }
  const double pos = (double)a.pos[w.row];
  float c[8], s[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) turn(pos * a.turns[i0 + e], &c[e], &s[e]);
  T* q = reinterpret_cast<T*>(a.q) + (size_t)w.row * a.ldq;
  T* k = reinterpret_cast<T*>(a.k) + (size_t)w.row * a.ldk;
  const int heads = a.nq + a.nkv;
  for (int h = w.head; h < heads; h += w.step) {
    float x[8], y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = u.get(e);
      y[e] = v.get(e);
    }
    if (h + w.step < heads) {                // the next head's, on their way meanwhile
      u.load(src + (h + w.step) * HD + i0);
      v.load(src + (h + w.step) * HD + H + i0);
    }
    if (a.gq) {
      float q2 = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) q2 += x[e] * x[e] + y[e] * y[e];
      const float r = 1.f / sqrtf(lanes_sum<LANES>(q2) * (1.f / HD) + a.eps);
      const float* g = (h < a.nq ? a.gq : a.gk) + i0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] *= r * g[e];
        y[e] *= r * g[H + e];
      }
    }
    float o[8], p[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      o[e] = x[e] * c[e] - y[e] * s[e];
      p[e] = y[e] * c[e] + x[e] * s[e];
    }
    T* dst = h < a.nq ? q + h * HD : k + (h - a.nq) * HD;
    Vec8<T>::store(dst + i0, o);
    Vec8<T>::store(dst + H + i0, p);
  }
}

template <typename T, int HD>
__global__ __launch_bounds__(256) void qk_backward_kernel(QkArgs a, int phases) {
  constexpr int H = HD / 2, LANES = HD / 16;
  __shared__ float red[2 * HD][256 / LANES];
  // sums of this lane's gains' gradients: [query or key][half][e]
  float dg[2][2][8] = {};
  const int rows = 256 / LANES / phases;     // rows of a workgroup's pass
  for (int block = blockIdx.x; block * rows < a.N; block += gridDim.x) {
    const Place w = place<HD>(phases, block);
    if (w.row >= a.N) break;
    const int i0 = 8 * w.lane, heads = a.nq + a.nkv;
    const T* src = reinterpret_cast<const T*>(a.qkv) + (size_t)w.row * a.ld;
    T* dst = reinterpret_cast<T*>(a.dqkv) + (size_t)w.row * a.ld;
    const T* dq = reinterpret_cast<const T*>(a.dq) + (size_t)w.row * a.ldq;
    const T* dk = reinterpret_cast<const T*>(a.dk) + (size_t)w.row * a.ldk;
    Vec8<T> du, dv, xu, xv;                  // of the head at hand, then of the next one
    auto load = [&](int h) {
      const T* dy = h < a.nq ? dq + h * HD : dk + (h - a.nq) * HD;
      du.load(dy + i0);
      dv.load(dy + H + i0);
      if (a.gq) {
        xu.load(src + h * HD + i0);
        xv.load(src + h * HD + H + i0);
      }
    };
    if (w.head < heads) load(w.head);
    const double pos = (double)a.pos[w.row];
    float c[8], s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) turn(pos * a.turns[i0 + e], &c[e], &s[e]);
    for (int h = w.head; h < heads; h += w.step) {
      const bool is_q = h < a.nq;
      const Vec8<T> u = xu, v = xv;
      float t[8], b[8];                      // the rotation undone: dn
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float p = du.get(e), q = dv.get(e);
        t[e] = p * c[e] + q * s[e];
        b[e] = q * c[e] - p * s[e];
      }
      if (h + w.step < heads) load(h + w.step);
      if (a.gq) {
        float q2 = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) q2 += u.get(e) * u.get(e) + v.get(e) * v.get(e);
        const float r = 1.f / sqrtf(lanes_sum<LANES>(q2) * (1.f / HD) + a.eps);
        const float* g = (is_q ? a.gq : a.gk) + i0;
        float tx = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float gx = t[e] * (u.get(e) * r), gy = b[e] * (v.get(e) * r);
          dg[0][0][e] += is_q ? gx : 0.f;
          dg[0][1][e] += is_q ? gy : 0.f;
          dg[1][0][e] += is_q ? 0.f : gx;
          dg[1][1][e] += is_q ? 0.f : gy;
          t[e] *= g[e];
          b[e] *= g[H + e];
          tx += t[e] * u.get(e) + b[e] * v.get(e);
        }
        const float m = lanes_sum<LANES>(tx) * (1.f / HD) * r * r;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          t[e] = r * (t[e] - u.get(e) * m);
          b[e] = r * (b[e] - v.get(e) * m);
        }
      }
      Vec8<T>::store(dst + h * HD + i0, t);
      Vec8<T>::store(dst + h * HD + H + i0, b);
    }
  }
  if (!a.gq) return;
  const int lane = threadIdx.x % LANES, col = threadIdx.x / LANES;
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (int f = 0; f < 2; ++f)
#pragma unroll
      for (int e = 0; e < 8; ++e) red[n * HD + f * H + 8 * lane + e][col] = dg[n][f][e];
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * HD; i += 256) {
    float sum = 0.f;
    for (int j = 0; j < 256 / LANES; ++j) sum += red[i][j];
    a.part[(size_t)blockIdx.x * 2 * HD + i] = sum;
  }
}

// The workgroups' sums: 8 entries per workgroup, 32 threads each.
__global__ __launch_bounds__(256) void qk_gain_kernel(const float* part, int blocks, int hd, float* dgq, float* dgk) {
  __shared__ double red[32][8];
  const int e = threadIdx.x & 7, g = threadIdx.x >> 3, i = 8 * blockIdx.x + e;
  double sum = 0.0;
#pragma unroll 8
  for (int b = g; b < blocks; b += 32) sum += (double)part[(size_t)b * 2 * hd + i];
  red[g][e] = sum;
  __syncthreads();
  if (g != 0) return;
  sum = 0.0;
#pragma unroll
  for (int j = 0; j < 32; ++j) sum += red[j][e];
  (i < hd ? dgq[i] : dgk[i - hd]) = (float)sum;
}

// Heads of a row side by side: a power of two that leaves each lane about four heads for
// its angles, more of them where the rows alone would not give the device four workgroups
// per compute unit.  4097 rows of 24 heads of 128, backward: 26 us with 4 side by side, 21
// with 8, 24 with 16.
int head_phases(int N, int nq, int nkv, int hd) {
  const int lanes = hd / 16;
  int p = 1;
  while (2 * p * lanes <= 256 && p < nq + nkv &&
         (8 * p <= nq + nkv ? 2 * p * lanes <= kWave : (int64_t)N * p * lanes < 1024 * 256))
    p *= 2;
  return p;
}

template <typename T, int HD>
hipError_t run(const QkArgs& a, hipStream_t st) {
  const int ph = head_phases(a.N, a.nq, a.nkv, HD);
  qk_kernel<T, HD><<<(unsigned)qk_blocks(a.N, a.nq, a.nkv, HD), 256, 0, st>>>(a, ph);
  return hipGetLastError();
}
template <typename T, int HD>
hipError_t run_backward(const QkArgs& a, hipStream_t st) {
  const int ph = head_phases(a.N, a.nq, a.nkv, HD), blocks = qk_backward_blocks(a.N, a.nq, a.nkv, HD);
  qk_backward_kernel<T, HD><<<blocks, 256, 0, st>>>(a, ph);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.gq) return e;
  qk_gain_kernel<<<2 * HD / 8, 256, 0, st>>>(a.part, blocks, HD, a.dgq, a.dgk);
  return hipGetLastError();
}

}  // namespace

int64_t qk_blocks(int N, int nq, int nkv, int hd) {
  const int rows = 256 / (hd / 16) / head_phases(N, nq, nkv, hd);
  return ((int64_t)N + rows - 1) / rows;
}
int qk_backward_blocks(int N, int nq, int nkv, int hd) {
  const int64_t most = N > 0 ? qk_blocks(N, nq, nkv, hd) : 1;        // no rows: one workgroup writes sums of 0
  return most < 1024 ? (int)most : 1024;
}

#define TANDEM_QK_DISPATCH(fn)                                             \
  switch (a.hd) {                                                          \
    case 32: return dtype == DT_BF16 ? fn<bf16_t, 32>(a, st) : fn<float, 32>(a, st);   \
    case 64: return dtype == DT_BF16 ? fn<bf16_t, 64>(a, st) : fn<float, 64>(a, st);   \
    case 128: return dtype == DT_BF16 ? fn<bf16_t, 128>(a, st) : fn<float, 128>(a, st); \
  }                                                                        \
  return hipErrorInvalidValue;

hipError_t launch_qk(const QkArgs& a, int dtype, hipStream_t st) { TANDEM_QK_DISPATCH(run) }
hipError_t launch_qk_backward(const QkArgs& a, int dtype, hipStream_t st) { TANDEM_QK_DISPATCH(run_backward) }

}  // namespace tandem
