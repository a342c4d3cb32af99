// k_flash.hip — causal grouped-query attention over packed sequences: the forward
// pass with its log-sum-exps, and the backward pass, which computes the
// probabilities again.
//
// Scores are formed with the 32 x 32 matrix instructions, on blocks of 32 queries by
// 32 keys.  Their result layout puts one column in a lane (column = lane % 32) and 16
// of the 32 rows in its registers (row = 8 (i / 4) + 4 (lane / 32) + i % 4 of
// register i); that is, up to the order of the summed index, the layout in which the
// next product takes its right operand.  So probabilities and their gradients go
// from one product into the next in registers, and only the left operands, which the
// waves of a workgroup share, pass through LDS: by rows (summed over the head
// dimension) and transposed (summed over positions).
//   forward   S^T = K Q^T, O^T += V^T P^T          a column is a query
//   dQ        S^T, dP^T = V dO^T, dQ^T += K^T dS^T  a column is a query
//   dK, dV    S = Q K^T, dP = dO V^T, dV^T += dO^T P, dK^T += Q^T dS   a column is a key
// dQ and dK/dV are separate passes: each output is summed by one wave in a fixed
// order (no atomics), for 7 products where one pass would take 5.
// float32 models run the same code on the float32 matrix instructions.
//
// In bf16 models the probabilities and score gradients are rounded to bf16 where the next
// product takes them (float32 operands run at a sixteenth of the rate), and dout . out takes the
// output as it was rounded: 1.7e-3 and 1.0e-3 of the norm of dQ and dK, beside the 1.7e-3 of
// their own rounding; 1.5e-3 of the output's norm for its probabilities, beside 1.6e-3.
// Scores, sums, maxima and accumulators are float32.
#include <algorithm>

#include "common.h"
#include "update.h"
#include "update_plan.h"

namespace tandem {
namespace {

typedef short s16x4_v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_v lds_s16x4_v;

constexpr int kRows = 64;        // rows of a staged tile
constexpr int kWaves = kFlashWaves;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ f32x16_t zero16() {
  f32x16_t z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.f;
  return z;
}
// row of register i in a 32 x 32 result, h = lane / 32
__device__ __forceinline__ int result_row(int i, int h) { return 8 * (i >> 2) + 4 * h + (i & 3); }

// A tile of rows of HD elements in LDS, in 16-byte chunks whose place is permuted by row
// (an exclusive or with `turn`) so that both readers spread over the 64 banks: 16
// consecutive rows' chunks c (rows as left operand), and 4 rows by 64 bytes (transposed).
// The permutation repeats after 16 rows, so a lane's places in a tile are a few offsets
// (Lanes) plus constants.
template <typename T, int HD> struct Ops;

template <int HD> struct Ops<bf16_t, HD> {
  static constexpr int CPR = HD / 8;                       // chunks per row
  static constexpr int ROW = HD * 2;                       // bytes per row
  static constexpr int WGS = 2;                            // workgroups per compute unit (registers): dQ
  static constexpr int FWD = HD == 128 ? 3 : 4;            // of the forward pass
  struct Right { bf16x8_t b[HD / 16]; };                   // 32 columns, summed over the head dimension
  struct Prob { bf16x8_t b[2]; };                          // 32 x 32, summed over its rows
  struct Lanes { int rows[HD / 16], cols[2][HD / 32]; };

  __device__ __forceinline__ static int turn(int row) {
    return HD == 128 ? ((row & 3) << 2) | ((row >> 2) & 3)
                     : HD == 64 ? (((row >> 1) & 1) << 2) | ((row >> 2) & 3) : (row >> 2) & 3;
  }
  __device__ __forceinline__ static int at(int row, int c) { return row * ROW + ((c ^ turn(row)) << 4); }
  __device__ __forceinline__ static Lanes lanes(int lane) {
    Lanes r;
#pragma unroll
    for (int k = 0; k < HD / 16; ++k) r.rows[k] = at(lane & 31, 2 * k + (lane >> 5));
    const int g = (lane >> 4) & 1, i = lane & 15;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
      for (int b = 0; b < 2; ++b)
        r.cols[b][d] = at(8 * b + 4 * (lane >> 5) + (i >> 2), 4 * d + 2 * g + ((i & 3) >> 1)) + (i & 1) * 8;
    return r;
  }
  // p: the column's row in memory
  __device__ __forceinline__ static void load_right(Right& r, const bf16_t* p, int h) {
#pragma unroll
    for (int k = 0; k < HD / 16; ++k) r.b[k] = *reinterpret_cast<const bf16x8_t*>(p + 16 * k + 8 * h);
  }
  __device__ __forceinline__ static Prob pack(const float* p) {
    Prob r;
#pragma unroll
    for (int i = 0; i < 16; ++i) r.b[i >> 3][i & 7] = (__bf16)p[i];
    return r;
  }
  // this lane's part of the sum of a b over the head dimension
  __device__ __forceinline__ static float dot(const Right& a, const Right& b) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < HD / 16; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) s += (float)a.b[k][e] * (float)b.b[k][e];
    return s;
  }
  // acc + tile rows r0 .. r0 + 31 by right; r0 is a multiple of 32
  __device__ __forceinline__ static f32x16_t by_rows(const char* tile, const Lanes& at, int r0, const Right& right,
                                                     f32x16_t acc = zero16()) {
#pragma unroll
    for (int k = 0; k < HD / 16; ++k) {
      const bf16x8_t a = *reinterpret_cast<const bf16x8_t*>(tile + at.rows[k] + r0 * ROW);
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, right.b[k], acc, 0, 0, 0);
    }
    return acc;
  }
  // acc[d / 32] += (tile rows r0 .. r0 + 31)^T by p.  A transposing read gives a lane four
  // positions of its dimension.
  __device__ __forceinline__ static void transposed(f32x16_t* acc, const char* tile, const Lanes& at, int r0,
                                                    const Prob& p) {
    typedef short s16x8_v __attribute__((ext_vector_type(8)));
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int d = 0; d < HD / 32; ++d) {
        const int to = (r0 + 16 * kb) * ROW;
        const s16x4_v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_v*)(tile + at.cols[0][d] + to));
        const s16x4_v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_v*)(tile + at.cols[1][d] + to));
        const s16x8_v a = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), p.b[kb], acc[d], 0, 0, 0);
      }
  }
};

template <int HD> struct Ops<float, HD> {
  static constexpr int CPR = HD / 4;
  static constexpr int ROW = HD * 4;
  static constexpr int WGS = HD == 128 ? 1 : 2;
  static constexpr int FWD = HD == 128 ? 2 : HD == 64 ? 3 : 4;
  struct Right { float b[HD / 2]; };
  struct Prob { float b[16]; };
  struct Lanes { int rows[HD / 8], cols[2][4]; };

  __device__ __forceinline__ static int turn(int row) {
    return HD == 32 ? (row >> 1) & 7 : (((row >> 2) & 1) << 3) | (((row >> 3) & 1) << 2) | (row & 3);
  }
  __device__ __forceinline__ static int at(int row, int c) { return row * ROW + ((c ^ turn(row)) << 4); }
  __device__ __forceinline__ static Lanes lanes(int lane) {
    Lanes r;
    const int h = lane >> 5, c = lane & 31;
#pragma unroll
    for (int k = 0; k < HD / 8; ++k) r.rows[k] = at(c, h * (HD / 8) + k);
    // row 8 b + 4 h + i, dimension c; 8 chunks on (32 dimensions) the permutation is the same
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) r.cols[b][i] = at(8 * b + 4 * h + i, c >> 2) + (c & 3) * 4;
    return r;
  }
  __device__ __forceinline__ static void load_right(Right& r, const float* p, int h) {
#pragma unroll
    for (int k = 0; k < HD / 8; ++k) {
      const f32x4_t v = *reinterpret_cast<const f32x4_t*>(p + h * (HD / 2) + 4 * k);
#pragma unroll
      for (int e = 0; e < 4; ++e) r.b[4 * k + e] = v[e];
    }
  }
  __device__ __forceinline__ static Prob pack(const float* p) {
    Prob r;
#pragma unroll
    for (int i = 0; i < 16; ++i) r.b[i] = p[i];
    return r;
  }
  __device__ __forceinline__ static float dot(const Right& a, const Right& b) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < HD / 2; ++k) s += a.b[k] * b.b[k];
    return s;
  }
  __device__ __forceinline__ static f32x16_t by_rows(const char* tile, const Lanes& at, int r0, const Right& right,
                                                     f32x16_t acc = zero16()) {
#pragma unroll
    for (int k = 0; k < HD / 8; ++k) {
      const f32x4_t a = *reinterpret_cast<const f32x4_t*>(tile + at.rows[k] + r0 * ROW);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], right.b[4 * k + e], acc, 0, 0, 0);
    }
    return acc;
  }
  __device__ __forceinline__ static void transposed(f32x16_t* acc, const char* tile, const Lanes& at, int r0,
                                                    const Prob& p) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
      for (int d = 0; d < HD / 32; ++d) {
        // the chunk 8 d + c, whose exclusive or reaches its fourth bit where rows are that long
        const int row = at.cols[(i >> 2) & 1][i & 3] + (r0 + 16 * (i >> 3)) * ROW;
        const float a = *reinterpret_cast<const float*>(tile + (HD == 32 ? row : (row ^ ((d & 1) << 7)) + (d >> 1) * 256));
        acc[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, p.b[i], acc[d], 0, 0, 0);
      }
  }
};

// Where a lane's chunks of a tile lie in memory.  A load instruction of a wave fills 1 KB
// of LDS in lane order, so the permutation of the chunks is made by the lanes' addresses,
// one for each of a wave's instructions within 16 rows.
template <typename T, int HD, int ROWS = kRows, int WAVES = kWaves> struct Stager {
  using O = Ops<T, HD>;
  static constexpr int TOTAL = ROWS * O::CPR / 64;                    // instructions of a tile
  static constexpr int COUNT = (TOTAL + WAVES - 1) / WAVES;           // of a wave, at most
  static constexpr int PASS = 64 * WAVES / O::CPR;                    // rows of one instruction of every wave
  static constexpr int KINDS = PASS < 16 ? 16 / PASS : 1;
  uint32_t at[KINDS], ld;        // bytes: this lane's chunks in memory; a row
  __device__ __forceinline__ Stager(int64_t stride, int lane, int wave) {
    ld = (uint32_t)stride * sizeof(T);
#pragma unroll
    for (int j = 0; j < KINDS; ++j) {
      const int chunk = 64 * (wave + WAVES * j) + lane, row = chunk / O::CPR, c = chunk % O::CPR;
      at[j] = row * ld + (O::at(row, c) - row * O::ROW);   // the permutation is its own inverse
    }
  }
  // Rows 0 .. ROWS-1 from g; rows at or past `valid` (>= 1) become 0.  Callers move g along
  // from tile to tile: a 64-bit product per tile would cost as much as a tenth of its work.
  __device__ __forceinline__ void load(char* tile, const T* g, int valid, int wave) const {
    const uint32_t bytes = (uint32_t)(min(valid, ROWS) - 1) * ld + HD * sizeof(T);
    const __amdgpu_buffer_rsrc_t r = buf_rsrc(g, bytes);
#pragma unroll
    for (int j = 0; j < COUNT; ++j)
      if (TOTAL % WAVES == 0 || wave + WAVES * j < TOTAL)
        buf_load_lds16(r, tile + (wave + WAVES * j) * 1024, (int)(at[j % KINDS] + (j / KINDS) * KINDS * PASS * ld), 0);
  }
};

// Which of the two buffers, known when the code is made: a lane's offsets then take it as a
// constant.
template <int N> struct Turn { static constexpr int value = N; };

// 64 floats from g; entries at or past `valid` (>= 1) become 0.  By one wave.
__device__ __forceinline__ void load_floats(float* dst, const float* g, int valid, int lane) {
  const __amdgpu_buffer_rsrc_t r = buf_rsrc(g, (uint32_t)min(valid, 64) * 4);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void_t*)dst, 4, lane * 4, 0, 0, 0);
}

// This wave's loads have arrived, its LDS reads and writes are done.
__device__ __forceinline__ void arrived() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }

// The same of every wave of the workgroup.
__device__ __forceinline__ void meet() {
  arrived();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

__device__ __forceinline__ void store4(bf16_t* p, float a, float b, float c, float d) {
  typedef __bf16 bf16x4_v __attribute__((ext_vector_type(4)));
  *reinterpret_cast<bf16x4_v*>(p) = bf16x4_v{(__bf16)a, (__bf16)b, (__bf16)c, (__bf16)d};
}
__device__ __forceinline__ void store4(float* p, float a, float b, float c, float d) {
  *reinterpret_cast<f32x4_t*>(p) = f32x4_t{a, b, c, d};
}
// The 32 columns of a wave's result, times `by`, as rows of memory: `valid` rows from g.  A lane
// holds parts of one row; through LDS (32 rows of this wave's own, laid out as a tile) they
// go out in whole rows.
template <typename T, int HD>
__device__ __forceinline__ void store_rows(char* own, T* g, int64_t ld, int valid, const f32x16_t* acc, float by,
                                           int lane) {
  using O = Ops<T, HD>;
  constexpr int EPC = 16 / sizeof(T);
  const int h = lane >> 5, col = lane & 31;
#pragma unroll
  for (int d = 0; d < HD / 32; ++d)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int e = 32 * d + 8 * j + 4 * h;
      store4(reinterpret_cast<T*>(own + O::at(col, e / EPC)) + e % EPC, acc[d][4 * j] * by, acc[d][4 * j + 1] * by,
             acc[d][4 * j + 2] * by, acc[d][4 * j + 3] * by);
    }
#pragma unroll
  for (int n = 0; n < 32 * O::CPR / 64; ++n) {
    const int p = 64 * n + lane, row = p / O::CPR, c = p % O::CPR;
    const u32x4_t v = *reinterpret_cast<const u32x4_t*>(own + O::at(row, c));
    if (row < valid) *reinterpret_cast<u32x4_t*>(g + row * ld + c * EPC) = v;
  }
}

// The tile of a workgroup, `per` positions of one sequence.  Up to 64 sequences are taken by
// length, the longest first, each one's tiles together (they read the same keys): the last
// workgroups to start are then short ones.  With more, sequence s owns the slots from
// off[s] / per + s on, which are enough for its tiles; the slots past its length are empty.
// A sequence's tiles come first to last, or with `last_first` the other way round.
struct Span {
  int start, len, first;         // first row and length of the sequence; first position of the tile (>= len: none)
};
__device__ __forceinline__ Span find_span(const int32_t* offs, int n_seqs, int N, int slot, int per, bool last_first) {
  const int lane = threadIdx.x & 63;
  Span r = {0, 0, 0};
  if (n_seqs <= kWave) {
    const int i = min(lane, n_seqs - 1);
    const int start = min(max(offs[i], 0), N), end = min(max(offs[i + 1], start), N);
    const int tiles = lane < n_seqs ? (end - start + per - 1) / per : 0;
    int before = 0;              // tiles of the sequences ahead of this lane's
    for (int k = 0; k < n_seqs; ++k) {
      const int t = __builtin_amdgcn_readlane(tiles, k);
      before += t > tiles || (t == tiles && k < lane) ? t : 0;
    }
    const uint64_t at = __ballot(slot >= before && slot < before + tiles);
    if (at == 0) return r;
    const int s = __builtin_ctzll(at), j = slot - __builtin_amdgcn_readlane(before, s);
    r.start = __builtin_amdgcn_readlane(start, s);
    r.len = __builtin_amdgcn_readlane(end, s) - r.start;
    r.first = (last_first ? __builtin_amdgcn_readlane(tiles, s) - 1 - j : j) * per;
    return r;
  }
  if (last_first) slot = N / per + n_seqs - 1 - slot;
  // a lane per sequence, its two offsets loaded together; the last sequence that begins at
  // or before the slot has it
  for (int b = 0; b < n_seqs; b += kWave) {
    const int i = min(b + lane, n_seqs - 1);
    const int start = min(max(offs[i], 0), N), end = min(max(offs[i + 1], start), N), first = start / per + i;
    const uint64_t at = __ballot(b + lane < n_seqs && first <= slot);
    if (at == 0) break;
    const int s = 63 - __builtin_clzll(at);
    r.start = __builtin_amdgcn_readlane(start, s);
    r.len = __builtin_amdgcn_readlane(end, s) - r.start;
    r.first = (slot - __builtin_amdgcn_readlane(first, s)) * per;
    if (~at != 0) break;
  }
  return r;
}

// The rows before the first sequence and behind the last one.
struct Rest {
  int before, behind, count;     // rows before; first row behind; rows in all
  __device__ __forceinline__ explicit Rest(const FlashArgs& a) {
    before = min(max(a.offs[0], 0), a.N);
    behind = min(max(a.offs[a.n_seqs], before), a.N);
    count = before + a.N - behind;
  }
  __device__ __forceinline__ int row(int i) const { return i < before ? i : behind + (i - before); }
};
// They become 0, by all workgroups of a launch of 256 threads in turn: `width` elements of each, and
// an entry of stat [heads][N].
template <typename T>
__device__ __forceinline__ void clear_rows(const FlashArgs& a, void* out, int64_t ld, int width) {
  const Rest r(a);
  for (int i = blockIdx.x; i < r.count; i += gridDim.x) {
    T* row = reinterpret_cast<T*>(out) + r.row(i) * ld;
    for (int c = threadIdx.x * (16 / (int)sizeof(T)); c < width; c += 256 * (16 / (int)sizeof(T)))
      *reinterpret_cast<u32x4_t*>(row + c) = u32x4_t{0, 0, 0, 0};
  }
}
__device__ __forceinline__ void clear_stat(const FlashArgs& a, float* stat) {
  const Rest r(a);
  for (int i = blockIdx.x; i < r.count; i += gridDim.x)
    for (int h = threadIdx.x; h < a.nq; h += 256) stat[(int64_t)h * a.N + r.row(i)] = 0.f;
}
// The outputs of the forward pass, and of the two passes of the backward one.
template <typename T, int HD>
__device__ __forceinline__ void clear_out(const FlashArgs& a) {
  if (a.clear & TANDEM_CLEAR_OUT) clear_rows<T>(a, a.out, a.ldo, a.nq * HD);
  if (a.clear & TANDEM_CLEAR_LSE) clear_stat(a, a.lse);
}
template <typename T, int HD>
__device__ __forceinline__ void clear_dq(const FlashArgs& a) {
  if (a.clear & TANDEM_CLEAR_DQ) clear_rows<T>(a, a.dq, a.lddq, a.nq * HD);
}
template <typename T, int HD>
__device__ __forceinline__ void clear_dkv(const FlashArgs& a) {
  if (a.clear & TANDEM_CLEAR_DK) clear_rows<T>(a, a.dk, a.lddk, a.nkv * HD);
  if (a.clear & TANDEM_CLEAR_DV) clear_rows<T>(a, a.dv, a.lddv, a.nkv * HD);
}

// The other half wave's value (lane l and l + 32 hold the same column).
__device__ __forceinline__ float other_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// The running softmax of a wave's 32 queries over blocks of 32 keys.  m2 is the maximum (in
// powers of two) that the sums are taken against; it is raised only where a score passes it
// by 2^8, which float32 sums and bf16's range bear, so that most blocks leave the
// accumulator alone.
template <typename T, int HD>
struct Softmax {
  using O = Ops<T, HD>;
  float m2 = -INFINITY, l = 0.f;
  f32x16_t o[HD / 32];

  // A block of keys, the first at n0.
  __device__ __forceinline__ void add(const char* __restrict__ tk, const char* __restrict__ tv,
                                      const typename O::Lanes& at, const typename O::Right& q, int n0, int q0, int qi,
                                      float s2, int h) {
    f32x16_t s = O::by_rows(tk, at, 0, q);
    if (n0 + 31 > q0) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (n0 + result_row(i, h) > qi) s[i] = -INFINITY;
    }
    float mx = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
    mx = other_max(mx) * s2;
    if (__any(mx > m2 + 8.f)) {
      const float m = fmaxf(m2, mx), f = __builtin_amdgcn_exp2f(m2 - m);
      m2 = m;
      l *= f;
#pragma unroll
      for (int d = 0; d < HD / 32; ++d) o[d] *= f;
    }
    float p[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], s2, -m2));
      l += p[i];
    }
    O::transposed(o, tv, at, 0, O::pack(p));
  }
};

// Bound by latency more than by any one pipe (the matrix pipe is busy 56% of the cycles): what
// counts is the waves a SIMD holds, so the tiles are of 32 keys and the code keeps nothing
// ahead.  Heads of 128 take 161 registers, three waves a SIMD: sixteen ragged rollouts (32 heads
// on 8) 275 us, 0.9 PFLOP/s.  Two waves with
// tiles of 64 and the scores, exponentials and value products of three blocks
// interleaved in each took 314, two without that 325.
template <typename T, int HD>
__global__ __launch_bounds__(64 * kWaves, (Ops<T, HD>::FWD)) void flash_kernel(FlashArgs a) {
  using O = Ops<T, HD>;
  constexpr int TILE = 32 * O::ROW;
  __shared__ __align__(16) char lds[2][2][TILE];           // [turn][keys, values]
  static_assert(sizeof(lds) >= kWaves * 32 * O::ROW, "room for the results");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5, col = lane & 31;
  const int group = a.nq / a.nkv, together = heads_together(group), per = 32 * (kWaves / together);
  const int kv = blockIdx.x % a.nkv, sub = blockIdx.x / a.nkv % (group / together);
  clear_out<T, HD>(a);
  // the last tiles of a sequence are its longest: they go first
  const Span w = find_span(a.offs, a.n_seqs, a.N, blockIdx.x / a.nkv / (group / together), per, true);
  if (w.first >= w.len) return;
  const int head = kv * group + sub * together + wave % together;
  const int q0 = w.first + 32 * (wave / together), qi = q0 + col;
  const int64_t row = w.start + min(qi, w.len - 1);
  const T* kb = reinterpret_cast<const T*>(a.k) + (int64_t)w.start * a.ldk + kv * HD;
  const T* vb = reinterpret_cast<const T*>(a.v) + (int64_t)w.start * a.ldv + kv * HD;
  const Stager<T, HD, 32> sk(a.ldk, lane, wave), sv(a.ldv, lane, wave);
  const int tiles = (min(w.len, w.first + per) + 31) / 32;          // that any row of the workgroup sees
  const int mine = q0 < w.len ? q0 / 32 + 1 : 0;                    // that this wave's rows see
  const int64_t dk = 32 * a.ldk, dv = 32 * a.ldv;
  auto load = [&](int t, int i) {
    sk.load(lds[t][0], kb, w.len - 32 * i, wave);
    sv.load(lds[t][1], vb, w.len - 32 * i, wave);
    kb += dk;
    vb += dv;
  };
  load(0, 0);
  typename O::Right q;
  O::load_right(q, reinterpret_cast<const T*>(a.q) + row * a.ldq + head * HD, h);
  const float s2 = a.scale * kLog2e;
  const typename O::Lanes at = O::lanes(lane);
  Softmax<T, HD> st;
#pragma unroll
  for (int d = 0; d < HD / 32; ++d) st.o[d] = zero16();
  auto step = [&](auto turn, int i) {
    constexpr int t = decltype(turn)::value;
    meet();
    if (i + 1 < tiles) load(t ^ 1, i + 1);
    if (i < mine) st.add(lds[t][0], lds[t][1], at, q, 32 * i, q0, qi, s2, h);
  };
  for (int i = 0; i < tiles; i += 2) {
    step(Turn<0>{}, i);
    if (i + 1 < tiles) step(Turn<1>{}, i + 1);
  }
  const float l = st.l + __shfl_xor(st.l, 32, kWave);
  meet();                                                  // the tiles' room takes the results
  if (mine == 0) return;
  store_rows<T, HD>(lds[0][0] + wave * 32 * O::ROW, reinterpret_cast<T*>(a.out) + (int64_t)(w.start + q0) * a.ldo + head * HD,
                    a.ldo, w.len - q0, st.o, 1.f / l, lane);
  if (h == 0 && qi < w.len) a.lse[(int64_t)head * a.N + row] = (st.m2 + __builtin_amdgcn_logf(l)) * kLn2;
}

// Where there are few tiles of queries, a workgroup's waves share 32 queries of one head and take
// every fourth tile of keys each, in LDS of their own and so without a meeting; what they
// have is joined through LDS.
template <typename T, int HD>
struct Alone {
  using O = Ops<T, HD>;
  static constexpr int TILE = 32 * O::ROW;
  static constexpr int TURNS = two_turns(HD, sizeof(T) == 2) ? 2 : 1;
  static constexpr int PART = 32 * HD * 4;                 // bytes of a wave's accumulator
  static constexpr int WGS = TURNS * TILE <= 8192 ? 2 : 1; // workgroups per compute unit (LDS: 64 KB, or 128)
  typedef char Room[kWaves][TURNS][2][TILE];
  static_assert(sizeof(Room) >= kWaves * PART && PART >= TILE, "room for the accumulators and the results");
  struct Work {                                            // of this workgroup
    Span w;
    int kv, head;
  };
  __device__ __forceinline__ static Work work(const FlashArgs& a) {
    const int group = a.nq / a.nkv, kv = blockIdx.x % a.nkv;
    return Work{find_span(a.offs, a.n_seqs, a.N, blockIdx.x / a.nq, 32, true), kv,
                kv * group + (int)(blockIdx.x / a.nkv) % group};
  }
  // use(keys, values, first key) for this wave's tiles of the keys that the queries see
  template <typename F>
  __device__ __forceinline__ static void tiles(Room& lds, const FlashArgs& a, const Work& x, int lane, int wave, F&& use) {
    const T* kb = reinterpret_cast<const T*>(a.k) + (int64_t)(x.w.start + 32 * wave) * a.ldk + x.kv * HD;
    const T* vb = reinterpret_cast<const T*>(a.v) + (int64_t)(x.w.start + 32 * wave) * a.ldv + x.kv * HD;
    const Stager<T, HD, 32, 1> sk(a.ldk, lane, 0), sv(a.ldv, lane, 0);
    auto load = [&](int t, int n0) {
      sk.load(lds[wave][t][0], kb, x.w.len - n0, 0);
      sv.load(lds[wave][t][1], vb, x.w.len - n0, 0);
      kb += 32 * kWaves * a.ldk;
      vb += 32 * kWaves * a.ldv;
    };
    int t = 0;
    if (TURNS == 2 && 32 * wave <= x.w.first) load(0, 32 * wave);
    for (int n0 = 32 * wave; n0 <= x.w.first; n0 += 32 * kWaves) {
      if (TURNS == 1) {
        arrived();                                         // the last tile has been read
        load(0, n0);
      }
      arrived();
      if (TURNS == 2 && n0 + 32 * kWaves <= x.w.first) load(t ^ 1, n0 + 32 * kWaves);
      use(lds[wave][t][0], lds[wave][t][1], n0);
      if (TURNS == 2) t ^= 1;
    }
  }
  // The waves' accumulators, each times its f, added up in the first wave's, in their order.
  __device__ __forceinline__ static void join(Room& lds, f32x16_t* acc, float f, int lane, int wave) {
    char* room = lds[0][0][0];
    f32x4_t* own = reinterpret_cast<f32x4_t*>(room + wave * PART) + lane;
    if (wave > 0) {
#pragma unroll
      for (int d = 0; d < HD / 32; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          own[64 * (4 * d + j)] =
              f32x4_t{acc[d][4 * j] * f, acc[d][4 * j + 1] * f, acc[d][4 * j + 2] * f, acc[d][4 * j + 3] * f};
    }
    meet();
    if (wave > 0) return;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d) acc[d] *= f;
    for (int o = 1; o < kWaves; ++o) {
      const f32x4_t* part = reinterpret_cast<const f32x4_t*>(room + o * PART) + lane;
#pragma unroll
      for (int d = 0; d < HD / 32; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f32x4_t v = part[64 * (4 * d + j)];
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[d][4 * j + e] += v[e];
        }
    }
  }
};

template <typename T, int HD>
__global__ __launch_bounds__(64 * kWaves, (Alone<T, HD>::WGS)) void flash_alone_kernel(FlashArgs a) {
  using O = Ops<T, HD>;
  using A = Alone<T, HD>;
  __shared__ __align__(16) typename A::Room lds;
  __shared__ float stat[kWaves][2][32];                    // maxima, sums
  clear_out<T, HD>(a);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5, col = lane & 31;
  const typename A::Work x = A::work(a);
  if (x.w.first >= x.w.len) return;
  const int q0 = x.w.first, qi = q0 + col;
  const int64_t row = x.w.start + min(qi, x.w.len - 1);
  typename O::Right q;
  O::load_right(q, reinterpret_cast<const T*>(a.q) + row * a.ldq + x.head * HD, h);
  const float s2 = a.scale * kLog2e;
  const typename O::Lanes at = O::lanes(lane);
  Softmax<T, HD> st;
#pragma unroll
  for (int d = 0; d < HD / 32; ++d) st.o[d] = zero16();
  A::tiles(lds, a, x, lane, wave, [&](const char* __restrict__ tk, const char* __restrict__ tv, int n0) {
    st.add(tk, tv, at, q, n0, q0, qi, s2, h);
  });
  const float own = st.l + __shfl_xor(st.l, 32, kWave);
  if (h == 0) {
    stat[wave][0][col] = st.m2;
    stat[wave][1][col] = own;
  }
  meet();                                                  // the tiles' room takes the accumulators
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int o = 0; o < kWaves; ++o) m = fmaxf(m, stat[o][0][col]);
#pragma unroll
  for (int o = 0; o < kWaves; ++o) l += stat[o][1][col] * __builtin_amdgcn_exp2f(stat[o][0][col] - m);
  A::join(lds, st.o, __builtin_amdgcn_exp2f(st.m2 - m), lane, wave);
  if (wave > 0) return;
  store_rows<T, HD>(lds[0][0][0], reinterpret_cast<T*>(a.out) + (int64_t)(x.w.start + q0) * a.ldo + x.head * HD, a.ldo,
                    x.w.len - q0, st.o, 1.f / l, lane);
  if (h == 0 && qi < x.w.len) a.lse[(int64_t)x.head * a.N + row] = (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// A block of 32 keys, the first at n0: the tile's rows from r0 on.
template <typename T, int HD>
__device__ __forceinline__ void dq_block(f32x16_t* dq, const char* __restrict__ tk, const char* __restrict__ tv, int r0,
                                         const typename Ops<T, HD>::Lanes& at, const typename Ops<T, HD>::Right& q,
                                         const typename Ops<T, HD>::Right& g, int n0, bool edge, int qi, float s2,
                                         float lse2, float delta, int h) {
  using O = Ops<T, HD>;
  const f32x16_t s = O::by_rows(tk, at, r0, q);
  const f32x16_t dp = O::by_rows(tv, at, r0, g);
  float ds[16];
#pragma unroll
  for (int i = 0; i < 16; ++i)
    ds[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], s2, -lse2)) * (dp[i] - delta);
  if (edge) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (n0 + result_row(i, h) > qi) ds[i] = 0.f;
  }
  O::transposed(dq, tk, at, r0, O::pack(ds));
}
template <typename T, int HD>
__device__ __forceinline__ void dq_tile(f32x16_t* dq, const char* __restrict__ tk, const char* __restrict__ tv,
                                        const typename Ops<T, HD>::Lanes& at, const typename Ops<T, HD>::Right& q,
                                        const typename Ops<T, HD>::Right& g, int n0, int q0, int qi, float s2,
                                        float lse2, float delta, int h) {
  const bool edge = n0 + kRows - 1 > q0;
#pragma unroll
  for (int b = 0; b < 2; ++b)
    dq_block<T, HD>(dq, tk, tv, 32 * b, at, q, g, n0 + 32 * b, edge, qi, s2, lse2, delta, h);
}

// The pairs' probabilities are held as 2^15 P, in float16 where they pass from wave to wave:
// 11 bits down to P = 2^-29, 8 times finer than the bf16 to which dS is rounded next (and
// rounding P itself to bf16 would round dS twice).  The results are scaled back exactly.
constexpr float kProbScale = 32768.f, kProbBits = 15.f;
template <typename T, int HD>
constexpr bool kByPairs = keys_by_pairs(HD, sizeof(T) == 2);

// What a lane holds of its query, and leaves for the pass over the keys (if `leave`): the delta
// dout . out (negated) and the log-sum-exp in powers of two.
template <typename T, int HD>
struct DqRows {
  using O = Ops<T, HD>;
  typename O::Right q, g;
  float delta, lse2;
  __device__ __forceinline__ DqRows(const FlashArgs& a, int head, int64_t row, int h, bool leave) {
    O::load_right(g, reinterpret_cast<const T*>(a.dout) + row * a.lddo + head * HD, h);
    O::load_right(q, reinterpret_cast<const T*>(a.out) + row * a.ldo + head * HD, h);
    delta = O::dot(g, q);
    delta += __shfl_xor(delta, 32, kWave);
    O::load_right(q, reinterpret_cast<const T*>(a.q) + row * a.ldq + head * HD, h);
    const int64_t stat = (int64_t)head * a.N + row;
    lse2 = a.lse[stat] * kLog2e;
    if (h == 0 && leave) {
      a.ndelta[stat] = -delta;
      a.lse2[stat] = kByPairs<T, HD> ? lse2 - kProbBits : lse2;
    }
  }
};

// dQ, and what the pass over the keys needs, each (row, head) being one lane pair's.
// The matrix pipe is busy 51% (heads of 128) and 66% (64) of the cycles: sixteen ragged rollouts
// 406 to 422 us as the clock allows, one sequence of 8703 236.  Two waves a SIMD; tiles of 32
// keys, or four waves a SIMD of heads of 64, take the same time.
template <typename T, int HD>
__global__ __launch_bounds__(64 * kWaves, (Ops<T, HD>::WGS)) void flash_dq_kernel(FlashArgs a) {
  using O = Ops<T, HD>;
  constexpr int TILE = kRows * O::ROW;
  __shared__ __align__(16) char lds[2][2][TILE];           // [turn][keys, values]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5, col = lane & 31;
  const int group = a.nq / a.nkv, together = heads_together(group), per = 32 * (kWaves / together);
  const int kv = blockIdx.x % a.nkv, sub = blockIdx.x / a.nkv % (group / together);
  clear_dq<T, HD>(a);
  const Span w = find_span(a.offs, a.n_seqs, a.N, blockIdx.x / a.nkv / (group / together), per, true);
  if (w.first >= w.len) return;
  const int head = kv * group + sub * together + wave % together;
  const int q0 = w.first + 32 * (wave / together), qi = q0 + col;
  const int64_t row = w.start + min(qi, w.len - 1);
  const T* kb = reinterpret_cast<const T*>(a.k) + (int64_t)w.start * a.ldk + kv * HD;
  const T* vb = reinterpret_cast<const T*>(a.v) + (int64_t)w.start * a.ldv + kv * HD;
  const Stager<T, HD> sk(a.ldk, lane, wave), sv(a.ldv, lane, wave);
  const int end = min(w.len, w.first + per);
  const int64_t dk = (int64_t)kRows * a.ldk, dv = (int64_t)kRows * a.ldv;
  auto load = [&](int t, int n0) {
    sk.load(lds[t][0], kb, w.len - n0, wave);
    sv.load(lds[t][1], vb, w.len - n0, wave);
    kb += dk;
    vb += dv;
  };
  load(0, 0);
  const DqRows<T, HD> r(a, head, row, h, qi < w.len);
  const float s2 = a.scale * kLog2e;
  f32x16_t dq[HD / 32];
#pragma unroll
  for (int d = 0; d < HD / 32; ++d) dq[d] = zero16();
  const typename O::Lanes at = O::lanes(lane);
  auto step = [&](auto turn, int n0) {
    constexpr int t = decltype(turn)::value;
    meet();
    if (n0 + kRows < end) load(t ^ 1, n0 + kRows);
    if (n0 <= q0 + 31) dq_tile<T, HD>(dq, lds[t][0], lds[t][1], at, r.q, r.g, n0, q0, qi, s2, r.lse2, r.delta, h);
  };
  for (int n0 = 0; n0 < end; n0 += 2 * kRows) {
    step(Turn<0>{}, n0);
    if (n0 + kRows < end) step(Turn<1>{}, n0 + kRows);
  }
  meet();                                                  // the tiles' room takes the results
  if (q0 >= w.len) return;
  store_rows<T, HD>(lds[0][0] + wave * 32 * O::ROW, reinterpret_cast<T*>(a.dq) + (int64_t)(w.start + q0) * a.lddq + head * HD,
                    a.lddq, w.len - q0, dq, a.scale, lane);
}

template <typename T, int HD>
__global__ __launch_bounds__(64 * kWaves, (Alone<T, HD>::WGS)) void flash_dq_alone_kernel(FlashArgs a) {
  using O = Ops<T, HD>;
  using A = Alone<T, HD>;
  __shared__ __align__(16) typename A::Room lds;
  clear_dq<T, HD>(a);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5, col = lane & 31;
  const typename A::Work x = A::work(a);
  if (x.w.first >= x.w.len) return;
  const int q0 = x.w.first, qi = q0 + col;
  const int64_t row = x.w.start + min(qi, x.w.len - 1);
  const DqRows<T, HD> r(a, x.head, row, h, wave == 0 && qi < x.w.len);
  const float s2 = a.scale * kLog2e;
  f32x16_t dq[HD / 32];
#pragma unroll
  for (int d = 0; d < HD / 32; ++d) dq[d] = zero16();
  const typename O::Lanes at = O::lanes(lane);
  A::tiles(lds, a, x, lane, wave, [&](const char* __restrict__ tk, const char* __restrict__ tv, int n0) {
    dq_block<T, HD>(dq, tk, tv, 0, at, r.q, r.g, n0, n0 + 31 > q0, qi, s2, r.lse2, r.delta, h);
  });
  meet();                                                  // the tiles' room takes the accumulators
  A::join(lds, dq, 1.f, lane, wave);
  if (wave > 0) return;
  store_rows<T, HD>(lds[0][0][0], reinterpret_cast<T*>(a.dq) + (int64_t)(x.w.start + q0) * a.lddq + x.head * HD, a.lddq,
                    x.w.len - q0, dq, a.scale, lane);
}

// A lane's column of a result, float32, 16 bytes at a time.
template <int HD>
__device__ __forceinline__ void store_column(float* p, const f32x16_t* acc, float by, int h) {
#pragma unroll
  for (int d = 0; d < HD / 32; ++d)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      store4(p + 32 * d + 8 * j + 4 * h, acc[d][4 * j] * by, acc[d][4 * j + 1] * by, acc[d][4 * j + 2] * by,
             acc[d][4 * j + 3] * by);
}

// One of the even parts of a list, of 2^26 steps (a launch over the queries has fewer than 2^24
// workgroups of 128 rows of a head) and 16 parts at most.
struct Share {
  int begin, count;
};
__device__ __forceinline__ Share share_of(int all, int part, int parts) {
  const int begin = (int)((uint32_t)(all * part) / (uint32_t)parts);
  return Share{begin, (int)((uint32_t)(all * (part + 1)) / (uint32_t)parts) - begin};
}

template <typename T, int HD>
__device__ __forceinline__ void dkv_tile(f32x16_t* dk, f32x16_t* dv, const char* __restrict__ tq,
                                         const char* __restrict__ tg, const float* __restrict__ t_lse2,
                                         const float* __restrict__ t_ndelta, const typename Ops<T, HD>::Lanes& at,
                                         const typename Ops<T, HD>::Right& k, const typename Ops<T, HD>::Right& v,
                                         int m0, int k0, int ki, float s2, int h) {
  using O = Ops<T, HD>;
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const int r0 = m0 + 32 * b;
    if (r0 + 31 < k0) continue;
    const f32x16_t s = O::by_rows(tq, at, 32 * b, k);
    const f32x16_t dp = O::by_rows(tg, at, 32 * b, v);
    float p[16], ds[16];
#pragma unroll
    for (int i = 0; i < 16; ++i)
      p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], s2, -t_lse2[32 * b + result_row(i, h)]));
    if (r0 < k0 + 31) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (r0 + result_row(i, h) < ki) p[i] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) ds[i] = p[i] * (dp[i] + t_ndelta[32 * b + result_row(i, h)]);
    O::transposed(dv, tg, at, 32 * b, O::pack(p));
    O::transposed(dk, tq, at, 32 * b, O::pack(ds));
  }
}

template <typename T, int HD>
__global__ __launch_bounds__(64 * kWaves, 1) void flash_dkv_kernel(FlashArgs a, int parts) {
  using O = Ops<T, HD>;
  constexpr int PER = 32 * kWaves, TILE = kRows * O::ROW;
  // a query past the sequence reads as 0, with log-sum-exp 0: probability 1 of a gradient of 0
  __shared__ __align__(16) char lds[2][2][TILE];           // [turn][queries, output gradients]
  __shared__ __align__(16) float stat[2][2][kRows];        // [turn][log-sum-exps, negated deltas]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5, col = lane & 31;
  const int group = a.nq / a.nkv;
  const int kv = blockIdx.x % a.nkv, part = blockIdx.x / a.nkv % parts, slot = blockIdx.x / a.nkv / parts;
  if (parts == 1) clear_dkv<T, HD>(a);
  const Span w = find_span(a.offs, a.n_seqs, a.N, slot, PER, false);
  if (w.first >= w.len) return;
  const int k0 = w.first + 32 * wave, ki = k0 + col;
  // the heads' tiles of queries, one after the other, and of those this part's
  const int tiles = (w.len - w.first + kRows - 1) / kRows;
  const Share mine = share_of(group * tiles, part, parts);
  int m0 = w.first + mine.begin % tiles * kRows, head = kv * group + mine.begin / tiles;
  const int64_t row = w.start + min(ki, w.len - 1);
  const Stager<T, HD> sq(a.ldq, lane, wave), sg(a.lddo, lane, wave);
  auto load = [&](int t, int head, int m0) {
    sq.load(lds[t][0], reinterpret_cast<const T*>(a.q) + (int64_t)(w.start + m0) * a.ldq + head * HD, w.len - m0, wave);
    sg.load(lds[t][1], reinterpret_cast<const T*>(a.dout) + (int64_t)(w.start + m0) * a.lddo + head * HD, w.len - m0,
            wave);
    const int64_t at = (int64_t)head * a.N + w.start + m0;
    if (wave == 0) load_floats(stat[t][0], a.lse2 + at, w.len - m0, lane);
    if (wave == 1) load_floats(stat[t][1], a.ndelta + at, w.len - m0, lane);
  };
  if (mine.count > 0) load(0, head, m0);
  typename O::Right k, v;
  O::load_right(k, reinterpret_cast<const T*>(a.k) + row * a.ldk + kv * HD, h);
  O::load_right(v, reinterpret_cast<const T*>(a.v) + row * a.ldv + kv * HD, h);
  const float s2 = a.scale * kLog2e;
  f32x16_t dk[HD / 32], dv[HD / 32];
#pragma unroll
  for (int d = 0; d < HD / 32; ++d) dk[d] = dv[d] = zero16();
  const typename O::Lanes at = O::lanes(lane);
  auto step = [&](auto turn, bool more) {
    constexpr int t = decltype(turn)::value;
    meet();
    const bool last = m0 + kRows >= w.len;
    const int m1 = last ? w.first : m0 + kRows, head1 = last ? head + 1 : head;
    if (more) load(t ^ 1, head1, m1);
    dkv_tile<T, HD>(dk, dv, lds[t][0], lds[t][1], stat[t][0], stat[t][1], at, k, v, m0, k0, ki, s2, h);
    m0 = m1;
    head = head1;
  };
  for (int i = 0; i < mine.count; i += 2) {
    step(Turn<0>{}, i + 1 < mine.count);
    if (i + 1 < mine.count) step(Turn<1>{}, i + 2 < mine.count);
  }
  meet();                                                  // the tiles' room takes the results
  if (k0 >= w.len) return;
  const int64_t row0 = w.start + k0;
  if (parts > 1) {
    if (ki >= w.len) return;
    const int64_t width = a.nkv * HD, plane = (int64_t)parts * a.N * width;
    float* sums = a.sums + ((int64_t)part * a.N + row0 + col) * width + kv * HD;
    store_column<HD>(sums, dv, 1.f, h);
    store_column<HD>(sums + plane, dk, a.scale, h);
    return;
  }
  char* room = lds[0][0] + wave * 32 * O::ROW;
  store_rows<T, HD>(room, reinterpret_cast<T*>(a.dk) + row0 * a.lddk + kv * HD, a.lddk, w.len - k0, dk, a.scale, lane);
  store_rows<T, HD>(room, reinterpret_cast<T*>(a.dv) + row0 * a.lddv + kv * HD, a.lddv, w.len - k0, dv, 1.f, lane);
}

typedef _Float16 f16x8_v __attribute__((ext_vector_type(8)));

// A step of the pairs below: 32 queries by a pair's 32 keys.  The first wave's half:
// P = e^(S - lse), dV^T += dO^T P.
template <int HD>
__device__ __forceinline__ void dv_step(f32x16_t* dv, const char* __restrict__ tq, const char* __restrict__ tg,
                                        const float* __restrict__ lse2, f16x8_v* __restrict__ prob,
                                        const typename Ops<bf16_t, HD>::Lanes& at,
                                        const typename Ops<bf16_t, HD>::Right& k, bool edge, int col, float s2, int h,
                                        int lane) {
  using O = Ops<bf16_t, HD>;
  const f32x16_t s = O::by_rows(tq, at, 0, k);
  float p[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], s2, -lse2[result_row(i, h)]));
  if (edge) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (result_row(i, h) < col) p[i] = 0.f;
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    f16x8_v v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (_Float16)p[8 * j + e];
    prob[64 * j + lane] = v;
  }
  O::transposed(dv, tg, at, 0, O::pack(p));
}
// The second wave's, first dP - delta of a step (the sum begins at -delta), one step later
// dS = P (dP - delta), dK^T += Q^T dS.
template <int HD>
__device__ __forceinline__ f32x16_t dp_step(const char* __restrict__ tg, const float* __restrict__ ndelta,
                                            const typename Ops<bf16_t, HD>::Lanes& at,
                                            const typename Ops<bf16_t, HD>::Right& v, int h) {
  f32x16_t dp;
#pragma unroll
  for (int i = 0; i < 16; ++i) dp[i] = ndelta[result_row(i, h)];
  return Ops<bf16_t, HD>::by_rows(tg, at, 0, v, dp);
}
template <int HD>
__device__ __forceinline__ void dk_step(f32x16_t* dk, const char* __restrict__ tq, const f16x8_v* __restrict__ prob,
                                        const f32x16_t& dp, const typename Ops<bf16_t, HD>::Lanes& at, int lane) {
  using O = Ops<bf16_t, HD>;
  float ds[16];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const f16x8_v p = prob[64 * j + lane];
#pragma unroll
    for (int e = 0; e < 8; ++e)              // with the 0 one instruction converts and multiplies: 1% of the time
      ds[8 * j + e] = __builtin_fmaf((float)p[e], dp[8 * j + e], 0.f);
  }
  O::transposed(dk, tq, at, 0, O::pack(ds));
}

// dK and dV of bf16 heads of 64 and 128 by pairs of waves: of each pair's 32 keys one wave
// forms the probabilities and dV, the other dP and dK.  Each then holds one operand and one
// accumulator: three waves of heads of 128 fit a SIMD, four of 64, where one wave with both
// has it alone.  The probabilities go through LDS, lane to lane, and the second wave uses
// those of the step behind, so that a step of 32 queries has one meeting: it forms dP of a
// step and keeps it over the meeting, and needs the step's queries one step longer.
//
// The matrix pipe is busy 50% of the cycles; waves wait at the meetings and for LDS.  What bounds
// a long run is power: the clock goes down to 1.7 GHz, and a form that took a quarter more
// cycles ran at 1.9.  Sixteen ragged rollouts, 32 heads of 128 on 8: 583 us; one sequence of
// 8703, 16 heads of 64 on 4: 358.  With float32 probabilities and both tiles a step longer, so two
// workgroups to a compute unit, 632 and 359; the second wave in the same step, at a second
// meeting, 676 and 383; four pairs to a workgroup 645 (90 us for the backward pass of 200
// sequences of at most 30, now 60), six 690.
//
// Where the tiles of keys are few, a workgroup takes one part of the steps and writes float32
// sums, which flash_join_kernel adds up.
constexpr int kPairs = 2;

template <int HD>
__global__ __launch_bounds__(128 * kPairs, (HD == 64 ? 4 : 3)) void flash_dkv_pair_kernel(FlashArgs a, int parts) {
  using O = Ops<bf16_t, HD>;
  using S = Stager<bf16_t, HD, 32, kPairs>;
  constexpr int TILE = 32 * O::ROW;
  // queries of the step behind, the current and the next one; output gradients of the current and
  // the next one
  __shared__ __align__(16) char lds[5][TILE];
  __shared__ __align__(16) f16x8_v prob[2][kPairs][128];   // [step's parity][pair]: probabilities in lane order
  __shared__ __align__(16) float stat[2][2 * kPairs][64];  // [step's parity][wave]: log-sum-exps, negated deltas
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool second = wave >= kPairs;
  const int h = lane >> 5, col = lane & 31, pair = second ? wave - kPairs : wave;
  const int kv = blockIdx.x % a.nkv, part = blockIdx.x / a.nkv % parts, slot = blockIdx.x / a.nkv / parts;
  const int group = a.nq / a.nkv;
  if (parts == 1) clear_dkv<bf16_t, HD>(a);
  const Span w = find_span(a.offs, a.n_seqs, a.N, slot, 32 * kPairs, false);
  if (w.first >= w.len) return;
  const int k0 = w.first + 32 * pair, ki = k0 + col;
  const int64_t row = w.start + min(ki, w.len - 1);
  // the first wave holds keys, loads queries; the second holds values, loads output gradients
  typename O::Right own;
  O::load_right(own, second ? reinterpret_cast<const bf16_t*>(a.v) + row * a.ldv + kv * HD
                            : reinterpret_cast<const bf16_t*>(a.k) + row * a.ldk + kv * HD, h);
  const int64_t ld = second ? a.lddo : a.ldq;
  const S stager(ld, lane, pair);
  // a step is 32 queries of one head; the heads one after the other, and of those steps this part's
  const int steps = (w.len - w.first + 31) / 32;
  const Share mine = share_of(group * steps, part, parts);
  const int total = mine.count, head0 = kv * group + mine.begin / steps, ahead = mine.begin % steps * 32;
  const bf16_t* head_src = reinterpret_cast<const bf16_t*>(second ? a.dout : a.q) +
                           (int64_t)(w.start + w.first) * ld + head0 * HD;
  const float* head_stat = (second ? a.ndelta : a.lse2) + (int64_t)head0 * a.N + w.start + w.first;
  const bf16_t* src = head_src + ahead * ld;               // of the next step to load
  const float* src_stat = head_stat + ahead;
  int left = w.len - w.first - ahead;                      // queries from there on
  auto load = [&](int i, int t) {                          // step i, t = i % 3
    stager.load(lds[second ? 3 + (i & 1) : t], src, left, pair);
    load_floats(stat[i & 1][wave], src_stat, left, lane);
    src += 32 * ld;
    src_stat += 32;
    left -= 32;
    if (left <= 0) {
      left = w.len - w.first;
      src = head_src += HD;
      src_stat = head_stat += a.N;
    }
  };
  if (total > 0) load(0, 0);
  const typename O::Lanes at = O::lanes(lane);
  const float s2 = a.scale * kLog2e;
  f32x16_t acc[HD / 32];
#pragma unroll
  for (int d = 0; d < HD / 32; ++d) acc[d] = zero16();
  int m0 = w.first + ahead;                                // queries of the step at hand
  auto next = [&]() {
    m0 += 32;
    if (m0 >= w.len) m0 = w.first;
  };
  // A step begins with a meeting: its tiles have arrived everywhere, the next ones are sent for.
  // One step more than there are: the second wave's last.
  if (second) {
    f32x16_t dp = zero16();
    bool before = false;                                   // the step behind has pairs that see each other
    for (int i = 0, t = 0, b = 2; i <= total; ++i) {
      const int n = t == 2 ? 0 : t + 1;
      meet();
      if (i + 1 < total) load(i + 1, n);
      if (before) dk_step<HD>(acc, lds[b], prob[(i - 1) & 1][pair], dp, at, lane);
      before = i < total && m0 >= k0;
      if (before) dp = dp_step<HD>(lds[3 + (i & 1)], stat[i & 1][wave], at, own, h);
      next();
      b = t;
      t = n;
    }
  } else {
    for (int i = 0, t = 0; i <= total; ++i) {
      const int n = t == 2 ? 0 : t + 1;
      meet();
      if (i == total) break;
      if (i + 1 < total) load(i + 1, n);
      if (m0 >= k0)
        dv_step<HD>(acc, lds[t], lds[3 + (i & 1)], stat[i & 1][wave], prob[i & 1][pair], at, own, m0 == k0, col, s2, h,
                    lane);
      next();
      t = n;
    }
  }
  meet();                                                  // the tiles' room takes the results
  if (k0 >= w.len) return;
  const int64_t row0 = w.start + k0;
  const float by = (second ? a.scale : 1.f) * (1.f / kProbScale);
  if (parts > 1) {
    float* sums = a.sums + (((int64_t)(second ? parts : 0) + part) * a.N + row0) * a.nkv * HD + kv * HD;
    if (ki < w.len) store_column<HD>(sums + (int64_t)(lane & 31) * a.nkv * HD, acc, by, h);
    return;
  }
  char* room = lds[wave];                                  // four waves, five tiles
  if (second)
    store_rows<bf16_t, HD>(room, reinterpret_cast<bf16_t*>(a.dk) + row0 * a.lddk + kv * HD, a.lddk, w.len - k0, acc, by, lane);
  else
    store_rows<bf16_t, HD>(room, reinterpret_cast<bf16_t*>(a.dv) + row0 * a.lddv + kv * HD, a.lddv, w.len - k0, acc, by, lane);
}

// dV (blockIdx.y 0) and dK (1) from the parts' sums, 8 elements per thread; rows of no
// sequence stay as they are, or become 0.
template <typename T>
__global__ __launch_bounds__(256) void flash_join_kernel(FlashArgs a, int width, int parts) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8, row = i / width;
  const int c = (int)(i % width);
  if (row >= a.N) return;
  const bool rest = row < a.offs[0] || row >= a.offs[a.n_seqs];
  if (rest && !(a.clear & (blockIdx.y ? TANDEM_CLEAR_DK : TANDEM_CLEAR_DV))) return;
  const int64_t plane = (int64_t)a.N * width;
  const float* p = a.sums + (int64_t)blockIdx.y * parts * plane + i;
  f32x4_t lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
  for (int j = 0; !rest && j < parts; ++j, p += plane) {
    lo += *reinterpret_cast<const f32x4_t*>(p);
    hi += *reinterpret_cast<const f32x4_t*>(p + 4);
  }
  T* out = blockIdx.y ? reinterpret_cast<T*>(a.dk) + row * a.lddk : reinterpret_cast<T*>(a.dv) + row * a.lddv;
  store4(out + c, lo[0], lo[1], lo[2], lo[3]);
  store4(out + c + 4, hi[0], hi[1], hi[2], hi[3]);
}

int64_t slots_of(const FlashArgs& a, int per) { return (int64_t)a.N / per + a.n_seqs; }

template <typename T, int HD>
bool shared_keys(const FlashArgs& a) { return few_queries(a.N, a.n_seqs, a.nq, a.nkv, HD, sizeof(T) == 2); }

// Workgroups, each of 256 threads, of the passes over the queries (forward, dQ) and over the keys, and
// of the parts' sums.
template <typename T, int HD>
int64_t query_blocks(const FlashArgs& a) {
  if (shared_keys<T, HD>(a)) return slots_of(a, 32) * a.nq;
  const int together = heads_together(a.nq / a.nkv);
  return slots_of(a, 32 * (kWaves / together)) * (a.nq / together);
}
template <typename T, int HD>
int parts_of(const FlashArgs& a) {
  return flash_parts(a.N, a.n_seqs, a.nq, a.nkv, HD, sizeof(T) == 2);
}
template <typename T, int HD>
int64_t key_blocks(const FlashArgs& a, int parts) {
  return slots_of(a, 32 * (kByPairs<T, HD> ? kPairs : kWaves)) * a.nkv * parts;
}
template <int HD>
int64_t join_blocks(const FlashArgs& a) { return ((int64_t)a.N * a.nkv * HD / 8 + 255) / 256; }

template <typename T, int HD>
int64_t most_blocks(const FlashArgs& a, bool backward) {
  const int64_t queries = query_blocks<T, HD>(a);
  if (!backward) return queries;
  const int parts = parts_of<T, HD>(a);
  return std::max({queries, key_blocks<T, HD>(a, parts), parts > 1 ? 2 * join_blocks<HD>(a) : 0});
}

template <typename T, int HD>
hipError_t run(const FlashArgs& a, hipStream_t st) {
  const unsigned grid = (unsigned)query_blocks<T, HD>(a);
  if (shared_keys<T, HD>(a))
    flash_alone_kernel<T, HD><<<grid, 64 * kWaves, 0, st>>>(a);
  else
    flash_kernel<T, HD><<<grid, 64 * kWaves, 0, st>>>(a);
  return hipGetLastError();
}

template <typename T, int HD>
hipError_t run_backward(const FlashArgs& a, hipStream_t st) {
  const unsigned queries = (unsigned)query_blocks<T, HD>(a);
  if (shared_keys<T, HD>(a))
    flash_dq_alone_kernel<T, HD><<<queries, 64 * kWaves, 0, st>>>(a);
  else
    flash_dq_kernel<T, HD><<<queries, 64 * kWaves, 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int parts = parts_of<T, HD>(a);
  const unsigned keys = (unsigned)key_blocks<T, HD>(a, parts);
  if constexpr (kByPairs<T, HD>)
    flash_dkv_pair_kernel<HD><<<keys, 128 * kPairs, 0, st>>>(a, parts);
  else
    flash_dkv_kernel<T, HD><<<keys, 64 * kWaves, 0, st>>>(a, parts);
  if (parts > 1) {
    const hipError_t f = hipGetLastError();
    if (f != hipSuccess) return f;
    flash_join_kernel<T><<<dim3((unsigned)join_blocks<HD>(a), 2), 256, 0, st>>>(a, a.nkv * HD, parts);
  }
  return hipGetLastError();
}

}  // namespace

int64_t flash_blocks(const FlashArgs& a, int hd, int dtype, bool backward) {
  if (a.N < 1 || a.n_seqs < 1) return 0;
  const bool b16 = dtype == DT_BF16;
  if (hd == 32) return b16 ? most_blocks<bf16_t, 32>(a, backward) : most_blocks<float, 32>(a, backward);
  if (hd == 64) return b16 ? most_blocks<bf16_t, 64>(a, backward) : most_blocks<float, 64>(a, backward);
  return b16 ? most_blocks<bf16_t, 128>(a, backward) : most_blocks<float, 128>(a, backward);
}

#define TANDEM_FLASH_DISPATCH(fn)                                                            \
  switch (hd) {                                                                              \
    case 32: return dtype == DT_BF16 ? fn<bf16_t, 32>(a, st) : fn<float, 32>(a, st);         \
    case 64: return dtype == DT_BF16 ? fn<bf16_t, 64>(a, st) : fn<float, 64>(a, st);         \
    case 128: return dtype == DT_BF16 ? fn<bf16_t, 128>(a, st) : fn<float, 128>(a, st);      \
  }                                                                                          \
  return hipErrorInvalidValue;

hipError_t launch_flash(const FlashArgs& a, int hd, int dtype, hipStream_t st) { TANDEM_FLASH_DISPATCH(run) }
hipError_t launch_flash_backward(const FlashArgs& a, int hd, int dtype, hipStream_t st) {
  TANDEM_FLASH_DISPATCH(run_backward)
}

}  // namespace tandem
