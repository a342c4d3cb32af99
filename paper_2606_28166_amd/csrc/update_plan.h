// Which form attention's launches take, from sizes and types alone.  Plain C++: the
// tests compile it for the host.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace tandem {

constexpr int kFlashWaves = 4;             // waves of a workgroup

// Query heads of a key head that share a workgroup (the rest of its waves take other
// positions): the largest power of two that divides the group, up to the waves.
constexpr int heads_together(int group) {
  int n = 1;
  while (2 * n <= kFlashWaves && group % (2 * n) == 0) n *= 2;
  return n;
}

// With the keys shared out, whether a wave holds two tiles of 32 keys and values in LDS, or one:
// 64 KB at most for the four waves' tiles, so two workgroups to a compute unit, but for
// float32 heads of 128, whose one tile takes 128 KB.  One sequence of 4000, 8 heads of 128 on 1, bf16,
// forward and backward 59 and 160 us; two in turn and one workgroup 86 and 182.
constexpr bool two_turns(int hd, bool bf16) { return 32 * hd * (bf16 ? 2 : 4) <= 4096; }

// Whether the tiles of queries are so few that the keys are shared out: below two workgroups per
// compute unit, if there are tiles enough to share (with one tile of a wave in LDS, more).
// Forward, us: one sequence of 2000, float32, 4 heads of 32 on 2, 86 and shared 34; bf16, one of 8703, 2 heads
// of 64 on 2, 135 and 53; one of 2000, 16 of 128 on 8, 47 and 42.  Not so few: 64 of at most 1000,
// float32, 108 and 139; one of 8703, 16 of 64 on 4, 191 and 271.  Short: eight of at most 373, 16 of
// 128 on 8, 19 and 23.  What the rule gives away: 20 of at most 299, 8 of 64 on 2, are shared and take 44 backward,
// not 39; four of at most 7998, float32, 4 of 32 on 2, are not and take 571 forward, not 319.
// The lengths are on the device: here, and in flash_parts, a sequence counts as N / n_seqs rows.  Rows of no
// sequence and empty sequences shift that mean, so a batch padded to a fixed size may take the
// form that suits its padded size: as exact, but slower.
inline bool few_queries(int N, int n_seqs, int nq, int nkv, int hd, bool bf16) {
  const int together = heads_together(nq / nkv);
  const int64_t workgroups = ((int64_t)N * together / (32 * kFlashWaves) + n_seqs / 2) * (nq / together);
  return workgroups < 512 && N / n_seqs >= (two_turns(hd, bf16) ? 160 : 512);
}

// dK and dV by pairs of waves, of 64 keys to a workgroup (the other form: 128).
constexpr bool keys_by_pairs(int hd, bool bf16) { return bf16 && hd >= 64; }

// How many parts the work on a tile of keys is cut into.
// Tiles of keys (64, or 128 of the other form) differ in work by as much as their sequence is
// long.  Below a workgroup per compute unit, and the longer the sequences below the more rounds
// of those that fit the device together, they are cut into parts that give `want`
// workgroups, four at least, unless a part would be shorter than about 8 steps.  Backward pass whole and
// in parts, us:
//   bf16    one sequence of 32768, 16 heads of 64 on 4, 8126 and 7310; four of 4096 753 and 570;
//           three of 2048, 32 of 128 on 8, 507 and 447; 20 of at most 1973, 8 of 64 on 2, 242 and 160
//   float32 four of at most 7998, 4 heads of 32 on 2, 2111 and 1344; one of 2000, 16 heads of 64
//           on 4, 1171 and 307
// Of short ones the sums cost more than the evenness gains: bf16, 24 of 1200, heads of 64 on 4, 375
// and 418; six of 1100, 32 of 128 on 8, 295 and 334; 32 of 2304, 16 of 64 on 4, 1518 and 1570.
inline int flash_parts(int N, int n_seqs, int nq, int nkv, int hd, bool bf16) {
  if (n_seqs < 1) return 1;
  const bool pairs = keys_by_pairs(hd, bf16);
  const int64_t tiles = (N / (pairs ? 64 : 128) + n_seqs / 2) * (int64_t)nkv, len = N / n_seqs;
  const int64_t want = pairs && hd == 128 ? 1024 : 2048;
  const int64_t few = std::min(want, want * len / (pairs ? 2048 : 512));
  if (tiles > std::max<int64_t>(256, few)) return 1;
  const int64_t most = std::min<int64_t>(16, len * (nq / nkv) / (pairs ? 256 : 64));
  return most < 2 ? 1 : (int)std::min(most, std::max<int64_t>(4, (want + tiles) / (tiles + 1)));
}

}  // namespace tandem
