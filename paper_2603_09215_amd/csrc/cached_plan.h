// How attention over a paged cache is cut (cached_attend.h): plain arithmetic on its sizes.
#pragma once
#include <algorithm>

namespace spark {

constexpr int MOST_SPLITS = 256;

// `tiles` tiles of `pairs` (row, head) pairs at most for each kv head, their tokens in `splits` parts
struct AttendPlan {
  int pairs, splits;
  long long tiles;
};

// Parts are joined by a workgroup for each vector where there are few of these (one step of 28 heads, 1537 slots in 13 parts, both launches: 9.5 us, by a
// group of lanes for each 11.2; 16 rows of it, 30000 slots in 64 parts: 30 and 37; but 1024 vectors of 4 parts 50.3 and 49.2, 3584 of 8 29.7 and 25.5).
inline bool join_by_workgroups(long long vectors) { return vectors <= 512; }

// Tiles are numbered by rows, or by pairs with one more for each sequence: whichever takes fewer numbers.  Neither is fewer than there are.
inline long long attend_numbers_by_row(int pairs, int group, int m) { return (long long)m * ((group + pairs - 1) / pairs); }
inline long long attend_numbers_by_pair(int pairs, int group, int m, int n) { return (long long)m * group / pairs + n; }
inline bool attend_tiles_by_row(int pairs, int group, int m, int n) { return attend_numbers_by_row(pairs, group, m) <= attend_numbers_by_pair(pairs, group, m, n); }

// A kernel's step over `tokens` tokens: us with one workgroup to a compute unit, and where some have more; and a workgroup's start and end
struct AttendKind { int pairs, tokens, room; float us_one, us_full, us_ends; };
// [head_dim 128][kernel]: streams of pieces (four waves' pieces a step), tiles of four waves and of eight (which heads of 64 gain nothing by: 95 us and 83 for
// 4000 rows of 16 heads; of 128: 528 and 545 for 8191 rows of 28)
constexpr AttendKind ATTEND_BF16[2][3] = {{{16, 128, 2, 1.2f, 2.0f, 2.0f}, {128, 64, 2, 1.3f, 1.35f, 3.0f}, {}},
                                          {{16, 128, 2, 1.55f, 3.2f, 2.0f}, {128, 64, 2, 1.83f, 2.2f, 3.0f}, {256, 64, 1, 2.17f, 2.17f, 5.0f}}};
constexpr AttendKind ATTEND_FP32[2] = {{16, 64, 2, 1.4f, 1.9f, 2.0f}, {16, 64, 2, 2.0f, 3.5f, 2.0f}};

// The plan whose estimate is shortest: rounds of workgroups, each as many steps as its share of the slots has; parts are written, read and
// joined by a launch of their own (4 us, 0.25 a part or by workgroups 0.04, and its bytes at 4 TB/s).  Slots and rows are what a call's tensors have room for: the
// host does not know lengths, so a batch of short sequences in long tables is cut finer than it need be.  Steps' times
// are fitted to sweeps of kernels and parts at 65 batches (1 to 64 sequences, 1 to 8191 rows, 300 to 60000 slots), with probabilities of one part.  With two, of which a tile's
// step takes 1.2 to 1.3 times as long, the plans of 46 batches are 5 % from the fastest on average, of heads of 64 8 %; the worst are 511 rows over 32768 slots
// (1.5 times) and 2 sequences of 300 rows over 7696 (1.4), and other constants of this form chose no better.
inline AttendPlan attend_plan(bool fp32, int head_dim, int n_kv_heads, int group, int m, int n, long long slots, int n_cu) {
  AttendPlan best{16, 1, 1};
  float best_us = 1e30f;
  const AttendKind *kinds = fp32 ? &ATTEND_FP32[head_dim == 128] : ATTEND_BF16[head_dim == 128];
  for (int i = 0; i < (fp32 ? 1 : 3); ++i) {
    const AttendKind &k = kinds[i];
    if (k.pairs == 0) continue;
    const long long tiles = std::min(attend_numbers_by_row(k.pairs, group, m), attend_numbers_by_pair(k.pairs, group, m, n));
    const float all = (float)(tiles * n_kv_heads), steps = (float)((slots + k.tokens - 1) / k.tokens);
    const long long vectors = (long long)m * group * n_kv_heads;
    const float part_us = (join_by_workgroups(vectors) ? 0.04f : 0.25f) + (float)vectors * head_dim * 8.0f / 4e6f;
    for (int s = 1; s <= MOST_SPLITS && (s == 1 || s <= steps); s += 1 + s / 32) {
      const float wgs = all * s;
      const float rounds = std::max(1.0f, wgs / (k.room * n_cu));
      const float us = rounds * ((float)(long long)((steps + s - 1) / s) * (wgs > n_cu ? k.us_full : k.us_one) + k.us_ends) +
                       (s > 1 ? 4.0f + s * part_us : 0.0f);
      if (us < best_us) {
        best_us = us;
        best = AttendPlan{k.pairs, s, tiles};
      }
    }
  }
  return best;
}

}  // namespace spark
