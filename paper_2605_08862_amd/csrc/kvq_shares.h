// How attention over the 8-bit cache is cut into equal shares, and in which order the parts of a unit are merged: the arithmetic, on the device as on the host.
#pragma once
#include "common.h"

constexpr int kStep = 4 * kTile;                       // tokens of a step: a tile for each wave

__host__ __device__ __forceinline__ int least_of(int a, int b) { return a < b ? a : b; }
__host__ __device__ __forceinline__ int most_of(int a, int b) { return a > b ? a : b; }
__host__ __device__ __forceinline__ int high_product(uint32_t a, uint32_t b) {
#if defined(__HIP_DEVICE_COMPILE__)
  return (int)__umulhi(a, b);
#else
  return (int)((uint64_t)a * b >> 32);
#endif
}

// All units in a row (sequence, KV head, block) have a length: kUnitHalf, step_cost for each of their steps, kUnitHalf, in units of 1/8 step of a launch that is bound
// by memory.  The workgroups cut that into W equal parts; a cut is moved to the next step's start, and to the unit's end or start where less than kSnap + 1
// steps would be left on that side.  So a share is a run of steps, and what a unit costs besides its steps (its queries, the merge of the waves) counts.
// Measured in the wide kernel, 128 sequences of 1 .. 17 rows and 500 .. 32000 tokens, 7B heads: a step of up to 32, 64 and more rows 0.97, 1.25 and 2.27 us, a unit
// besides its steps 10 us.  With 12 for the last, and 8 for both others, this batch took 227 us and 100 sequences around 3000 tokens 114; with 14 211 and 107, with 15 209
// and 103; kUnitHalf 24, 28, 32, 36: 211, 210, 209, 211 and 106, 104, 103, 105.
// Of the kernel for few rows 4, 8, 12: 64 x 1 row of 500 .. 32000 tokens 88, 86, 87 us; 1.5B heads, 256 x 1 .. 5 rows around 1500 tokens 79, 76, 76.
constexpr int kSnap = 2;
template <bool WIDE> constexpr int kUnitHalf = WIDE ? 32 : 8;             // on either side of a unit's steps
template <bool WIDE> __host__ __device__ __forceinline__ int step_cost(int R) { return !WIDE ? 8 : R > 64 ? 15 : R > 32 ? 8 : 6; }
template <bool WIDE> constexpr int kBlock = WIDE ? 128 : 32;          // rows of a block
// Query heads of a KV head.  x / g by a product with 2^32 / g rounded up: exact for x below 2^32 / g, i.e. any packed row.
struct Group {
  int g;
  uint32_t recip;
  __host__ __device__ __forceinline__ int div(int x) const { return g == 1 ? x : high_product((uint32_t)x, recip); }
};
inline Group make_group(int g) { return Group{g, g == 1 ? 0 : (uint32_t)((((uint64_t)1 << 32) + g - 1) / g)}; }
// Steps of the block qb of a sequence of n rows behind c tokens: of the tokens that its last row sees.
template <int RP> __host__ __device__ __forceinline__ int block_steps(int c, int n, Group G, int qb) { return (c + least_of(n - 1, G.div((qb + 1) * RP - 1)) + kStep) / kStep; }

struct Shares {
  int total, W;                                         // length of everything, workgroups that have a share
  unsigned long long per;                               // length of a share, 16 bits of fraction
  float inv;                                            // its reciprocal
  __host__ __device__ __forceinline__ int bound(int w) const { return w >= W ? total : (int)((w * per) >> 16); }
  // the largest w with bound(w) <= p
  __host__ __device__ __forceinline__ int of(int p) const {
    int w = least_of(W - 1, (int)((float)p * inv));
    while (w > 0 && bound(w) > p) --w;
    while (w + 1 < W && bound(w + 1) <= p) ++w;
    return w;
  }
};

// Of `total` for a launch of `grid` workgroups.  A share is no shorter than kLeastShare, and longer than two steps, so that every share between two others of a
// unit has a step of it.
constexpr int kLeastShare = 32;
__host__ __device__ __forceinline__ Shares make_shares(int total, int grid) {
  Shares sh;
  sh.total = total;
  sh.W = least_of(grid, most_of(1, total / kLeastShare));
  sh.per = (unsigned long long)((double)sh.total * 65536.0 / (double)sh.W);    // the same in every workgroup; (W - 1) per is below the total
  sh.inv = (float)sh.W / (float)most_of(sh.total, 1);
  return sh;
}
// Blocks of 32 rows on four waves, two workgroups on a CU, or of up to 128 rows on eight waves.  The second reads K/V once for four times the rows, but has
// more to do before and behind its steps, so it needs many units (of 128 rows) and much to read; the block table's width is what the host knows of the lengths.
// Narrow and wide, us: 7B heads, 17 rows, 32 units of 20000 tokens 69 and 80, 36 of 20000 122 and 80; 64 units of 1000 tokens (1024 pages) 22 and 27, 2800 (2816)
// 38 and 38, 4000 (4032) 48 and 44, 8000 84 and 61; 512 units of 100 (1024) 29 and 27, 250 (2560) 39 and 36; 9 rows, 512 units of 250 tokens (2560) 23 and 28, 500 (4096) 30
// and 30, 1000 52 and 45; 1.5B heads, 9 rows, 128 units of 1000 tokens (2048) 22 and 22, 2000 (4096) 30 and 26; prompts of 7B heads, 500 rows (896) 19 and 23, 1000
// rows (3520) 40 and 33.
constexpr int kWideUnits = 32, kWidePages = 2560;
inline bool is_wide(long long rows) { return rows > kBlock<false>; }         // rows: the most (query row x head) of a sequence and KV head
inline bool runs_wide(int B, int Hkv, long long rows, int max_pages) {
  const long long units = B * Hkv * ((rows + kBlock<true> - 1) / kBlock<true>);
  return is_wide(rows) && units > kWideUnits && units * max_pages > kWidePages;
}
// Workgroups of a launch: no more than shares, of sequences as long as the block table is wide.
inline int share_workgroups(bool wide) { return (wide ? 1 : 2) * kCUs; }
inline int share_grid(bool wide, int B, int Hkv, long long rows, int max_pages) {
  const int RP = wide ? kBlock<true> : kBlock<false>, half = wide ? kUnitHalf<true> : kUnitHalf<false>;
  const long long most = (long long)B * Hkv * ((rows + RP - 1) / RP) * (2 * half + 15 * (max_pages / 2 + 1)) / kLeastShare + 1;
  return (int)(most < share_workgroups(wide) ? most : share_workgroups(wide));
}

template <bool WIDE>
struct Unit {
  int b, h, qb, blocks;                                 // sequence, KV head, block of its blocks
  int n, c, row0, slot;                                 // rows of the sequence, tokens before them, first packed row
  int first, steps, step;                               // where the unit begins, its steps, what one costs
  __host__ __device__ __forceinline__ int end() const { return first + 2 * kUnitHalf<WIDE> + step * steps; }
  // step at which a cut at p is made
  __host__ __device__ __forceinline__ int cut(int p) const {
    const int x = most_of(p - first - kUnitHalf<WIDE>, 0) + step - 1, j = high_product((uint32_t)x, step == 8 ? 536870912u : step == 15 ? 286331154u : 715827883u);   // / step
    return p >= end() ? steps : p <= first + kUnitHalf<WIDE> + kSnap * step ? 0 : steps - j <= kSnap ? steps : j;
  }
  // the first and the last workgroup that have steps of the unit
  __host__ __device__ __forceinline__ int first_share(const Shares& sh) const { return sh.of(least_of(first + kUnitHalf<WIDE> + kSnap * step, sh.total - 1)); }
  __host__ __device__ __forceinline__ int last_share(const Shares& sh) const { return sh.of(first + kUnitHalf<WIDE> + most_of(step * (steps - kSnap - 1), kSnap * step)); }
};
template <bool WIDE>
__host__ __device__ __forceinline__ void fill_unit(Unit<WIDE>& u, Group G) {
  constexpr int RP = kBlock<WIDE>;
  u.steps = block_steps<RP>(u.c, u.n, G, u.qb);
  u.step = step_cost<WIDE>(u.n * G.g - u.qb * RP);
}

// ---- merge of the n parts of a unit ----------------------------------------------------------------------------------------------
// On level L the parts 0, F^L, 2 F^L, .. are left; F neighbours of them make a group, which its last to arrive merges into its first (F = 2^log_f).  A part that
// has no neighbour on a level, the last one, goes on to the next with nothing done: its maximum and sum stay on the level that they were written on, and whoever
// merges it looks for them there.
// Level on which part i, left on `level`, has its maximum and sum: behind the last level on which its group had a second part.
__host__ __device__ __forceinline__ int pair_level(int i, int n, int level, int log_f) {
  while (level > 0 && i + (1 << (log_f * (level - 1))) >= n) --level;
  return level;
}
// The way of the workgroup that has stored part i: arrive(level, i0, count) publishes what it has stored and says whether it is the last of the group of `count`
// parts that begins at i0; merge(level, i0, stride, count, lone_level, last) merges them, the last of them from lone_level (all others from `level`).
template <typename Arrive, typename Merge>
__host__ __device__ __forceinline__ void merge_levels(int i, int n, int log_f, const Arrive& arrive, const Merge& merge) {
  for (int level = 0, stride = 1; stride < n; ++level, stride <<= log_f) {
    i &= -(stride << log_f);
    const int count = least_of(1 << log_f, (n - i + stride - 1) / stride);
    if (count == 1) continue;
    if (!arrive(level, i, count)) return;
    merge(level, i, stride, count, pair_level(i + (count - 1) * stride, n, level, log_f), (stride << log_f) >= n);
  }
}
