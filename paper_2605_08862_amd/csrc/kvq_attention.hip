// Ragged causal attention over the 8-bit cache (codes, scales and element order: kvq.h).
//
// No work list.  A unit is (sequence, KV head, block of packed query rows); its K/V stream is cut into steps of 128 tokens, and the steps of all units, in a
// row, into equal shares, one for each workgroup (a multiple of the CUs).  Every workgroup finds its share from a prefix sum over the sequences that it makes
// itself.  A share can begin and end inside a unit: the workgroup then leaves a partial (rows, maximum, sum), and the last of a unit's workgroups to arrive
// merges them, in groups of four or eight where there are many (publish_arrival, common.h; nobody waits).
//   * Few rows: blocks of 32, four waves take a 32-token tile each of every step, with an online softmax of their own (attn_softmax.h), merged at the unit's end.
//     Many: blocks of 128, eight waves, kvq_wide_kernel.
//   * S^T = K Q^T and O^T = V^T P^T on the 32 x 32 x 16 f16 MFMA.  A lane's sixteen bytes of codes are operands of two K-steps: one conversion with the block's
//     scale gives two exact float16 values, so nothing is rounded that the 16-bit cache would not round.
#include "kvq.h"
#include "attn_softmax.h"
#include "kvq_shares.h"
#include <type_traits>

namespace {

struct KvqOut { void* p; int ld; };                    // ld > 0: float16 rows in chunk order (act_index); 0: bf16 [rows][Hq][D]

__device__ __forceinline__ f16x8 values8(uint32_t a, uint32_t b, float scale) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef _Float16 h2 __attribute__((ext_vector_type(2)));
  const h2 x = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)a, scale, false), y = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)a, scale, true);
  const h2 z = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)b, scale, false), w = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)b, scale, true);
  return f16x8{x[0], x[1], y[0], y[1], z[0], z[1], w[0], w[1]};
#else
  return f16x8{};
#endif
}
__device__ __forceinline__ f32x16 mfma32(f16x8 a, f16x8 b, f32x16 c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
#else
  return c;
#endif
}

// ---- the shares ------------------------------------------------------------------------------------------------------------------
// A sequence that the thread which counted it leaves for the others: the one that this workgroup's share begins in.
struct Seq { int b, n, c, slot; };
// Sum over the lanes up to this one.
__device__ __forceinline__ int wave_scan(int v) {
#if defined(__HIP_DEVICE_COMPILE__)
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);            // row_shr 1, 2, 4, 8: in rows of sixteen lanes
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);            // row_bcast 15 to rows 1 and 3, row_bcast 31 to rows 2 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
#endif
  return v;
}

// Called by all threads.  s_start, s_row [B + 1]: where every sequence begins, and its first packed row; s_scan: 2 words for each wave; s_seq: see above.
template <int THREADS, bool WIDE>
__device__ __forceinline__ Shares find_shares(const int32_t* __restrict__ seq_slot, const int32_t* __restrict__ seq_pos, const int32_t* __restrict__ seq_n, int n_add,
                                              int n_max, int B, int n_slots, int max_pages, Group G, int Hkv, int* s_start, int* s_row, int* s_scan, Seq* s_seq,
                                              int32_t* __restrict__ status) {
  constexpr int NW = THREADS / 64, RP = kBlock<WIDE>;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // few sequences: up to 64 threads share the blocks of one; many: a thread has a run of them
  int subs = 1;
  while (subs < 64 && 2 * subs * B <= THREADS) subs *= 2;
  const int per = subs > 1 ? 1 : (B + THREADS - 1) / THREADS, sub = tid & (subs - 1), at = tid / subs;
  const int lo = min(at * per, B), hi = min(lo + per, B);
  int cost = 0, rows = 0, fault = 0, n = 0, slot = 0, c = 0;
  for (int b = lo; b < hi; ++b) {
    if (sub == 0) { s_start[b] = cost; s_row[b] = rows; }
    n = seq_n[b] + n_add; slot = seq_slot[b]; c = seq_pos[b];
    if (n < 0 || n > n_max) { fault |= BS_FAULT_DRAFT_LEN; continue; }
    if (n == 0) continue;
    if (sub == 0) rows += n;
    if (slot < 0 || slot >= n_slots) { fault |= BS_FAULT_SLOT; continue; }
    if (c < 0 || (long long)c + n > (long long)max_pages * kPage) { fault |= BS_FAULT_KV_PAGES; continue; }
    int s = 0;
    for (int qb = sub; qb * RP < n * G.g; qb += subs) s += 2 * kUnitHalf<WIDE> + step_cost<WIDE>(n * G.g - qb * RP) * block_steps<RP>(c, n, G, qb);
    cost += s * Hkv;
  }
  if (fault && blockIdx.x == 0 && status) atomicOr(status, fault);
  const int is = wave_scan(cost), ir = wave_scan(rows);
  if (lane == 63) { s_scan[wave] = is; s_scan[NW + wave] = ir; }
  __syncthreads();
  int bs = is - cost, br = ir - rows, total = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    if (w < wave) { bs += s_scan[w]; br += s_scan[NW + w]; }
    total += s_scan[w];
  }
  const Shares sh = make_shares(__builtin_amdgcn_readfirstlane(total), (int)gridDim.x);
  const int p0 = sh.bound(blockIdx.x);
  const bool mine = bs <= p0 && p0 < bs + cost;
  if (mine && per == 1) *s_seq = Seq{at, n, c, slot};
  if (sub == 0)
    for (int b = lo; b < hi; ++b) {
      const int first = s_start[b] + bs, end = b + 1 < hi ? s_start[b + 1] + bs : bs + cost;
      s_start[b] = first;
      s_row[b] += br;
      if (mine && per > 1 && first <= p0 && p0 < end) *s_seq = Seq{b, seq_n[b] + n_add, seq_pos[b], seq_slot[b]};
    }
  if (tid == 0) s_start[B] = total;
  __syncthreads();
  return sh;
}

template <bool WIDE>
__device__ __forceinline__ void enter_sequence(Unit<WIDE>& u, const int* s_start, const int* s_row, const int32_t* __restrict__ seq_slot, const int32_t* __restrict__ seq_pos, const int32_t* __restrict__ seq_n, int n_add, Group G) {
  u.b = __builtin_amdgcn_readfirstlane(u.b);
  u.n = seq_n[u.b] + n_add;
  u.c = seq_pos[u.b];
  u.slot = seq_slot[u.b];
  u.row0 = __builtin_amdgcn_readfirstlane(s_row[u.b]);
  u.first = __builtin_amdgcn_readfirstlane(s_start[u.b]);
  u.blocks = (u.n * G.g + kBlock<WIDE> - 1) / kBlock<WIDE>;
  u.h = u.qb = 0;
  fill_unit<WIDE>(u, G);
}
// The unit that p lies in, of the sequence that p lies in.
template <bool WIDE>
__device__ __forceinline__ Unit<WIDE> unit_at(int p, const Seq& s, const int* s_start, const int* s_row, Group G, int Hkv) {
  Unit<WIDE> u;
  auto same = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  u.b = same(s.b); u.n = same(s.n); u.c = same(s.c); u.slot = same(s.slot); u.row0 = same(s_row[u.b]); u.first = same(s_start[u.b]);
  u.blocks = (u.n * G.g + kBlock<WIDE> - 1) / kBlock<WIDE>;
  u.h = u.qb = 0;
  fill_unit<WIDE>(u, G);
  const int head = u.blocks == 1 ? u.end() - u.first : (same(s_start[u.b + 1]) - u.first) / Hkv;
  int h = min(Hkv - 1, (int)((float)(p - u.first) / (float)head));
  while (h > 0 && h * head > p - u.first) --h;
  while (h + 1 < Hkv && (h + 1) * head <= p - u.first) ++h;
  u.h = same(h);
  u.first += u.h * head;
  while (u.end() <= p) { u.first = u.end(); ++u.qb; fill_unit<WIDE>(u, G); }
  return u;
}
// The unit behind; false behind the last one.
template <bool WIDE>
__device__ __forceinline__ bool next_unit(Unit<WIDE>& u, int B, int Hkv, const int* s_start, const int* s_row, const int32_t* __restrict__ seq_slot, const int32_t* __restrict__ seq_pos,
                                          const int32_t* __restrict__ seq_n, int n_add, Group G) {
  u.first = u.end();
  if (++u.qb < u.blocks) { fill_unit<WIDE>(u, G); return true; }
  u.qb = 0;
  if (++u.h < Hkv) { fill_unit<WIDE>(u, G); return true; }
  do { if (++u.b >= B) return false; } while (s_start[u.b + 1] == s_start[u.b]);
  enter_sequence<WIDE>(u, s_start, s_row, seq_slot, seq_pos, seq_n, n_add, G);
  return true;
}
// What a workgroup does of a unit.
struct Part {
  int slot, h, row0, qr0, R, c, s_lo, s_hi, n_tiles, c_all;   // qr0: first row (query row x head) of the block in the sequence; c_all: last position that every row sees
  int w_first, w_last;                                     // workgroups that have a part
  bool whole;
};
template <bool WIDE>
__device__ __forceinline__ Part part_of(const Unit<WIDE>& u, const Shares& sh, int s_lo, int s_hi, Group G) {
  constexpr int RP = kBlock<WIDE>;
  Part t;
  t.slot = u.slot; t.h = u.h; t.row0 = u.row0; t.c = u.c;
  t.qr0 = u.qb * RP;
  t.R = min(u.n * G.g - t.qr0, RP);
  t.s_lo = s_lo; t.s_hi = s_hi;
  t.n_tiles = (u.c + min(u.n - 1, G.div(t.qr0 + RP - 1))) / kTile + 1;
  t.c_all = u.c + G.div(t.qr0);
  t.whole = s_lo == 0 && s_hi == u.steps;
  t.w_first = t.w_last = blockIdx.x;
  if (!t.whole) {
    t.w_first = __builtin_amdgcn_readfirstlane(s_lo == 0 ? (int)blockIdx.x : u.first_share(sh));
    t.w_last = __builtin_amdgcn_readfirstlane(s_hi == u.steps ? (int)blockIdx.x : u.last_share(sh));
  }
  return t;
}
// Calls f(part) for every part of this workgroup's share.
template <bool WIDE, typename F>
__device__ __forceinline__ void for_parts(const Shares& sh, int B, const int* s_start, const int* s_row, const int32_t* __restrict__ seq_slot, const int32_t* __restrict__ seq_pos,
                                          const int32_t* __restrict__ seq_n, int n_add, Group G, int Hkv, const Seq& s_seq, const F& f) {
  const int w = blockIdx.x;
  if (w >= sh.W || sh.total == 0) return;
  const int p0 = __builtin_amdgcn_readfirstlane(sh.bound(w)), p1 = __builtin_amdgcn_readfirstlane(sh.bound(w + 1));
  Unit<WIDE> u = unit_at<WIDE>(p0, s_seq, s_start, s_row, G, Hkv);
  int s_lo = u.cut(p0);
  while (true) {
    const bool last = u.end() >= p1;
    const int s_hi = last ? u.cut(p1) : u.steps;
    const bool any = s_lo < s_hi;
    const Part part = part_of<WIDE>(u, sh, s_lo, s_hi, G);
    // the next unit is looked up in front of this one's work, which covers the trip to memory
    const bool more = !last && next_unit<WIDE>(u, B, Hkv, s_start, s_row, seq_slot, seq_pos, seq_n, n_add, G);
    if (any) f(part);
    s_lo = 0;
    if (!more) break;
  }
}
// Partial rows: two places for each workgroup, for a unit that began before its share and for one that goes on behind it.
template <int RP> __device__ __forceinline__ uint32_t partial_row(int w, bool began_here) { return (uint32_t)(2 * w + (began_here ? 1 : 0)) * RP; }

template <int D, bool STEP>
__device__ __forceinline__ void store4(const KvqOut& out, int Hq, int row, int col, f32x4 v, float inv, int32_t* status) {
  if constexpr (STEP) {
    *(f16x4*)((f16*)out.p + act_index(row, col, out.ld)) = to_f16x4_guarded(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv, status);
  } else {
    typedef bf16 b4 __attribute__((ext_vector_type(4)));
    *(b4*)((bf16*)out.p + (size_t)row * Hq * D + col) = b4{(bf16)(v[0] * inv), (bf16)(v[1] * inv), (bf16)(v[2] * inv), (bf16)(v[3] * inv)};
  }
}

// Four columns of row r of a block.
template <int D, bool STEP>
__device__ __forceinline__ void store_row(const KvqOut& out, int Hq, const Part& un, Group G, int r, int col, f32x4 v, float inv, int32_t* status) {
  const int qr = un.qr0 + r, i = G.div(qr);
  store4<D, STEP>(out, Hq, un.row0 + i, (un.h * G.g + qr - i * G.g) * D + col, v, inv, status);
}

// ---- merge of a unit's parts -------------------------------------------------------------------------------------------------------
// Partial rows: part_o [2 W][RP][D], and (maximum, sum) part_ml [kLevels][2 W][RP][2].  Parts are merged in groups of F neighbours by the last of a group to
// arrive, into the place of the group's first part, the merged parts again, and so on (merge_levels): a unit of 64 parts of 119 rows is 4 MB, which one workgroup alone read in
// 70 us of a launch of 88.  Maxima and sums of a level have a place of their own, since several threads read those of a row.
// counters [kLevels][kMaxShares], zero between launches; a workgroup is the first of at most one group of more than one part on every level.
constexpr int kLevels = 5, kMaxShares = 2 * kCUs;
struct Parts { float *o, *ml; int32_t* counters; };
template <int RP> constexpr uint32_t kMlLevel = (uint32_t)2 * kMaxShares * RP;      // rows of a level

// Merges `count` parts, `stride` apart from part i0 of the unit on, on level `level` (merge_levels).  An item is four columns of a row; the loads of NI items and GC parts are in
// flight together.
template <int THREADS, int RP, int D, bool STEP, int NI, int GC>
__device__ __forceinline__ void merge_group(const Part& un, const Parts& p, int level, int i0, int stride, int count, int lone_level, bool last, const KvqOut& out,
                                            int Hq, Group G, int32_t* status) {
  constexpr int CH = D / 4;
  const wt_buf bo = wt_buffer(p.o), bm = wt_buffer(p.ml);
  const int items = un.R * CH;
  const uint32_t to = partial_row<RP>(un.w_first + i0, i0 == 0);
  for (int it0 = threadIdx.x; it0 < items; it0 += THREADS * NI) {
    float m[NI], l[NI];
    f32x4 acc[NI];
#pragma unroll
    for (int k = 0; k < NI; ++k) { m[k] = -INFINITY; l[k] = 0.f; acc[k] = f32x4{0.f, 0.f, 0.f, 0.f}; }
    for (int c0 = 0; c0 < count; c0 += GC) {
      wt_f32x2 ml[GC][NI];
      f32x4 v[GC][NI];
#pragma unroll
      for (int u = 0; u < GC; ++u) {
        const int nth = min(c0 + u, count - 1), i = i0 + nth * stride;
        const uint32_t row = partial_row<RP>(un.w_first + i, i == 0), ml_row = (nth == count - 1 ? lone_level : level) * kMlLevel<RP> + row;
#pragma unroll
        for (int k = 0; k < NI; ++k) {                  // (an item behind the last one: the last one)
          const int it = min(it0 + k * THREADS, items - 1);
          ml[u][k] = wt_load2(bm, (ml_row + it / CH) * 8);
          v[u][k] = wt_load4(bo, ((row + it / CH) * D + it % CH * 4) * 4);
        }
      }
#pragma unroll
      for (int k = 0; k < NI; ++k) {
        float mg = m[k];
#pragma unroll
        for (int u = 0; u < GC; ++u) { if (c0 + u >= count) ml[u][k] = wt_f32x2{-INFINITY, 0.f}; mg = fmaxf(mg, ml[u][k][0]); }
        if (mg == -INFINITY) continue;
        const float f0 = __builtin_amdgcn_exp2f(m[k] - mg);
        l[k] *= f0;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[k][e] *= f0;
#pragma unroll
        for (int u = 0; u < GC; ++u) {
          const float f = __builtin_amdgcn_exp2f(ml[u][k][0] - mg);
          l[k] += ml[u][k][1] * f;
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[k][e] += v[u][k][e] * f;
        }
        m[k] = mg;
      }
    }
#pragma unroll
    for (int k = 0; k < NI; ++k) {
      const int it = it0 + k * THREADS;
      if (it >= items) continue;
      const int r = it / CH, ch = it % CH;
      if (!last) {
        wt_store4(bo, ((to + r) * D + ch * 4) * 4, acc[k]);
        if (ch == 0) wt_store2(bm, ((level + 1) * kMlLevel<RP> + to + r) * 8, m[k], l[k]);
      } else if (m[k] != INFINITY) {                    // (infinite: a bad page, the row stays as it is)
        store_row<D, STEP>(out, Hq, un, G, r, ch * 4, acc[k], 1.0f / l[k], status);
      }
    }
  }
}
// Called by all threads of a workgroup that has stored its part of a cut unit on level 0.
template <int THREADS, int RP, int D, bool STEP>
__device__ __forceinline__ void merge_unit(const Part& un, const Parts& p, const KvqOut& out, int Hq, Group G, int32_t* status, int* s_flag) {
  const bool few = un.R * (D / 4) <= THREADS;           // few rows, as of one long sequence: groups of eight
  merge_levels((int)blockIdx.x - un.w_first, un.w_last - un.w_first + 1, few ? 3 : 2,
               [&](int level, int i, int count) { return publish_arrival(p.counters + level * kMaxShares + un.w_first + i, count, s_flag); },
               [&](int level, int i, int stride, int count, int lone_level, bool last) {
                 if (count == 2 && !few) merge_group<THREADS, RP, D, STEP, 8, 2>(un, p, level, i, stride, count, lone_level, last, out, Hq, G, status);
                 else if (few) merge_group<THREADS, RP, D, STEP, 1, 8>(un, p, level, i, stride, count, lone_level, last, out, Hq, G, status);
                 else merge_group<THREADS, RP, D, STEP, 4, 4>(un, p, level, i, stride, count, lone_level, last, out, Hq, G, status);
               });
}

// Online softmax of one tile of scores (attn_softmax.h): the scores become probabilities in float16, the running maximum, sum and accumulators follow.
template <int DT>
__device__ __forceinline__ void softmax_tile(const f32x16& st, bool full, int tok0, int lim, float scale_log2e, float& m_run, float& l_run, f32x16 (&o)[DT], f16x8 (&pf)[2]) {
  float y[16];
  if (full) {                                           // the same for the wave
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = st[i];
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = tok0 + i <= lim ? st[i] : -INFINITY;
  }
  float mloc = y[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) mloc = fmaxf(mloc, y[i]);
  mloc = max_halves(mloc) * scale_log2e;                // scale > 0 commutes with max
  if (__any(mloc > m_run + kLateRescale)) {
    const float m_new = fmaxf(m_run, mloc);
    const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
    l_run *= alpha;
    m_run = m_new;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[dt][i] *= alpha;
  }
  const float m_safe = m_run == -INFINITY ? 0.f : m_run;
  float psum = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    y[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(y[i], scale_log2e, -m_safe));
    psum += y[i];
  }
  l_run += psum;                                        // per half of the wave; the halves are added at the end
#pragma unroll
  for (int i = 0; i < 16; ++i) pf[i / 8][i % 8] = (f16)y[i];
}

// Sixteen bytes of a query row as float16.
template <bool STEP> __device__ __forceinline__ u32x4 query8(u32x4 v, bool& range) {
  if constexpr (STEP) return v;
  float y[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) { y[2 * e] = __uint_as_float(v[e] << 16); y[2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u); }
  f16x4 lo = f16x4{(f16)y[0], (f16)y[1], (f16)y[2], (f16)y[3]}, hi = f16x4{(f16)y[4], (f16)y[5], (f16)y[6], (f16)y[7]};
  if (f16x4_out_of_range(lo) || f16x4_out_of_range(hi)) {
    range = true;
    lo = f16x4{(f16)f16_saturate(y[0]), (f16)f16_saturate(y[1]), (f16)f16_saturate(y[2]), (f16)f16_saturate(y[3])};
    hi = f16x4{(f16)f16_saturate(y[4]), (f16)f16_saturate(y[5]), (f16)f16_saturate(y[6]), (f16)f16_saturate(y[7])};
  }
  const u32x2 a = __builtin_bit_cast(u32x2, lo), b = __builtin_bit_cast(u32x2, hi);
  return u32x4{a[0], a[1], b[0], b[1]};
}

#define BS_KVQ_PARAMS                                                                                                                                     \
  const int32_t *__restrict__ seq_slot, const int32_t *__restrict__ seq_pos, const int32_t *__restrict__ seq_n, int n_add, int n_max, int B,                \
      const int32_t *__restrict__ block_table, int n_slots, int max_pages, int n_pages, const uint8_t *__restrict__ k_pages, const uint8_t *__restrict__ v_pages, \
      const float *__restrict__ k_scale, const float *__restrict__ v_scale, int Hq, int Hkv, int g_n, uint32_t g_recip, float scale_log2e, const uint16_t *__restrict__ q, size_t q_stride, \
      KvqOut out, Parts parts, int32_t *__restrict__ status

// Blocks of up to 32 rows, four waves, two workgroups on a CU.  STEP: inside bs_verify_step (float16 queries, output in chunk order).  Every wave has two tiles of K
// and V codes in registers and loads the next but one behind the products that read them.
// What bounds it: memory, where there are steps enough (7B heads, 64 sequences of 4096 tokens, one row: 56 us, 4.8 TB/s); else the way to the first tile and the
// merges (1.5B heads, one row of 30001 tokens: 14.9 us).
template <int D, bool STEP>
__global__ void __launch_bounds__(256, 2) kvq_attention_kernel(BS_KVQ_PARAMS) {
  constexpr int KS = D / 16, DT = D / 32, RP = 32, CH = D / 4;
  constexpr int LDO = D + 4;                            // row stride (floats) of an accumulator in LDS
  extern __shared__ __align__(16) char lds_raw[];
  __shared__ int s_scan[8], s_flag;
  __shared__ Seq s_seq;
  u32x4* const s_q = (u32x4*)lds_raw;                   // [KS][64] query fragments; behind a unit's last product, the waves' accumulators
  float* const s_o = (float*)lds_raw;                   // [4][32][LDO]
  float* const s_m = s_o + 4 * 32 * LDO;                // [4][32]
  float* const s_l = s_m + 4 * RP;
  int* const s_start = (int*)(s_l + 4 * RP);            // [B + 1]
  int* const s_row = s_start + B + 1;                   // [B + 1]
  const int tid = threadIdx.x, w_id = blockIdx.x;
  const Group G{g_n, g_recip};
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, ln = lane & 31, lg = lane >> 5;
  const Shares sh = find_shares<256, false>(seq_slot, seq_pos, seq_n, n_add, n_max, B, n_slots, max_pages, G, Hkv, s_start, s_row, s_scan, &s_seq, status);
  for_parts<false>(sh, B, s_start, s_row, seq_slot, seq_pos, seq_n, n_add, G, Hkv, s_seq, [&](const Part& un) {
    const int32_t* __restrict__ bt = block_table + (size_t)un.slot * max_pages;
    const int t0 = 4 * un.s_lo + wave, t_end = min(4 * un.s_hi, un.n_tiles);
    const int n_my = t0 < t_end ? (t_end - t0 + 3) / 4 : 0, t_last = t0 + (n_my - 1) * 4;
    bool bad = false;

    struct At { size_t off; float ks, vs; };
    auto place = [&](int t) -> At {
      int page = bt[t * kTile / kPage];
      if ((unsigned)page >= (unsigned)n_pages) { page = 0; bad = true; }
      return At{(size_t)page * ((size_t)Hkv * kPage * D) + (size_t)(un.h * 2 + (t & 1)) * (kTile * D) + lane * 16, k_scale[(size_t)page * Hkv + un.h],
                v_scale[(size_t)page * Hkv + un.h]};
    };
    auto load_tile = [&](const uint8_t* base, size_t off, u32x4 (&f)[DT]) {
#pragma unroll
      for (int i = 0; i < DT; ++i) f[i] = *(const u32x4*)(base + off + i * 1024);
    };

    // queries first, the first two tiles behind them
    constexpr int QF = KS / 4;                          // fragments of each wave
    u32x4 qv[QF];
    {
      const int qr = un.qr0 + min(ln, un.R - 1), i = G.div(qr);              // rows behind the last one are masked
      const uint16_t* src = q + (size_t)(un.row0 + i) * q_stride + (size_t)(un.h * G.g + qr - i * G.g) * D + lg * (D / 2);
#pragma unroll
      for (int j = 0; j < QF; ++j) qv[j] = *(const u32x4*)(src + (wave + 4 * j) * 8);
    }
    u32x4 k0[DT], v0[DT], k1[DT], v1[DT];
    At a0 = place(n_my > 0 ? t0 : un.n_tiles - 1), a1 = place(n_my > 1 ? t0 + 4 : n_my > 0 ? t0 : un.n_tiles - 1);
    load_tile(k_pages, a0.off, k0);
    load_tile(v_pages, a0.off, v0);
    load_tile(k_pages, a1.off, k1);
    load_tile(v_pages, a1.off, v1);
    bool range = false;
#pragma unroll
    for (int j = 0; j < QF; ++j) s_q[(wave + 4 * j) * 64 + lane] = query8<STEP>(qv[j], range);
    if (range && status) atomicOr(status, BS_FAULT_RANGE);
    __syncthreads();
    const u32x4* my_q = s_q + lane;

    f32x16 o[DT];
    float m_run = -INFINITY, l_run = 0.f;
    const int lim = ln < un.R ? un.c + G.div(un.qr0 + ln) : -1;              // last visible position of the lane's row
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;

    auto tile = [&](auto pref, int t, int t_pref, u32x4 (&kc)[DT], u32x4 (&vc)[DT], At& at) {
      constexpr bool PREF = decltype(pref)::value;
      At next{0, 1.f, 1.f};
      if (PREF) next = place(t_pref);
      f32x16 st;
#pragma unroll
      for (int i = 0; i < 16; ++i) st[i] = 0.f;
#pragma unroll
      for (int s = 0; s < KS; ++s) st = mfma32(values8(kc[s / 2][2 * (s % 2)], kc[s / 2][2 * (s % 2) + 1], at.ks), as_f16x8(my_q[s * 64]), st);
      __builtin_amdgcn_sched_barrier(0);
      if (PREF) load_tile(k_pages, next.off, kc);
      __builtin_amdgcn_sched_barrier(0);
      f16x8 pf[2];                                       // accumulator register i <-> token t * kTile + 16 lg + i
      softmax_tile<DT>(st, (t + 1) * kTile - 1 <= un.c_all, t * kTile + 16 * lg, lim, scale_log2e, m_run, l_run, o, pf);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int t2 = 0; t2 < 2; ++t2) o[dt] = mfma32(values8(vc[dt][2 * t2], vc[dt][2 * t2 + 1], at.vs), pf[t2], o[dt]);
      __builtin_amdgcn_sched_barrier(0);
      if (PREF) load_tile(v_pages, next.off, vc);
      at = next;
      __builtin_amdgcn_sched_barrier(0);
    };
    {
      int i = 0;
      for (; i + 2 <= n_my; i += 2) {
        const int t = t0 + i * 4;
        tile(std::true_type{}, t, min(t + 8, t_last), k0, v0, a0);
        tile(std::true_type{}, t + 4, min(t + 12, t_last), k1, v1, a1);
      }
      if (i < n_my) tile(std::false_type{}, t0 + i * 4, 0, k0, v0, a0);
    }

    // ---- merge of the waves
    const uint32_t part = partial_row<RP>(w_id, w_id == un.w_first);
    const wt_buf bo = wt_buffer(parts.o), bm = wt_buffer(parts.ml);
    if (bad && lane == 0 && status) atomicOr(status, BS_FAULT_KV_PAGES);
    l_run = sum_halves(l_run);
    if (lg == 0) { s_m[wave * RP + ln] = bad ? INFINITY : m_run; s_l[wave * RP + ln] = l_run; }
    __syncthreads();                                    // the fragments are no longer read
    float* mine = s_o + (size_t)wave * 32 * LDO;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4)
        *(f32x4*)(mine + ln * LDO + dt * 32 + 8 * i4 + 4 * lg) = f32x4{o[dt][4 * i4], o[dt][4 * i4 + 1], o[dt][4 * i4 + 2], o[dt][4 * i4 + 3]};
    __syncthreads();
    for (int it = tid; it < un.R * CH; it += 256) {
      const int r = it / CH, ch = it % CH;
      float mw[4], mt = -INFINITY, lt = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) { mw[w] = s_m[w * RP + r]; mt = fmaxf(mt, mw[w]); }
      f32x4 acc{0.f, 0.f, 0.f, 0.f};
      if (mt != -INFINITY && mt != INFINITY)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float f = __builtin_amdgcn_exp2f(mw[w] - mt);
          lt += s_l[w * RP + r] * f;
          const f32x4 v = *(const f32x4*)(s_o + ((size_t)w * 32 + r) * LDO + ch * 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[e] += v[e] * f;
        }
      if (!un.whole) {
        wt_store4(bo, ((part + r) * D + ch * 4) * 4, acc);
        if (ch == 0) wt_store2(bm, (part + r) * 8, mt, lt);
      } else if (mt != INFINITY) {
        store_row<D, STEP>(out, Hq, un, G, r, ch * 4, acc, 1.0f / lt, status);
      }
    }
    if (!un.whole) merge_unit<256, RP, D, STEP>(un, parts, out, Hq, G, status, &s_flag);
    __syncthreads();                                    // LDS is the next unit's
  });
}

// Waits until at most N of this wave's requests are in flight (and for its LDS accesses), then for the other waves.
template <int N> __device__ __forceinline__ void wait_requests() {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
#endif
}
// A word or sixteen bytes of each lane from memory to LDS (dst: the same in all lanes, the first lane's place).
__device__ __forceinline__ void copy_word_to_lds(const void* src, char* dst) {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src, (__attribute__((address_space(3))) void*)dst, 4, 0, 0);
#endif
}
__device__ __forceinline__ void copy_to_lds(const uint8_t* src, char* dst) {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src, (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
#endif
}

// Blocks of up to 128 rows, eight waves: NQT = 2 or 4 query tiles by the rows of the unit and NPH = 8 / NQT token phases, which work on different token tiles; wave
// w has phase w % NPH of query tile w / NPH, so that the waves of a SIMD (w % 4) are of different query tiles.  The waves of a phase share a tile of codes in LDS:
// the memory pipeline copies it there (global -> LDS loads, a share of the 1 KiB pieces by each wave), NB buffers for each phase, NB - 1 tiles in flight and one
// barrier per tile.
// What bounds it: two query tiles, memory; four, that matrix and vector instructions of the two waves of a SIMD overlap in part only.  7B heads, 32 sequences of 8192
// tokens (memory 57 us), 9 rows 64 .. 68 us, 17 rows 98 .. 103.  Of the latter, at 105 then, with parts left out: the way to the first tile and the merges 22, copying the tiles
// alone 69, matrix instructions alone 84 (half of their nominal rate, as a large matrix product has it too), everything but them 87, everything but the softmax 90,
// everything but the conversions 100.  Two tiles per barrier, a tile of K read ahead, requests behind the scores: the same or slower; twelve waves with three phases:
// 12 us more; scores of the next tile multiplied while this one's become probabilities: 10 us more; the two waves of a SIMD held half a tile apart by barriers: 10 us more;
// two query tiles in a wave, which halves the conversions, with queries in LDS: 17 rows 101, 9 rows 70.  Scores from 8-bit products (queries split into e4m3 terms) took
// 17 rows to 96 us, but the matrix unit sums those eight at a time at the place of the largest and drops what is below 2^-13 of it: K with one large channel is then
// read wrongly.
template <int D> constexpr int kWideStage = 96 * 1024 * D / 128;
constexpr int kWideScales = 6 * 8 * 256;                // [buffers][waves] K and V scale in the first two words
template <int D, bool STEP>
__global__ void __launch_bounds__(512) kvq_wide_kernel(BS_KVQ_PARAMS) {
  constexpr int KS = D / 16, DT = D / 32, RP = 128, CH = D / 4;
  constexpr int DH = D / 2, LDO = DH + 4;               // the accumulators are merged in two halves of the columns
  extern __shared__ __align__(16) char lds_raw[];
  __shared__ int s_scan[16], s_bad, s_flag;
  __shared__ Seq s_seq;
  float* const s_o = (float*)lds_raw;                   // [8][32][LDO], on top of the codes
  char* const s_scale = lds_raw + kWideStage<D>;
  float* const s_m = (float*)(s_scale + kWideScales);   // [8][32]
  float* const s_l = s_m + 8 * 32;
  int* const s_start = (int*)(s_l + 8 * 32);            // [B + 1]
  int* const s_row = s_start + B + 1;                   // [B + 1]
  const int tid = threadIdx.x, w_id = blockIdx.x;
  const Group G{g_n, g_recip};
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, ln = lane & 31, lg = lane >> 5;
  const Shares sh = find_shares<512, true>(seq_slot, seq_pos, seq_n, n_add, n_max, B, n_slots, max_pages, G, Hkv, s_start, s_row, s_scan, &s_seq, status);

  auto run = [&](auto nqt_tag, const Part& un) {
    constexpr int NQT = decltype(nqt_tag)::value, NPH = 8 / NQT;
    constexpr int NF = 2 * DT, LPW = NF / NQT;          // 1 KiB pieces of a tile, K then V; of those a wave moves
    constexpr int NB = kWideStage<D> / (NPH * NF * 1024);     // buffers: 3 or 6
    const int32_t* __restrict__ bt = block_table + (size_t)un.slot * max_pages;
    const int qt = wave / NPH, ph = wave % NPH;
    const bool has_rows = qt * 32 < un.R;               // a wave without query rows only moves data
    const int t_begin = 4 * un.s_lo, t_end = min(4 * un.s_hi, un.n_tiles), n_it = (t_end - t_begin + NPH - 1) / NPH;
    bool bad = false;
    auto tile_of = [&](int i) { return min(t_begin + ph + NPH * i, un.n_tiles - 1); };   // a phase without a tile moves the last one again
    auto page_of = [&](int i) { return bt[tile_of(i) * kTile / kPage]; };
    const size_t head = (size_t)un.h * (kPage * D) + lane * 16;
    auto request = [&](int page, int i, int buf) {      // this wave's share: pieces qt, qt + NQT, ..
      if ((unsigned)page >= (unsigned)n_pages) { bad = true; page = 0; }
      const size_t off = (size_t)page * ((size_t)Hkv * kPage * D) + (size_t)(tile_of(i) & 1) * (kTile * D) + head;
#pragma unroll
      for (int j = 0; j < LPW; ++j) {
        const int f = qt + NQT * j;
        const bool is_k = NQT * (j + 1) <= DT ? true : NQT * j >= DT ? false : f < DT;
        copy_to_lds((is_k ? k_pages : v_pages) + off + (is_k ? f : f - DT) * 1024, lds_raw + ((size_t)(buf * NPH + ph) * NF + f) * 1024);
      }
      // the scales the same way: as scalar loads they were a trip to memory that every iteration waited for
      copy_word_to_lds((lane == 0 ? k_scale : v_scale) + (size_t)page * Hkv + un.h, s_scale + (buf * 8 + wave) * 256);
    };
    const int qr = qt * 32 + ln;
    const int lim = qr < un.R ? un.c + G.div(un.qr0 + qr) : -1;
    u32x4 qf[KS];
    {
      const int qc = un.qr0 + min(qr, un.R - 1), i = G.div(qc);
      const uint16_t* src = q + (size_t)(un.row0 + i) * q_stride + (size_t)(un.h * G.g + qc - i * G.g) * D + lg * (D / 2);
#pragma unroll
      for (int s = 0; s < KS; ++s) qf[s] = *(const u32x4*)(src + s * 8);
    }
    // the query loads in front and the requests unconditional, so that the wait for the queries leaves the requests in flight
    int first_pages[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) first_pages[i] = page_of(i);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < NB - 1; ++i) request(first_pages[i], i, i);
    int next_page = first_pages[NB - 1];
    __builtin_amdgcn_sched_barrier(0);
    bool range = false;
#pragma unroll
    for (int s = 0; s < KS; ++s) { asm volatile("" : "+v"(qf[s])); qf[s] = query8<STEP>(qf[s], range); }
    f32x16 o[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;
    int buf = 0;
    // matrix instructions and what feeds them go first: the other wave of the SIMD takes the vector instructions of its softmax meanwhile (17 rows 105 -> 99 us)
    __builtin_amdgcn_s_setprio(1);
    for (int i = 0; i < n_it; ++i) {
      // this wave's share of tile i has arrived (the up to NB - 2 requested behind it may be in flight), then everybody's; nobody reads tile i - 1 any more,
      // whose buffer takes tile i + NB - 1.  Behind the end the last one is requested again: the counts hold all the way.
      wait_requests<(NB - 2) * (LPW + 1)>();
      __builtin_amdgcn_sched_barrier(0);
      request(next_page, i + NB - 1, buf == 0 ? NB - 1 : buf - 1);
      next_page = page_of(i + NB);
      __builtin_amdgcn_sched_barrier(0);
      const int t = t_begin + ph + NPH * i;
      if (has_rows && t < t_end) {
        const char* at = lds_raw + (size_t)(buf * NPH + ph) * NF * 1024 + lane * 16;
        const u32x2 scales = *(const u32x2*)(s_scale + (buf * 8 + wave) * 256);
        const float ks = __uint_as_float(scales[0]), vs = __uint_as_float(scales[1]);
        u32x4 kc[DT], vc[DT];
#pragma unroll
        for (int s = 0; s < DT; ++s) kc[s] = *(const u32x4*)(at + s * 1024);
        __builtin_amdgcn_sched_barrier(0);
        f32x16 st;
#pragma unroll
        for (int r = 0; r < 16; ++r) st[r] = 0.f;
#pragma unroll
        for (int s = 0; s < KS; ++s) st = mfma32(values8(kc[s / 2][2 * (s % 2)], kc[s / 2][2 * (s % 2) + 1], ks), as_f16x8(qf[s]), st);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int s = 0; s < DT; ++s) vc[s] = *(const u32x4*)(at + (DT + s) * 1024);
        __builtin_amdgcn_sched_barrier(0);
        f16x8 pf[2];
        __builtin_amdgcn_s_setprio(0);
        softmax_tile<DT>(st, (t + 1) * kTile - 1 <= un.c_all, t * kTile + 16 * lg, lim, scale_log2e, m_run, l_run, o, pf);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int t2 = 0; t2 < 2; ++t2) o[dt] = mfma32(values8(vc[dt][2 * t2], vc[dt][2 * t2 + 1], vs), pf[t2], o[dt]);
      }
      buf = buf == NB - 1 ? 0 : buf + 1;
    }
    __builtin_amdgcn_s_setprio(0);
    if (bad && lane == 0) s_bad = 1;
    if (range && status) atomicOr(status, BS_FAULT_RANGE);
    wait_requests<0>();                                 // the codes' buffers become the accumulators'

    // ---- merge of the phases of every query tile, half of the columns at a time
    const uint32_t part = partial_row<RP>(w_id, w_id == un.w_first);
    const wt_buf bo = wt_buffer(parts.o), bm = wt_buffer(parts.ml);
    const bool bad_unit = s_bad != 0;
    if (bad_unit && tid == 0 && status) atomicOr(status, BS_FAULT_KV_PAGES);
    l_run = sum_halves(l_run);
    if (lg == 0) { s_m[wave * 32 + ln] = m_run; s_l[wave * 32 + ln] = l_run; }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      if (half) __syncthreads();
      float* mine = s_o + (size_t)wave * 32 * LDO;
#pragma unroll
      for (int d2 = 0; d2 < DT / 2; ++d2)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
          const f32x16& a = o[half * (DT / 2) + d2];
          *(f32x4*)(mine + ln * LDO + d2 * 32 + 8 * i4 + 4 * lg) = f32x4{a[4 * i4], a[4 * i4 + 1], a[4 * i4 + 2], a[4 * i4 + 3]};
        }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < NQT * 32 * (CH / 2) / 512; ++j) {                 // all rows of the query tiles, so that the loads are in flight together
        const int it = tid + 512 * j, r = it / (CH / 2), ch = it % (CH / 2), tq = r / 32, lr = r % 32;
        float mw[NPH], mt = -INFINITY, lt = 0.f;
#pragma unroll
        for (int w = 0; w < NPH; ++w) { mw[w] = s_m[(tq * NPH + w) * 32 + lr]; mt = fmaxf(mt, mw[w]); }
        f32x4 acc{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NPH; ++w) {
          const float f = mw[w] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw[w] - mt);
          lt += s_l[(tq * NPH + w) * 32 + lr] * f;
          const f32x4 v = *(const f32x4*)(s_o + ((size_t)(tq * NPH + w) * 32 + lr) * LDO + ch * 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[e] += v[e] * f;
        }
        const int col = half * DH + ch * 4;
        if (r >= un.R) continue;
        if (!un.whole) {
          wt_store4(bo, ((part + r) * D + col) * 4, acc);
          if (half == 0 && ch == 0) wt_store2(bm, (part + r) * 8, bad_unit ? INFINITY : mt, lt);
        } else if (!bad_unit) {
          store_row<D, STEP>(out, Hq, un, G, r, col, acc, 1.0f / lt, status);
        }
      }
    }
  };

  for_parts<true>(sh, B, s_start, s_row, seq_slot, seq_pos, seq_n, n_add, G, Hkv, s_seq, [&](const Part& un) {
    if (tid == 0) s_bad = 0;
    __syncthreads();                                    // LDS of the unit before is no longer read
    if (un.R > 64) run(std::integral_constant<int, 4>{}, un);
    else run(std::integral_constant<int, 2>{}, un);
    if (!un.whole) merge_unit<512, RP, D, STEP>(un, parts, out, Hq, G, status, &s_flag);
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");    // the next unit counts its own requests
#endif
    __syncthreads();
  });
}

size_t workspace_bytes(bool wide, int D) {
  const size_t rows = (size_t)2 * (wide ? 128 : 32);
  return kLevels * kMaxShares * sizeof(int32_t) + rows * sizeof(float) * (kLevels * kMaxShares * 2 + (size_t)share_workgroups(wide) * D);
}

template <int D, bool STEP>
void launch(const KvqView& kv, const KvqSeqs& s, int Hq, const void* q, size_t q_stride, KvqOut out, int32_t* status, void* workspace, hipStream_t st) {
  const int G = Hq / kv.Hkv;
  const bool wide = runs_wide(s.B, kv.Hkv, (long long)s.n_max * G, kv.max_pages);
  const int RP = wide ? 128 : 32;
  const int grid = share_grid(wide, s.B, kv.Hkv, (long long)s.n_max * G, kv.max_pages);
  const uint32_t g_recip = make_group(G).recip;
  int32_t* counters = (int32_t*)workspace;
  float* ml = (float*)(counters + kLevels * kMaxShares);
  const Parts parts{ml + (size_t)kLevels * 2 * kMaxShares * RP * 2, ml, counters};
  const size_t lists = (size_t)(s.B + 1) * 8;
  const size_t lds = wide ? kWideStage<D> + kWideScales + 2 * 8 * 32 * 4 + lists : (size_t)4 * 32 * (D + 4) * 4 + 2 * 4 * 32 * 4 + lists;
  auto kern = wide ? kvq_wide_kernel<D, STEP> : kvq_attention_kernel<D, STEP>;
  static const hipError_t set[2] = {hipFuncSetAttribute((const void*)kvq_wide_kernel<D, STEP>, hipFuncAttributeMaxDynamicSharedMemorySize, 144 * 1024),
                                    hipFuncSetAttribute((const void*)kvq_attention_kernel<D, STEP>, hipFuncAttributeMaxDynamicSharedMemorySize, 112 * 1024)};
  (void)set;
  const float scale_log2e = 1.4426950408889634f / sqrtf((float)D);
  hipLaunchKernelGGL(kern, dim3(grid), dim3(wide ? 512 : 256), lds, st, s.slot, s.pos, s.n, s.n_add, s.n_max, s.B, kv.block_table, kv.n_slots, kv.max_pages, kv.n_pages,
                     kv.k, kv.v, kv.ks, kv.vs, Hq, kv.Hkv, G, g_recip, scale_log2e, (const uint16_t*)q, q_stride, out, parts, status);
}
}  // namespace

size_t kvq_attention_workspace(int Hq, int Hkv, int D, int q_max) {
  const size_t few = workspace_bytes(false, D), many = is_wide((long long)q_max * (Hq / Hkv)) ? workspace_bytes(true, D) : 0;
  return few > many ? few : many;
}

void launch_kvq_attention(const KvqView& kv, const KvqSeqs& s, int Hq, const void* qrows, size_t q_stride, void* out, int32_t* status, void* workspace, hipStream_t st) {
  const KvqOut o{out, 0};
  if (kv.D == 128) launch<128, false>(kv, s, Hq, qrows, q_stride, o, status, workspace, st);
  else launch<64, false>(kv, s, Hq, qrows, q_stride, o, status, workspace, st);
}
void launch_kvq_step_attention(const KvqView& kv, const KvqSeqs& s, int Hq, const void* qrows, void* out, int out_ld, int32_t* status, void* workspace, hipStream_t st) {
  const KvqOut o{out, out_ld};
  if (kv.D == 128) launch<128, true>(kv, s, Hq, qrows, (size_t)Hq * kv.D, o, status, workspace, st);
  else launch<64, true>(kv, s, Hq, qrows, (size_t)Hq * kv.D, o, status, workspace, st);
}
