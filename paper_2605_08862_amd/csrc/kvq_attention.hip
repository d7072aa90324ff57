// Ragged causal attention over the 8-bit cache (codes, scales and element order: kvq.h).
//
// One launch and no work list.  A unit is (sequence, KV head, block of at most 32 NQ packed query rows); its K/V stream is cut into steps of 128 tokens, and
// the steps of all units, in order, into equal shares, one per workgroup (a multiple of the CUs).  Every workgroup finds its share from a prefix sum over the
// sequences that it makes itself.  A share can begin and end inside a unit: the workgroup then leaves a partial (rows, maximum, sum), and the last of a
// unit's workgroups to arrive merges them (publish_arrival, common.h; nobody waits).
//   * The four waves of a workgroup take a 32-token tile each of every step, with an online softmax of their own (attn_softmax.h), merged at a unit's end.
//   * S^T = K Q^T and O^T = V^T P^T on the 32 x 32 x 16 f16 MFMA.  A lane's sixteen bytes of codes are operands of two K-steps: one conversion with the block's
//     scale gives two exact float16 values, so nothing is rounded that the 16-bit cache would not round.
//   * Query fragments lie in LDS; K/V tiles are loaded two ahead into registers.
#include "kvq.h"
#include "attn_softmax.h"
#include <type_traits>

namespace {

constexpr int kStep = 4 * kTile;                       // tokens of a step: a tile for each wave
constexpr int kCounters = 1024;                        // one per workgroup, rounded up

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

// STEP: inside bs_verify_step (float16 queries, output in chunk order).
template <int NQ, int D, bool STEP>
__global__ void __launch_bounds__(256, NQ == 1 ? 2 : 1)
kvq_attention_kernel(const int32_t* __restrict__ seq_slot, const int32_t* __restrict__ seq_pos, const int32_t* __restrict__ seq_n, int n_add, int n_max, int B,
                     const int32_t* __restrict__ block_table, int n_slots, int max_pages, int n_pages, const uint8_t* __restrict__ k_pages,
                     const uint8_t* __restrict__ v_pages, const float* __restrict__ k_scale, const float* __restrict__ v_scale, int Hq, int Hkv,
                     float scale_log2e, const uint16_t* __restrict__ q, size_t q_stride, KvqOut out, int share_min_num, float* __restrict__ part_o,
                     float* __restrict__ part_ml, int32_t* __restrict__ counters, int32_t* __restrict__ status) {
  constexpr int KS = D / 16, DT = D / 32, RP = 32 * NQ, CH = D / 4;
  constexpr int LDO = D + 4;                            // row stride (floats) of an accumulator in LDS
  extern __shared__ __align__(16) char lds_raw[];
  __shared__ int s_scan[12], s_flag;
  u32x4* const s_q = (u32x4*)lds_raw;                   // [NQ][KS][64] query fragments; behind a unit's last product, the waves' accumulators
  float* const s_o = (float*)lds_raw;                   // [4][32][LDO]
  constexpr size_t kOBytes = (size_t)4 * 32 * LDO * 4, kQBytes = (size_t)NQ * KS * 1024;
  float* const s_m = (float*)(lds_raw + (kOBytes > kQBytes ? kOBytes : kQBytes));   // [4][NQ * 32]
  float* const s_l = s_m + 4 * RP;
  int* const s_start = (int*)(s_l + 4 * RP);            // [B + 1] first step of every sequence
  int* const s_row = s_start + B + 1;                   // [B + 1] first packed row
  const int tid = threadIdx.x, G = Hq / Hkv;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, ln = lane & 31, lg = lane >> 5;

  // ---- the shares --------------------------------------------------------------------------------------------------------------
  auto block_steps = [&](int c, int n, int qb) { return (c + min(n - 1, ((qb + 1) * RP - 1) / G) + kStep) / kStep; };   // of the tokens that the block's last row sees
  int most = 0;
  {
    const int per = (B + 255) / 256, lo = min(tid * per, B), hi = min(lo + per, B);
    int steps = 0, rows = 0, fault = 0;
    for (int b = lo; b < hi; ++b) {
      s_start[b] = steps;
      s_row[b] = rows;
      const int n = seq_n[b] + n_add;
      if (n < 0 || n > n_max) { fault |= BS_FAULT_DRAFT_LEN; continue; }
      if (n == 0) continue;
      rows += n;
      const int slot = seq_slot[b], c = seq_pos[b];
      if (slot < 0 || slot >= n_slots) { fault |= BS_FAULT_SLOT; continue; }
      if (c < 0 || (long long)c + n > (long long)max_pages * kPage) { fault |= BS_FAULT_KV_PAGES; continue; }
      const int blocks = (n * G + RP - 1) / RP;
      int s = 0;
      for (int qb = 0; qb < blocks; ++qb) s += block_steps(c, n, qb);
      most = max(most, block_steps(c, n, blocks - 1));
      steps += s * Hkv;
    }
    if (fault && blockIdx.x == 0 && status) atomicOr(status, fault);
    // exclusive prefix over the threads
    int is = steps, ir = rows;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int a = __shfl_up(is, o), r = __shfl_up(ir, o);
      if (lane >= o) { is += a; ir += r; }
      most = max(most, __shfl_xor(most, o));
    }
    if (lane == 63) { s_scan[wave] = is; s_scan[4 + wave] = ir; }
    if (lane == 0) s_scan[8 + wave] = most;
    __syncthreads();
    int bs = is - steps, br = ir - rows;
#pragma unroll
    for (int w = 0; w < 3; ++w) if (w < wave) { bs += s_scan[w]; br += s_scan[4 + w]; }
    for (int b = lo; b < hi; ++b) { s_start[b] += bs; s_row[b] += br; }
    if (tid == 0) { s_start[B] = s_scan[0] + s_scan[1] + s_scan[2] + s_scan[3]; s_row[B] = 0; }
    most = max(max(s_scan[8], s_scan[9]), max(s_scan[10], s_scan[11]));
    __syncthreads();
  }
  const int total = __builtin_amdgcn_readfirstlane(s_start[B]);
  // a share is no shorter than sqrt(steps of the longest unit * share_min_num / 16): its partials have to be merged by one workgroup
  int share = (total + (int)gridDim.x - 1) / (int)gridDim.x;
  share = max(share, (int)sqrtf((float)most * (float)share_min_num * 0.0625f));
  share = __builtin_amdgcn_readfirstlane(max(share, 1));
  const int w_id = blockIdx.x;
  int x = w_id * share;
  const int x_end = min(x + share, total);
  if (x >= x_end) return;
  int b = 0;
  {
    int hi = B;                                         // largest b with s_start[b] <= x (sequences without steps are passed over)
    while (hi - b > 1) { const int mid = (b + hi) >> 1; if (s_start[mid] <= x) b = mid; else hi = mid; }
    b = __builtin_amdgcn_readfirstlane(b);
  }

  auto store4 = [&](int row, int col, f32x4 v) {
    if constexpr (STEP) {
      *(f16x4*)((f16*)out.p + act_index(row, col, out.ld)) = to_f16x4_guarded(v[0], v[1], v[2], v[3], status);
    } else {
      typedef bf16 b4 __attribute__((ext_vector_type(4)));
      *(b4*)((bf16*)out.p + (size_t)row * Hq * D + col) = b4{(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
    }
  };

  // Merges the partials of a unit, workgroups w0 .. w1: an item is four columns of a row.
  auto merge_unit = [&](int w0, int w1, int R, int row0, int qr0, int h) {
    const wt_buf bo = wt_buffer(part_o), bm = wt_buffer(part_ml);
    for (int it = tid; it < R * CH; it += 256) {
      const int r = it / CH, ch = it % CH;
      float m = -INFINITY, l = 0.f;
      f32x4 acc{0.f, 0.f, 0.f, 0.f};
      constexpr int GC = 8;
      for (int c0 = w0; c0 <= w1; c0 += GC) {
        wt_f32x2 ml[GC];
        f32x4 v[GC];
#pragma unroll
        for (int u = 0; u < GC; ++u) {
          const int c = min(c0 + u, w1);
          const uint32_t pr = (uint32_t)(2 * c + (c == w0 ? 1 : 0)) * RP + r;
          ml[u] = wt_load2(bm, pr * 8);
          v[u] = wt_load4(bo, (pr * D + ch * 4) * 4);
        }
        float mg = m;
#pragma unroll
        for (int u = 0; u < GC; ++u) mg = fmaxf(mg, ml[u][0]);
        if (mg == -INFINITY) continue;
        const float f0 = __builtin_amdgcn_exp2f(m - mg);
        l *= f0;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] *= f0;
#pragma unroll
        for (int u = 0; u < GC; ++u) {
          if (c0 + u > w1) break;
          const float f = __builtin_amdgcn_exp2f(ml[u][0] - mg);
          l += ml[u][1] * f;
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[e] += v[u][e] * f;
        }
        m = mg;
      }
      if (m == INFINITY) continue;                      // a bad page: the row stays as it is
      const float inv = 1.0f / l;
      const int qr = qr0 + r;
      store4(row0 + qr / G, (h * G + qr % G) * D + ch * 4, f32x4{acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv});
    }
  };

  // ---- the units of the share --------------------------------------------------------------------------------------------------
  while (x < x_end) {
    while (s_start[b + 1] <= x) ++b;
    b = __builtin_amdgcn_readfirstlane(b);
    const int n = seq_n[b] + n_add, c = seq_pos[b], row0 = __builtin_amdgcn_readfirstlane(s_row[b]);
    const int first = __builtin_amdgcn_readfirstlane(s_start[b]);
    const int per_head = __builtin_amdgcn_readfirstlane((s_start[b + 1] - first) / Hkv);
    const int h = (x - first) / per_head;
    int unit = first + h * per_head, qb = 0;            // first step of the unit
    for (int s; unit + (s = block_steps(c, n, qb)) <= x; ++qb) unit += s;
    const int steps = block_steps(c, n, qb), s_lo = x - unit, s_hi = min(steps, x_end - unit);
    const int qr0 = qb * RP, R = min(n * G - qr0, RP);  // packed query rows of the block
    const int32_t* __restrict__ bt = block_table + (size_t)seq_slot[b] * max_pages;
    const int n_tok = c + min(n - 1, (qr0 + RP - 1) / G) + 1, n_tiles = (n_tok + kTile - 1) / kTile;
    const int t0 = 4 * s_lo + wave, t_end = min(4 * s_hi, n_tiles);
    const int n_my = t0 < t_end ? (t_end - t0 + 3) / 4 : 0, t_last = t0 + (n_my - 1) * 4;
    const int c_all = c + qr0 / G;                      // last position that every row sees
    bool bad = false;

    struct At { size_t off; float ks, vs; };
    auto place = [&](int t) -> At {
      int page = bt[t * kTile / kPage];
      if ((unsigned)page >= (unsigned)n_pages) { page = 0; bad = true; }
      return At{(size_t)page * ((size_t)Hkv * kPage * D) + (size_t)(h * 2 + (t & 1)) * (kTile * D) + lane * 16, k_scale[(size_t)page * Hkv + h], v_scale[(size_t)page * Hkv + h]};
    };
    auto load_tile = [&](const uint8_t* base, size_t off, u32x4 (&f)[DT]) {
#pragma unroll
      for (int i = 0; i < DT; ++i) f[i] = *(const u32x4*)(base + off + i * 1024);
    };

    // queries first, the first two tiles behind them
    constexpr int QF = NQ * KS / 4;                     // fragments of each wave
    u32x4 qv[QF];
#pragma unroll
    for (int j = 0; j < QF; ++j) {
      const int f = wave + 4 * j, qt = f / KS, s = f % KS;
      const int qr = qr0 + min(qt * 32 + ln, R - 1);    // rows behind the last one are masked
      qv[j] = *(const u32x4*)(q + (size_t)(row0 + qr / G) * q_stride + (size_t)(h * G + qr % G) * D + lg * (D / 2) + s * 8);
    }
    u32x4 k0[DT], v0[DT], k1[DT], v1[DT];
    At a0 = place(n_my > 0 ? t0 : n_tiles - 1), a1 = place(n_my > 1 ? t0 + 4 : n_my > 0 ? t0 : n_tiles - 1);
    load_tile(k_pages, a0.off, k0);
    load_tile(v_pages, a0.off, v0);
    load_tile(k_pages, a1.off, k1);
    load_tile(v_pages, a1.off, v1);
    bool range = false;
#pragma unroll
    for (int j = 0; j < QF; ++j) {
      if constexpr (!STEP) {
        const bf16x8 y = __builtin_bit_cast(bf16x8, qv[j]);
        f16x8 z;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float f = (float)y[e];
          if (!(fabsf(f) <= 65504.f)) { f = f16_saturate(f); range = true; }
          z[e] = (f16)f;
        }
        qv[j] = __builtin_bit_cast(u32x4, z);
      }
      s_q[(wave + 4 * j) * 64 + lane] = qv[j];
    }
    if (range && status) atomicOr(status, BS_FAULT_RANGE);
    __syncthreads();
    const u32x4* my_q = s_q + lane;

    f32x16 o[NQ][DT];
    float m_run[NQ], l_run[NQ];
    int lim[NQ];                                        // last visible position of the lane's row
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) {
      m_run[qt] = -INFINITY;
      l_run[qt] = 0.f;
      lim[qt] = qt * 32 + ln < R ? c + (qr0 + qt * 32 + ln) / G : -1;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[qt][dt][i] = 0.f;
    }

    auto tile = [&](auto pref, int t, int t_pref, u32x4 (&kc)[DT], u32x4 (&vc)[DT], At& at) {
      constexpr bool PREF = decltype(pref)::value;
      At next{0, 1.f, 1.f};
      if (PREF) next = place(t_pref);
      const int tok0 = t * kTile + 16 * lg;             // accumulator register i <-> token tok0 + i
      const bool full = (t + 1) * kTile - 1 <= c_all;
      f32x16 st[NQ];
#pragma unroll
      for (int qt = 0; qt < NQ; ++qt)
#pragma unroll
        for (int i = 0; i < 16; ++i) st[qt][i] = 0.f;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const f16x8 kh = values8(kc[s / 2][2 * (s % 2)], kc[s / 2][2 * (s % 2) + 1], at.ks);
#pragma unroll
        for (int qt = 0; qt < NQ; ++qt) st[qt] = mfma32(kh, as_f16x8(my_q[(qt * KS + s) * 64]), st[qt]);
      }
      __builtin_amdgcn_sched_barrier(0);
      if (PREF) load_tile(k_pages, next.off, kc);
      __builtin_amdgcn_sched_barrier(0);
      f16x8 pf[NQ][2];
#pragma unroll
      for (int qt = 0; qt < NQ; ++qt) {
        float y[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = full || tok0 + i <= lim[qt] ? st[qt][i] : -INFINITY;
        float mloc = y[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mloc = fmaxf(mloc, y[i]);
        mloc = max_halves(mloc) * scale_log2e;          // scale > 0 commutes with max
        if (__any(mloc > m_run[qt] + kLateRescale)) {
          const float m_new = fmaxf(m_run[qt], mloc);
          const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run[qt] - m_new);
          l_run[qt] *= alpha;
          m_run[qt] = m_new;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[qt][dt][i] *= alpha;
        }
        const float m_safe = m_run[qt] == -INFINITY ? 0.f : m_run[qt];
        float psum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          y[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(y[i], scale_log2e, -m_safe));
          psum += y[i];
        }
        l_run[qt] += psum;                              // per half of the wave; the halves are added at the end
#pragma unroll
        for (int i = 0; i < 16; ++i) pf[qt][i / 8][i % 8] = (f16)y[i];
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int t2 = 0; t2 < 2; ++t2) {
          const f16x8 vh = values8(vc[dt][2 * t2], vc[dt][2 * t2 + 1], at.vs);
#pragma unroll
          for (int qt = 0; qt < NQ; ++qt) o[qt][dt] = mfma32(vh, pf[qt][t2], o[qt][dt]);
        }
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

    // ---- merge of the waves, one query tile at a time --------------------------------------------------------------------------
    const bool whole = s_lo == 0 && s_hi == steps;
    const int w_first = unit / share, w_last = (unit + steps - 1) / share;
    const uint32_t part = (uint32_t)(2 * w_id + (s_lo == 0 ? 1 : 0)) * RP;
    const wt_buf bo = wt_buffer(part_o), bm = wt_buffer(part_ml);
    if (bad && lane == 0 && status) atomicOr(status, BS_FAULT_KV_PAGES);
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) {
      l_run[qt] = sum_halves(l_run[qt]);
      if (lg == 0) { s_m[wave * RP + qt * 32 + ln] = bad ? INFINITY : m_run[qt]; s_l[wave * RP + qt * 32 + ln] = l_run[qt]; }
    }
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) {
      if (qt * 32 >= R) break;
      __syncthreads();                                  // the fragments, or the accumulators of the tile before, are no longer read
      float* mine = s_o + (size_t)wave * 32 * LDO;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4)
          *(f32x4*)(mine + ln * LDO + dt * 32 + 8 * i4 + 4 * lg) = f32x4{o[qt][dt][4 * i4], o[qt][dt][4 * i4 + 1], o[qt][dt][4 * i4 + 2], o[qt][dt][4 * i4 + 3]};
      __syncthreads();
      for (int it = tid; it < min(R - qt * 32, 32) * CH; it += 256) {
        const int r = it / CH, ch = it % CH, rr = qt * 32 + r;
        float mw[4], mt = -INFINITY, lt = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) { mw[w] = s_m[w * RP + rr]; mt = fmaxf(mt, mw[w]); }
        f32x4 acc{0.f, 0.f, 0.f, 0.f};
        if (mt != -INFINITY && mt != INFINITY)
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const float f = __builtin_amdgcn_exp2f(mw[w] - mt);
            lt += s_l[w * RP + rr] * f;
            const f32x4 v = *(const f32x4*)(s_o + ((size_t)w * 32 + r) * LDO + ch * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] += v[e] * f;
          }
        if (!whole) {
          wt_store4(bo, ((part + rr) * D + ch * 4) * 4, acc);
          if (ch == 0) wt_store2(bm, (part + rr) * 8, mt, lt);
        } else if (mt != INFINITY) {
          const float inv = 1.0f / lt;
          const int qr = qr0 + rr;
          store4(row0 + qr / G, (h * G + qr % G) * D + ch * 4, f32x4{acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv});
        }
      }
    }
    if (!whole && publish_arrival(counters + w_first, w_last - w_first + 1, &s_flag)) merge_unit(w_first, w_last, R, row0, qr0, h);
    x = unit + s_hi;
    __syncthreads();                                    // LDS is the next unit's
  }
}

// Query tiles of a block: what the rows of a sequence need, at most four (accumulators of four tiles of 32 rows x 128 fill half of the registers).
int query_tiles(int G, int q_max) {
  const long long rows = (long long)q_max * G;
  return rows <= 32 ? 1 : rows <= 64 ? 2 : 4;
}
int workgroups(int NQ) { return (NQ == 1 ? 2 : 1) * kCUs; }

template <int NQ, int D, bool STEP>
void launch(const KvqView& kv, const KvqSeqs& s, int Hq, const void* q, size_t q_stride, KvqOut out, int32_t* status, void* workspace, hipStream_t st) {
  constexpr int RP = 32 * NQ;
  const int grid = workgroups(NQ);
  float* part_ml = (float*)((char*)workspace + kCounters * sizeof(int32_t));
  float* part_o = part_ml + (size_t)2 * grid * RP * 2;
  const size_t o = (size_t)4 * 32 * (D + 4) * 4, qb = (size_t)NQ * (D / 16) * 1024;
  const size_t lds = (o > qb ? o : qb) + (size_t)2 * 4 * RP * 4 + (size_t)(s.B + 1) * 8;
  auto kern = kvq_attention_kernel<NQ, D, STEP>;
  static const hipError_t set = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, 120 * 1024);
  (void)set;
  const float scale_log2e = 1.4426950408889634f / sqrtf((float)D);
  hipLaunchKernelGGL(kern, dim3(grid), dim3(256), lds, st, s.slot, s.pos, s.n, s.n_add, s.n_max, s.B, kv.block_table, kv.n_slots, kv.max_pages, kv.n_pages, kv.k, kv.v,
                     kv.ks, kv.vs, Hq, kv.Hkv, scale_log2e, (const uint16_t*)q, q_stride, out, 2, part_o, part_ml, (int32_t*)workspace, status);
}
}  // namespace

size_t kvq_attention_workspace(int Hq, int Hkv, int D, int q_max) {
  const int NQ = query_tiles(Hq / Hkv, q_max);
  size_t most = 0;
  for (int n = 1; n <= NQ; n *= 2) { const size_t b = (size_t)2 * workgroups(n) * 32 * n * (D + 2) * sizeof(float); most = b > most ? b : most; }
  return kCounters * sizeof(int32_t) + most;
}

void launch_kvq_attention(const KvqView& kv, const KvqSeqs& s, int Hq, const void* qrows, size_t q_stride, void* out, int32_t* status, void* workspace, hipStream_t st) {
  const int NQ = query_tiles(Hq / kv.Hkv, s.n_max);
  const KvqOut o{out, 0};
#define BS_KVQ(NQ_, D_) launch<NQ_, D_, false>(kv, s, Hq, qrows, q_stride, o, status, workspace, st)
  if (kv.D == 128) { if (NQ == 1) BS_KVQ(1, 128); else if (NQ == 2) BS_KVQ(2, 128); else BS_KVQ(4, 128); }
  else { if (NQ == 1) BS_KVQ(1, 64); else if (NQ == 2) BS_KVQ(2, 64); else BS_KVQ(4, 64); }
#undef BS_KVQ
}
