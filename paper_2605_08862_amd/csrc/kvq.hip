// Rows of K and V <-> the pages of the 8-bit cache (scales and element order: kvq.h).
#include "kvq.h"

namespace {

// What a workgroup knows of its (sequence, page): tokens [lo, hi) of the page are rows row .. of the batch.
struct Span { int page, lo, hi, row; bool live; };

// The sequence's rows are checked as a whole, by every workgroup that has a page of it alike: a sequence with a bad count, slot, position or page, or
// (writes) with the slot of an earlier sequence that has rows, is skipped.  s_red: one word per wave.
template <bool WRITE>
__device__ __forceinline__ Span find_span(const KvqView& kv, const KvqSeqs& q, int b, int page_at, int* s_red, int32_t* status) {
  Span sp{0, 0, 0, 0, false};
  const int n = (q.n ? q.n[b] : 0) + q.n_add;
  const int slot = q.slot ? q.slot[b] : q.slot0, pos = q.pos ? q.pos[b] : q.pos0;
  int fault = 0;
  if (n < 0 || n > q.n_max) fault |= BS_FAULT_DRAFT_LEN;
  if (n == 0 || fault) {
    if (fault && page_at == 0 && threadIdx.x == 0 && status) atomicOr(status, fault);
    return sp;
  }
  if (slot < 0 || slot >= kv.n_slots) fault |= BS_FAULT_SLOT;
  if (pos < 0 || (long long)pos + n > (long long)kv.max_pages * kPage) fault |= BS_FAULT_KV_PAGES;
  const int first = pos / kPage, last = fault ? first : (pos + n - 1) / kPage;
  if (!fault && page_at > last - first) return sp;
  const int32_t* bt = kv.block_table + (size_t)slot * kv.max_pages;
  int before = 0, bad = fault;
  if (!fault)
    for (int p = first + (int)threadIdx.x; p <= last; p += 256) if ((unsigned)bt[p] >= (unsigned)kv.n_pages) bad |= BS_FAULT_KV_PAGES;
  if (q.slot)
    for (int c = threadIdx.x; c < b; c += 256) {
      const int m = WRITE || !q.row_start ? q.n[c] + q.n_add : 0;
      const bool rows = m > 0 && m <= q.n_max;           // (a padded entry may have any slot)
      before += rows ? m : 0;
      if (WRITE && rows && q.slot[c] == slot) bad |= BS_FAULT_SLOT;
    }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) { before += __shfl_xor(before, o); bad |= __shfl_xor(bad, o); }
  if ((threadIdx.x & 63) == 0) { s_red[threadIdx.x >> 6] = before; s_red[4 + (threadIdx.x >> 6)] = bad; }
  __syncthreads();
  before = s_red[0] + s_red[1] + s_red[2] + s_red[3];
  bad = s_red[4] | s_red[5] | s_red[6] | s_red[7];
  if (bad) {
    if (page_at == 0 && threadIdx.x == 0 && status) atomicOr(status, bad);
    return sp;
  }
  const int p = first + page_at;
  sp.page = bt[p];
  sp.lo = max(pos - p * kPage, 0);
  sp.hi = min(pos + n - p * kPage, kPage);
  sp.row = (q.row_start ? q.row_start[b] : before) + p * kPage + sp.lo - pos;
  sp.live = true;
  return sp;
}

// Where rows come from: a caller's bf16 rows (VEC: on sixteen bytes), or the float16 pages that a verify step leaves its rows in (staged: row r is token
// r % 64 of page r / 64, element order of the 16-bit cache).
enum Source { ROWS, ROWS_VEC, STAGED };
template <Source S> struct Elem { typedef bf16 T; };
template <> struct Elem<STAGED> { typedef f16 T; };
// bits of 57344 in the source type: magnitudes compare as integers, infinities and NaN are above
template <Source S> constexpr uint32_t kMostBits = S == STAGED ? 0x7b00 : 0x4760;

template <Source S> __device__ __forceinline__ void unpack2(uint32_t w, float& a, float& b) {
  if constexpr (S == STAGED) {
    typedef f16 h2 __attribute__((ext_vector_type(2)));
    const h2 h = __builtin_bit_cast(h2, w);
    a = (float)h[0]; b = (float)h[1];
  } else {
    a = __uint_as_float(w << 16); b = __uint_as_float(w & 0xffff0000u);
  }
}
// largest magnitude of two pairs, as bits
__device__ __forceinline__ uint32_t max_pairs(uint32_t m, uint32_t w) {
  typedef uint16_t us2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(us2, m), __builtin_bit_cast(us2, w & 0x7fff7fffu)));
}
__device__ __forceinline__ float bounded(float f) { return f != f ? 0.f : fminf(fmaxf(f, -kKvqMost), kKvqMost); }

// One workgroup per (page of a sequence, KV head): two waves have K, two V.  All of a thread's rows are loaded before the scale is known and stay in registers.
// K: a thread has sixteen d of a token, which are sixteen bytes of the page; V: four d of sixteen tokens, transposed in registers into four times sixteen bytes.
// No two threads write the same sixteen bytes, so older rows that have to be rounded again need no barrier.  Many rows: bound by memory, 32016 rows x 4 heads x 128
// (16 prompts of the 7B heads) written and read back 53 us, 3.7 TB/s of rows and codes.  A row each of 64 sequences: 6 us, a chain of trips to memory (the batch's numbers, the
// page's id, its scale and the row) and the launch.
template <Source S, int D>
__global__ void __launch_bounds__(256) kvq_write_kernel(KvqView kv, KvqSeqs q, int pages_each, const void* __restrict__ k_rows, const void* __restrict__ v_rows,
                                                        size_t stride, int32_t* __restrict__ status) {
  typedef typename Elem<S>::T T;
  __shared__ int s_red[8];
  __shared__ uint32_t s_max[4];
  constexpr int PK = D / 32, KD = D / 16, VD = D / 4;   // K pieces of a thread, of a row; threads for the d of V
  const int nth = (int)(blockIdx.z * gridDim.y + blockIdx.y), b = nth / pages_each, h = blockIdx.x, is_v = __builtin_amdgcn_readfirstlane(threadIdx.x >> 7), t = threadIdx.x & 127;
  if (b >= q.B) return;
  const Span sp = find_span<true>(kv, q, b, nth - b * pages_each, s_red, h == 0 ? status : nullptr);
  if (!sp.live) return;
  const T* rows = (const T*)(is_v ? v_rows : k_rows);
  uint8_t* page = (is_v ? kv.v : kv.k) + (size_t)sp.page * kvq_page_bytes(kv.Hkv, D);
  float* scale = (is_v ? kv.vs : kv.ks) + (size_t)sp.page * kv.Hkv + h;
  const int e_old = kvq_exp_of(*scale);
  const int tg = t / VD, dq = t % VD;                   // V: tokens 16 tg .. 16 tg + 15, d from 4 dq
  uint32_t x[32];                                       // K: [piece][8 pairs of d]; V: [token][2 pairs of d]
#pragma unroll
  for (int i = 0; i < 32; ++i) x[i] = 0;
  if (!is_v) {
#pragma unroll
    for (int j = 0; j < PK; ++j) {
      const int i = t + 128 * j, tok = i / KD, d0 = i % KD * 16;
      if (tok < sp.lo || tok >= sp.hi) continue;
      const int r = sp.row + tok - sp.lo;
      if constexpr (S == STAGED) {
        const T* src = rows + (size_t)(r / kPage) * kv_page_elems(kv.Hkv, D);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const u32x4 v = *(const u32x4*)(src + k_index_bf16(D, h, r % kPage, d0 + 8 * u));
#pragma unroll
          for (int e = 0; e < 4; ++e) x[j * 8 + u * 4 + e] = v[e];
        }
      } else {
        const T* src = rows + (size_t)r * stride + h * D + d0;
        if constexpr (S == ROWS_VEC) {
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const u32x4 v = *(const u32x4*)(src + 8 * u);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[j * 8 + u * 4 + e] = v[e];
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[j * 8 + e] = (uint32_t)((const uint16_t*)src)[2 * e] | (uint32_t)((const uint16_t*)src)[2 * e + 1] << 16;
        }
      }
    }
  } else if (tg < 4) {
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const int tok = tg * 16 + j;
      if (tok < sp.lo || tok >= sp.hi) continue;
      const int r = sp.row + tok - sp.lo;
      if constexpr (S == STAGED) {
        const uint16_t* src = (const uint16_t*)rows + (size_t)(r / kPage) * kv_page_elems(kv.Hkv, D) + v_index_bf16(D, h, r % kPage, dq * 4);
        x[2 * j] = (uint32_t)src[0] | (uint32_t)src[8] << 16;      // consecutive d are eight elements apart
        x[2 * j + 1] = (uint32_t)src[16] | (uint32_t)src[24] << 16;
      } else {
        const T* src = rows + (size_t)r * stride + h * D + dq * 4;
        if constexpr (S == ROWS_VEC) {
          const u32x2 v = *(const u32x2*)src;
          x[2 * j] = v[0];
          x[2 * j + 1] = v[1];
        } else {
#pragma unroll
          for (int e = 0; e < 2; ++e) x[2 * j + e] = (uint32_t)((const uint16_t*)src)[2 * e] | (uint32_t)((const uint16_t*)src)[2 * e + 1] << 16;
        }
      }
    }
  }
  uint32_t m2 = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i) m2 = max_pairs(m2, x[i]);
  uint32_t m = max(m2 & 0xffff, m2 >> 16);
  const bool out_of_range = m > kMostBits<S>;
  if (out_of_range) {                                   // (never for sane models) the magnitude that is left of this thread's elements
    float a = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      float f, g;
      unpack2<S>(x[i], f, g);
      a = fmaxf(a, fmaxf(fabsf(bounded(f)), fabsf(bounded(g))));
    }
    if constexpr (S == STAGED) m = __builtin_bit_cast(uint16_t, (f16)a); else m = __float_as_uint(a) >> 16;
    if (status) atomicOr(status, BS_FAULT_RANGE);
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
  if ((threadIdx.x & 63) == 0) s_max[threadIdx.x >> 6] = m;
  __syncthreads();
  m = max(s_max[2 * is_v], s_max[2 * is_v + 1]);
  float a, unused;
  unpack2<S>(m, a, unused);
  int e = kvq_exp_for(a);
  const bool again = sp.lo > 0 && e > e_old;            // rows that are there already are rounded again
  if (sp.lo > 0) e = max(e, e_old);
  if (t == 0) *scale = kvq_scale(e);
  const float f = kvq_scale(-e), f_old = kvq_scale(e_old - e);
  auto codes = [&](uint32_t lo, uint32_t hi) {
    float v[4];
    unpack2<S>(lo, v[0], v[1]);
    unpack2<S>(hi, v[2], v[3]);
    if (out_of_range) {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = bounded(v[i]);
    }
    return kvq_codes4(v[0] * f, v[1] * f, v[2] * f, v[3] * f);
  };
  auto rounded_again = [&](u32x4 w) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { const f32x4 v = kvq_values4(w[i]); w[i] = kvq_codes4(v[0] * f_old, v[1] * f_old, v[2] * f_old, v[3] * f_old); }
    return w;
  };
  if (!is_v) {
#pragma unroll
    for (int j = 0; j < PK; ++j) {
      const int i = t + 128 * j, tok = i / KD, d0 = i % KD * 16;
      u32x4* at = (u32x4*)(page + kvq_k_piece(D, h, tok, d0));
      if (tok >= sp.lo && tok < sp.hi) {
        u32x4 w;
#pragma unroll
        for (int u = 0; u < 4; ++u) w[u] = codes(x[j * 8 + 2 * u], x[j * 8 + 2 * u + 1]);
        *at = w;
      } else if (again && tok < sp.lo) {
        *at = rounded_again(*at);
      }
    }
    return;
  }
  const int g0 = tg * 16;
  if (tg >= 4 || g0 >= sp.hi || (g0 + 16 <= sp.lo && !again)) return;
  u32x4* at = (u32x4*)(page + kvq_v_piece(D, h, g0, dq * 4));        // of d = 4 dq; the next three d follow
  if (g0 + 16 <= sp.lo) {
#pragma unroll
    for (int d = 0; d < 4; ++d) at[d] = rounded_again(at[d]);
    return;
  }
  const bool part = g0 < sp.lo || g0 + 16 > sp.hi;      // tokens of the sixteen that are not this call's stay
  u32x4 w[4];                                           // [d][four tokens]
#pragma unroll
  for (int k = 0; k < 4; ++k) {                         // four tokens x four d of codes, transposed
    uint32_t r[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = codes(x[2 * (4 * k + j)], x[2 * (4 * k + j) + 1]);
    const uint32_t a0 = __builtin_amdgcn_perm(r[1], r[0], 0x05010400), a1 = __builtin_amdgcn_perm(r[3], r[2], 0x05010400);   // d 0, 1 of tokens 0 1, 2 3
    const uint32_t b0 = __builtin_amdgcn_perm(r[1], r[0], 0x07030602), b1 = __builtin_amdgcn_perm(r[3], r[2], 0x07030602);   // d 2, 3
    w[0][k] = __builtin_amdgcn_perm(a1, a0, 0x05040100);
    w[1][k] = __builtin_amdgcn_perm(a1, a0, 0x07060302);
    w[2][k] = __builtin_amdgcn_perm(b1, b0, 0x05040100);
    w[3][k] = __builtin_amdgcn_perm(b1, b0, 0x07060302);
  }
  if (part) {
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const u32x4 old = again ? rounded_again(at[d]) : at[d];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint32_t mask = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) { const int tok = g0 + 4 * k + j; if (tok >= sp.lo && tok < sp.hi) mask |= 0xffu << (8 * j); }
        w[d][k] = (w[d][k] & mask) | (old[k] & ~mask);
      }
    }
  }
#pragma unroll
  for (int d = 0; d < 4; ++d) at[d] = w[d];
}

__device__ __forceinline__ uint32_t bf16_pair(float a, float b) { return __float_as_uint(a) >> 16 | (__float_as_uint(b) & 0xffff0000u); }   // exact: four significant bits

// As kvq_write_kernel, the other way.
template <bool VEC, int D>
__global__ void __launch_bounds__(256) kvq_read_kernel(KvqView kv, KvqSeqs q, int pages_each, bf16* __restrict__ k_rows, bf16* __restrict__ v_rows,
                                                       size_t stride, int32_t* __restrict__ status) {
  __shared__ int s_red[8];
  constexpr int PK = D / 32, KD = D / 16, VD = D / 4;
  const int nth = (int)(blockIdx.z * gridDim.y + blockIdx.y), b = nth / pages_each, h = blockIdx.x, is_v = __builtin_amdgcn_readfirstlane(threadIdx.x >> 7), t = threadIdx.x & 127;
  if (b >= q.B) return;
  const Span sp = find_span<false>(kv, q, b, nth - b * pages_each, s_red, h == 0 ? status : nullptr);
  if (!sp.live) return;
  const uint8_t* page = (is_v ? kv.v : kv.k) + (size_t)sp.page * kvq_page_bytes(kv.Hkv, D);
  const float f = kvq_scale(kvq_exp_of((is_v ? kv.vs : kv.ks)[(size_t)sp.page * kv.Hkv + h]));
  if (!is_v) {
    u32x4 w[PK];
#pragma unroll
    for (int j = 0; j < PK; ++j) { const int i = t + 128 * j; w[j] = *(const u32x4*)(page + kvq_k_piece(D, h, i / KD, i % KD * 16)); }
#pragma unroll
    for (int j = 0; j < PK; ++j) {
      const int i = t + 128 * j, tok = i / KD, d0 = i % KD * 16;
      if (tok < sp.lo || tok >= sp.hi) continue;
      bf16* dst = k_rows + (size_t)(sp.row + tok - sp.lo) * stride + h * D + d0;
      uint32_t y[8];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const f32x4 v = kvq_values4(w[j][u]);
        y[2 * u] = bf16_pair(v[0] * f, v[1] * f);
        y[2 * u + 1] = bf16_pair(v[2] * f, v[3] * f);
      }
      if constexpr (VEC) {
        *(u32x4*)dst = u32x4{y[0], y[1], y[2], y[3]};
        *(u32x4*)(dst + 8) = u32x4{y[4], y[5], y[6], y[7]};
      } else {
#pragma unroll
        for (int u = 0; u < 8; ++u) { ((uint16_t*)dst)[2 * u] = (uint16_t)y[u]; ((uint16_t*)dst)[2 * u + 1] = (uint16_t)(y[u] >> 16); }
      }
    }
    return;
  }
  const int tg = t / VD, dq = t % VD, g0 = tg * 16;
  if (tg >= 4 || g0 >= sp.hi || g0 + 16 <= sp.lo) return;
  u32x4 w[4];
#pragma unroll
  for (int d = 0; d < 4; ++d) w[d] = ((const u32x4*)(page + kvq_v_piece(D, h, g0, dq * 4)))[d];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    f32x4 v[4];                                         // [d] four tokens
#pragma unroll
    for (int d = 0; d < 4; ++d) v[d] = kvq_values4(w[d][k]);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int tok = g0 + 4 * k + j;
      if (tok < sp.lo || tok >= sp.hi) continue;
      bf16* dst = v_rows + (size_t)(sp.row + tok - sp.lo) * stride + h * D + dq * 4;
      const u32x2 y{bf16_pair(v[0][j] * f, v[1][j] * f), bf16_pair(v[2][j] * f, v[3][j] * f)};
      if constexpr (VEC) *(u32x2*)dst = y;
      else {
#pragma unroll
        for (int u = 0; u < 2; ++u) { ((uint16_t*)dst)[2 * u] = (uint16_t)y[u]; ((uint16_t*)dst)[2 * u + 1] = (uint16_t)(y[u] >> 16); }
      }
    }
  }
}

int pages_each(const KvqSeqs& q) { return (q.n_max + 2 * kPage - 2) / kPage; }   // pages that n_max rows touch at most
// The heads of a page side by side: their rows are neighbours in memory (16 prompts 53 us, with the heads far apart 58).
dim3 grid_of(const KvqView& kv, const KvqSeqs& q) {
  const long long pages = (long long)q.B * pages_each(q), z = (pages + 65534) / 65535;
  return dim3(kv.Hkv, (unsigned)((pages + z - 1) / z), (unsigned)z);
}
}  // namespace

void launch_kvq_write(const KvqView& kv, const KvqSeqs& q, const void* k_rows, const void* v_rows, size_t stride, int32_t* status, hipStream_t st) {
  const dim3 grid = grid_of(kv, q);
  const bool vec = (((uintptr_t)k_rows | (uintptr_t)v_rows) & 15) == 0 && stride % 8 == 0;
#define BS_KVQ(S_, D_) hipLaunchKernelGGL((kvq_write_kernel<S_, D_>), grid, dim3(256), 0, st, kv, q, pages_each(q), k_rows, v_rows, stride, status)
  if (kv.D == 128) { if (vec) BS_KVQ(ROWS_VEC, 128); else BS_KVQ(ROWS, 128); }
  else { if (vec) BS_KVQ(ROWS_VEC, 64); else BS_KVQ(ROWS, 64); }
#undef BS_KVQ
}
void launch_kvq_write_staged(const KvqView& kv, const KvqSeqs& q, const void* k_pages, const void* v_pages, int32_t* status, hipStream_t st) {
  const dim3 grid = grid_of(kv, q);
  if (kv.D == 128) hipLaunchKernelGGL((kvq_write_kernel<STAGED, 128>), grid, dim3(256), 0, st, kv, q, pages_each(q), k_pages, v_pages, (size_t)0, status);
  else hipLaunchKernelGGL((kvq_write_kernel<STAGED, 64>), grid, dim3(256), 0, st, kv, q, pages_each(q), k_pages, v_pages, (size_t)0, status);
}
void launch_kvq_read(const KvqView& kv, const KvqSeqs& q, void* k_rows, void* v_rows, size_t stride, int32_t* status, hipStream_t st) {
  const dim3 grid = grid_of(kv, q);
  const bool vec = (((uintptr_t)k_rows | (uintptr_t)v_rows) & 15) == 0 && stride % 8 == 0;
#define BS_KVQ(V_, D_) hipLaunchKernelGGL((kvq_read_kernel<V_, D_>), grid, dim3(256), 0, st, kv, q, pages_each(q), (bf16*)k_rows, (bf16*)v_rows, stride, status)
  if (kv.D == 128) { if (vec) BS_KVQ(true, 128); else BS_KVQ(false, 128); }
  else { if (vec) BS_KVQ(true, 64); else BS_KVQ(false, 64); }
#undef BS_KVQ
}
