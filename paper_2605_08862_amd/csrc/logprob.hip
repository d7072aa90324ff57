// Log probabilities of given tokens, entropy and best alternatives of rows of logits.
//
// With m = max z and y = (z - m) / T:  log p(t) = y_t - log sum e^y,  H = log sum e^y - sum e^y y / sum e^y.  A masked token (-inf) has e^y = 0 and adds
// nothing to either sum.  A row in which everything is masked has no law: log p = -inf, H = 0, no alternatives.
//
// One pass over the logits, bound by memory.  A row is cut into segments, a workgroup each, which keeps its segment in registers: every wave sums against its own
// maximum, and the best alternatives come from a bound.  The largest of 64 groups of threads are known from the maxima; the n-th largest of these is no larger
// than the n-th largest logit, and hardly any other logit reaches it, so that one comparison per logit leaves a short list (a few more than n), which is ranked by
// counting.  Where more than kList of a segment reach it (logits that are all alike, or within 2^-7 of each other), the alternatives are looked for one after the
// other in n passes over the segment: 1152 rows of 152064 such float32 words 4350 us, bf16 3270, instead of 142 and 104.  The last segment of a row to arrive (publish_arrival, common.h) merges maxima, sums and lists the same way.
#include "logprob.h"

namespace {

constexpr int kThreads = 256, kEach = 64, kList = 512;  // elements of a thread; places of the list of candidates
constexpr int kSegment = kThreads * kEach, kMaxSegs = kLogprobMaxVocab / kSegment;       // (a lane for each in the merge: at most 64)
constexpr int kMergeEach = kMaxSegs * kLogprobMaxTop / kThreads;     // list entries of a thread in the merge

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <typename T> constexpr int kPer = 16 / sizeof(T);                    // elements of a vector of sixteen bytes
template <typename T> constexpr int kVecs = kEach / kPer<T>;                 // vectors of a thread
template <typename T> struct Vec;                                            // a vector that starts on any element
template <> struct Vec<float> { typedef uint32_t V __attribute__((ext_vector_type(4), aligned(4))); };
template <> struct Vec<bf16> { typedef uint32_t V __attribute__((ext_vector_type(4), aligned(2))); };
// element e of a vector
template <typename T> __device__ __forceinline__ float element(const u32x4& v, int e);
template <> __device__ __forceinline__ float element<float>(const u32x4& v, int e) { return __uint_as_float(v[e]); }
template <> __device__ __forceinline__ float element<bf16>(const u32x4& v, int e) { return __uint_as_float(e & 1 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16); }

// Over the 64 lanes, in registers: neighbours, halves of rows of sixteen lanes, then the rows.
template <int CTRL> __device__ __forceinline__ float dpp(float v) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, true)); }
template <typename F> __device__ __forceinline__ float wave_reduce(float v, const F& f) {
  v = f(v, dpp<0xB1>(v));                               // quad_perm 1 0 3 2
  v = f(v, dpp<0x4E>(v));                               // quad_perm 2 3 0 1
  v = f(v, dpp<0x141>(v));                              // row_half_mirror
  v = f(v, dpp<0x140>(v));                              // row_mirror
#if defined(__HIP_DEVICE_COMPILE__)
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = f(__uint_as_float(b[0]), __uint_as_float(b[1]));
#endif
  return v;
}
__device__ __forceinline__ float wave_max(float v) { return wave_reduce(v, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float wave_sum(float v) { return wave_reduce(v, [](float a, float b) { return a + b; }); }

// What a lane wrote to LDS, others of its wave read behind this.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

struct Top { float z; int j; };
__device__ __forceinline__ bool better(float za, int ja, float zb, int jb) { return za > zb || (za == zb && ja < jb); }

constexpr int kOwners = 4;                              // threads of a wave whose elements are looked at together
struct SelectShared {
  float group[4][64];
  Top list[kList];
  int rank[kList];
  int n;
  Top best[4];
};
// Behind it, one after the other: elements of those threads, [wave][kOwners][vector]; in the merge, the segments' alternatives.
constexpr size_t kStageBytes = (size_t)4 * kOwners * kEach * sizeof(float);
size_t select_bytes(int segs, int n_top) {
  const size_t parts = segs > 1 ? (size_t)segs * n_top * sizeof(Top) : 0;
  return n_top == 0 ? 0 : parts > kStageBytes ? parts : kStageBytes;
}

// The n best of the elements that the threads have, E each; -inf and NaN are none.  zmax: the thread's largest.  src.own(e): element e of the calling thread.  Many
// elements (Source::kMany): src.show(p), called by the threads with a candidate, up to kOwners of a wave, puts the thread's elements in place p; src.value(p, e):
// element e of place p, whose thread is `owner`, src.index(owner, e): its token.  out(rank, z, j) is called once for every rank that is taken; returns how many are.
template <int E, typename Source, typename Out>
__device__ __forceinline__ int select_top(float zmax, int n, const Source& src, const Out& out, SelectShared& s) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  s.group[wave][lane] = zmax;
  if (tid == 0) s.n = 0;
  __syncthreads();
  // bound: no larger than the n-th largest of 64 groups (a lane of all four waves), off by less than 2^-7 of it: the first sixteen bits of its ranking key
  const uint32_t g = filter_key(fmaxf(fmaxf(s.group[0][lane], s.group[1][lane]), fmaxf(s.group[2][lane], s.group[3][lane])));
  uint32_t key = 0;
#pragma unroll
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t t = key | 1u << bit;
    if (__popcll(__ballot(g >= t)) >= n) key = t;
  }
  const float bound = key <= 0x007fffffu ? -INFINITY : __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
  // candidates go to the list a wave at a time
  auto put = [&](bool hit, unsigned long long hits, int at, float z, int j) {
    const int k = at + __popcll(hits & ((1ull << lane) - 1));
    if (hit && k < kList) { s.list[k] = Top{z, j}; s.rank[k] = 0; }
  };
  auto reserve = [&](int count) {
    int at = 0;
    if (lane == 0) at = atomicAdd(&s.n, count);
    return __builtin_amdgcn_readfirstlane(at);
  };
  auto hit = [&](float z) { return z >= bound && z > -INFINITY; };
  if constexpr (Source::kMany) {
    // the elements of the few threads that have one, one by each lane
    constexpr int C = E / 64;
    for (unsigned long long have = __ballot(hit(zmax)); have;) {
      const int p = __popcll(have & ((1ull << lane) - 1));
      if ((have >> lane & 1) && p < kOwners) src.show(p);
      wave_fence();
      float z[kOwners][C];
#pragma unroll
      for (int o = 0; o < kOwners; ++o)
#pragma unroll
        for (int c = 0; c < C; ++c) z[o][c] = src.value(o, c * 64 + lane);
      const int shown = min((int)__popcll(have), kOwners);
      int count = 0;
#pragma unroll
      for (int o = 0; o < kOwners; ++o)
#pragma unroll
        for (int c = 0; c < C; ++c) {
          if (o >= shown) z[o][c] = -INFINITY;           // (what was shown there before)
          count += __popcll(__ballot(hit(z[o][c])));
        }
      int at = reserve(count);
#pragma unroll
      for (int o = 0; o < kOwners; ++o) {
        const int owner = wave * 64 + __ffsll((long long)have) - 1;
        have &= have - 1;                                // (0 stays 0)
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const unsigned long long hits = __ballot(hit(z[o][c]));
          if (!hits) continue;
          put(hit(z[o][c]), hits, at, z[o][c], src.index(owner, c * 64 + lane));
          at += __popcll(hits);
        }
      }
      wave_fence();
    }
  } else {
    for (int e = 0; e * kThreads < src.n; ++e) {
      const Top t = src.own(e);
      const unsigned long long hits = __ballot(hit(t.z));
      if (hits) put(hit(t.z), hits, reserve(__popcll(hits)), t.z, t.j);
    }
  }
  __syncthreads();
  const int found = s.n;
  if (found <= kList) {                                 // a wave counts against a quarter of the list
    const int o0 = found * wave / 4, o1 = found * (wave + 1) / 4;
    for (int k = lane; k < found; k += 64) {
      const Top t = s.list[k];
      int rank = 0;
#pragma unroll 4
      for (int o = o0; o < o1; ++o) { const Top x = s.list[o]; rank += better(x.z, x.j, t.z, t.j) ? 1 : 0; }
      if (rank) atomicAdd(&s.rank[k], rank);
    }
    __syncthreads();
    for (int k = tid; k < found; k += kThreads) if (s.rank[k] < n) out(s.rank[k], s.list[k].z, s.list[k].j);
    return min(found, n);
  }
  // more than the list holds reach the bound (a segment of equal logits, say): one after the other
  Top last{INFINITY, -1};
  for (int r = 0; r < n; ++r) {
    Top best{-INFINITY, 0x7fffffff};
    for (int e = 0; e < E; ++e) {
      const Top t = src.own(e);
      if (better(last.z, last.j, t.z, t.j) && better(t.z, t.j, best.z, best.j)) best = t;
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const float x = __shfl_xor(best.z, o);
      const int j = __shfl_xor(best.j, o);
      if (better(x, j, best.z, best.j)) best = Top{x, j};
    }
    __syncthreads();
    if (lane == 0) s.best[wave] = best;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) if (better(s.best[w].z, s.best[w].j, best.z, best.j)) best = s.best[w];
    last = best;
    if (tid == 0) out(r, best.z, best.j);
  }
  return n;
}

// A segment: element e of a thread is j0 + (e / P * kThreads + thread) * P + e % P, in vector e / P.
template <typename T> struct SegmentSource {
  static constexpr bool kMany = true;
  const u32x4 (&v)[kVecs<T>];
  const T* z0;
  int j0, j1;
  u32x4* stage;                                        // the wave's
  __device__ __forceinline__ int index(int thread, int e) const { return j0 + (e / kPer<T> * kThreads + thread) * kPer<T> + e % kPer<T>; }
  __device__ __forceinline__ void show(int p) const {
#pragma unroll
    for (int u = 0; u < kVecs<T>; ++u) stage[p * (kEach / 4) + u] = v[u];
  }
  __device__ __forceinline__ float value(int p, int e) const { return to_f32<T>(((const T*)(stage + p * (kEach / 4)))[e]); }
  __device__ __forceinline__ Top own(int e) const {
    const int j = index(threadIdx.x, e);
    return Top{j < j1 ? to_f32<T>(z0[j]) : -INFINITY, j};
  }
};
// The alternatives of a row's segments, in LDS.
struct PartsSource {
  static constexpr bool kMany = false;
  int n;
  const Top* parts;
  __device__ __forceinline__ Top own(int e) const {
    const int i = e * kThreads + threadIdx.x;
    return i < n ? parts[i] : Top{-INFINITY, 0x7fffffff};
  }
};

// Maximum and sums of a part of a row, in units of log2: t = (z - m) c with c = log2(e) / T;  s = sum 2^t, q = sum 2^t t.
struct Stats { float m, s, q; };
__device__ __forceinline__ Stats merge_stats(Stats a, Stats b, float c) {
  const float m = fmaxf(a.m, b.m);
  if (m == -INFINITY) return Stats{m, a.s + b.s, a.q + b.q};                  // both empty (or NaN alone, which the sums carry)
  // a shift of the maximum by d moves every t by d c
  const float da = a.m == -INFINITY ? 0.f : (a.m - m) * c, db = b.m == -INFINITY ? 0.f : (b.m - m) * c;
  const float fa = a.m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(da), fb = b.m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(db);
  const float qa = fmaxf(da, -1e4f), qb = fmaxf(db, -1e4f);                  // 0 * -inf is 0 here
  return Stats{m, a.s * fa + b.s * fb, fa * (a.q + a.s * qa) + fb * (b.q + b.s * qb)};
}

// `entry`: the row's place in the outputs; false: it has no row, and its outputs are written.
__device__ __forceinline__ bool find_row(const LogprobArgs& a, int entry, bool write, int* s_i, size_t& row, int& tok) {
  const int width = a.k_max + 1, b = entry / width, i = entry - b * width, tid = threadIdx.x;
  const int k = a.draft_len ? a.draft_len[b] : a.k_max, n = a.n_tokens ? a.n_tokens[b] : k + 1;
  const bool bad = k < 0 || k > a.k_max || n < 0 || n > k + 1;
  tok = !bad && i < n ? a.tokens[entry] : 0;
  const bool wrong = tok < 0 || tok >= a.vocab;
  if (bad || i >= n || wrong) {
    if (!write) return false;
    if (tid == 0) {
      if (bad && i == 0 && a.status) atomicOr(a.status, BS_FAULT_DRAFT_LEN);
      if (wrong && a.status) atomicOr(a.status, BS_FAULT_TOKEN_ID);
      a.logprob[entry] = 0.f;
      if (a.entropy) a.entropy[entry] = 0.f;
    }
    for (int j = tid; j < a.n_top; j += kThreads) { a.top_tokens[(size_t)entry * a.n_top + j] = -1; a.top_logprobs[(size_t)entry * a.n_top + j] = 0.f; }
    return false;
  }
  if (!a.draft_len) { row = entry; return true; }
  int before = 0;
  for (int x = tid; x < b; x += kThreads) { const int d = a.draft_len[x]; before += d >= 0 && d <= a.k_max ? d + 1 : 0; }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) before += __shfl_xor(before, o);
  if ((tid & 63) == 0) s_i[tid >> 6] = before;
  __syncthreads();
  row = (size_t)(s_i[0] + s_i[1] + s_i[2] + s_i[3]) + i;
  return true;
}

// 1152 rows of 152064 float32 logits, the 20 best: 142 us, 4.7 TB/s (130 without alternatives); of bf16 104 us, where the workgroups' chains of selection bound
// it (78 without alternatives).  Registers for five waves on a SIMD: float32 160 us with four; for eight: bf16 108 us with seven.
// seg: elements of a segment, a multiple of 8; segs of them cover a row.  Partials: [entry][segs] statistics, [entry][segs][n_top] alternatives.
template <typename T, bool TOP>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 4 ? 5 : 8) logprob_kernel(LogprobArgs a, int seg, int segs, wt_f32x4* __restrict__ part, Top* __restrict__ part_top,
                                                           int32_t* __restrict__ counters) {
  extern __shared__ __align__(16) char s_more[];
  __shared__ SelectShared s_sel;
  __shared__ Stats s_stats[4];
  __shared__ Top s_top[kLogprobMaxTop];
  __shared__ int s_i[4], s_flag;
  constexpr int P = kPer<T>;                            // elements of a vector
  const int entry = blockIdx.x / segs, sg = blockIdx.x - entry * segs, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = a.vocab;
  size_t row;
  int tok;
  if (!find_row(a, entry, sg == 0, s_i, row, tok)) return;
  const T* z0 = (const T*)a.logits + row * V;
  const int j0 = sg * seg, j1 = min(j0 + seg, V);
  const float z_tok = to_f32<T>(z0[tok]);

  // ---- the segment: element e of a thread is j0 + (e / P * kThreads + tid) * P + e % P
  u32x4 v[kVecs<T>];
  const uint32_t none = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;           // -inf
#pragma unroll
  for (int u = 0; u < kVecs<T>; ++u) {
    const int j = j0 + (u * kThreads + tid) * P;
    v[u] = u32x4{none, none, none, none};
    if (j0 + u * kThreads * P >= j1) continue;          // the same for all threads
    if (j + P <= j1) {
      v[u] = *(const typename Vec<T>::V*)(z0 + j);
    } else {
#pragma unroll
      for (int e = 0; e < P; ++e)
        if (j + e < j1) {
          if constexpr (P == 4) v[u][e] = ((const uint32_t*)z0)[j + e];
          else v[u][e / 2] = e & 1 ? (v[u][e / 2] & 0xffffu) | (uint32_t)((const uint16_t*)z0)[j + e] << 16 : (v[u][e / 2] & 0xffff0000u) | ((const uint16_t*)z0)[j + e];
        }
    }
  }
  float zmax = -INFINITY;                               // (of NaN alone: no maximum)
#pragma unroll
  for (int u = 0; u < kVecs<T>; ++u)
#pragma unroll
    for (int e = 0; e < P; ++e) zmax = fmaxf(zmax, element<T>(v[u], e));
  const float m = wave_max(zmax);
  if constexpr (P == 8) {                               // unpacked again below: kept, the elements would take 128 registers
#pragma unroll
    for (int u = 0; u < kVecs<T>; ++u) asm volatile("" : "+v"(v[u]));
  }
  const float c = a.inv_temp * 1.44269504088896341f, m0 = m == -INFINITY ? 0.f : m;
  float sum = 0.f, q = 0.f;
#pragma unroll
  for (int u = 0; u < kVecs<T>; ++u) {
    if (j0 + u * kThreads * P >= j1) break;
#pragma unroll
    for (int e = 0; e < P; ++e) {
      const float t = (element<T>(v[u], e) - m0) * c, x = __builtin_amdgcn_exp2f(t);      // (m c - z c would overflow where logits are near the type's lowest value)
      sum += x;
      q += x * fmaxf(t, -1e4f);                         // a masked one: 0 * -1e4
    }
  }
  sum = wave_sum(sum);
  q = wave_sum(q);
  if (lane == 0) s_stats[wave] = Stats{m, sum, q};
  int n_found = 0;
  if constexpr (TOP)
    n_found = select_top<kEach>(zmax, a.n_top, SegmentSource<T>{v, z0, j0, j1, (u32x4*)s_more + wave * (kOwners * kEach / 4)}, [&](int r, float x, int j) { s_top[r] = Top{x, j}; }, s_sel);
  __syncthreads();
  Stats st = s_stats[0];
#pragma unroll
  for (int w = 1; w < 4; ++w) st = merge_stats(st, s_stats[w], c);

  if (segs > 1) {
    const wt_buf bp = wt_buffer(part + (size_t)entry * segs), bt = wt_buffer(part_top + (size_t)entry * segs * a.n_top);
    if (tid == 0) wt_store4(bp, sg * 16, wt_f32x4{st.m, st.s, st.q, 0.f});
    if constexpr (TOP)
      for (int r = tid; r < a.n_top; r += kThreads) {
        const bool is = r < n_found;
        wt_store2(bt, (sg * a.n_top + r) * 8, is ? s_top[r].z : -INFINITY, __int_as_float(is ? s_top[r].j : 0x7fffffff));
      }
    if (!publish_arrival(counters + entry, segs, &s_flag)) return;
    // the last segment of the row: all of them, in their order
    const wt_f32x4 mine = wt_load4(bp, min(lane, segs - 1) * 16);      // a lane for each, in every wave
    st = lane < segs ? Stats{mine[0], mine[1], mine[2]} : Stats{-INFINITY, 0.f, 0.f};
    float tmax = -INFINITY;
    if constexpr (TOP) {
      const int n = segs * a.n_top;
      for (int i = tid; i < n; i += kThreads) {
        const wt_f32x2 p = wt_load2(bt, i * 8);
        ((Top*)s_more)[i] = Top{p[0], __float_as_int(p[1])};
        tmax = fmaxf(tmax, p[0]);
      }
    }
    for (int o = 1; o < segs; o <<= 1) st = merge_stats(st, Stats{__shfl_xor(st.m, o), __shfl_xor(st.s, o), __shfl_xor(st.q, o)}, c);
    auto first = [](float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); };
    st = Stats{first(st.m), first(st.s), first(st.q)};
    __syncthreads();
    if constexpr (TOP) {
      n_found = select_top<kMergeEach>(tmax, a.n_top, PartsSource{segs * a.n_top, (const Top*)s_more}, [&](int r, float x, int j) { s_top[r] = Top{x, j}; }, s_sel);
      __syncthreads();
    }
  }
  const bool empty = st.m == -INFINITY && st.s == 0.f;
  const float lse = logf(st.s), ln2 = 0.693147180559945309f;
  auto logp = [&](float x) { return st.s != st.s ? st.s : empty || x == -INFINITY ? -INFINITY : (x - st.m) * a.inv_temp - lse; };
  if (tid == 0) {
    a.logprob[entry] = logp(z_tok);
    if (a.entropy) a.entropy[entry] = empty ? 0.f : lse - st.q * ln2 / st.s;
  }
  if constexpr (TOP)
    for (int r = tid; r < a.n_top; r += kThreads) {
      const bool is = r < n_found;
      a.top_tokens[(size_t)entry * a.n_top + r] = is ? s_top[r].j : -1;
      a.top_logprobs[(size_t)entry * a.n_top + r] = is ? logp(s_top[r].z) : -INFINITY;
    }
}

// Segments of a row: as few as fit (64 elements of a thread in registers), of the same length.  More of them for few rows: the merge of one more costs what its
// shorter pass saves (9 rows of 151936 bf16 words in segments of 2048 words 22.7 us, 4096 18.8, 8192 16.4, 16384 16.1; 64 rows of float32 23.0, 22.9, 22.9, 21.3; 500
// rows of 8000 26.9, 20.4, 13.4, 13.5).  Segments of twice the length for bf16: 1152 rows 101 us, with the 20 best,
// instead of 104, but 64 rows 19.6 instead of 17.8 and 9 rows 14.3 instead of 13.6.
struct Cutting { int seg, segs; };
Cutting cut_rows(int vocab) {
  const int segs = (vocab + kSegment - 1) / kSegment;
  return Cutting{((vocab + segs - 1) / segs + 7) / 8 * 8, segs};
}
}  // namespace

size_t logprob_workspace(int B, int k_max, int vocab, int n_top) {
  return (size_t)kLogprobMaxRows * sizeof(int32_t) + (size_t)B * (k_max + 1) * cut_rows(vocab).segs * (sizeof(wt_f32x4) + (size_t)n_top * sizeof(Top));
}

void launch_logprob(const LogprobArgs& a, int B, int dtype, void* workspace, hipStream_t st) {
  const long long rows = (long long)B * (a.k_max + 1);
  const Cutting cut = cut_rows(a.vocab);
  int32_t* counters = (int32_t*)workspace;
  wt_f32x4* part = (wt_f32x4*)(counters + kLogprobMaxRows);
  Top* part_top = (Top*)(part + rows * cut.segs);
  const dim3 grid((unsigned)(rows * cut.segs));
#define BS_LOGPROB(T_, TOP_) hipLaunchKernelGGL((logprob_kernel<T_, TOP_>), grid, dim3(kThreads), select_bytes(cut.segs, a.n_top), st, a, cut.seg, cut.segs, part, part_top, counters)
  if (dtype == BS_F32) { if (a.n_top > 0) BS_LOGPROB(float, true); else BS_LOGPROB(float, false); }
  else { if (a.n_top > 0) BS_LOGPROB(bf16, true); else BS_LOGPROB(bf16, false); }
#undef BS_LOGPROB
}
