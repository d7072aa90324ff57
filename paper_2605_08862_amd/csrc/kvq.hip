// Rows of K and V <-> the pages of the 8-bit cache (scales and element order: kvq.h).
#include "kvq.h"

namespace {

// What a workgroup knows of its (sequence, page): tokens [lo, hi) of the page are rows row .. of the batch.
struct Span { int page, lo, hi, row; bool live; };

// The sequence's rows are checked as a whole, by every workgroup that has a page of it alike: a sequence with a bad count, slot, position or page, or
// (writes) with the slot of an earlier sequence, is skipped.  s_red: one word per wave.
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
      if (!q.row_start) { const int m = q.n[c] + q.n_add; before += m >= 0 && m <= q.n_max ? m : 0; }
      if (WRITE && q.slot[c] == slot) bad |= BS_FAULT_SLOT;
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

__device__ __forceinline__ float bounded(bf16 x, bool& out_of_range) {
  const float f = to_f32<bf16>(x);
  if (fabsf(f) <= kKvqMost) return f;
  out_of_range = true;
  return f != f ? 0.f : copysignf(kKvqMost, f);
}

// One workgroup per (page of a sequence, KV head, K or V).
__global__ void __launch_bounds__(256) kvq_write_kernel(KvqView kv, KvqSeqs q, int pages_each, const bf16* __restrict__ k_rows, const bf16* __restrict__ v_rows,
                                                        size_t stride, int32_t* __restrict__ status) {
  __shared__ int s_red[8];
  __shared__ float s_max[4];
  const int b = blockIdx.x / pages_each, h = blockIdx.y >> 1, is_v = blockIdx.y & 1, D = kv.D;
  const Span sp = find_span<true>(kv, q, b, blockIdx.x % pages_each, s_red, blockIdx.y == 0 ? status : nullptr);
  if (!sp.live) return;
  const bf16* rows = (is_v ? v_rows : k_rows) + (size_t)sp.row * stride + h * D;
  uint8_t* page = (is_v ? kv.v : kv.k) + (size_t)sp.page * kvq_page_bytes(kv.Hkv, D);
  float* scale = (is_v ? kv.vs : kv.ks) + (size_t)sp.page * kv.Hkv + h;
  const int n = sp.hi - sp.lo;
  bool out_of_range = false;
  float a = 0.f;
  for (int i = threadIdx.x; i < n * D; i += 256) a = fmaxf(a, fabsf(bounded(rows[(size_t)(i / D) * stride + i % D], out_of_range)));
  if (out_of_range && status) atomicOr(status, BS_FAULT_RANGE);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) a = fmaxf(a, __shfl_xor(a, o));
  if ((threadIdx.x & 63) == 0) s_max[threadIdx.x >> 6] = a;
  const int e_old = kvq_exp_of(*scale);
  __syncthreads();
  int e = kvq_exp_for(fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3])));
  if (sp.lo > 0) {
    if (e > e_old) {                                   // rows that are there already are rounded again
      const float f = kvq_scale(e_old - e);
      uint32_t* w = (uint32_t*)(page + (size_t)h * kPage * D);
      for (int i = threadIdx.x; i < kPage * D / 4; i += 256) {
        const f32x4 x = kvq_values4(w[i]);
        w[i] = kvq_codes4(x[0] * f, x[1] * f, x[2] * f, x[3] * f);
      }
      __syncthreads();
    }
    e = max(e, e_old);
  }
  if (threadIdx.x == 0) *scale = kvq_scale(e);
  const float f = kvq_scale(-e);
  bool dummy;
  for (int i = threadIdx.x; i < n * D; i += 256) {
    const int t = i / D, d = i % D, tok = sp.lo + t;
    const uint32_t c = kvq_codes4(bounded(rows[(size_t)t * stride + d], dummy) * f, 0.f, 0.f, 0.f);
    page[is_v ? kvq_v_piece(D, h, tok & ~15, d) + (tok & 15) : kvq_k_piece(D, h, tok, d & ~15) + (d & 15)] = (uint8_t)c;
  }
}

__global__ void __launch_bounds__(256) kvq_read_kernel(KvqView kv, KvqSeqs q, int pages_each, bf16* __restrict__ k_rows, bf16* __restrict__ v_rows,
                                                       size_t stride, int32_t* __restrict__ status) {
  __shared__ int s_red[8];
  const int b = blockIdx.x / pages_each, h = blockIdx.y >> 1, is_v = blockIdx.y & 1, D = kv.D;
  const Span sp = find_span<false>(kv, q, b, blockIdx.x % pages_each, s_red, blockIdx.y == 0 ? status : nullptr);
  if (!sp.live) return;
  bf16* rows = (is_v ? v_rows : k_rows) + (size_t)sp.row * stride + h * D;
  const uint8_t* page = (is_v ? kv.v : kv.k) + (size_t)sp.page * kvq_page_bytes(kv.Hkv, D);
  const float f = kvq_scale(kvq_exp_of((is_v ? kv.vs : kv.ks)[(size_t)sp.page * kv.Hkv + h]));
  for (int i = threadIdx.x; i < (sp.hi - sp.lo) * D; i += 256) {
    const int t = i / D, d = i % D, tok = sp.lo + t;
    const uint32_t c = page[is_v ? kvq_v_piece(D, h, tok & ~15, d) + (tok & 15) : kvq_k_piece(D, h, tok, d & ~15) + (d & 15)];
    rows[(size_t)t * stride + d] = from_f32<bf16>(kvq_values4(c)[0] * f);
  }
}

int pages_each(const KvqSeqs& q) { return (q.n_max + 2 * kPage - 2) / kPage; }   // pages that n_max rows touch at most
}  // namespace

void launch_kvq_write(const KvqView& kv, const KvqSeqs& q, const void* k_rows, const void* v_rows, size_t stride, int32_t* status, hipStream_t st) {
  hipLaunchKernelGGL(kvq_write_kernel, dim3(q.B * pages_each(q), 2 * kv.Hkv), dim3(256), 0, st, kv, q, pages_each(q), (const bf16*)k_rows, (const bf16*)v_rows,
                     stride, status);
}
void launch_kvq_read(const KvqView& kv, const KvqSeqs& q, void* k_rows, void* v_rows, size_t stride, int32_t* status, hipStream_t st) {
  hipLaunchKernelGGL(kvq_read_kernel, dim3(q.B * pages_each(q), 2 * kv.Hkv), dim3(256), 0, st, kv, q, pages_each(q), (bf16*)k_rows, (bf16*)v_rows, stride, status);
}
