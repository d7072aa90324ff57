// Ragged causal attention over the 8-bit cache.
#include "kvq.h"

namespace {
// One workgroup per (packed row, query head): softmax over chunks of 256 tokens with the running maximum and sum.
__global__ void __launch_bounds__(256) kvq_attention_kernel(KvqView kv, KvqSeqs s, int Hq, const bf16* __restrict__ q, size_t q_stride, bf16* __restrict__ out,
                                                            float scale, int32_t* __restrict__ status) {
  __shared__ float s_q[128], s_p[256], s_red[4], s_o[256];
  __shared__ int s_i[8];
  const int b = blockIdx.x / s.n_max, i = blockIdx.x % s.n_max, hq = blockIdx.y, D = kv.D, h = hq / (Hq / kv.Hkv), tid = threadIdx.x;
  const int n = s.n[b] + s.n_add, slot = s.slot[b], c = s.pos[b];
  int bad = 0, before = 0;
  if (n < 0 || n > s.n_max) bad |= BS_FAULT_DRAFT_LEN;
  if (n != 0 && !bad) {
    if (slot < 0 || slot >= kv.n_slots) bad |= BS_FAULT_SLOT;
    if (c < 0 || (long long)c + n > (long long)kv.max_pages * kPage) bad |= BS_FAULT_KV_PAGES;
  }
  const int32_t* bt = kv.block_table + (size_t)slot * kv.max_pages;
  if (!bad && n > 0)
    for (int p = tid; p <= (c + n - 1) / kPage; p += 256) if ((unsigned)bt[p] >= (unsigned)kv.n_pages) bad |= BS_FAULT_KV_PAGES;
  for (int x = tid; x < b; x += 256) { const int m = s.n[x] + s.n_add; before += m >= 0 && m <= s.n_max ? m : 0; }
  for (int o = 1; o < 64; o <<= 1) { before += __shfl_xor(before, o); bad |= __shfl_xor(bad, o); }
  if ((tid & 63) == 0) { s_i[tid >> 6] = before; s_i[4 + (tid >> 6)] = bad; }
  __syncthreads();
  before = s_i[0] + s_i[1] + s_i[2] + s_i[3];
  bad = s_i[4] | s_i[5] | s_i[6] | s_i[7];
  if (bad) { if (tid == 0 && i == 0 && status) atomicOr(status, bad); return; }
  if (i >= n) return;
  const size_t row = before + i;
  if (tid < D) s_q[tid] = to_f32<bf16>(q[row * q_stride + (size_t)hq * D + tid]) * scale;
  __syncthreads();
  float m = -INFINITY, l = 0.f, o = 0.f;
  const int d = tid % D, grp = tid / D, per = 256 / (256 / D);
  for (int t0 = 0; t0 <= c + i; t0 += 256) {
    const int t = t0 + tid;
    float x = -INFINITY;
    if (t <= c + i) {
      const int page = bt[t / kPage];
      const uint8_t* kp = kv.k + (size_t)page * kvq_page_bytes(kv.Hkv, D);
      x = 0.f;
      for (int d0 = 0; d0 < D; d0 += 16) {
        const u32x4 w = *(const u32x4*)(kp + kvq_k_piece(D, h, t % kPage, d0));
        for (int e = 0; e < 4; ++e) {
          const f32x4 k = kvq_values4(w[e]);
          for (int j = 0; j < 4; ++j) x += s_q[d0 + 4 * e + j] * k[j];
        }
      }
      x *= kvq_scale(kvq_exp_of(kv.ks[(size_t)page * kv.Hkv + h]));
    }
    float mx = x;
    for (int k = 1; k < 64; k <<= 1) mx = fmaxf(mx, __shfl_xor(mx, k));
    if ((tid & 63) == 0) s_red[tid >> 6] = mx;
    __syncthreads();
    const float m_new = fmaxf(m, fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3])));
    const float f = __expf(m - m_new), p = __expf(x - m_new);
    m = m_new;
    s_p[tid] = p;
    __syncthreads();
    l *= f; o *= f;
    for (int k = 0; k < 256; ++k) l += s_p[k];
    for (int k = grp * per; k < (grp + 1) * per && t0 + k <= c + i; ++k) {
      const int page = bt[(t0 + k) / kPage], tok = (t0 + k) % kPage;
      const uint32_t code = kv.v[(size_t)page * kvq_page_bytes(kv.Hkv, D) + kvq_v_piece(D, h, tok & ~15, d) + (tok & 15)];
      o += s_p[k] * kvq_values4(code)[0] * kvq_scale(kvq_exp_of(kv.vs[(size_t)page * kv.Hkv + h]));
    }
    __syncthreads();
  }
  s_o[tid] = o;
  __syncthreads();
  if (tid < D) {
    float sum = 0.f;
    for (int g = 0; g < 256 / D; ++g) sum += s_o[g * D + tid];
    out[row * (size_t)Hq * D + (size_t)hq * D + tid] = from_f32<bf16>(sum / l);
  }
}
}  // namespace

size_t kvq_attention_workspace(int, int, int, int) { return 256; }

void launch_kvq_attention(const KvqView& kv, const KvqSeqs& s, int Hq, const void* qrows, size_t q_stride, void* out, int32_t* status, void*, hipStream_t st) {
  hipLaunchKernelGGL(kvq_attention_kernel, dim3(s.B * s.n_max, Hq), dim3(256), 0, st, kv, s, Hq, (const bf16*)qrows, q_stride, (bf16*)out,
                     1.0f / sqrtf((float)kv.D), status);
}
