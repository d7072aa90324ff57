// Log probabilities of given tokens, entropy and best alternatives of rows of logits.
//
// With m = max z and y = (z - m) / T:  log p(t) = y_t - log sum e^y,  H = log sum e^y - sum e^y y / sum e^y.  A masked token (-inf) has e^y = 0 and adds
// nothing to either sum.  A row in which everything is masked has no law: log p = -inf, H = 0, no alternatives.
#include "logprob.h"

namespace {
template <typename T>
__global__ void __launch_bounds__(256) logprob_kernel(LogprobArgs a) {
  __shared__ float s_f[12];
  __shared__ unsigned long long s_u[4];
  __shared__ int s_i[4];
  const int b = blockIdx.x / (a.k_max + 1), i = blockIdx.x % (a.k_max + 1), tid = threadIdx.x, V = a.vocab;
  int before = 0;
  for (int x = tid; x < b; x += 256) { const int k = a.draft_len ? a.draft_len[x] : a.k_max; before += k >= 0 && k <= a.k_max ? k + 1 : 0; }
  for (int o = 1; o < 64; o <<= 1) before += __shfl_xor(before, o);
  if ((tid & 63) == 0) s_i[tid >> 6] = before;
  __syncthreads();
  before = s_i[0] + s_i[1] + s_i[2] + s_i[3];
  const int k = a.draft_len ? a.draft_len[b] : a.k_max, n = a.n_tokens ? a.n_tokens[b] : k + 1;
  const size_t at = blockIdx.x;
  const bool bad = k < 0 || k > a.k_max || n < 0 || n > k + 1;
  if (bad && i == 0 && tid == 0 && a.status) atomicOr(a.status, BS_FAULT_DRAFT_LEN);
  const int tok = !bad && i < n ? a.tokens[at] : -1;
  const bool wrong = !bad && i < n && (tok < 0 || tok >= V);
  if (wrong && tid == 0 && a.status) atomicOr(a.status, BS_FAULT_TOKEN_ID);
  if (bad || i >= n || wrong) {
    if (tid == 0) { a.logprob[at] = 0.f; if (a.entropy) a.entropy[at] = 0.f; }
    for (int j = tid; j < a.n_top; j += 256) { a.top_tokens[at * a.n_top + j] = -1; a.top_logprobs[at * a.n_top + j] = 0.f; }
    return;
  }
  const T* z = (const T*)a.logits + (size_t)(before + i) * V;
  float m = -INFINITY;
  for (int j = tid; j < V; j += 256) m = fmaxf(m, to_f32<T>(z[j]));
  for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
  if ((tid & 63) == 0) s_f[tid >> 6] = m;
  __syncthreads();
  m = fmaxf(fmaxf(s_f[0], s_f[1]), fmaxf(s_f[2], s_f[3]));
  float sum = 0.f, sy = 0.f;
  for (int j = tid; j < V; j += 256) {
    const float x = to_f32<T>(z[j]);
    if (x == -INFINITY) continue;
    const float y = (x - m) * a.inv_temp, e = expf(y);
    sum += e;
    if (e != 0.f) sy += e * y;
  }
  for (int o = 1; o < 64; o <<= 1) { sum += __shfl_xor(sum, o); sy += __shfl_xor(sy, o); }
  __syncthreads();
  if ((tid & 63) == 0) { s_f[4 + (tid >> 6)] = sum; s_f[8 + (tid >> 6)] = sy; }
  __syncthreads();
  sum = s_f[4] + s_f[5] + s_f[6] + s_f[7];
  sy = s_f[8] + s_f[9] + s_f[10] + s_f[11];
  const bool empty = m == -INFINITY && sum == 0.f;
  const float lse = logf(sum);
  auto logp = [&](float x) { return empty || x == -INFINITY ? -INFINITY : (x - m) * a.inv_temp - lse; };
  if (tid == 0) {
    a.logprob[at] = sum != sum ? sum : logp(to_f32<T>(z[tok]));
    if (a.entropy) a.entropy[at] = empty ? 0.f : lse - sy / sum;
  }
  unsigned long long last = ~0ull;
  for (int j = 0; j < a.n_top; ++j) {                  // the largest key below the last one
    unsigned long long best = 0;
    for (int x = tid; x < V; x += 256) {
      const unsigned long long key = logprob_key(to_f32<T>(z[x]), x);
      if (key < last && key > best) best = key;
    }
    for (int o = 1; o < 64; o <<= 1) { const unsigned long long y = __shfl_xor(best, o); best = y > best ? y : best; }
    __syncthreads();
    if ((tid & 63) == 0) s_u[tid >> 6] = best;
    __syncthreads();
    for (int w = 0; w < 4; ++w) best = s_u[w] > best ? s_u[w] : best;
    last = best;
    if (tid == 0) {
      const int x = best ? (int)(0xffffffffu - (uint32_t)best) : -1;
      a.top_tokens[at * a.n_top + j] = x;
      a.top_logprobs[at * a.n_top + j] = x < 0 ? -INFINITY : sum != sum ? sum : logp(to_f32<T>(z[x]));
    }
  }
}
}  // namespace

size_t logprob_workspace(int, int, int, int) { return 256; }

void launch_logprob(const LogprobArgs& a, int B, int dtype, void*, hipStream_t st) {
  const dim3 grid(B * (a.k_max + 1));
  if (dtype == BS_F32) hipLaunchKernelGGL(logprob_kernel<float>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(logprob_kernel<bf16>, grid, dim3(256), 0, st, a);
}
