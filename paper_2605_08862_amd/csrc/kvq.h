// The KV cache in 8 bits (bs_kvq_*): scales, element order inside a page, what the kernels and launchers share.
//
// A block is one page (64 tokens) of one KV head, K and V apart.  It holds e4m3 codes and a scale 2^e, value = code * 2^e, e in -15 .. 7: every value is
// then a multiple of 2^-24 and at most 57344, i.e. exact in float16 (and, with four significant bits, in bfloat16), so codes become operands of the f16
// MFMA with no rounding.  A power of two as the scale makes a later, larger scale harmless: codes of rows that are there already move to a smaller exponent
// and are rounded again only where they become subnormal.
#pragma once
#include "gemm_mfma.h"

constexpr int kKvqMinExp = -15, kKvqMaxExp = 7;
constexpr float kKvqMost = 57344.f;                    // 448 * 2^7
typedef uint8_t u8x16 __attribute__((ext_vector_type(16)));

struct KvqView {
  int n_pages, n_slots, max_pages, Hkv, D;
  const int32_t* block_table;
  uint8_t *k, *v;
  float *ks, *vs;                                      // [n_pages][Hkv]
};
// Packed rows of a batch: sequence b has n[b] + n_add rows for positions pos[b] .. of slot slot[b] (a count outside 0 .. n_max counts as none).
// row_start: first packed row of every sequence; null: the kernels add the counts up.  slot == null: one sequence, the scalars.
struct KvqSeqs {
  int B, n_max, n_add;
  const int32_t *slot, *pos, *n, *row_start;
  int slot0, pos0;
};

// Element order inside a page.  Per head two tiles of 32 tokens in the operand order of the 32 x 32 x 16 MFMA (as the 16-bit pages, common.h), two
// K-steps to a lane's sixteen bytes, so that a wave's load is one contiguous KiB.
//   K tile: S^T = K Q^T; lane (m, g) has, for steps 2 s and 2 s + 1, sixteen consecutive d from g * D/2 + 16 s of the token of A-row m (k_tile_row).
//   V tile: O^T = V^T P^T; lane (d % 32, g) has the sixteen tokens 16 g .. 16 g + 15 of one d.
__host__ __device__ __forceinline__ size_t kvq_page_bytes(int Hkv, int D) { return (size_t)Hkv * kPage * D; }
// the sixteen bytes of K that hold d0 .. d0 + 15 (d0 % 16 == 0) of a token
__host__ __device__ __forceinline__ int kvq_k_piece(int D, int h, int tok, int d0) {
  const int tile = tok / kTile, g = d0 / (D / 2), s = d0 % (D / 2) / 16;
  return ((((h * 2 + tile) * (D / 32) + s) * 2 + g) * 32 + k_tile_row(tok % kTile)) * 16;
}
// the sixteen bytes of V that hold tokens tok0 .. tok0 + 15 (tok0 % 16 == 0) of a d
__host__ __device__ __forceinline__ int kvq_v_piece(int D, int h, int tok0, int d) {
  const int tile = tok0 / kTile, g = tok0 % kTile / 16;
  return ((((h * 2 + tile) * (D / 32) + d / 32) * 2 + g) * 32 + d % 32) * 16;
}

__device__ __forceinline__ float kvq_scale(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// exponent of a stored scale (memory that was never written: a valid one all the same)
__device__ __forceinline__ int kvq_exp_of(float scale) {
  const int e = (int)(__float_as_uint(scale) >> 23 & 255) - 127;
  return min(max(e, kKvqMinExp), kKvqMaxExp);
}
// least e with a <= 448 * 2^e = 1.75 * 2^(e + 8)
__device__ __forceinline__ int kvq_exp_for(float a) {
  const uint32_t u = __float_as_uint(a);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return min(max(e, kKvqMinExp), kKvqMaxExp);
}
__device__ __forceinline__ uint32_t kvq_codes4(float a, float b, float c, float d) {
#if defined(__HIP_DEVICE_COMPILE__)
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
#else
  return 0;
#endif
}
__device__ __forceinline__ f32x4 kvq_values4(uint32_t c) {
#if defined(__HIP_DEVICE_COMPILE__)
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
  return f32x4{lo[0], lo[1], hi[0], hi[1]};
#else
  return f32x4{0.f, 0.f, 0.f, 0.f};
#endif
}

// kvq.hip   rows -> pages and back.  stride: elements from one row to the next.
void launch_kvq_write(const KvqView& kv, const KvqSeqs& q, const void* k_rows, const void* v_rows, size_t stride, int32_t* status, hipStream_t st);
// Rows that a verify step left in staging pages (16-bit page order): packed row r is token r % kPage of page r / kPage.
void launch_kvq_write_staged(const KvqView& kv, const KvqSeqs& q, const void* k_pages, const void* v_pages, int32_t* status, hipStream_t st);
void launch_kvq_read(const KvqView& kv, const KvqSeqs& q, void* k_rows, void* v_rows, size_t stride, int32_t* status, hipStream_t st);
// kvq_attention.hip   q, out: [rows][Hq][D] bf16, q_stride elements from one row of q to the next
size_t kvq_attention_workspace(int Hq, int Hkv, int D, int q_max);
void launch_kvq_attention(const KvqView& kv, const KvqSeqs& q, int Hq, const void* qrows, size_t q_stride, void* out, int32_t* status, void* workspace,
                          hipStream_t st);
// of a verify step: float16 queries [rows][Hq][D], output in chunk order (act_index, out_ld)
void launch_kvq_step_attention(const KvqView& kv, const KvqSeqs& q, int Hq, const void* qrows, void* out, int out_ld, int32_t* status, void* workspace, hipStream_t st);
// Whether the lengths of all units (at most 96 for each step of 128 tokens and 128 rows) can be counted in 32 bits.
inline bool kvq_attention_counts(int B, int Hkv, int G, int max_pages, int q_max) {
  return (int64_t)B * Hkv * (max_pages / 2 + 1) <= ((int64_t)1 << 24) / ((int64_t)q_max * G / 128 + 1);
}
