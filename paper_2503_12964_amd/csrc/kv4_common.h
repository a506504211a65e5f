// Shared by the kernels of the 4-bit key/value cache (gfx950).
//
// A row (token, K/V head) of head_dim elements is held as blocks of 32 consecutive elements: E2M1 codes (sign, two
// exponent bits, one mantissa bit: 0, 1/2, 1, 3/2, 2, 3, 4, 6), two to a byte, first element in the low half, and
// one byte b per block for the factor 2^(b - 127).  A power-of-two factor makes every step but the rounding to a code
// exact, and the conversion instructions of this chip take it as an operand: a row goes back to bf16 at one
// instruction per two elements, products and all.  b is 7 .. 252 (every code times the factor is a normal bf16); 255 marks a block that
// held a NaN or an infinity.
#pragma once

#include "vfm_common.h"

namespace vfm {

constexpr int kKv4Block = 32;
constexpr uint32_t kKv4Nan = 255;

// The cache as kernels see it.  Pages of 2^shift tokens: [n_pages][n_kv_heads][page][head_dim / 2] codes and
// [n_pages][n_kv_heads][page][head_dim / 32] factors.
struct Kv4Cache {
  uint8_t *k4, *v4, *ks, *vs;
  const int32_t* pages;      // [n_seqs][max_pages]
  const int32_t* lens;       // [n_seqs], or null (gather)
  int n_pages, max_pages, shift, n_kv_heads;
};

// New tokens of every sequence of a run, in packed order (host array, by value).
struct Kv4Table {
  int n;
  int cu[VFM_MAX_SEQS + 1];
};

__device__ __forceinline__ int kv4_seq_of(const Kv4Table& t, int tok) {   // the last s with cu[s] <= tok
  int lo = 0, hi = t.n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (t.cu[mid] <= tok) lo = mid; else hi = mid;
  }
  return lo;
}

// Page that holds place `pos` of sequence s, or -1: past the table, or an entry that names no page of the cache.
__device__ __forceinline__ int kv4_page(const Kv4Cache& c, int s, long long pos) {
  if (pos < 0 || (pos >> c.shift) >= c.max_pages) return -1;
  const int p = c.pages[(size_t)s * c.max_pages + (size_t)(pos >> c.shift)];
  return p >= 0 && p < c.n_pages ? p : -1;
}
__device__ __forceinline__ size_t kv4_row(const Kv4Cache& c, int page, int kvh, long long pos) {
  return (((size_t)page * c.n_kv_heads + kvh) << c.shift) + (size_t)(pos & ((1 << c.shift) - 1));
}

// 8 codes (one word) as bf16, times the factor
__device__ __forceinline__ bf16x8 kv4_values(uint32_t w, float factor) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, factor, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, factor, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, factor, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, factor, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ float kv4_factor(uint32_t b) { return __builtin_bit_cast(float, b << 23); }

hipError_t launch_kv4_append(const void* k, uint32_t k_row, const void* v, uint32_t v_row, const Kv4Table& t,
                             const Kv4Cache& c, int head_dim, hipStream_t stream);
hipError_t launch_kv4_gather(const Kv4Table& t, const Kv4Cache& c, int head_dim, void* k, void* v, hipStream_t stream);
hipError_t launch_kv4_attn(const void* q, uint32_t q_row, const Kv4Table& t, const Kv4Cache& c, int n_heads, int total,
                           int head_dim, float scale, void* out, float* lse, void* workspace, hipStream_t stream);
size_t kv4_attn_workspace(const int32_t* cu_seqlens, int n_seqs, int n_heads, int n_kv_heads, int head_dim);

}  // namespace vfm
