// Keys and rows that hold a NaN or an infinity, for those that do not see them.  Included by the causal attention kernels.
//
// A pair (row, key) that is not seen has weight 0 in the second products, but 0 times a NaN or an infinity is a NaN.  The only
// such pairs that are multiplied at all lie in the units that cross the diagonal, or next to it in a wavefront's tile, and among the
// copies of the last row or key that fill a last tile.  Where it comes from is not asked: besides the operands themselves it may be a
// product of finite ones that overflows (dP or Delta).  To look at the pairs would cost the loops; so every wavefront looks at its
// sums once, at the end.  Where they hold a NaN it forms them again: pair by pair from memory, with
// plain multiplications, over the pairs that are seen, until every NaN has been met again.  That is slow, some microseconds per key
// or row (12,007 tokens x 32/8 heads x 128 with one query of NaNs in the middle: the backward 674 ms, 3.8 without), and lasts only where
// NaNs did come from what is not seen (with all values NaN in one column: 8.1 ms).
// The look itself (an addition per sum) and the code beside the loops cost a call about 1 % (8,000 tokens x 16/1 heads x 128, backward:
// 860 us without, 868 with).
#pragma once

#include "cattn_common.h"

namespace vfm {

// A wave-uniform value that the compiler takes for a new one: what is rarely needed is worked out from it where it is needed, and
// nothing of that is kept in registers through the loops.
__device__ __forceinline__ int anew(int x) {
  x = __builtin_amdgcn_readfirstlane(x);
  asm volatile("" : "+s"(x));
  return x;
}
__device__ __forceinline__ CausalShape shape_anew(const CausalShape& sh) {
  CausalShape s = sh;
  s.group = anew(s.group);
  s.n_kv_heads = anew(s.n_kv_heads);
  return s;
}

template <int N>
__device__ __forceinline__ bool any_nan(const f32x16 (&a)[N]) {   // in any lane (sums that overflow count too)
  float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e & 3] += a[i][e];
  const float t = (s[0] + s[1]) + (s[2] + s[3]);
  return __builtin_amdgcn_ballot_w64(t != t) != 0;
}
// How many of this lane's sums are NaN.  Sums formed again hold none where the first ones do not: as many are the same ones, and then
// the first ones stand, whatever is still to be added.
__device__ __forceinline__ int count_nans(const f32x16& a) {
  int n = 0;
#pragma unroll
  for (int e = 0; e < 16; ++e) n += a[e] != a[e] ? 1 : 0;
  return n;
}
__device__ __forceinline__ bool as_many_nans(const f32x16& again, int nans) { return __builtin_amdgcn_ballot_w64(count_nans(again) < nans) == 0; }
// This lane's half (elements 16 ks + 8 g + e) of the product of two rows, summed with the other half's
template <int D>
__device__ __forceinline__ float row_dot(const char* a, const char* b) {
  float s = 0.f;
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) {
    const bf16x8 x = *reinterpret_cast<const bf16x8*>(a + ks * 32), y = *reinterpret_cast<const bf16x8*>(b + ks * 32);
#pragma unroll
    for (int e = 0; e < 8; ++e) s = __builtin_fmaf((float)x[e], (float)y[e], s);
  }
  return pair_sum(s);
}
// acc += w * row, 32 columns as the accumulators lie (elements 8 q + 4 g + e; row: this lane's first, 4 g)
__device__ __forceinline__ void add_row(f32x16& acc, float w, const char* row) {
#pragma unroll
  for (int q4 = 0; q4 < 4; ++q4) {
    const bf16x4 x = *reinterpret_cast<const bf16x4*>(row + q4 * 16);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[4 * q4 + e] = __builtin_fmaf(w, (float)x[e], acc[4 * q4 + e]);
  }
}

// The sums are formed again 32 columns at a time: a second set of all of them would not fit beside the first.

// out's sums of 32 rows over keys [j0, j1).  q_row: this lane's; k, v: the sequence's first; lim: last key that the row sees; m: the
// reference that the sum of its exponentials has.
template <int D>
__device__ __forceinline__ void fwd_again(f32x16 (&acc)[D / 32], const char* q_row, const char* k, uint32_t k_row, const char* v,
                                          uint32_t v_row, int j0, int j1, int lim, float m, float scale_log2) {
  const int g = lane_anew() >> 5;
#pragma unroll
  for (int db = 0; db < D / 32; ++db) {
    const int nans = count_nans(acc[db]);
    f32x16 sum = {};
    int j = j0;
#pragma unroll 1
    for (; j < j1; ++j) {
      if ((j & 31) == 0 && as_many_nans(sum, nans)) break;
      const float s = row_dot<D>(q_row + 16 * g, k + (size_t)j * k_row + 16 * g);
      if (j <= lim) add_row(sum, fast_exp2(s * scale_log2 - m), v + (size_t)j * v_row + 64 * db + 8 * g);
    }
    if (j >= j1) acc[db] = sum;
  }
}

// dq's sums of 32 rows over the 32-key blocks b0, b0 + step .. below key j1.
template <int D>
__device__ __forceinline__ void dq_again(f32x16 (&acc)[D / 32], const char* q_row, const char* do_row, const char* k, uint32_t k_row,
                                         const char* v, uint32_t v_row, int b0, int step, int j1, int lim, float lse2, float delta,
                                         float scale_log2) {
  const int g = lane_anew() >> 5;
#pragma unroll
  for (int db = 0; db < D / 32; ++db) {
    const int nans = count_nans(acc[db]);
    f32x16 sum = {};
    int j = 32 * b0;
#pragma unroll 1
    for (; j < j1; j += (j & 31) == 31 ? 32 * step - 31 : 1) {
      if ((j & 31) == 0 && as_many_nans(sum, nans)) break;
      const char* kj = k + (size_t)j * k_row;
      const float s = row_dot<D>(q_row + 16 * g, kj + 16 * g), dp = row_dot<D>(do_row + 16 * g, v + (size_t)j * v_row + 16 * g);
      if (j <= lim) add_row(sum, fast_exp2(s * scale_log2 - lse2) * (dp - delta), kj + 64 * db + 8 * g);
    }
    if (j >= j1) acc[db] = sum;
  }
}

// dk's and dv's sums of 32 keys over the rows of the 32-row blocks that take(block) takes, from r1 - 1 back to r0.  k_row, v_row: this
// lane's key; q_at(r), do_at(r), stat_at(r): addresses of row r and index of its statistics; row_min: the first row that sees the key.
template <int D, class Take, class QAt, class DoAt, class StatAt>
__device__ __forceinline__ void dkdv_again(f32x16 (&dk)[D / 32], f32x16 (&dv)[D / 32], const char* k_row, const char* v_row, int r0, int r1,
                                           Take take, QAt q_at, DoAt do_at, StatAt stat_at, const float* lse2, const float* delta,
                                           int row_min, float scale_log2) {
  const int g = lane_anew() >> 5;
#pragma unroll
  for (int db = 0; db < D / 32; ++db) {
    const int k_nans = count_nans(dk[db]), v_nans = count_nans(dv[db]);
    f32x16 sk = {}, sv = {};
    int r = r1 - 1;
#pragma unroll 1
    for (; r >= r0; --r) {
      if (!take(r >> 5)) { r &= ~31; continue; }
      if ((r & 31) == 31 && as_many_nans(sk, k_nans) && as_many_nans(sv, v_nans)) break;
      const char *qr = q_at(r), *dr = do_at(r);
      const size_t at = stat_at(r);
      const float s = row_dot<D>(qr + 16 * g, k_row + 16 * g), dp = row_dot<D>(dr + 16 * g, v_row + 16 * g);
      if (r >= row_min) {
        const float p = fast_exp2(s * scale_log2 - lse2[at]);
        add_row(sk, p * (dp - delta[at]), qr + 64 * db + 8 * g);
        add_row(sv, p, dr + 64 * db + 8 * g);
      }
    }
    if (r < r0) { dk[db] = sk; dv[db] = sv; }
  }
}

}  // namespace vfm
