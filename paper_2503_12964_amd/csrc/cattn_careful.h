// Keys and rows that hold a NaN or an infinity, for those that do not see them.  Included by the causal attention kernels.
//
// A pair (row, key) that is not seen has weight 0 in the second products, but 0 times a NaN or an infinity is a NaN.  The only
// such pairs that are multiplied at all lie in the units that cross the diagonal, or next to it in a wavefront's tile, and among the
// copies of the last row or key that fill a last tile.  Where it comes from is not asked: besides the operands themselves it may be a
// product of finite ones that overflows (dP or Delta).  To look at the pairs would cost the loops; so every wavefront looks at its
// sums once, at the end.  Where they hold a NaN it goes through the blocks of its walk that have pairs which are not seen, and if one
// of those can have made a NaN, it forms its sums again over the pairs that are seen, block by block with operands straight
// from memory, and pair by pair only for the rows of those blocks that hold something that is not finite.
// A block takes about 2 us, ten times the loop's; all wavefronts together are bound by their loads.  12,007 tokens x 32/8 heads x 128,
// forward and backward in ms, 1.1 and 3.8 without: one query of NaN in the middle 1.1, 6.7; one key whose value holds a NaN 1.5, 28; a
// column of NaN in all values 6.8, 30; a column of infinities in dout 1.1, 33.
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
// Which of 32 rows hold anything that is not finite (a bit each); row: this lane's (lane & 31), the half that its lane >> 5 looks at.
template <int D>
__device__ __forceinline__ uint32_t rows_not_finite(const char* row) {
  bool bad = false;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(row + 16 * i);
#pragma unroll
    for (int x = 0; x < 4; ++x) bad |= (w[x] & 0x7f80u) == 0x7f80u || (w[x] & 0x7f800000u) == 0x7f800000u;
  }
  const uint64_t m = __builtin_amdgcn_ballot_w64(bad);
  return (uint32_t)m | (uint32_t)(m >> 32);
}
// Products of 32 rows with 32 columns; a, b: this lane's row of either, from its half's first 8 elements (16 g bytes) on.  Element e
// of the result: row block_row(e, g), column lane & 31.
__device__ __forceinline__ int block_row(int e, int g) { return 8 * (e >> 2) + 4 * g + (e & 3); }
template <int D>
__device__ __forceinline__ f32x16 block_dot(const char* a, const char* b) {
  f32x16 s = {};
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks)
    s = mfma32(*reinterpret_cast<const bf16x8*>(a + ks * 32), *reinterpret_cast<const bf16x8*>(b + ks * 32), s);
  return s;
}
// acc += X^T w for the 32 rows X of a block, w as block_dot leaves it; base + at: this lane's row (lane & 31).  Rows of `skip` count as
// zeros (and have weights 0).
template <int D>
__device__ __forceinline__ void add_block(f32x16 (&acc)[D / 32], const f32x16& w, const char* base, uint32_t at, uint32_t skip) {
  const int lane = lane_anew(), c = lane & 31, g = lane >> 5;
#pragma unroll
  for (int s2 = 0; s2 < 2; ++s2) {
    f32x8 x;
    uint32_t from[8];
    bool none[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int r = block_row(8 * s2 + e, g);
      x[e] = w[8 * s2 + e];
      from[e] = (uint32_t)__shfl((int)at, r) + 2 * c;
      none[e] = (skip >> r) & 1;
    }
    const bf16x8 b = to_bf16x8(x);
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
      bf16x8 a;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const __bf16 y = *reinterpret_cast<const __bf16*>(base + from[e] + 64 * db);
        a[e] = none[e] ? (__bf16)0.f : y;
      }
      acc[db] = mfma32(a, b, acc[db]);
    }
    __builtin_amdgcn_sched_barrier(0);    // (all of a block's elements on their way at once take registers from the kernel)
  }
}
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
// acc += w * row, as the accumulators lie (elements 32 db + 8 q + 4 g + e; row: this lane's first, 4 g)
template <int D>
__device__ __forceinline__ void add_row(f32x16 (&acc)[D / 32], float w, const char* row) {
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      const bf16x4 x = *reinterpret_cast<const bf16x4*>(row + 64 * db + 16 * q4);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[db][4 * q4 + e] = __builtin_fmaf(w, (float)x[e], acc[db][4 * q4 + e]);
    }
}

template <int D>
__device__ __forceinline__ void clear(f32x16 (&acc)[D / 32]) {
#pragma unroll
  for (int db = 0; db < D / 32; ++db) acc[db] = f32x16{};
}
__device__ __forceinline__ bool finite(float x) { return __builtin_fabsf(x) < INFINITY; }

// The three below look at the 32-key (or 32-row) blocks of a wavefront's walk in which some pair is not seen.  If none of those pairs
// can have made a NaN the sums stand.  Otherwise they are formed again, block by block: where all see all of a block, it is weighed as
// in the loops; elsewhere the weights of pairs that are not seen are set to 0 after all else, and the block's rows that hold
// something that is not finite are left out of the products and added one by one, to those who see them.

// out's sums of 32 rows over the keys [j0, end), j0 a multiple of 32; the loop went on to key `walked`, past the last key with copies of
// it.  q_row: this lane's; k, v: the sequence's first; lim: last key that the row sees; all_see: last key that every row sees; m: the
// reference that the sum of its exponentials has.
template <int D>
__device__ __forceinline__ void fwd_again(f32x16 (&acc)[D / 32], const char* q_row, const char* k, uint32_t k_row, const char* v,
                                          uint32_t v_row, int j0, int end, int walked, int lim, int all_see, float m, float scale_log2) {
  const int lane = lane_anew(), c = lane & 31, g = lane >> 5;
  bool met = false;
#pragma unroll 1
  for (int j = j0; j < walked; j += 32)
    if (j + 31 > all_see) met |= rows_not_finite<D>(v + (uint32_t)min(j + c, end - 1) * v_row + g * D) != 0;
  if (!met) return;
  clear<D>(acc);
#pragma unroll 1
  for (int j = j0; j < end; j += 32) {
    const uint32_t key = (uint32_t)min(j + c, end - 1), v_at = key * v_row;
    f32x16 w = block_dot<D>(k + key * k_row + 16 * g, q_row + 16 * g);
    const bool all = j + 31 <= all_see;      // (wave-uniform)
    const uint32_t bad = all ? 0 : rows_not_finite<D>(v + v_at + g * D);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      w[e] = fast_exp2(w[e] * scale_log2 - m);
      const int r = block_row(e, g);
      if (!all && (j + r > lim || ((bad >> r) & 1))) w[e] = 0.f;
    }
    add_block<D>(acc, w, v, v_at, bad);
#pragma unroll 1
    for (uint32_t left = bad; left; left &= left - 1) {
      const int x = j + __builtin_ctz(left);
      if (x >= end) break;                   // (copies of the last key)
      const float s = row_dot<D>(q_row + 16 * g, k + (uint32_t)x * k_row + 16 * g);
      if (x <= lim) add_row<D>(acc, fast_exp2(s * scale_log2 - m), v + (uint32_t)x * v_row + 8 * g);
    }
  }
}

// dq's sums of 32 rows over the 32-key blocks b0, b0 + step .. below key `end`, the loop's below `walked`; last_key: the sequence's.
template <int D>
__device__ __forceinline__ void dq_again(f32x16 (&acc)[D / 32], const char* q_row, const char* do_row, const char* k, uint32_t k_row,
                                         const char* v, uint32_t v_row, int b0, int step, int end, int walked, int last_key, int lim,
                                         int all_see, float lse2, float delta, float scale_log2) {
  const int lane = lane_anew(), c = lane & 31, g = lane >> 5;
  bool met = false;
#pragma unroll 1
  for (int j = 32 * b0; j < walked; j += 32 * step) {
    if (j + 31 <= all_see) continue;
    const uint32_t key = (uint32_t)min(j + c, last_key);
    const f32x16 dp = block_dot<D>(v + key * v_row + 16 * g, do_row + 16 * g);
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 16; ++e) bad |= j + block_row(e, g) > lim && !finite(dp[e] - delta);
    met |= rows_not_finite<D>(k + key * k_row + g * D) != 0 || __builtin_amdgcn_ballot_w64(bad) != 0;
  }
  if (!met) return;
  clear<D>(acc);
#pragma unroll 1
  for (int j = 32 * b0; j < end; j += 32 * step) {
    const uint32_t key = (uint32_t)min(j + c, last_key), k_at = key * k_row;
    f32x16 w = block_dot<D>(k + k_at + 16 * g, q_row + 16 * g);
    const f32x16 dp = block_dot<D>(v + key * v_row + 16 * g, do_row + 16 * g);
    const bool all = j + 31 <= all_see;
    const uint32_t bad = all ? 0 : rows_not_finite<D>(k + k_at + g * D);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      w[e] = fast_exp2(w[e] * scale_log2 - lse2) * (dp[e] - delta);
      const int r = block_row(e, g);
      if (!all && (j + r > lim || ((bad >> r) & 1))) w[e] = 0.f;
    }
    add_block<D>(acc, w, k, k_at, bad);
#pragma unroll 1
    for (uint32_t left = bad; left; left &= left - 1) {
      const int x = j + __builtin_ctz(left);
      if (x >= end) break;                   // (past all limits)
      const char* kx = k + (uint32_t)x * k_row;
      const float s = row_dot<D>(q_row + 16 * g, kx + 16 * g), d = row_dot<D>(do_row + 16 * g, v + (uint32_t)x * v_row + 16 * g);
      if (x <= lim) add_row<D>(acc, fast_exp2(s * scale_log2 - lse2) * (d - delta), kx + 8 * g);
    }
  }
}

// Where row r of a (sequence, K/V head) lies: bytes from its first row in q and in dout, index of its statistics.
struct RowAt { uint32_t q, dout; size_t stat; };

// dk's and dv's sums of 32 keys over the rows [r0, end) in the 32-row blocks that take(block) takes, r0 a multiple of 32; the loop began at
// row `walked`, past the last row with copies of it.  k_row, v_row: this lane's key; at(r): where row r lies; row_min: the first
// row that sees the key; all_see: the first that sees every key.
template <int D, class Take, class At>
__device__ __forceinline__ void dkdv_again(f32x16 (&dk)[D / 32], f32x16 (&dv)[D / 32], const char* k_row, const char* v_row, int r0, int end,
                                           int walked, Take take, const char* q, const char* dout, At at, const float* lse2,
                                           const float* delta, int row_min, int all_see, float scale_log2) {
  const int lane = lane_anew(), c = lane & 31, g = lane >> 5;
  bool met = false;
#pragma unroll 1
  for (int r = r0; r < walked; r += 32) {
    if (!take(r >> 5) || (r >= all_see && r + 32 <= end)) continue;
    const RowAt own = at(min(r + c, end - 1));
    const f32x16 dp = block_dot<D>(dout + own.dout + 16 * g, v_row + 16 * g);
    const float l = lse2[own.stat], d = delta[own.stat];
    bool bad = l != l || !finite(d);
#pragma unroll
    for (int e = 0; e < 16; ++e) bad |= (r + block_row(e, g) < row_min || r + block_row(e, g) >= end) && !finite(dp[e]);
    met |= (rows_not_finite<D>(q + own.q + g * D) | rows_not_finite<D>(dout + own.dout + g * D)) != 0 || __builtin_amdgcn_ballot_w64(bad) != 0;
  }
  if (!met) return;
  clear<D>(dk);
  clear<D>(dv);
#pragma unroll 1
  for (int r = r0; r < end; r += 32) {
    if (!take(r >> 5)) continue;
    const RowAt own = at(min(r + c, end - 1));
    f32x16 p = block_dot<D>(q + own.q + 16 * g, k_row + 16 * g), ds = block_dot<D>(dout + own.dout + 16 * g, v_row + 16 * g);
    const float l = lse2[own.stat], d = delta[own.stat];
    const bool all = r >= all_see && r + 32 <= end;
    const uint32_t bad = all ? 0 : rows_not_finite<D>(q + own.q + g * D) | rows_not_finite<D>(dout + own.dout + g * D);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int x = block_row(e, g);
      p[e] = fast_exp2(p[e] * scale_log2 - __shfl(l, x));
      ds[e] = p[e] * (ds[e] - __shfl(d, x));
      if (!all && (r + x < row_min || r + x >= end || ((bad >> x) & 1))) p[e] = ds[e] = 0.f;
    }
    add_block<D>(dv, p, dout, own.dout, bad);
    add_block<D>(dk, ds, q, own.q, bad);
#pragma unroll 1
    for (uint32_t left = bad; left; left &= left - 1) {
      const int x = r + __builtin_ctz(left);
      if (x >= end) break;                   // (copies of the last row)
      const RowAt w = at(x);
      const float s = row_dot<D>(q + w.q + 16 * g, k_row + 16 * g), dp = row_dot<D>(dout + w.dout + 16 * g, v_row + 16 * g);
      if (x >= row_min) {
        const float pe = fast_exp2(s * scale_log2 - lse2[w.stat]);
        add_row<D>(dk, pe * (dp - delta[w.stat]), q + w.q + 8 * g);
        add_row<D>(dv, pe, dout + w.dout + 8 * g);
      }
    }
  }
}

}  // namespace vfm
