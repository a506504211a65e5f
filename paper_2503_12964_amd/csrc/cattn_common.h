// Shared by the causal attention kernels with grouped heads (gfx950).
//
// Row space.  The `group` query heads that share a K/V head are treated as rows of one matrix: row r of a
// (sequence, K/V head) is query token r / group, head kv_head * group + r % group.  All of a group's
// products then read a staged K/V tile once, and the sums of dK, dV over the group are sums over rows.  Rows
// stay in token order, so the causal limit is monotone in r: row r sees keys j <= r / group + off, off = keys - queries
// (the last query sees the last key), and key j is seen by the rows r >= (j - off) * group.
#pragma once

#include "vfm_common.h"

namespace vfm {

struct CausalShape {
  int total_q, n_heads, n_kv_heads, group;
  uint32_t q_row, k_row, v_row;      // bytes between consecutive tokens
  float scale, scale_log2;
};

// One (sequence, K/V head) as a workgroup sees it.
struct CausalSeq {
  int qs, ql, ks, kl;   // first query token, queries, first key, keys
  int off;              // row r sees keys <= r / group + off
  int rows;             // ql * group
};
template <class Segs>
__device__ __forceinline__ CausalSeq causal_seq(const Segs& t, int s, int group) {
  CausalSeq c;
  c.qs = t.q_start(s); c.ql = t.q_len(s); c.ks = t.kv_start(s); c.kl = t.kv_len(s);
  c.off = c.kl - c.ql;
  c.rows = c.ql * group;
  return c;
}

// Tiles of the sequences before s: of the rows (query heads of a group times queries) or of the keys.
template <bool KV>
inline TileIndex make_causal_index(const XSegTable& segs, int group, int rows_per_tile) {
  TileIndex ti;
  int tiles = 0;
  for (int s = 0; s <= VFM_MAX_SEQS; ++s) {
    ti.cu[s] = tiles;
    if (s < segs.n)
      tiles += (int)(((KV ? (long long)segs.kl[s] : (long long)segs.ql[s] * group) + rows_per_tile - 1) / rows_per_tile);
  }
  return ti;
}

// locate_tile for a whole wavefront that asks for one tile: every lane looks at the boundaries that it holds, one round of loads
// where the binary search takes a dependent one per step.  cu has `room` + 1 entries, those past n repeating the total or unused.
template <int ROOM>
__device__ __forceinline__ void locate_tile_wave(const int* cu, int n, int tile, int& s, int& t) {
  const int lane = threadIdx.x & 63;
  int below = 0;
#pragma unroll
  for (int x = 0; x < ROOM; x += 64) {
    const int i = x + lane;
    const bool le = i < n && cu[i < n ? i : 0] <= tile;
    below += __builtin_popcountll(__builtin_amdgcn_ballot_w64(le));
  }
  s = __builtin_amdgcn_readfirstlane(below - 1);     // the last sequence that begins at or before it
  t = tile - cu[s];
}

// The lane's number, formed where it is asked for: what is rarely needed takes no register in between.
__device__ __forceinline__ int lane_anew() {
  uint32_t zero = 0;
  asm volatile("" : "+s"(zero));
  return __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, zero));
}

// store_tile_rows for rows that lie anywhere: dst(r) is the address of row r of the wavefront's tile (first column), asked
// only for rows < rows_valid.
template <int D, class Dst>
__device__ __forceinline__ void store_tile_rows_at(char* turn, const f32x16 (&acc)[D / 32], float mul, int rows_valid, Dst dst) {
  constexpr int CPR = D / 8, RB = D * 2;
  const int lane = threadIdx.x & 63, c = lane & 31, g = lane >> 5;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      f32x4 a;
#pragma unroll
      for (int e = 0; e < 4; ++e) a[e] = acc[db][q4 * 4 + e] * mul;
      *reinterpret_cast<bf16x4*>(turn + c * RB + (((db * 4 + q4) ^ (c & (CPR - 1))) << 4) + 8 * g) = to_bf16x4(a);
    }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const int rr = lane / CPR, cx = lane % CPR;
#pragma unroll
  for (int i = 0; i < 32 * CPR / 64; ++i) {
    const int r = i * (64 / CPR) + rr;
    const u32x4 w = *reinterpret_cast<const u32x4*>(turn + r * RB + ((cx ^ (r & (CPR - 1))) << 4));
    if (r < rows_valid) *reinterpret_cast<u32x4*>(dst(r) + cx * 8) = w;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

hipError_t launch_cattn_fwd(const void* q, const void* k, const void* v, const XSegTable& segs, const CausalShape& sh,
                            int head_dim, void* out, float* lse, void* workspace, hipStream_t stream);
size_t cattn_fwd_workspace(const XSegTable& segs, const CausalShape& sh, int head_dim);   // bytes that the run needs
hipError_t launch_cattn_bwd(const void* q, const void* k, const void* v, const void* out, const float* lse,
                            const void* dout, const XSegTable& segs, const CausalShape& sh, int head_dim,
                            void* dq, uint32_t dq_row, void* dk, uint32_t dk_row, void* dv, uint32_t dv_row,
                            float* delta, float* lse2, float* sentinel, float* parts, hipStream_t stream);
size_t cattn_bwd_parts(const XSegTable& segs, const CausalShape& sh, int head_dim);        // bytes of `parts` that the run needs

}  // namespace vfm
