// dK, dV of causal attention with grouped heads: one workgroup owns 128 keys of one (sequence, K/V head), 32 per wavefront.
// Included by cattn_bwd.hip.
//
// The loop is that of the bidirectional pass (bwd_dkdv_unit in attn_bwd.hip, where its choices are explained with
// their measurements): row blocks of 32 in a software pipeline, S/dP products of block b+1 under the exponentials of block b,
// tiles of 64 rows in a ring of three LDS stages requested two ahead, score products as assembly at head_dim 128 with K and V in
// AGPRs.  What the causal order and the groups add:
//  - A tile's rows are (query, head) pairs (cattn_common.h); a lane steps the addresses of its rows by a tile with one
//    conditional correction, no division.
//  - The walk goes from the sequence's last rows, which see all keys, back to the first row that sees any of the workgroup's keys
//    (a wavefront's to the first that sees any of its own).  So the workgroups of an XCD, whose keys differ, begin at the same rows
//    and stay on them together, in their L2: walked forwards, every key tile begins at its own diagonal and all are apart
//    (8,000 tokens x 16/1 heads, four splits, whole backward: forwards 2,000 us, backwards 1,161).
//  - With K/V heads shared by a group there are few of them, and a call of a few sequences may be fewer workgroups than the chip has
//    room for, the longest taking as long as its rows are many.  RG = 2 or 4: the four wavefronts own 64 or 32 keys, RG of
//    them the same ones; each takes one 32-row block of every tile, and their sums are added in order at the end.  With one block
//    per tile the row operands of a block are read two tiles ahead, so that the ring has a fourth stage.
//  - Where that is not enough (one K/V head for all query heads, long sequences) the walk itself is cut: `splits` workgroups take
//    a share each of a key tile's rows and leave their sums in fp32, as they lie, in the workspace; cattn_dkdv_join_kernel adds
//    them in order.
//  - Scores of pairs that are not seen become -inf before their exponentials, in the blocks that cross the diagonal only.
// Bound by the matrix pipe, whose clock the power limit sets: 12,007 tokens x 32/8 heads x 128 in 2,070 us, 1.14 PFLOP/s of its four
// products over the pairs that are seen.
#pragma once

#include "cattn_careful.h"
#include "cattn_common.h"
#include "cattn_plan.h"

namespace vfm {

constexpr int kCBwdWaves = 4;
constexpr int kSgbValu = 0x002, kSgbMfma = 0x008, kSgbDsRead = 0x100;

template <int D, int RG>
struct CKvCfg {
  static constexpr int kBC = kCBwdBC / RG;                               // keys per workgroup
  static constexpr int kBQ = RG == 4 ? 128 : 64;                         // rows per LDS tile
  static constexpr int kBlocks = kBQ / 32 / RG;                          // row blocks of a tile that a wavefront takes
  static constexpr int kRing = RG == 1 ? 3 : 4;                          // LDS stages
  static constexpr int kAhead = kRing - 1;                               // tiles requested ahead
  static constexpr int kTileBytes = kBQ * D * 2;                         // one Q or dO tile
  static constexpr int kStageBytes = 2 * kTileBytes;
  static constexpr int kStatBytes = 4 * kBQ * 4;                         // lse2, Delta (+ spare) of one stage
  static constexpr int kStatBase = kRing * kStageBytes;
  // K and V rows on their way into registers: over the ring's last stage, which fills after the prologue (RG = 1: V behind the
  // statistics; else wavefronts of the same keys share a copy)
  static constexpr int kOwnK = (kRing - 1) * kStageBytes;
  static constexpr int kOwnV = RG == 1 ? kStatBase + kRing * kStatBytes : kOwnK + kBC * D * 2;
  static constexpr int kLdsBytes = RG == 1 ? kOwnV + kCBwdBC * D * 2 : kStatBase + kRing * kStatBytes;
  static constexpr int kTurn = 4 / RG * 32 * D * 2;                      // results on their way out, then (RG > 1) the others' sums
  static_assert(kBC * D * 2 * (RG == 1 ? 1 : 2) <= kStageBytes && kOwnV % 1024 == 0 && kLdsBytes <= 160 * 1024, "own rows fit a stage; LDS of one CU");
  static_assert(kTurn + (RG - 1) * (4 / RG) * 2 * 32 * D * 4 <= kStatBase, "the others' sums");
  static constexpr int kChunksPerRow = D / 8;
  static constexpr int kLoadsPerWave = kBQ * kChunksPerRow / (kCBwdWaves * 64);
};

// The row that is the first to see key j
__device__ __forceinline__ int first_row_of(const CausalSeq& cs, int group, int j) {
  const long long r = ((long long)j - cs.off) * group;
  return r < 0 ? 0 : r > 0x7fffffffLL ? 0x7fffffff : (int)r;
}
// What a workgroup takes: a sequence's first keys, which most rows see, first.
struct KvWalk {
  CausalSeq cs;
  int kvh, split, j0;     // first key
  int rt0, n_tiles;       // rows: n_tiles tiles from rt0 on
};
template <int D, int RG>
__device__ __forceinline__ KvWalk kv_walk(int block, const XSegTable& segs, const TileIndex& ti, const CausalShape& sh, int splits) {
  constexpr int kBQ = CKvCfg<D, RG>::kBQ;
  KvWalk w;
  w.kvh = block % sh.n_kv_heads;
  int seq, tk;
  locate_tile_wave<VFM_MAX_XSEQS>(ti.cu, segs.n, block / sh.n_kv_heads / splits, seq, tk);
  w.split = block / sh.n_kv_heads % splits;
  w.cs = causal_seq(segs, seq, sh.group);
  w.j0 = tk * CKvCfg<D, RG>::kBC;
  w.rt0 = first_row_of(w.cs, sh.group, w.j0) / kBQ * kBQ;
  w.n_tiles = w.rt0 < w.cs.rows ? (w.cs.rows - w.rt0 + kBQ - 1) / kBQ : 0;
  if (splits > 1) {
    const int t0 = (int)((long long)w.n_tiles * w.split / splits), t1 = (int)((long long)w.n_tiles * (w.split + 1) / splits);
    w.rt0 += t0 * kBQ;
    w.n_tiles = t1 - t0;
  }
  return w;
}

// A wavefront's sums hold a NaN: they are formed again over the rows that see each key, if those that do not may have made one.
template <int D, int RG>
__device__ __forceinline__ void dkdv_checked(f32x16 (&dk)[D / 32], f32x16 (&dv)[D / 32], int wave, const __bf16* q, const __bf16* k,
                                             const __bf16* v, const __bf16* dout, const float* lse2, const float* delta,
                                             const XSegTable& segs, const TileIndex& ti, const CausalShape& sh, int splits) {
  constexpr int RB = D * 2, kBQ = CKvCfg<D, RG>::kBQ;
  const KvWalk w = kv_walk<D, RG>(anew(blockIdx.x), segs, ti, sh, splits);
  const CausalSeq& cs = w.cs;
  const int rg = wave / (kCBwdWaves / RG), jw = w.j0 + wave % (kCBwdWaves / RG) * 32;
  const int row0 = first_row_of(cs, sh.group, jw), r_first = row0 <= w.rt0 ? w.rt0 : row0 / kBQ * kBQ;
  const int r_end = min(w.rt0 + w.n_tiles * kBQ, cs.rows);
  auto at = [&](int r) -> RowAt {
    const int tok = r / sh.group, sub = r - tok * sh.group;
    return {(uint32_t)tok * sh.q_row + (uint32_t)sub * RB, ((uint32_t)tok * sh.n_heads + sub) * RB,
            (size_t)(w.kvh * sh.group + sub) * sh.total_q + cs.qs + tok};
  };
  const int key = min(jw + (lane_anew() & 31), cs.kl - 1);
  dkdv_again<D>(dk, dv, (const char*)k + (size_t)(cs.ks + key) * sh.k_row + (size_t)w.kvh * RB,
                (const char*)v + (size_t)(cs.ks + key) * sh.v_row + (size_t)w.kvh * RB, r_first, r_end,
                w.rt0 + w.n_tiles * kBQ, [&](int block) { return RG == 1 || block % RG == rg; },
                (const char*)q + (size_t)cs.qs * sh.q_row + (size_t)w.kvh * sh.group * RB,
                (const char*)dout + ((size_t)cs.qs * sh.n_heads + (size_t)w.kvh * sh.group) * RB, at, lse2, delta,
                first_row_of(cs, sh.group, key), first_row_of(cs, sh.group, jw + 31), sh.scale_log2);
}

template <int D, int RG>
__global__ __launch_bounds__(kCBwdWaves * 64, D == 64 && RG < 4 ? 2 : 1)
void cattn_dkdv_kernel(const __bf16* __restrict__ q, const __bf16* __restrict__ k, const __bf16* __restrict__ v,
                       const __bf16* __restrict__ dout, const float* __restrict__ lse2, const float* __restrict__ delta,
                       const float* __restrict__ sentinel, __bf16* __restrict__ dk, __bf16* __restrict__ dv,
                       const XSegTable segs, const TileIndex ti, const CausalShape sh, uint32_t dk_row, uint32_t dv_row,
                       int splits, float* __restrict__ parts) {
  using Cfg = CKvCfg<D, RG>;
  constexpr int kBQ = Cfg::kBQ;
  constexpr int KS = D / 16, DB = D / 32;
  constexpr int LPW = Cfg::kLoadsPerWave;
  constexpr int SB = Cfg::kStageBytes;
  constexpr int TB = Cfg::kTileBytes;
  constexpr int RB = D * 2;
  constexpr bool kAsm = D == 128;   // more than 256 registers (see mfma32_v)

  extern __shared__ __attribute__((aligned(16))) char smem[];

  const KvWalk walk = kv_walk<D, RG>(blockIdx.x, segs, ti, sh, splits);
  const int kvh = walk.kvh, split = walk.split, j0 = walk.j0, rt0 = walk.rt0, n_tiles = walk.n_tiles;
  const CausalSeq cs = walk.cs;

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63;
  const int c = lane & 31;
  const int g = lane >> 5;
  const int rg = wave / (kCBwdWaves / RG);             // which of a tile's row blocks it takes (RG > 1)
  const int jw = j0 + wave % (kCBwdWaves / RG) * 32;   // the wavefront's first key
  const int keys_valid = cs.kl - jw;
  auto kv_row0 = [&](__bf16* base, uint32_t row_bytes) {
    return reinterpret_cast<__bf16*>(reinterpret_cast<char*>(base) + (size_t)(cs.ks + jw) * row_bytes) + kvh * D;
  };

  auto first_row = [&](int j) { return first_row_of(cs, sh.group, j); };
  // where this wavefront's sums go if the rows are split: 32 keys of dK, then of dV, as the accumulators lie
  f32x4* part = nullptr;
  if (splits > 1) {
    // blocks of 32 keys, tile by tile (a sequence's last tile may have some past its end)
    const size_t block = (size_t)(blockIdx.x / sh.n_kv_heads / splits) * (Cfg::kBC / 32) + wave % (kCBwdWaves / RG);
    part = reinterpret_cast<f32x4*>(parts) + ((block * sh.n_kv_heads + kvh) * splits + split) * (16 * D);
    if (n_tiles == 0) {
      if (rg == 0 && keys_valid > 0)
        for (int i = lane; i < 16 * D; i += 64) part[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      return;
    }
  }
  if (n_tiles == 0) {      // keys of a sequence without queries
    if (rg == 0 && c < keys_valid) {
      const u32x2 z = {0u, 0u};
#pragma unroll
      for (int x = 0; x < D / 8; ++x) {
        *reinterpret_cast<u32x2*>(kv_row0(dk, dk_row) + (size_t)c * (dk_row / 2) + 4 * g + 8 * x) = z;
        *reinterpret_cast<u32x2*>(kv_row0(dv, dv_row) + (size_t)c * (dv_row / 2) + 4 * g + 8 * x) = z;
      }
    }
    return;
  }
  const int row_min = first_row(jw + c);               // of this lane's key
  const int wave_all = __builtin_amdgcn_readfirstlane(first_row(jw + 31));   // rows from here on see all of the wavefront's keys
  const int rt_last = rt0 + (n_tiles - 1) * kBQ;       // tile t of the walk is rows rt_last - t * kBQ ..
  // tiles of the walk until its rows see none of the wavefront's keys; none for a wavefront without keys
  const int first_tile = first_row(jw) <= rt0 ? 0 : (first_row(jw) - rt0) / kBQ;
  const int wave_tiles = __builtin_amdgcn_readfirstlane(keys_valid <= 0 || first_tile >= n_tiles ? 0 : n_tiles - first_tile);

  // ---- tile requests (direct global->LDS).  Lane L of wave instruction (x, wave) owns LDS chunk (x*waves + wave)*64 + L:
  // row P / chunks_per_row, physical chunk P % chunks_per_row (the swizzle has a period of 16 rows, so the logical chunk
  // does not depend on x).  Offsets count from the sequence's first query and step back by a tile; past the last row
  // they clamp to it, and so do those that the requests ahead of the walk's end bring below row 0 (wrapped, they are large).
  // Waves 0/2 fetch lse2, waves 1/3 Delta: 0 and 1 of a tile's first 64 rows, 2 and 3 of the others (of the same into spare LDS
  // where there are none).
  const uint32_t do_row = (uint32_t)sh.n_heads * RB;
  const int d_tok = kBQ / sh.group, d_sub = kBQ - d_tok * sh.group;
  const uint32_t q_step = (uint32_t)d_tok * sh.q_row + (uint32_t)d_sub * RB, q_wrap = sh.q_row - (uint32_t)sh.group * RB;
  const uint32_t do_step = (uint32_t)d_tok * do_row + (uint32_t)d_sub * RB, do_wrap = do_row - (uint32_t)sh.group * RB;
  const uint32_t q_last = (uint32_t)(cs.ql - 1) * sh.q_row + (uint32_t)(sh.group - 1) * RB;
  const uint32_t do_last = (uint32_t)(cs.ql - 1) * do_row + (uint32_t)(sh.group - 1) * RB;
  const char* qbase = uniform_ptr((const char*)q + (size_t)cs.qs * sh.q_row + (size_t)kvh * sh.group * RB);
  const char* dobase = uniform_ptr((const char*)dout + ((size_t)cs.qs * sh.n_heads + (size_t)kvh * sh.group) * RB);
  static_assert(kCBwdWaves * 64 / Cfg::kChunksPerRow % 16 == 0, "rows of consecutive x: whole periods of the swizzle apart");
  constexpr int kRowsX = kCBwdWaves * 64 / Cfg::kChunksPerRow;     // rows from one x to the next
  const int x_tok = kRowsX / sh.group, x_sub = kRowsX - x_tok * sh.group;
  const uint32_t qx_step = (uint32_t)x_tok * sh.q_row + (uint32_t)x_sub * RB, dox_step = (uint32_t)x_tok * do_row + (uint32_t)x_sub * RB;
  const int own_row = (wave * 64 + lane) / Cfg::kChunksPerRow;
  const uint32_t colb = (uint32_t)(((lane % Cfg::kChunksPerRow) ^ swz<D>(own_row)) * 16);
  int sub;                              // of the lane's row at x = 0
  uint32_t q_off, do_off;
  {
    const int row = rt_last + own_row, tok = row / sh.group;
    sub = row - tok * sh.group;
    q_off = (uint32_t)tok * sh.q_row + (uint32_t)sub * RB;
    do_off = (uint32_t)tok * do_row + (uint32_t)sub * RB;
  }
  const bool is_lse = (wave & 1) == 0;
  const int stat_half = kBQ == 128 ? wave >> 1 : 0;
  const float* stat_src = uniform_ptr(is_lse ? lse2 : delta);
  const uint32_t stat_sentinel = (uint32_t)((const char*)(sentinel + (is_lse ? 0 : 1)) - (const char*)stat_src);
  int stat_row = rt_last + 64 * stat_half + lane, stat_sub = stat_row % sh.group;
  uint32_t stat_off = ((uint32_t)(kvh * sh.group + stat_sub) * sh.total_q + cs.qs + stat_row / sh.group) * 4u;
  const uint32_t stat_step = ((uint32_t)d_sub * sh.total_q + d_tok) * 4u, stat_wrap = 4u - (uint32_t)sh.group * sh.total_q * 4u;
  const uint32_t smem_addr = lds_addr_of(smem);
  const uint32_t wave_lds = __builtin_amdgcn_readfirstlane(smem_addr + wave * 1024);
  const uint32_t stat_lds = __builtin_amdgcn_readfirstlane(
      smem_addr + Cfg::kStatBase + (kBQ == 128 ? (wave & 1) * 128 + stat_half * 64 : wave * 64) * 4);
  auto issue_tile = [&](int stage) {
    uint32_t qo = q_off, dd = do_off;
    int sb = sub;
#pragma unroll
    for (int x = 0; x < LPW; ++x) {
      const uint32_t dst = wave_lds + stage * SB + x * kCBwdWaves * 1024;
      lds_dma16(qbase, min(qo, q_last) + colb, dst);
      lds_dma16(dobase, min(dd, do_last) + colb, dst + TB);
      sb += x_sub;
      const bool wrap = sb >= sh.group;
      qo += qx_step + (wrap ? q_wrap : 0u);
      dd += dox_step + (wrap ? do_wrap : 0u);
      sb -= wrap ? sh.group : 0;
    }
    sub -= d_sub;
    const bool back = sub < 0;
    q_off -= q_step + (back ? q_wrap : 0u);
    do_off -= do_step + (back ? do_wrap : 0u);
    sub += back ? sh.group : 0;
    lds_dma4(stat_src, (uint32_t)stat_row < (uint32_t)cs.rows ? stat_off : stat_sentinel, stat_lds + stage * Cfg::kStatBytes);
    stat_row -= kBQ;
    stat_sub -= d_sub;
    const bool wrap = stat_sub < 0;
    stat_off -= stat_step + (wrap ? stat_wrap : 0u);
    stat_sub += wrap ? sh.group : 0;
  };

  // ---- per-lane LDS addresses within a tile (as in bwd_dkdv_unit): rows as A operand, transposing reads of the same rows
  const int rbase = tile_off<D>(c, 8 * g);
  int tbase[2];
#pragma unroll
  for (int t = 0; t < 2; ++t)
    tbase[t] = tile_off<D>(8 * t + 4 * g + ((lane & 15) >> 2), 16 * ((lane >> 4) & 1) + 4 * (lane & 3));
  constexpr int SETS = Cfg::kRing * SB > 65536 ? 2 : 1;   // set 1: stages 2 and 3, beyond the 64 KB an immediate reaches
  uint32_t rb[SETS][KS], tb[SETS][2][DB];
#pragma unroll
  for (int hs = 0; hs < SETS; ++hs) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      rb[hs][ks] = smem_addr + hs * 2 * SB + (rbase ^ (ks << 5)) + rg * 32 * RB;
      asm volatile("" : "+v"(rb[hs][ks]));
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        tb[hs][t][db] = smem_addr + hs * 2 * SB + (tbase[t] ^ (db << 6)) + rg * 32 * RB;
        asm volatile("" : "+v"(tb[hs][t][db]));
      }
  }

  const f32x16 zero16 = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  f32x16 dkacc[DB], dvacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) { dkacc[db] = zero16; dvacc[db] = zero16; }

  auto read_rows = [&](int stage, int ib, bf16x8 (&qa)[KS], bf16x8 (&da)[KS]) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const uint32_t a = rb[SETS == 2 ? stage >> 1 : 0][ks] + (SETS == 2 ? stage & 1 : stage) * SB + ib * 32 * RB;
      qa[ks] = lds_read_b128_at(a);
      da[ks] = lds_read_b128_at(a + TB);
    }
  };

  // ---- prologue: K, V rows, tiles 0 and 1 requested
  const uint32_t own = smem_addr + wave % (kCBwdWaves / RG) * (32 * RB);   // this wavefront's rows, from kOwnK and kOwnV on
  {
    const char* kbase = uniform_ptr((const char*)k + (size_t)cs.ks * sh.k_row + (size_t)kvh * RB);
    const char* vbase = uniform_ptr((const char*)v + (size_t)cs.ks * sh.v_row + (size_t)kvh * RB);
    const uint32_t own_s = __builtin_amdgcn_readfirstlane(own);
#pragma unroll
    for (int x = 0; x < 32 * RB / 1024; ++x) {
      const int p = x * 64 + lane, r = p / Cfg::kChunksPerRow;
      const uint32_t key = (uint32_t)min(jw + r, cs.kl - 1), col = (uint32_t)(((p % Cfg::kChunksPerRow) ^ swz<D>(r)) * 16);
      lds_dma16(kbase, key * sh.k_row + col, own_s + Cfg::kOwnK + x * 1024);
      lds_dma16(vbase, key * sh.v_row + col, own_s + Cfg::kOwnV + x * 1024);
    }
  }
#pragma unroll
  for (int t = 0; t < Cfg::kAhead; ++t) issue_tile(t);
  wait_vmcnt<0>();
  bf16x8 kreg[KS], vreg[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    kreg[ks] = lds_read_b128_at(own + Cfg::kOwnK + (rbase ^ (ks << 5)));
    vreg[ks] = lds_read_b128_at(own + Cfg::kOwnV + (rbase ^ (ks << 5)));
    if constexpr (kAsm) { to_agpr(kreg[ks]); to_agpr(vreg[ks]); }
    else { settle(kreg[ks]); settle(vreg[ks]); }
  }
  __syncthreads();

  // tiles that the wavefront does not compute: its share of the requests, the waits and barriers
  auto idle_from = [&](int t) {
    for (; t < n_tiles; ++t) {
      wait_vmcnt<0>();
      __syncthreads();
      issue_tile((t + Cfg::kAhead) % Cfg::kRing);
    }
    wait_vmcnt<0>();   // no load may still be writing LDS when the workgroup ends
    __syncthreads();   // the ring is free
  };
  // With no tile of its own a wavefront with keys still writes zeros (sums of a split walk, or none of its keys are seen here)
  if (keys_valid <= 0) {
    idle_from(0);
    if constexpr (RG > 1) __syncthreads();
    return;
  }

  bf16x8 qa_n[KS], da_n[KS];      // row operands of block b+1
  f32x16 s_cur, dp_cur;           // S(b), dP(b)
  {
    bf16x8 q0r[KS], d0r[KS];
    read_rows(0, 0, q0r, d0r);
    if constexpr (Cfg::kBlocks == 2) read_rows(0, 1, qa_n, da_n); else read_rows(1, 0, qa_n, da_n);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if constexpr (kAsm) {
        mfma32_v(s_cur, q0r[ks], kreg[ks], ks == 0);
        mfma32_v(dp_cur, d0r[ks], vreg[ks], ks == 0);
      } else {
        s_cur = mfma32(q0r[ks], kreg[ks], ks == 0 ? zero16 : s_cur);
        dp_cur = mfma32(d0r[ks], vreg[ks], ks == 0 ? zero16 : dp_cur);
      }
    }
    if constexpr (kAsm) wait_mfma_v(s_cur, dp_cur);
  }

  // One pipeline iteration; POS = b % (3 blocks of a tile) fixes every LDS stage at compile time.  row0: first row of block b.
  auto iteration = [&](auto pos_c, int row0) {
    constexpr int POS = decltype(pos_c)::value;
    constexpr int NB = Cfg::kBlocks;
    constexpr int IB = POS % NB;                            // block b within its tile
    constexpr int ST_CUR = (POS / NB) % Cfg::kRing;          // stage of block b's tile
    constexpr int ST_ROW = ((POS + 2) / NB) % Cfg::kRing;    // stage of block b+2's tile
    constexpr int IB_ROW = (POS + 2) % NB;
    if constexpr (IB == 0) {
      // Start of tile t: what was requested has landed for every wave before anyone reads block b+2's rows (tile t+1;
      // one block per tile: t+2), and every wave is past tile t-1, whose stage takes the next.
      wait_vmcnt<0>();
      __syncthreads();
      issue_tile((ST_CUR + Cfg::kAhead) % Cfg::kRing);
    }
    if (row0 < wave_all) {   // (wave-uniform) the block crosses the diagonal: rows that do not see this lane's key
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (row0 + 8 * (e >> 2) + 4 * g + (e & 3) < row_min) s_cur[e] = -INFINITY;
    }
    const float* lse_s = reinterpret_cast<const float*>(smem + Cfg::kStatBase + ST_CUR * Cfg::kStatBytes) + rg * 32;
    const float* delta_s = lse_s + kBQ;

    // ---- phase A: S(b+1), dP(b+1) | P(b) | statistics and transposed-operand reads of block b (one group per product)
    constexpr int NG = 2 * KS;
    f32x4 l4[4], d4[4];
    s16x4 dlo[2][DB], dhi[2][DB], qlo[2][DB], qhi[2][DB];
    f32x16 s_next, dp_next, p;
    u32x8 pw;
#pragma unroll
    for (int gi = 0; gi < NG; ++gi) {
      const int ks = gi >> 1;
      if constexpr (kAsm) {
        if ((gi & 1) == 0) mfma32_v(s_next, qa_n[ks], kreg[ks], ks == 0, s_cur, p, pw);
        else mfma32_v(dp_next, da_n[ks], vreg[ks], ks == 0, s_cur, p, pw);
      } else {
        if ((gi & 1) == 0) s_next = mfma32(qa_n[ks], kreg[ks], ks == 0 ? zero16 : s_next);
        else dp_next = mfma32(da_n[ks], vreg[ks], ks == 0 ? zero16 : dp_next);
      }
      if (gi == 0) {
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) l4[q4] = *reinterpret_cast<const f32x4*>(lse_s + IB * 32 + 8 * q4 + 4 * g);
      }
#pragma unroll
      for (int r = 2 * gi; r < 2 * gi + 2; ++r) {
        const int rr = r % (4 * DB), s2 = rr / (2 * DB), db = (rr >> 1) % DB, hi = rr & 1;
        const uint32_t o = tb[SETS == 2 ? ST_CUR >> 1 : 0][hi][db] + (SETS == 2 ? ST_CUR & 1 : ST_CUR) * SB + (IB * 32 + 16 * s2) * RB;
        if (r < 4 * DB) { if (hi) dhi[s2][db] = lds_read_tr_at(o + TB); else dlo[s2][db] = lds_read_tr_at(o + TB); }
        else { if (hi) qhi[s2][db] = lds_read_tr_at(o); else qlo[s2][db] = lds_read_tr_at(o); }
      }
      if (gi >= NG - 2) {
#pragma unroll
        for (int q4 = 2 * (gi - (NG - 2)); q4 < 2 * (gi - (NG - 2)) + 2; ++q4)
          d4[q4] = *reinterpret_cast<const f32x4*>(delta_s + IB * 32 + 8 * q4 + 4 * g);
      }
      // P for rows 8*(e/4) + 4g + e%4 of the block, column = this lane's key; a pair is converted one group after its
      // exponentials
#pragma unroll
      for (int e = 1; e < 16; e += 2)
        if (e * (NG - 2) / 16 + 3 == gi) {
          const f32x2 pr = {p[e - 1], p[e]};
          pw[e >> 1] = __builtin_bit_cast(uint32_t, __builtin_convertvector(pr, bf16x2));
        }
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (e * (NG - 2) / 16 + 2 == gi) p[e] = fast_exp2(s_cur[e] * sh.scale_log2 - l4[e >> 2][e & 3]);
      __builtin_amdgcn_sched_barrier(0);
    }
    {
      const f32x2 pr = {p[14], p[15]};   // the last pair's group would be NG
      pw[7] = __builtin_bit_cast(uint32_t, __builtin_convertvector(pr, bf16x2));
    }
    bf16x8 pb[2];
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2) {
      const u32x4 w = {pw[4 * s2], pw[4 * s2 + 1], pw[4 * s2 + 2], pw[4 * s2 + 3]};
      pb[s2] = __builtin_bit_cast(bf16x8, w);
    }

    // ---- phase B: dV^T += dO(b)^T P(b) | dS(b) = P(b) o (dP(b) - Delta)
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
      for (int db = 0; db < DB; ++db)
        dvacc[db] = mfma32(join_tr(dlo[s2][db], dhi[s2][db]), pb[s2], dvacc[db]);
    bf16x8 dsb[2];
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2) {
      f32x8 a;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int r = 8 * s2 + e;
        a[e] = p[r] * (dp_cur[r] - d4[r >> 2][r & 3]);
      }
      dsb[s2] = to_bf16x8(a);
    }
#pragma unroll
    for (int i = 0; i < 2 * DB; ++i) {
      __builtin_amdgcn_sched_group_barrier(kSgbMfma, 1, 0);
      __builtin_amdgcn_sched_group_barrier(kSgbValu, 5, 0);
    }
    __builtin_amdgcn_sched_barrier(0);

    // ---- phase C: dK^T += Q(b)^T dS(b) | row operands of block b+2
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
      for (int db = 0; db < DB; ++db)
        dkacc[db] = mfma32(join_tr(qlo[s2][db], qhi[s2][db]), dsb[s2], dkacc[db]);
    bf16x8 qa_2[KS], da_2[KS];
    read_rows(ST_ROW, IB_ROW, qa_2, da_2);
#pragma unroll
    for (int i = 0; i < 2 * DB; ++i) {
      __builtin_amdgcn_sched_group_barrier(kSgbMfma, 1, 0);
      __builtin_amdgcn_sched_group_barrier(kSgbDsRead, (2 * KS + 2 * DB - 1) / (2 * DB), 0);
    }
    __builtin_amdgcn_sched_barrier(0);

    s_cur = s_next;
    dp_cur = dp_next;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) { qa_n[ks] = qa_2[ks]; da_n[ks] = da_2[ks]; }
  };

  for (int t = 0; t < wave_tiles; t += Cfg::kRing) {
    const int row = rt_last - t * kBQ;
    if constexpr (RG == 1) {
      iteration(IntC<0>{}, row);
      iteration(IntC<1>{}, row + 32);
      if (t + 1 < wave_tiles) { iteration(IntC<2>{}, row - 64); iteration(IntC<3>{}, row - 32); }
      if (t + 2 < wave_tiles) { iteration(IntC<4>{}, row - 128); iteration(IntC<5>{}, row - 96); }
    } else {
      iteration(IntC<0>{}, row + rg * 32);
      if (t + 1 < wave_tiles) iteration(IntC<1>{}, row - kBQ + rg * 32);
      if (t + 2 < wave_tiles) iteration(IntC<2>{}, row - 2 * kBQ + rg * 32);
      if (t + 3 < wave_tiles) iteration(IntC<3>{}, row - 3 * kBQ + rg * 32);
    }
  }
  idle_from(wave_tiles);

  if (wave_tiles > 0 && (any_nan(dkacc) || any_nan(dvacc)))   // (rare)
    dkdv_checked<D, RG>(dkacc, dvacc, wave, q, k, v, dout, lse2, delta, segs, ti, shape_anew(sh), splits);

  // ---- epilogue: dK (scaled) and dV of this wavefront's keys; each wavefront turns its tiles through a piece of the ring
  if constexpr (RG > 1) {
    const int ln = lane_anew(), kb = wave % (kCBwdWaves / RG);
    auto sums = [&](int r) { return reinterpret_cast<f32x4*>(smem + Cfg::kTurn) + (size_t)((r - 1) * (kCBwdWaves / RG) + kb) * (2 * 8 * D); };
    if (rg > 0) {
      f32x4* to = sums(rg);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          to[(db * 4 + q4) * 64 + ln] = f32x4{dkacc[db][4 * q4], dkacc[db][4 * q4 + 1], dkacc[db][4 * q4 + 2], dkacc[db][4 * q4 + 3]};
          to[((DB + db) * 4 + q4) * 64 + ln] = f32x4{dvacc[db][4 * q4], dvacc[db][4 * q4 + 1], dvacc[db][4 * q4 + 2], dvacc[db][4 * q4 + 3]};
        }
    }
    __syncthreads();
    if (rg > 0) return;
#pragma unroll
    for (int r = 1; r < RG; ++r) {
      const f32x4* from = sums(r);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const f32x4 a = from[(db * 4 + q4) * 64 + ln], b = from[((DB + db) * 4 + q4) * 64 + ln];
#pragma unroll
          for (int e = 0; e < 4; ++e) { dkacc[db][4 * q4 + e] += a[e]; dvacc[db][4 * q4 + e] += b[e]; }
        }
    }
  }
  if (splits > 1) {
    const int ln = lane_anew();
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        part[(db * 4 + q4) * 64 + ln] = f32x4{dkacc[db][4 * q4], dkacc[db][4 * q4 + 1], dkacc[db][4 * q4 + 2], dkacc[db][4 * q4 + 3]};
        part[((DB + db) * 4 + q4) * 64 + ln] = f32x4{dvacc[db][4 * q4], dvacc[db][4 * q4 + 1], dvacc[db][4 * q4 + 2], dvacc[db][4 * q4 + 3]};
      }
    return;
  }
  char* turn = smem + wave * (32 * RB);
  store_tile_rows<D>(turn, dkacc, sh.scale, kv_row0(dk, dk_row), dk_row / 2, keys_valid);
  store_tile_rows<D>(turn, dvacc, 1.0f, kv_row0(dv, dv_row), dv_row / 2, keys_valid);
}

// Adds the shares of 32 keys in order; wavefront 0 dK, wavefront 1 dV.  blockIdx.x: (32-key block as above, K/V head).
template <int D>
__global__ __launch_bounds__(128)
void cattn_dkdv_join_kernel(__bf16* __restrict__ dk, __bf16* __restrict__ dv, const XSegTable segs, const TileIndex ti,
                            const CausalShape sh, uint32_t dk_row, uint32_t dv_row, int keys_per_tile, int splits,
                            const float* __restrict__ parts) {
  constexpr int DB = D / 32;
  __shared__ __attribute__((aligned(16))) char smem[2 * 32 * D * 2];
  const int kvh = blockIdx.x % sh.n_kv_heads, block = blockIdx.x / sh.n_kv_heads, per = keys_per_tile / 32;
  int seq, tk;
  locate_tile_wave<VFM_MAX_XSEQS>(ti.cu, segs.n, block / per, seq, tk);
  const CausalSeq cs = causal_seq(segs, seq, sh.group);
  const int j0 = tk * keys_per_tile + block % per * 32, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (j0 >= cs.kl) return;
  const f32x4* part = reinterpret_cast<const f32x4*>(parts) + ((size_t)block * sh.n_kv_heads + kvh) * splits * (16 * D) + wave * (8 * D);
  f32x16 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = f32x16{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < splits; ++s, part += 16 * D)
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const f32x4 a = part[(db * 4 + q4) * 64 + lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[db][4 * q4 + e] += a[e];
      }
  const uint32_t row = wave == 0 ? dk_row : dv_row;
  __bf16* to = reinterpret_cast<__bf16*>(reinterpret_cast<char*>(wave == 0 ? dk : dv) + (size_t)(cs.ks + j0) * row) + kvh * D;
  store_tile_rows<D>(smem + wave * (32 * D * 2), acc, wave == 0 ? sh.scale : 1.0f, to, row / 2, cs.kl - j0);
}

}  // namespace vfm
