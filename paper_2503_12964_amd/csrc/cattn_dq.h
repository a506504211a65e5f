// dQ of causal attention with grouped heads at head_dim 128: one workgroup owns 256 rows of one (sequence, K/V head), 64 per
// wavefront.  Included by cattn_bwd.hip.
//
// The loop is that of the bidirectional pass (bwd_dq2_unit in attn_bwd.hip, where its choices are explained with
// their measurements): two 32-row blocks per wavefront, so that every operand read from LDS feeds two products, the blocks
// alternating in half-steps, Q, dO and the dQ^T accumulators in AGPRs, all products written as assembly, K/V tiles of 64 keys in
// a ring of three LDS stages.  What the causal order and the groups add:
//  - Rows are (query, head) pairs (cattn_common.h).  The walk ends with the last key that the tile's last row sees, a
//    wavefront's with its own last row's.
//  - Scores of pairs that are not seen (which takes in the keys past the sequence's end) become -inf before their
//    exponentials, in the blocks that cross the diagonal only.
//  - The pass runs before dK/dV and leaves Delta and lse in log2 units for it.  Delta_i = dO_i . O_i comes from the rows on
//    their way into registers.  For a row that sees at most 32 keys |O| is as large as |V| and dS cancels, so that the
//    rounding of `out` would show in dq, dk (see bwd_short_delta_kernel in attn_bwd.hip); in causal order every sequence begins with
//    such rows.  Their Delta is formed as sum_j P_ij dP_ij from the scores of the first 32 keys.
// Bound by the matrix pipe: 12,007 tokens x 32/8 heads x 128 in 1,390 us, 1.28 PFLOP/s of its three products over the pairs that are seen.
#pragma once

#include "cattn_careful.h"
#include "cattn_common.h"

namespace vfm {

constexpr int kCDqWaves = 4;
constexpr int kCDqRing = 3;
constexpr int kCDqBC = 64;      // keys per LDS tile
constexpr int kCFewKeys = 32;   // rows that see at most so many keys have their Delta formed from P and dP
constexpr float kCLog2eB = 1.4426950408889634f;

// Delta of this lane's row from its products with the first 32 keys (accumulator layout: lane's row, keys 8*(e/4) + 4g + e%4).
__device__ __forceinline__ float few_delta(const f32x16& s, const f32x16& dp, float scale_log2, float lse2, int lim) {
  const int g = (threadIdx.x >> 5) & 1;
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e)
    if (8 * (e >> 2) + 4 * g + (e & 3) <= lim) sum += fast_exp2(s[e] * scale_log2 - lse2) * dp[e];
  return pair_sum(sum);
}

// The sums of a wavefront's 32 rows over the 32-key blocks b0, b0 + step .. below key j1 hold a NaN: they are formed again over the
// keys that each row sees, if those that it does not see may have made one.
template <int D>
__device__ __forceinline__ void dq_checked(f32x16 (&acc)[D / 32], const __bf16* q, const __bf16* k, const __bf16* v, const __bf16* dout,
                                           const CausalSeq& cs, const CausalShape& sh, int kvh, int row_w, int b0, int step, int j1,
                                           float lse2, float delta) {
  constexpr int RB = D * 2;
  const char* kbase = (const char*)k + (size_t)cs.ks * sh.k_row + (size_t)kvh * RB;
  const char* vbase = (const char*)v + (size_t)cs.ks * sh.v_row + (size_t)kvh * RB;
  const int row = min(row_w + (lane_anew() & 31), cs.rows - 1), tok = row / sh.group, head = kvh * sh.group + row - tok * sh.group;
  dq_again<D>(acc, (const char*)q + (size_t)(cs.qs + tok) * sh.q_row + (size_t)head * RB,
              (const char*)(dout + ((size_t)(cs.qs + tok) * sh.n_heads + head) * D), kbase, sh.k_row, vbase, sh.v_row, b0, step,
              (min(row_w + 32, cs.rows) - 1) / sh.group + cs.off + 1, j1, cs.kl - 1, tok + cs.off,
              min(row_w, cs.rows - 1) / sh.group + cs.off, lse2, delta, sh.scale_log2);
}

template <int D>
struct CDq2Cfg {
  static constexpr int kBR = kCDqWaves * 64;                 // rows per workgroup
  static constexpr int kTileBytes = kCDqBC * D * 2;          // one K or V tile
  static constexpr int kStageBytes = 2 * kTileBytes;         // K tile, V tile
  // a wavefront's 64 rows of Q and of dO on their way into registers: behind the ring's first stage
  static constexpr int kOwnBase = kStageBytes;
  static constexpr int kOwnBytes = 2 * 64 * D * 2;
  static constexpr int kLdsBytes = kOwnBase + kCDqWaves * kOwnBytes;
  static_assert(kLdsBytes >= kCDqRing * kStageBytes && kLdsBytes <= 160 * 1024, "ring, LDS of one CU");
  static constexpr int kChunksPerRow = D / 8;
  static constexpr int kChunksPerThread = kCDqBC * kChunksPerRow / (kCDqWaves * 64);
};

template <int D>
__global__ __launch_bounds__(kCDqWaves * 64, 1)
void cattn_dq2_kernel(const __bf16* __restrict__ q, const __bf16* __restrict__ k, const __bf16* __restrict__ v,
                      const __bf16* __restrict__ dout, const __bf16* __restrict__ out, const float* __restrict__ lse,
                      float* __restrict__ lse2g, float* __restrict__ delta, float* __restrict__ sentinel,
                      __bf16* __restrict__ dq, const XSegTable segs, const TileIndex ti, const CausalShape sh, uint32_t dq_row) {
  using Cfg = CDq2Cfg<D>;
  constexpr int KS = D / 16, DB = D / 32;
  constexpr int CPT = Cfg::kChunksPerThread;
  constexpr int RB = D * 2;
  constexpr int TB = Cfg::kTileBytes;
  constexpr int SB = Cfg::kStageBytes;
  constexpr int NG = 2 * KS + 2 * DB;   // MFMAs (groups) per half-step
  static_assert(D == 128, "tuned for head_dim 128");

  extern __shared__ __attribute__((aligned(16))) char smem[];

  const int kvh = blockIdx.x % sh.n_kv_heads;
  int seq, tq;
  locate_tile(ti, segs.n, blockIdx.x / sh.n_kv_heads, seq, tq);
  const CausalSeq cs = causal_seq(segs, seq, sh.group);
  tq = (cs.rows + Cfg::kBR - 1) / Cfg::kBR - 1 - tq;           // a sequence's last rows, which see most, first
  const int r0 = tq * Cfg::kBR;

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63;
  const int c = lane & 31;
  const int g = lane >> 5;
  const int row_w = r0 + wave * 64;
  if (blockIdx.x == 0 && tid == 0) {   // statistics of rows past a sequence's end, for the dK/dV pass
    sentinel[0] = INFINITY;
    sentinel[1] = 0.f;
  }
  auto row_tok = [&](int r) { return r / sh.group; };
  auto head_row = [&](int r) {          // (token, head) row of q's, out's and dout's packed order
    const int tok = row_tok(r);
    return (size_t)(cs.qs + tok) * sh.n_heads + (size_t)kvh * sh.group + (r - tok * sh.group);
  };
  auto dq_at = [&](int r) {
    const int tok = row_tok(r);
    return reinterpret_cast<__bf16*>(reinterpret_cast<char*>(dq) + (size_t)(cs.qs + tok) * dq_row) +
           (size_t)(kvh * sh.group + (r - tok * sh.group)) * D;
  };
  int lim[2], wave_min[2];              // last key that this lane's rows see, and the blocks' first rows
  size_t stat[2];
#pragma unroll
  for (int ib = 0; ib < 2; ++ib) {
    const int r = min(row_w + ib * 32 + c, cs.rows - 1), tok = row_tok(r);
    lim[ib] = tok + cs.off;
    stat[ib] = (size_t)(kvh * sh.group + (r - tok * sh.group)) * sh.total_q + cs.qs + tok;
    wave_min[ib] = __builtin_amdgcn_readfirstlane(row_tok(min(row_w + ib * 32, cs.rows - 1)) + cs.off);
  }

  const int n_keys = row_tok(min(r0 + Cfg::kBR, cs.rows) - 1) + cs.off + 1;
  const int n_tiles = n_keys > 0 ? (n_keys + kCDqBC - 1) / kCDqBC : 0;
  if (n_tiles == 0) {                   // rows that see no key
    const u32x4 z = {0u, 0u, 0u, 0u};
    for (int i = lane; i < 64 * Cfg::kChunksPerRow; i += 64) {
      const int r = row_w + i / Cfg::kChunksPerRow;
      if (r < cs.rows) *reinterpret_cast<u32x4*>(dq_at(r) + (i % Cfg::kChunksPerRow) * 8) = z;
    }
#pragma unroll
    for (int ib = 0; ib < 2; ++ib)
      if (g == 0 && row_w + ib * 32 + c < cs.rows) { lse2g[stat[ib]] = INFINITY; delta[stat[ib]] = 0.f; }
    return;
  }
  // tiles up to the last key of the wavefront's last row
  const int wave_last = row_tok(min(row_w + 64, cs.rows) - 1) + cs.off;
  const int wave_tiles = __builtin_amdgcn_readfirstlane(row_w >= cs.rows ? 0 : wave_last < 0 ? 1 : wave_last / kCDqBC + 1);

  // ---- K/V staging with direct global->LDS loads; tiles are requested in sequence.  (The swizzle has a period of 16 rows, so
  // a lane's logical chunk is the same in all of its rows.)
  const char* kbase = uniform_ptr((const char*)k + (size_t)cs.ks * sh.k_row + (size_t)kvh * RB);
  const char* vbase = uniform_ptr((const char*)v + (size_t)cs.ks * sh.v_row + (size_t)kvh * RB);
  static_assert(kCDqWaves * 64 / Cfg::kChunksPerRow % 16 == 0, "rows of consecutive x: whole periods of the swizzle apart");
  const int own_row = (wave * 64 + lane) / Cfg::kChunksPerRow;
  const uint32_t colb = (uint32_t)(((lane % Cfg::kChunksPerRow) ^ swz<D>(own_row)) * 16);
  const uint32_t k_off = own_row * sh.k_row + colb, v_off = own_row * sh.v_row + colb;
  const uint32_t smem_addr = lds_addr_of(smem);
  const uint32_t wave_lds = __builtin_amdgcn_readfirstlane(smem_addr + wave * 1024);
  int next_tile = 0;                    // (wave-uniform; asked for past the last one, the last one again)
  auto issue_tile = [&](int stage) {
    const int key0 = __builtin_amdgcn_readfirstlane(min(next_tile, (cs.kl - 1) / kCDqBC)) * kCDqBC;
    ++next_tile;
    const char* kt = kbase + (size_t)key0 * sh.k_row;
    const char* vt = vbase + (size_t)key0 * sh.v_row;
    constexpr int kStep = kCDqWaves * 64 / Cfg::kChunksPerRow;
    if (key0 + kCDqBC <= cs.kl) {
#pragma unroll
      for (int x = 0; x < CPT; ++x) {
        const uint32_t dst = wave_lds + stage * SB + x * kCDqWaves * 1024;
        lds_dma16(kt + (size_t)(x * kStep) * sh.k_row, k_off, dst);
        lds_dma16(vt + (size_t)(x * kStep) * sh.v_row, v_off, dst + TB);
      }
    } else {                            // keys past the last one: copies of it (no row sees them)
      const int row = (wave * 64 + lane_anew()) / Cfg::kChunksPerRow;   // (not kept in registers for this)
      const uint32_t col = (uint32_t)(((lane_anew() % Cfg::kChunksPerRow) ^ swz<D>(row)) * 16);
#pragma unroll
      for (int x = 0; x < CPT; ++x) {
        const uint32_t dst = wave_lds + stage * SB + x * kCDqWaves * 1024;
        const uint32_t r = min(x * kStep + row, cs.kl - 1 - key0);
        lds_dma16(kt, r * sh.k_row + col, dst);
        lds_dma16(vt, r * sh.v_row + col, dst + TB);
      }
    }
  };
  // tiles that the wavefront does not compute: per tile from the second on the wait, the barrier, the request
  auto idle_from = [&](int t) {
    for (; t < n_tiles; ++t) {
      wait_vmcnt<0>();
      __syncthreads();
      if (t + 1 < n_tiles) issue_tile((t + 1) % kCDqRing);
    }
  };

  if (wave_tiles == 0) {                // a wavefront past the last row
    issue_tile(0);
    wait_vmcnt<0>();
    __syncthreads();
    issue_tile(1);
    idle_from(1);
    wait_vmcnt<0>();
    __syncthreads();
    return;
  }

  // ---- swizzled LDS addresses, one register each (a second set for the third stage, beyond an immediate's 64 KB)
  uint32_t rb[KS], tb[2][DB], rb2[KS], tb2[2][DB];
  {
    const int rbase = tile_off<D>(c, 8 * g);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      rb[ks] = smem_addr + (rbase ^ (ks << 5));
      rb2[ks] = rb[ks] + 2 * SB;
      asm volatile("" : "+v"(rb[ks]), "+v"(rb2[ks]));
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int tbase = tile_off<D>(8 * t + 4 * g + ((lane & 15) >> 2), 16 * ((lane >> 4) & 1) + 4 * (lane & 3));
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        tb[t][db] = smem_addr + (tbase ^ (db << 6));
        tb2[t][db] = tb[t][db] + 2 * SB;
        asm volatile("" : "+v"(tb[t][db]), "+v"(tb2[t][db]));
      }
    }
  }

  const f32x16 zero16 = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  f32x16 dqacc[2][DB];
#pragma unroll
  for (int ib = 0; ib < 2; ++ib)
#pragma unroll
    for (int db = 0; db < DB; ++db) dqacc[ib][db] = zero16;

  // ---- this wavefront's Q and dO rows as B operands (AGPRs), through LDS in whole rows; Delta from dO and out
  const uint32_t own = smem_addr + Cfg::kOwnBase + wave * Cfg::kOwnBytes;   // Q rows, then dO rows
  {
    const char* qbase = uniform_ptr((const char*)q + (size_t)cs.qs * sh.q_row + (size_t)kvh * sh.group * RB);
    const char* dobase = uniform_ptr((const char*)dout + ((size_t)cs.qs * sh.n_heads + (size_t)kvh * sh.group) * RB);
    const uint32_t own_s = __builtin_amdgcn_readfirstlane(own);
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      const int r = x * 4 + (lane >> 4), row = min(row_w + r, cs.rows - 1), tok = row_tok(row);
      const uint32_t col = (uint32_t)(row - tok * sh.group) * RB + (uint32_t)(((lane & 15) ^ swz<D>(r)) * 16);
      lds_dma16(qbase, (uint32_t)tok * sh.q_row + col, own_s + x * 1024);
      lds_dma16(dobase, (uint32_t)tok * (uint32_t)(sh.n_heads * RB) + col, own_s + 64 * RB + x * 1024);
    }
  }
  issue_tile(0);
  bf16x8 qreg[2][KS], doreg[2][KS];
  float lse2[2], dlt[2];
  {
    bf16x8 orow[16];
#pragma unroll
    for (int x = 0; x < 16; ++x)
      orow[x] = *reinterpret_cast<const bf16x8*>(out + head_row(min(row_w + x * 4 + (lane >> 4), cs.rows - 1)) * D + (lane & 15) * 8);
#pragma unroll
    for (int ib = 0; ib < 2; ++ib) {
      const float l = lse[stat[ib]];
      lse2[ib] = l == -INFINITY ? INFINITY : l * kCLog2eB;     // (a row without keys: P = 0)
    }
    wait_vmcnt<0>();
    float s[16];
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      const bf16x8 d = lds_read_b128_at(own + 64 * RB + tile_off<D>(x * 4 + (lane >> 4), (lane & 15) * 8));
      s[x] = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) s[x] = __builtin_fmaf((float)orow[x][e], (float)d[e], s[x]);
      s[x] = row16_sum(s[x]);
    }
#pragma unroll
    for (int ib = 0; ib < 2; ++ib)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const uint32_t a = own + (tile_off<D>(c, 8 * g) ^ (ks << 5)) + ib * 32 * RB;
        qreg[ib][ks] = lds_read_b128_at(a);
        doreg[ib][ks] = lds_read_b128_at(a + 64 * RB);
        to_agpr(qreg[ib][ks]);
        to_agpr(doreg[ib][ks]);
      }
    asm volatile("" ::: "memory");   // (the sums take the place of rows read above)
    if ((lane & 15) == 0)
#pragma unroll
      for (int x = 0; x < 16; ++x)
        *reinterpret_cast<__attribute__((address_space(3))) float*>(own + (x * 4 + (lane >> 4)) * 4) = s[x];
#pragma unroll
    for (int ib = 0; ib < 2; ++ib)
      dlt[ib] = *reinterpret_cast<const __attribute__((address_space(3))) float*>(own + (ib * 32 + c) * 4);
  }
#pragma unroll
  for (int ib = 0; ib < 2; ++ib) asm volatile("" :: "v"(lse2[ib]), "v"(dlt[ib]));
  __syncthreads();            // tile 0 has landed, everyone has its rows
  issue_tile(1);              // (re-requests the last rows when there is a single tile)

  // ---- state carried between half-steps
  f32x16 sacc[2], dpacc[2];   // S^T, dP^T of the current key block, per row block
  f32x16 dsf;                 // dS^T of the half-step at hand, fp32
  u32x8 pw[2];                // dS^T as bf16 pairs, per row block: B operands of the update
  bf16x8 ka[KS], va[KS];      // row operands of the key block whose scores come next
  s16x4 klo[2][DB], khi[2][DB];   // K^T operands of the key block whose update comes next
#pragma unroll
  for (int i = 0; i < 8; ++i) { pw[0][i] = 0u; pw[1][i] = 0u; }
#pragma unroll
  for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
    for (int db = 0; db < DB; ++db) { klo[s2][db] = s16x4{0, 0, 0, 0}; khi[s2][db] = s16x4{0, 0, 0, 0}; }
  dsf = zero16;

  // prologue: row operands of key block 0, S^T and dP^T of (key block 0, row block 0); where rows see few keys, row block 1's too
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    ka[ks] = lds_read_b128_at(rb[ks]);
    va[ks] = lds_read_b128_at(rb[ks] + TB);
  }
  sacc[1] = zero16;
  dpacc[1] = zero16;
  if (wave_min[0] < kCFewKeys) {
#pragma unroll
    for (int ib = 0; ib < 2; ++ib) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        mfma32_v(sacc[0], ka[ks], qreg[ib][ks], ks == 0);
        mfma32_v(dpacc[0], va[ks], doreg[ib][ks], ks == 0);
      }
      wait_mfma_v(sacc[0], dpacc[0]);
      if (lim[ib] < kCFewKeys) dlt[ib] = few_delta(sacc[0], dpacc[0], sh.scale_log2, lse2[ib], lim[ib]);
    }
  }
#pragma unroll
  for (int ib = 0; ib < 2; ++ib)
    if (g == 0 && row_w + ib * 32 + c < cs.rows) {
      lse2g[stat[ib]] = lse2[ib];
      delta[stat[ib]] = dlt[ib];
    }
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    mfma32_v(sacc[0], ka[ks], qreg[0][ks], ks == 0);
    mfma32_v(dpacc[0], va[ks], doreg[0][ks], ks == 0);
  }
  wait_mfma_v(sacc[0], dpacc[0]);

  int lim_g[2];               // lim against the first of the keys that this lane holds of a block
#pragma unroll
  for (int ib = 0; ib < 2; ++ib) lim_g[ib] = lim[ib] - 4 * g;

  // One half-step.  POSB = b % 6 fixes every LDS stage at compile time; IB is the row block
  // whose dS^T the VALU forms.
  auto half_step = [&](auto posb_c, auto ib_c, int b) {
    constexpr int POSB = decltype(posb_c)::value;
    constexpr int IB = decltype(ib_c)::value;
    constexpr int OB = 1 - IB;                               // the block the matrix pipe works for
    constexpr int ST_CUR = (POSB / 2) % kCDqRing;            // stage of key block b
    constexpr int ST_NEXT = ((POSB + 1) / 2) % kCDqRing;     // stage of key block b+1
    constexpr int JB_CUR = POSB & 1, JB_NEXT = (POSB + 1) & 1;
    if (b * 32 + 31 > wave_min[IB]) {   // (wave-uniform) the block crosses the diagonal: keys that this lane's row does not see
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (b * 32 + 8 * (e >> 2) + (e & 3) > lim_g[IB]) sacc[IB][e] = -INFINITY;
    }
    const float lse_i = lse2[IB];
    // Delta is made a new value here: the subtractions dP - Delta then cannot be moved up into the previous
    // half-step, where the MFMAs that produce dP are still running
    float dlt_i = dlt[IB];
    asm volatile("" : "+v"(dlt_i));
#pragma unroll
    for (int gi = 0; gi < NG; ++gi) {
      // ---- matrix pipe
      if (gi < 2 * KS) {
        const int ks = gi >> 1;
        if ((gi & 1) == 0) mfma32_v(sacc[OB], ka[ks], qreg[OB][ks], ks == 0, sacc[IB], dsf, pw[IB]);
        else mfma32_v(dpacc[OB], va[ks], doreg[OB][ks], ks == 0, sacc[IB], dsf, pw[IB]);
      } else {
        const int s2 = (gi - 2 * KS) / DB, db = (gi - 2 * KS) % DB;
        const u32x4 w = {pw[OB][4 * s2], pw[OB][4 * s2 + 1], pw[OB][4 * s2 + 2], pw[OB][4 * s2 + 3]};
        mfma32_acc(dqacc[OB][db], join_tr(klo[s2][db], khi[s2][db]), __builtin_bit_cast(bf16x8, w),
                   sacc[IB], dsf, pw[IB]);
      }
      // ---- LDS reads
      if (IB == 0) {
        // row operands of key block b+1, once the score MFMAs have consumed those of block b
        if (gi >= 2 * KS) {
          constexpr int per = (2 * KS) / (2 * DB);   // reads per group: 16 / 8
#pragma unroll
          for (int x = (gi - 2 * KS) * per; x < (gi - 2 * KS + 1) * per; ++x) {
            const int ks = x >> 1;
            const uint32_t a = (ST_NEXT == 2 ? rb2[ks] : rb[ks] + ST_NEXT * SB) + JB_NEXT * 32 * RB;
            if ((x & 1) == 0) ka[ks] = lds_read_b128_at(a); else va[ks] = lds_read_b128_at(a + TB);
          }
        }
      } else {
        // K^T operands of key block b (the updates of block b-1 were all issued a half-step ago)
        if (gi < 2 * DB) {
#pragma unroll
          for (int x = 2 * gi; x < 2 * gi + 2; ++x) {
            const int s2 = x / (2 * DB), db = (x >> 1) % DB, hi = x & 1;
            const uint32_t a = (ST_CUR == 2 ? tb2[hi][db] : tb[hi][db] + ST_CUR * SB) + (JB_CUR * 32 + 16 * s2) * RB;
            if (hi) khi[s2][db] = lds_read_tr_at(a); else klo[s2][db] = lds_read_tr_at(a);
          }
        }
      }
      // ---- VALU: one element of dS^T per group: the exponential in group G(e), the product one group later, the
      // conversion of a pair one group after that
#pragma unroll
      for (int e = 1; e < 16; e += 2)
        if (1 + e * (NG - 2) / 16 + 2 == gi) {
          const f32x2 pr = {dsf[e - 1], dsf[e]};
          pw[IB][e >> 1] = __builtin_bit_cast(uint32_t, __builtin_convertvector(pr, bf16x2));
        }
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (1 + e * (NG - 2) / 16 + 1 == gi) dsf[e] = dsf[e] * (dpacc[IB][e] - dlt_i);
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (1 + e * (NG - 2) / 16 == gi) dsf[e] = fast_exp2(sacc[IB][e] * sh.scale_log2 - lse_i);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto block = [&](auto posb_c, int b) {
    constexpr int POSB = decltype(posb_c)::value;
    if constexpr ((POSB & 1) == 1) {
      // key block 2t-1: tile t has landed for every wave, every wave is done with tile t-2,
      // whose stage takes tile t+1
      const int t = (b + 1) >> 1;
      if (t < n_tiles) {
        wait_vmcnt<0>();
        __syncthreads();
        if (t + 1 < n_tiles) issue_tile(((POSB + 1) / 2 + 1) % kCDqRing);
      }
    }
    half_step(posb_c, IntC<0>{}, b);
    half_step(posb_c, IntC<1>{}, b);
  };
  const int n_blocks = 2 * wave_tiles;
  for (int b = 0; b < n_blocks; b += 6) {
    block(IntC<0>{}, b);
    block(IntC<1>{}, b + 1);
    if (b + 2 < n_blocks) { block(IntC<2>{}, b + 2); block(IntC<3>{}, b + 3); }
    if (b + 4 < n_blocks) { block(IntC<4>{}, b + 4); block(IntC<5>{}, b + 5); }
  }
  // drain: the last key block's update for row block 1
#pragma unroll
  for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      const u32x4 w = {pw[1][4 * s2], pw[1][4 * s2 + 1], pw[1][4 * s2 + 2], pw[1][4 * s2 + 3]};
      mfma32_acc(dqacc[1][db], join_tr(klo[s2][db], khi[s2][db]), __builtin_bit_cast(bf16x8, w));
    }
  idle_from(wave_tiles + 1);
  wait_vmcnt<0>();   // no load may still be writing LDS when the workgroup ends
  // the accumulators were written by assembly: wait out the last MFMA before they are read
#pragma unroll
  for (int ib = 0; ib < 2; ++ib) wait_mfma_a(dqacc[ib][0], dqacc[ib][1], dqacc[ib][2], dqacc[ib][3]);

  auto checked = [&](auto ib_c) {       // (rare)
    constexpr int ib = decltype(ib_c)::value;
    if (any_nan(dqacc[ib]))
      dq_checked<D>(dqacc[ib], q, k, v, dout, cs, shape_anew(sh), kvh, row_w + ib * 32, 0, 1, wave_tiles * kCDqBC, lse2[ib], dlt[ib]);
  };
  checked(IntC<0>{});
  checked(IntC<1>{});

  // ---- epilogue: dq = bf16(scale * dQ^T), whole rows per store
  __syncthreads();   // the ring is free: each wavefront turns its tiles through a piece of it
#pragma unroll
  for (int ib = 0; ib < 2; ++ib) {
    const int row0 = row_w + ib * 32;
    store_tile_rows_at<D>(smem + wave * (32 * D * 2), dqacc[ib], sh.scale, cs.rows - row0, [&](int r) { return dq_at(row0 + r); });
  }
}

}  // namespace vfm
