// Causal packed attention backward with grouped heads for gfx950 (bf16 MFMA, fp32 accumulate).
//
//     P_ij = exp(S_ij - lse_i) where j <= i + off, else 0;   Delta_i = sum_d dO_id O_id
//     dV_j = sum_i P_ij dO_i;   dS_ij = P_ij (dO_i . v_j - Delta_i);   dQ_i = scale sum_j dS_ij K_j;   dK_j = scale sum_i dS_ij Q_i
//
// The sums of dK, dV run over all rows of the K/V head: queries times the heads of its group (cattn_common.h).  Two launches, no
// atomics, every output written once:
//   dq   : a workgroup owns a tile of rows and walks the keys that its last row sees; it forms Delta and lse in log2 units
//          (+inf for a row that sees no key, so that its P is 0) on the way and leaves them for the second.
//   dkdv : a workgroup owns 128 keys and walks the rows that see any of them.
// S and dP are formed in both (7 products instead of 5): sums of dQ over key tiles would need device-wide atomics, which are
// executed at the memory side on this chip.
// P and dS are rounded to bf16 as operands of the second products (half a step, 2^-9 relative at most; in 32 bits they would take
// the vector pipe's rate): dq, dk, dv are off by 0.0024 in the RMS, of which their own rounding is 0.0017.
#include "cattn_careful.h"
#include "cattn_common.h"
#include "cattn_dkdv.h"
#include "cattn_dq.h"
#include "cattn_plan.h"

namespace vfm {

// ---------------------------------------------------------------- dQ, 32 rows per wavefront
// At head_dim 64 three workgroups of four wavefronts share a CU: with the exponentials weighing twice as much against the products
// as at head_dim 128, wavefronts of other workgroups fill the gaps.  KG = 2 or 4, at either head_dim: KG of the
// wavefronts own the same 32 rows and take a 32-key block each of every tile; their sums are added in order at the end.
// For calls of few sequences, where the longest row tile outlasts an even share of the work (as RG in cattn_dkdv.h).  Delta and
// the statistics as in cattn_dq2_kernel.
template <int D, int KG>
struct CDqCfg {
  static constexpr int kBR = 128 / KG;                        // rows per workgroup
  static constexpr int kBC = KG == 4 ? 128 : 64;              // keys per LDS tile
  static constexpr int kBlocks = kBC / 32 / KG;               // key blocks of a tile that a wavefront takes
  static constexpr int kTileBytes = kBC * D * 2;              // K or V rows of one tile
  static constexpr int kStageBytes = 2 * kTileBytes;
  static constexpr int kRing = kStageBytes <= 32 * 1024 ? 3 : 2;
  static constexpr int kLdsBytes = kRing * kStageBytes;
  static constexpr int kTurn = 4 / KG * 32 * D * 2;           // results on their way out, then (KG > 1) the others' sums
  static_assert(kTurn + (KG - 1) * (4 / KG) * 32 * D * 4 <= kLdsBytes, "the others' sums");
  static constexpr int kChunksPerRow = D / 8;
  static constexpr int kLoadsPerWave = kBC * kChunksPerRow / 256;
  static constexpr int kWaves = D == 64 ? (KG == 4 ? 1 : 3) : 1;   // per SIMD
};

template <int D, int KG>
__global__ __launch_bounds__(256, (CDqCfg<D, KG>::kWaves))
void cattn_dq_kernel(const __bf16* __restrict__ q, const __bf16* __restrict__ k, const __bf16* __restrict__ v,
                     const __bf16* __restrict__ dout, const __bf16* __restrict__ out, const float* __restrict__ lse,
                     float* __restrict__ lse2g, float* __restrict__ delta, float* __restrict__ sentinel,
                     __bf16* __restrict__ dq, const XSegTable segs, const TileIndex ti, const CausalShape sh, uint32_t dq_row) {
  using Cfg = CDqCfg<D, KG>;
  constexpr int KS = D / 16, DB = D / 32, RB = D * 2;
  constexpr int LPW = Cfg::kLoadsPerWave;
  extern __shared__ __attribute__((aligned(16))) char smem[];

  const int kvh = blockIdx.x % sh.n_kv_heads;
  int seq, tq;
  locate_tile_wave<VFM_MAX_XSEQS>(ti.cu, segs.n, blockIdx.x / sh.n_kv_heads, seq, tq);
  const CausalSeq cs = causal_seq(segs, seq, sh.group);
  tq = (cs.rows + Cfg::kBR - 1) / Cfg::kBR - 1 - tq;           // a sequence's last rows, which see most, first
  const int r0 = tq * Cfg::kBR;

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63;
  const int c = lane & 31;
  const int g = lane >> 5;
  if (blockIdx.x == 0 && tid == 0) {   // statistics of rows past a sequence's end, for the dK/dV pass
    sentinel[0] = INFINITY;
    sentinel[1] = 0.f;
  }
  const int kg = wave / (4 / KG), rw = wave % (4 / KG);         // which of a tile's key blocks it takes; which rows
  const int row_w = r0 + rw * 32;
  const int rows_valid = cs.rows - row_w;
  const int row = min(row_w + c, cs.rows - 1), tok = row / sh.group, head = kvh * sh.group + row - tok * sh.group;
  const int lim = tok + cs.off;
  const int wave_min = __builtin_amdgcn_readfirstlane(min(row_w, cs.rows - 1) / sh.group + cs.off);
  const int n_keys = (min(r0 + Cfg::kBR, cs.rows) - 1) / sh.group + cs.off + 1;
  const int n_tiles = n_keys > 0 ? (n_keys + Cfg::kBC - 1) / Cfg::kBC : 0;

  const size_t stat = (size_t)head * sh.total_q + cs.qs + tok;
  const bool keeps = kg == 0 && g == 0 && row_w + c < cs.rows;             // this lane leaves its row's statistics
  if (n_tiles == 0 && keeps) { lse2g[stat] = INFINITY; delta[stat] = 0.f; }

  const f32x16 zero16 = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  f32x16 dqacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) dqacc[db] = zero16;

  if (n_tiles > 0) {
    bf16x8 qreg[KS], doreg[KS];
    const size_t qtok = cs.qs + tok;
    const char* qp = (const char*)q + qtok * sh.q_row + (size_t)head * RB + 16 * g;
    const __bf16* dp_ = dout + (qtok * sh.n_heads + head) * D + 8 * g;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) { qreg[ks] = *(const bf16x8*)(qp + ks * 32); doreg[ks] = *(const bf16x8*)(dp_ + ks * 16); }
    const __bf16* op = out + (qtok * sh.n_heads + head) * D + 8 * g;
    float dlt = 0.f, lse2 = lse[stat];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const bf16x8 o = *(const bf16x8*)(op + ks * 16);
#pragma unroll
      for (int e = 0; e < 8; ++e) dlt = __builtin_fmaf((float)o[e], (float)doreg[ks][e], dlt);
    }
    dlt = pair_sum(dlt);
    lse2 = lse2 == -INFINITY ? INFINITY : lse2 * kCLog2eB;     // (a row without keys: P = 0)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) { settle(qreg[ks]); settle(doreg[ks]); }
    asm volatile("" :: "v"(lse2), "v"(dlt));

    const char* kbase = uniform_ptr((const char*)k + (size_t)cs.ks * sh.k_row + (size_t)kvh * RB);
    const char* vbase = uniform_ptr((const char*)v + (size_t)cs.ks * sh.v_row + (size_t)kvh * RB);
    const uint32_t smem_addr = __builtin_amdgcn_readfirstlane(lds_addr_of(smem));
    auto issue_tile = [&](int stage, int t) {
      const uint32_t dst = smem_addr + stage * Cfg::kStageBytes + wave * 1024;
#pragma unroll
      for (int x = 0; x < LPW; ++x) {
        const int p = (x * 4 + wave) * 64 + lane;
        const int r = p / Cfg::kChunksPerRow;
        const uint32_t col = (uint32_t)(((p % Cfg::kChunksPerRow) ^ swz<D>(r)) * 16);
        const uint32_t key = (uint32_t)min(t * Cfg::kBC + r, cs.kl - 1);
        lds_dma16(kbase, key * sh.k_row + col, dst + x * 4096);
        lds_dma16(vbase, key * sh.v_row + col, dst + Cfg::kTileBytes + x * 4096);
      }
    };
    const int rbase = tile_off<D>(c, 8 * g);
    int tbase[2];
#pragma unroll
    for (int t = 0; t < 2; ++t)
      tbase[t] = tile_off<D>(8 * t + 4 * g + ((lane & 15) >> 2), 16 * ((lane >> 4) & 1) + 4 * (lane & 3));

    issue_tile(0, 0);
    if (Cfg::kRing == 3) issue_tile(1, 1);
    int stage = 0;
    for (int t = 0; t < n_tiles; ++t) {
      // tile t is there for everyone (with three stages the next one may be on its way; the statistics' stores are waited
      // out once), and everyone is done with tile t - 1, whose stage takes the next
      if (Cfg::kRing == 3 && t > 1) wait_vmcnt<2 * LPW>(); else wait_vmcnt<0>();
      __syncthreads();
      issue_tile(stage == 0 ? Cfg::kRing - 1 : stage - 1, t + Cfg::kRing - 1);
      if (t == 0) {
        if (wave_min < kCFewKeys) {     // (wave-uniform)
          f32x16 s, dp;
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            s = mfma32(lds_read_b128(smem, rbase ^ (ks << 5)), qreg[ks], ks == 0 ? zero16 : s);
            dp = mfma32(lds_read_b128(smem + Cfg::kTileBytes, rbase ^ (ks << 5)), doreg[ks], ks == 0 ? zero16 : dp);
          }
          if (lim < kCFewKeys) dlt = few_delta(s, dp, sh.scale_log2, lse2, lim);
        }
        if (keeps) { lse2g[stat] = lse2; delta[stat] = dlt; }
      }
      const char* kt = smem + stage * Cfg::kStageBytes;
      const char* vt = kt + Cfg::kTileBytes;
      stage = stage + 1 == Cfg::kRing ? 0 : stage + 1;
#pragma unroll
      for (int x = 0; x < Cfg::kBlocks; ++x) {
        const int jb = KG == 1 ? x : kg;
        const int j0 = t * Cfg::kBC + jb * 32;
        f32x16 s, dp, ds;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const int off = (rbase ^ (ks << 5)) + jb * 32 * RB;
          s = mfma32(lds_read_b128(kt, off), qreg[ks], ks == 0 ? zero16 : s);
          dp = mfma32(lds_read_b128(vt, off), doreg[ks], ks == 0 ? zero16 : dp);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) ds[e] = fast_exp2(s[e] * sh.scale_log2 - lse2) * (dp[e] - dlt);
        if (j0 + 31 > wave_min) {
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (j0 + 8 * (e >> 2) + 4 * g + (e & 3) > lim) ds[e] = 0.f;
        }
        bf16x8 dsb[2];
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) {
          f32x8 a;
#pragma unroll
          for (int e = 0; e < 8; ++e) a[e] = ds[8 * s2 + e];
          dsb[s2] = to_bf16x8(a);
        }
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
          for (int db = 0; db < DB; ++db) {
            const bf16x8 kta = join_tr(lds_read_tr(kt, (tbase[0] ^ (db << 6)) + (jb * 32 + 16 * s2) * RB),
                                       lds_read_tr(kt, (tbase[1] ^ (db << 6)) + (jb * 32 + 16 * s2) * RB));
            dqacc[db] = mfma32(kta, dsb[s2], dqacc[db]);
          }
      }
    }
    wait_vmcnt<0>();
    __syncthreads();
    if (any_nan(dqacc))       // (rare)
      dq_checked<D>(dqacc, q, k, v, dout, cs, shape_anew(sh), kvh, row_w, kg, KG, n_tiles * Cfg::kBC, lse2, dlt);
  }
  if constexpr (KG > 1) {
    auto sums = [&](int x) { return reinterpret_cast<f32x4*>(smem + Cfg::kTurn) + (size_t)((x - 1) * (4 / KG) + rw) * (8 * D); };
    if (kg > 0) {
      f32x4* to = sums(kg);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4)
          to[(db * 4 + q4) * 64 + lane] = f32x4{dqacc[db][4 * q4], dqacc[db][4 * q4 + 1], dqacc[db][4 * q4 + 2], dqacc[db][4 * q4 + 3]};
    }
    __syncthreads();
    if (kg > 0) return;
#pragma unroll
    for (int x = 1; x < KG; ++x) {
      const f32x4* from = sums(x);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const f32x4 a = from[(db * 4 + q4) * 64 + lane];
#pragma unroll
          for (int e = 0; e < 4; ++e) dqacc[db][4 * q4 + e] += a[e];
        }
    }
  }
  store_tile_rows_at<D>(smem + rw * (32 * RB), dqacc, sh.scale, rows_valid, [&](int r) {
    const int at = row_w + r, tk = at / sh.group;
    return reinterpret_cast<__bf16*>(reinterpret_cast<char*>(dq) + (size_t)(cs.qs + tk) * dq_row) +
           (kvh * sh.group + at - tk * sh.group) * D;
  });
}

// ---------------------------------------------------------------- launch
size_t cattn_bwd_parts(const XSegTable& segs, const CausalShape& sh, int head_dim) {
  const KeysPlan plan = keys_plan(segs, sh, head_dim, compute_unit_count());
  if (plan.splits == 1) return 0;
  const int per = kCBwdBC / plan.rg;
  size_t blocks = 0;
  for (int s = 0; s < segs.n; ++s) blocks += (size_t)((segs.kl[s] + per - 1) / per) * (per / 32);
  return blocks * sh.n_kv_heads * plan.splits * 64 * head_dim * sizeof(float);
}

template <int D>
static hipError_t launch_bwd_dim(const __bf16* q, const __bf16* k, const __bf16* v, const __bf16* out, const float* lse,
                                 const __bf16* dout, const XSegTable& segs, const CausalShape& sh, __bf16* dq,
                                 uint32_t dq_row, __bf16* dk, uint32_t dk_row, __bf16* dv, uint32_t dv_row, float* delta,
                                 float* lse2, float* sentinel, float* parts, hipStream_t stream) {
  auto rows_pass = [&](auto kern, int rows, int lds) -> hipError_t {
    const TileIndex tq = make_causal_index<false>(segs, sh.group, rows);
    const int n = count_tiles(tq);
    if (n == 0) return hipSuccess;
    hipError_t e = allow_lds(kern, lds);
    if (e != hipSuccess) return e;
    return launch(kern, dim3((unsigned)n * sh.n_kv_heads), dim3(256), lds, stream, q, k, v, dout, out, lse, lse2, delta, sentinel, dq,
                  segs, tq, sh, dq_row);
  };
  const int kg = dq_shares(segs, sh, D, compute_unit_count());
  hipError_t e;
  if (kg == 4) e = rows_pass(cattn_dq_kernel<D, 4>, CDqCfg<D, 4>::kBR, CDqCfg<D, 4>::kLdsBytes);
  else if (kg == 2) e = rows_pass(cattn_dq_kernel<D, 2>, CDqCfg<D, 2>::kBR, CDqCfg<D, 2>::kLdsBytes);
  else if constexpr (D == 128) e = rows_pass(cattn_dq2_kernel<D>, CDq2Cfg<D>::kBR, CDq2Cfg<D>::kLdsBytes);
  else e = rows_pass(cattn_dq_kernel<D, 1>, CDqCfg<D, 1>::kBR, CDqCfg<D, 1>::kLdsBytes);
  if (e != hipSuccess) return e;
  const KeysPlan plan = keys_plan(segs, sh, D, compute_unit_count());
  auto keys_pass = [&](auto rg_c) -> hipError_t {
    constexpr int RG = decltype(rg_c)::value;
    using Cfg = CKvCfg<D, RG>;
    const TileIndex tk = make_causal_index<true>(segs, sh.group, Cfg::kBC);
    const int n = count_tiles(tk);
    if (n == 0) return hipSuccess;
    hipError_t e = allow_lds(cattn_dkdv_kernel<D, RG>, Cfg::kLdsBytes);
    if (e != hipSuccess) return e;
    e = launch(cattn_dkdv_kernel<D, RG>, dim3((unsigned)n * sh.n_kv_heads * plan.splits), dim3(256), Cfg::kLdsBytes, stream, q, k, v, dout,
                  lse2, delta, sentinel, dk, dv, segs, tk, sh, dk_row, dv_row, plan.splits, parts);
    if (e != hipSuccess || plan.splits == 1) return e;
    return launch(cattn_dkdv_join_kernel<D>, dim3((unsigned)n * (Cfg::kBC / 32) * sh.n_kv_heads), dim3(128), 0, stream, dk, dv, segs, tk,
                  sh, dk_row, dv_row, Cfg::kBC, plan.splits, (const float*)parts);
  };
  if constexpr (D == 64)
    if (plan.rg == 4) return keys_pass(IntC<4>{});
  return plan.rg == 1 ? keys_pass(IntC<1>{}) : keys_pass(IntC<2>{});
}

hipError_t launch_cattn_bwd(const void* q, const void* k, const void* v, const void* out, const float* lse,
                            const void* dout, const XSegTable& segs, const CausalShape& sh, int head_dim,
                            void* dq, uint32_t dq_row, void* dk, uint32_t dk_row, void* dv, uint32_t dv_row,
                            float* delta, float* lse2, float* sentinel, float* parts, hipStream_t stream) {
  auto run = head_dim == 128 ? launch_bwd_dim<128> : launch_bwd_dim<64>;
  return run((const __bf16*)q, (const __bf16*)k, (const __bf16*)v, (const __bf16*)out, lse, (const __bf16*)dout, segs, sh,
             (__bf16*)dq, dq_row, (__bf16*)dk, dk_row, (__bf16*)dv, dv_row, delta, lse2, sentinel, parts, stream);
}

}  // namespace vfm
