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
#include "cattn_common.h"
#include "cattn_dkdv.h"
#include "cattn_dq.h"

namespace vfm {

// ---------------------------------------------------------------- dQ at head_dim 64
// 128 rows per workgroup, 32 per wavefront, three workgroups per CU: with the exponentials weighing twice as much against the products
// as at head_dim 128, wavefronts of other workgroups fill the gaps.  Delta and the statistics as in cattn_dq2_kernel.
template <int D>
struct CDqCfg {
  static constexpr int kBR = 128;                             // rows per workgroup
  static constexpr int kBC = 64;                              // keys per LDS tile
  static constexpr int kTileBytes = kBC * D * 2;              // K or V rows of one tile
  static constexpr int kLdsBytes = 4 * kTileBytes;
  static constexpr int kChunksPerRow = D / 8;
  static constexpr int kLoadsPerWave = kBC * kChunksPerRow / 256;
};

template <int D>
__global__ __launch_bounds__(256, D == 64 ? 3 : 1)
void cattn_dq_kernel(const __bf16* __restrict__ q, const __bf16* __restrict__ k, const __bf16* __restrict__ v,
                     const __bf16* __restrict__ dout, const __bf16* __restrict__ out, const float* __restrict__ lse,
                     float* __restrict__ lse2g, float* __restrict__ delta, float* __restrict__ sentinel, __bf16* __restrict__ dq, const XSegTable segs, const TileIndex ti, const CausalShape sh, uint32_t dq_row) {
  using Cfg = CDqCfg<D>;
  constexpr int KS = D / 16, DB = D / 32, RB = D * 2;
  constexpr int LPW = Cfg::kLoadsPerWave;
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
  if (blockIdx.x == 0 && tid == 0) {   // statistics of rows past a sequence's end, for the dK/dV pass
    sentinel[0] = INFINITY;
    sentinel[1] = 0.f;
  }
  const int row_w = r0 + wave * 32;
  const int rows_valid = cs.rows - row_w;
  const int row = min(row_w + c, cs.rows - 1), tok = row / sh.group, head = kvh * sh.group + row - tok * sh.group;
  const int lim = tok + cs.off;
  const int wave_min = __builtin_amdgcn_readfirstlane(min(row_w, cs.rows - 1) / sh.group + cs.off);
  const int n_keys = (min(r0 + Cfg::kBR, cs.rows) - 1) / sh.group + cs.off + 1;
  const int n_tiles = n_keys > 0 ? (n_keys + Cfg::kBC - 1) / Cfg::kBC : 0;

  const size_t stat = (size_t)head * sh.total_q + cs.qs + tok;
  const bool keeps = g == 0 && row_w + c < cs.rows;             // this lane leaves its row's statistics
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
      const uint32_t dst = smem_addr + stage * 2 * Cfg::kTileBytes + wave * 1024;
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
    for (int t = 0; t < n_tiles; ++t) {
      wait_vmcnt<0>();
      __syncthreads();
      if (t + 1 < n_tiles) issue_tile((t + 1) & 1, t + 1);
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
      const char* kt = smem + (t & 1) * 2 * Cfg::kTileBytes;
      const char* vt = kt + Cfg::kTileBytes;
#pragma unroll
      for (int jb = 0; jb < 2; ++jb) {
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
  }
  store_tile_rows_at<D>(smem + wave * (32 * RB), dqacc, sh.scale, rows_valid, [&](int r) {
    const int rw = row_w + r, tk = rw / sh.group;
    return reinterpret_cast<__bf16*>(reinterpret_cast<char*>(dq) + (size_t)(cs.qs + tk) * dq_row) +
           (kvh * sh.group + rw - tk * sh.group) * D;
  });
}

// ---------------------------------------------------------------- launch
// Wavefronts that share the keys of a dK/dV workgroup (RG of cattn_dkdv_kernel): 1 where the workgroups of 128 keys keep the chip
// busy; more where the longest of them, which walks all of its sequence's rows, takes longer than an even share of the
// work.
static int dkdv_shares(const XSegTable& segs, const CausalShape& sh, int head_dim, int cus) {
  long long longest = 0, work = 0;                 // in 64-row tiles
  for (int s = 0; s < segs.n; ++s) {
    const long long tiles = ((long long)segs.ql[s] * sh.group + 63) / 64, n = (segs.kl[s] + kCBwdBC - 1) / kCBwdBC;
    // keys before the first query are seen by all rows, the others by half of them on average
    const long long before = segs.kl[s] > segs.ql[s] ? (segs.kl[s] - segs.ql[s]) / kCBwdBC : 0;
    longest = longest > tiles ? longest : tiles;
    work += before * tiles + (n - before) * (tiles + 1) / 2;
  }
  const long long share = work * sh.n_kv_heads / cus;
  if (longest <= share + share / 2 + 4) return 1;
  return head_dim == 64 && longest > 3 * share ? 4 : 2;
}

template <int D>
static hipError_t launch_bwd_dim(const __bf16* q, const __bf16* k, const __bf16* v, const __bf16* out, const float* lse,
                                 const __bf16* dout, const XSegTable& segs, const CausalShape& sh, __bf16* dq,
                                 uint32_t dq_row, __bf16* dk, uint32_t dk_row, __bf16* dv, uint32_t dv_row, float* delta,
                                 float* lse2, float* sentinel, hipStream_t stream) {
  constexpr int kRows = D == 128 ? CDq2Cfg<128>::kBR : CDqCfg<64>::kBR;
  constexpr int kLds = D == 128 ? CDq2Cfg<128>::kLdsBytes : CDqCfg<64>::kLdsBytes;
  const TileIndex tq = make_causal_index<false>(segs, sh.group, kRows);
  if (const int n = count_tiles(tq)) {
    auto kern = [] { if constexpr (D == 128) return cattn_dq2_kernel<128>; else return cattn_dq_kernel<64>; }();
    hipError_t e = allow_lds(kern, kLds);
    if (e != hipSuccess) return e;
    e = launch(kern, dim3((unsigned)n * sh.n_kv_heads), dim3(256), kLds, stream, q, k, v, dout, out, lse, lse2, delta, sentinel, dq,
               segs, tq, sh, dq_row);
    if (e != hipSuccess) return e;
  }
  auto keys_pass = [&](auto rg_c) -> hipError_t {
    constexpr int RG = decltype(rg_c)::value;
    using Cfg = CKvCfg<D, RG>;
    const TileIndex tk = make_causal_index<true>(segs, sh.group, Cfg::kBC);
    const int n = count_tiles(tk);
    if (n == 0) return hipSuccess;
    hipError_t e = allow_lds(cattn_dkdv_kernel<D, RG>, Cfg::kLdsBytes);
    if (e != hipSuccess) return e;
    return launch(cattn_dkdv_kernel<D, RG>, dim3((unsigned)n * sh.n_kv_heads), dim3(256), Cfg::kLdsBytes, stream, q, k, v, dout,
                  lse2, delta, sentinel, dk, dv, segs, tk, sh, dk_row, dv_row);
  };
  const int rg = dkdv_shares(segs, sh, D, compute_unit_count());
  if constexpr (D == 64)
    if (rg == 4) return keys_pass(IntC<4>{});
  return rg == 1 ? keys_pass(IntC<1>{}) : keys_pass(IntC<2>{});
}

hipError_t launch_cattn_bwd(const void* q, const void* k, const void* v, const void* out, const float* lse,
                            const void* dout, const XSegTable& segs, const CausalShape& sh, int head_dim,
                            void* dq, uint32_t dq_row, void* dk, uint32_t dk_row, void* dv, uint32_t dv_row,
                            float* delta, float* lse2, float* sentinel, hipStream_t stream) {
  auto run = head_dim == 128 ? launch_bwd_dim<128> : launch_bwd_dim<64>;
  return run((const __bf16*)q, (const __bf16*)k, (const __bf16*)v, (const __bf16*)out, lse, (const __bf16*)dout, segs, sh,
             (__bf16*)dq, dq_row, (__bf16*)dk, dk_row, (__bf16*)dv, dv_row, delta, lse2, sentinel, stream);
}

}  // namespace vfm
