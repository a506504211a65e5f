// Causal packed attention backward with grouped heads for gfx950 (bf16 MFMA, fp32 accumulate).
//
//     P_ij = exp(S_ij - lse_i) where j <= i + off, else 0;   Delta_i = sum_d dO_id O_id
//     dV_j = sum_i P_ij dO_i;   dS_ij = P_ij (dO_i . v_j - Delta_i);   dQ_i = scale sum_j dS_ij K_j;   dK_j = scale sum_i dS_ij Q_i
//
// The sums of dK, dV run over all rows of the K/V head: queries times the heads of its group (cattn_common.h).  No atomics: one
// pass per output kind, every output written once.
//   prepare : Delta and lse in log2 units (+inf for a row that sees no key, so that its P is 0).
//   dkdv    : a workgroup owns 128 keys (32 per wavefront: K, V rows and the dK^T, dV^T accumulators in registers) and walks
//             the rows that see any of them, staged through LDS.
//   dq      : a workgroup owns 128 rows and walks the keys that its last row sees.
#include "cattn_common.h"

namespace vfm {

constexpr int kCBwdBC = 128;   // keys per dK/dV workgroup
constexpr int kCBwdBQ = 64;    // rows per LDS tile
constexpr int kCFewKeys = 32;  // rows that see at most so many keys have their Delta formed from P and dP
constexpr float kCLog2eB = 1.4426950408889634f;

// ---------------------------------------------------------------- prepare
template <int D>
__global__ __launch_bounds__(256) void cattn_prepare_kernel(const u32x4* __restrict__ out, const u32x4* __restrict__ dout,
                                                            const float* __restrict__ lse, float* __restrict__ delta,
                                                            float* __restrict__ lse2, float* __restrict__ sentinel,
                                                            int total, int n_heads) {
  constexpr int kLanesPerRow = D / 8;
  constexpr int kRowsPerBlock = 256 / kLanesPerRow;
  const size_t row = (size_t)blockIdx.x * kRowsPerBlock + threadIdx.x / kLanesPerRow;   // token * n_heads + head
  const int chunk = threadIdx.x % kLanesPerRow;
  const size_t rows = (size_t)total * n_heads;
  if (blockIdx.x == 0 && threadIdx.x == 0) {   // statistics of rows past a sequence's end: P = 0, Delta = 0
    sentinel[0] = INFINITY;
    sentinel[1] = 0.f;
  }
  const size_t rr = row < rows ? row : rows - 1;
  const u32x4 a = out[rr * kLanesPerRow + chunk], b = dout[rr * kLanesPerRow + chunk];
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    s = __builtin_fmaf(__builtin_bit_cast(float, a[e] << 16), __builtin_bit_cast(float, b[e] << 16), s);
    s = __builtin_fmaf(__builtin_bit_cast(float, a[e] & 0xffff0000u), __builtin_bit_cast(float, b[e] & 0xffff0000u), s);
  }
#pragma unroll
  for (int o = kLanesPerRow / 2; o > 0; o >>= 1) s += __shfl_xor(s, o, kLanesPerRow);
  if (row < rows && chunk == 0) {
    const size_t at = (row % n_heads) * total + row / n_heads;
    const float l = lse[at];
    const bool none = l == -INFINITY;
    delta[at] = none ? 0.f : s;
    lse2[at] = none ? INFINITY : l * kCLog2eB;
  }
}

// Delta_i = sum_j P_ij dP_ij for rows that see at most kCFewKeys keys.  With so few keys |O| is as large as |V| and dS cancels, so
// that the rounding of `out` would show in dq, dk (see bwd_short_delta_kernel); in causal order every sequence
// begins with such rows.  One wavefront per 32 rows: one MFMA tile each of S^T and dP^T.
__host__ __device__ inline int few_first(const CausalSeq& c, int group) { return (c.off < 0 ? -c.off : 0) * group; }
__host__ __device__ inline int few_end(const CausalSeq& c, int group) {
  const int tok = kCFewKeys - c.off;
  return tok <= 0 ? 0 : (tok < c.ql ? tok : c.ql) * group;
}

template <int D>
__global__ __launch_bounds__(64) void cattn_few_delta_kernel(const __bf16* __restrict__ q, const __bf16* __restrict__ k,
                                                             const __bf16* __restrict__ v, const __bf16* __restrict__ dout,
                                                             const float* __restrict__ lse, float* __restrict__ delta,
                                                             const XSegTable segs, const TileIndex ti, const CausalShape sh) {
  constexpr int KS = D / 16;
  int seq, t;
  locate_tile(ti, segs.n, blockIdx.x, seq, t);
  const CausalSeq cs = causal_seq(segs, seq, sh.group);
  const int kvh = blockIdx.y;
  const int lane = threadIdx.x, c = lane & 31, g = lane >> 5;
  const int end = few_end(cs, sh.group);
  const int r = few_first(cs, sh.group) + t * 32 + c;
  const int row = min(r, end - 1), tok = row / sh.group, head = kvh * sh.group + row - tok * sh.group;
  const int lim = tok + cs.off;
  const size_t qtok = cs.qs + tok;
  const char* qp = (const char*)q + qtok * sh.q_row + (size_t)head * D * 2 + 16 * g;
  const __bf16* dp_ = dout + (qtok * sh.n_heads + head) * D + 8 * g;
  const size_t ktok = cs.ks + min(c, cs.kl - 1);
  const char* kp = (const char*)k + ktok * sh.k_row + (size_t)kvh * D * 2 + 16 * g;
  const char* vp = (const char*)v + ktok * sh.v_row + (size_t)kvh * D * 2 + 16 * g;
  const size_t stat = (size_t)head * sh.total_q + qtok;
  const float lse_i = lse[stat] * kCLog2eB;
  f32x16 s = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  f32x16 dp = s;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    s = mfma32(*(const bf16x8*)(kp + ks * 32), *(const bf16x8*)(qp + ks * 32), s);
    dp = mfma32(*(const bf16x8*)(vp + ks * 32), *(const bf16x8*)(dp_ + ks * 16), dp);
  }
  float acc = 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e)
    if (8 * (e >> 2) + 4 * g + (e & 3) <= lim) acc += fast_exp2(s[e] * sh.scale_log2 - lse_i) * dp[e];
  acc = pair_sum(acc);
  if (r < end && g == 0) delta[stat] = acc;
}

// ---------------------------------------------------------------- dK, dV
template <int D>
struct CKvCfg {
  static constexpr int kTileBytes = kCBwdBQ * D * 2;          // Q or dO rows of one tile
  static constexpr int kStatBytes = 4 * kCBwdBQ * 4;          // lse2, Delta (two spare copies)
  static constexpr int kStageBytes = 2 * kTileBytes + kStatBytes;
  static constexpr int kLdsBytes = 2 * kStageBytes;
  static constexpr int kChunksPerRow = D / 8;
  static constexpr int kLoadsPerWave = kCBwdBQ * kChunksPerRow / 256;
};

template <int D>
__global__ __launch_bounds__(256, D == 64 ? 2 : 1)
void cattn_dkdv_kernel(const __bf16* __restrict__ q, const __bf16* __restrict__ k, const __bf16* __restrict__ v,
                       const __bf16* __restrict__ dout, const float* __restrict__ lse2, const float* __restrict__ delta,
                       const float* __restrict__ sentinel, __bf16* __restrict__ dk, __bf16* __restrict__ dv,
                       const XSegTable segs, const TileIndex ti, const CausalShape sh, uint32_t dk_row, uint32_t dv_row) {
  using Cfg = CKvCfg<D>;
  constexpr int KS = D / 16, DB = D / 32, RB = D * 2;
  constexpr int LPW = Cfg::kLoadsPerWave;
  extern __shared__ __attribute__((aligned(16))) char smem[];

  const int kvh = blockIdx.x % sh.n_kv_heads;
  int seq, tk;
  locate_tile(ti, segs.n, blockIdx.x / sh.n_kv_heads, seq, tk);   // a sequence's first keys, which most rows see, first
  const CausalSeq cs = causal_seq(segs, seq, sh.group);
  const int j0 = tk * kCBwdBC;

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63;
  const int c = lane & 31;
  const int g = lane >> 5;
  const int jw = j0 + wave * 32;                       // the wavefront's first key
  const int keys_valid = cs.kl - jw;
  auto kv_row = [&](__bf16* base, uint32_t row_bytes, int r) {
    return reinterpret_cast<__bf16*>(reinterpret_cast<char*>(base) + (size_t)(cs.ks + jw + r) * row_bytes) + kvh * D;
  };

  // rows [first, cs.rows) see key j0; tiles of 64 from the one that holds the first
  const long long first = (long long)(j0 - cs.off) * sh.group;
  const int rt0 = first <= 0 ? 0 : (int)(first / kCBwdBQ) * kCBwdBQ;
  const int n_tiles = rt0 < cs.rows ? (cs.rows - rt0 + kCBwdBQ - 1) / kCBwdBQ : 0;

  const f32x16 zero16 = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  f32x16 dkacc[DB], dvacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) { dkacc[db] = zero16; dvacc[db] = zero16; }

  if (n_tiles > 0) {
    // K and V rows as B operands (lane: row c, columns ks*16 + 8g)
    bf16x8 kreg[KS], vreg[KS];
    {
      const size_t tok = cs.ks + min(jw + c, cs.kl - 1);
      const char* kp = (const char*)k + tok * sh.k_row + (size_t)kvh * RB + 16 * g;
      const char* vp = (const char*)v + tok * sh.v_row + (size_t)kvh * RB + 16 * g;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) { kreg[ks] = *(const bf16x8*)(kp + ks * 32); vreg[ks] = *(const bf16x8*)(vp + ks * 32); }
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) { settle(kreg[ks]); settle(vreg[ks]); }
    }
    // the first row that sees this lane's key
    const long long see = ((long long)(jw + c) - cs.off) * sh.group;
    const int row_min = see < 0 ? 0 : see > 0x7fffffffLL ? 0x7fffffff : (int)see;
    const long long see_w = ((long long)(jw + 31) - cs.off) * sh.group;   // ... all of the wavefront's keys
    const int wave_all = __builtin_amdgcn_readfirstlane(see_w < 0 ? 0 : see_w > 0x7fffffffLL ? 0x7fffffff : (int)see_w);

    const uint32_t smem_addr = __builtin_amdgcn_readfirstlane(lds_addr_of(smem));
    const char* qbase = uniform_ptr((const char*)q + (size_t)cs.qs * sh.q_row + (size_t)kvh * sh.group * RB);
    const char* dobase = uniform_ptr((const char*)dout + ((size_t)cs.qs * sh.n_heads + (size_t)kvh * sh.group) * RB);
    const uint32_t do_row = (uint32_t)sh.n_heads * RB;
    const bool is_lse = (wave & 1) == 0;
    const float* stat_src = uniform_ptr(is_lse ? lse2 : delta);
    const uint32_t stat_sentinel = (uint32_t)((const char*)(sentinel + (is_lse ? 0 : 1)) - (const char*)stat_src);
    auto issue_tile = [&](int stage, int t) {
      const int rt = rt0 + t * kCBwdBQ;
      const uint32_t dst = smem_addr + stage * Cfg::kStageBytes;
#pragma unroll
      for (int x = 0; x < LPW; ++x) {
        const int p = (x * 4 + wave) * 64 + lane;
        const int r = p / Cfg::kChunksPerRow;
        const uint32_t col = (uint32_t)(((p % Cfg::kChunksPerRow) ^ swz<D>(r)) * 16);
        const int row = min(rt + r, cs.rows - 1), tok = row / sh.group;
        const uint32_t sub = (uint32_t)(row - tok * sh.group) * RB + col;
        lds_dma16(qbase, (uint32_t)tok * sh.q_row + sub, dst + wave * 1024 + x * 4096);
        lds_dma16(dobase, (uint32_t)tok * do_row + sub, dst + Cfg::kTileBytes + wave * 1024 + x * 4096);
      }
      const int row = rt + lane, tok = row / sh.group;
      const uint32_t at = (uint32_t)(((size_t)(kvh * sh.group + row - tok * sh.group) * sh.total_q + cs.qs + tok) * 4);
      lds_dma4(stat_src, row < cs.rows ? at : stat_sentinel, dst + 2 * Cfg::kTileBytes + wave * (kCBwdBQ * 4));
    };

    const int rbase = tile_off<D>(c, 8 * g);
    int tbase[2];
#pragma unroll
    for (int t = 0; t < 2; ++t)
      tbase[t] = tile_off<D>(8 * t + 4 * g + ((lane & 15) >> 2), 16 * ((lane >> 4) & 1) + 4 * (lane & 3));

    issue_tile(0, 0);
    for (int t = 0; t < n_tiles; ++t) {
      wait_vmcnt<0>();
      __syncthreads();           // tile t is there for everyone, and everyone is done with tile t - 1
      if (t + 1 < n_tiles) issue_tile((t + 1) & 1, t + 1);
      const char* qt = smem + (t & 1) * Cfg::kStageBytes;
      const char* dt = qt + Cfg::kTileBytes;
      const float* st = reinterpret_cast<const float*>(dt + Cfg::kTileBytes);
#pragma unroll
      for (int ib = 0; ib < 2; ++ib) {
        const int rb = rt0 + t * kCBwdBQ + ib * 32;
        f32x16 s, dp;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          s = mfma32(lds_read_b128(qt, (rbase ^ (ks << 5)) + ib * 32 * RB), kreg[ks], ks == 0 ? zero16 : s);
          dp = mfma32(lds_read_b128(dt, (rbase ^ (ks << 5)) + ib * 32 * RB), vreg[ks], ks == 0 ? zero16 : dp);
        }
        f32x16 p, ds;
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const f32x4 l4 = *reinterpret_cast<const f32x4*>(st + ib * 32 + 8 * q4 + 4 * g);
          const f32x4 d4 = *reinterpret_cast<const f32x4*>(st + kCBwdBQ + ib * 32 + 8 * q4 + 4 * g);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            p[q4 * 4 + e] = fast_exp2(s[q4 * 4 + e] * sh.scale_log2 - l4[e]);
            ds[q4 * 4 + e] = p[q4 * 4 + e] * (dp[q4 * 4 + e] - d4[e]);
          }
        }
        if (rb < wave_all) {      // rows that do not see this lane's key
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (rb + 8 * (e >> 2) + 4 * g + (e & 3) < row_min) p[e] = ds[e] = 0.f;
        }
        bf16x8 pb[2], dsb[2];
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) {
          f32x8 a, b;
#pragma unroll
          for (int e = 0; e < 8; ++e) { a[e] = p[8 * s2 + e]; b[e] = ds[8 * s2 + e]; }
          pb[s2] = to_bf16x8(a);
          dsb[s2] = to_bf16x8(b);
        }
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
          for (int db = 0; db < DB; ++db) {
            const int o0 = (tbase[0] ^ (db << 6)) + (ib * 32 + 16 * s2) * RB, o1 = (tbase[1] ^ (db << 6)) + (ib * 32 + 16 * s2) * RB;
            dvacc[db] = mfma32(join_tr(lds_read_tr(dt, o0), lds_read_tr(dt, o1)), pb[s2], dvacc[db]);
            dkacc[db] = mfma32(join_tr(lds_read_tr(qt, o0), lds_read_tr(qt, o1)), dsb[s2], dkacc[db]);
          }
      }
    }
    wait_vmcnt<0>();
    __syncthreads();             // the tiles are free: each wavefront turns its results through a piece of them
  }
  char* turn = smem + wave * (32 * RB);
  store_tile_rows_at<D>(turn, dkacc, sh.scale, keys_valid, [&](int r) { return kv_row(dk, dk_row, r); });
  store_tile_rows_at<D>(turn, dvacc, 1.0f, keys_valid, [&](int r) { return kv_row(dv, dv_row, r); });
}

// ---------------------------------------------------------------- dQ
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
                     const __bf16* __restrict__ dout, const float* __restrict__ lse2g, const float* __restrict__ delta,
                     __bf16* __restrict__ dq, const XSegTable segs, const TileIndex ti, const CausalShape sh, uint32_t dq_row) {
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
  const int row_w = r0 + wave * 32;
  const int rows_valid = cs.rows - row_w;
  const int row = min(row_w + c, cs.rows - 1), tok = row / sh.group, head = kvh * sh.group + row - tok * sh.group;
  const int lim = tok + cs.off;
  const int wave_min = __builtin_amdgcn_readfirstlane(min(row_w, cs.rows - 1) / sh.group + cs.off);
  const int n_keys = (min(r0 + Cfg::kBR, cs.rows) - 1) / sh.group + cs.off + 1;
  const int n_tiles = n_keys > 0 ? (n_keys + Cfg::kBC - 1) / Cfg::kBC : 0;

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
    const size_t stat = (size_t)head * sh.total_q + qtok;
    const float lse2 = lse2g[stat], dlt = delta[stat];
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
template <int D>
static hipError_t launch_bwd_dim(const __bf16* q, const __bf16* k, const __bf16* v, const __bf16* out, const float* lse,
                                 const __bf16* dout, const XSegTable& segs, const CausalShape& sh, __bf16* dq,
                                 uint32_t dq_row, __bf16* dk, uint32_t dk_row, __bf16* dv, uint32_t dv_row, float* delta,
                                 float* lse2, hipStream_t stream, float* sentinel) {
  TileIndex few;
  int n_few = 0;
  for (int s = 0; s <= VFM_MAX_SEQS; ++s) {
    few.cu[s] = n_few;
    if (s < segs.n && segs.kl[s] > 0) {
      CausalSeq c;
      c.ql = segs.ql[s];
      c.off = segs.kl[s] - segs.ql[s];
      const int n = few_end(c, sh.group) - few_first(c, sh.group);
      if (n > 0) n_few += (n + 31) / 32;
    }
  }
  hipError_t e;
  if (n_few > 0) {
    e = launch(cattn_few_delta_kernel<D>, dim3(n_few, sh.n_kv_heads), dim3(64), 0, stream, q, k, v, dout, lse, delta, segs, few, sh);
    if (e != hipSuccess) return e;
  }
  const TileIndex tk = make_causal_index<true>(segs, sh.group, kCBwdBC);
  if (const int n = count_tiles(tk)) {
    using Cfg = CKvCfg<D>;
    e = allow_lds(cattn_dkdv_kernel<D>, Cfg::kLdsBytes);
    if (e != hipSuccess) return e;
    e = launch(cattn_dkdv_kernel<D>, dim3((unsigned)n * sh.n_kv_heads), dim3(256), Cfg::kLdsBytes, stream, q, k, v, dout, lse2,
               delta, sentinel, dk, dv, segs, tk, sh, dk_row, dv_row);
    if (e != hipSuccess) return e;
  }
  const TileIndex tq = make_causal_index<false>(segs, sh.group, CDqCfg<D>::kBR);
  if (const int n = count_tiles(tq)) {
    using Cfg = CDqCfg<D>;
    e = allow_lds(cattn_dq_kernel<D>, Cfg::kLdsBytes);
    if (e != hipSuccess) return e;
    return launch(cattn_dq_kernel<D>, dim3((unsigned)n * sh.n_kv_heads), dim3(256), Cfg::kLdsBytes, stream, q, k, v, dout, lse2,
                  delta, dq, segs, tq, sh, dq_row);
  }
  return hipSuccess;
}

hipError_t launch_cattn_prepare(const void* out, const void* dout, const float* lse, float* delta, float* lse2,
                                float* sentinel, int total_q, int n_heads, int head_dim, hipStream_t stream) {
  const size_t rows = (size_t)total_q * n_heads, per = 256 / (head_dim / 8);
  auto kern = head_dim == 128 ? cattn_prepare_kernel<128> : cattn_prepare_kernel<64>;
  return launch(kern, dim3((unsigned)((rows + per - 1) / per)), dim3(256), 0, stream, (const u32x4*)out, (const u32x4*)dout,
                lse, delta, lse2, sentinel, total_q, n_heads);
}

hipError_t launch_cattn_bwd(const void* q, const void* k, const void* v, const void* out, const float* lse,
                            const void* dout, const XSegTable& segs, const CausalShape& sh, int head_dim,
                            void* dq, uint32_t dq_row, void* dk, uint32_t dk_row, void* dv, uint32_t dv_row,
                            float* delta, float* lse2, float* sentinel, hipStream_t stream) {
  auto run = head_dim == 128 ? launch_bwd_dim<128> : launch_bwd_dim<64>;
  return run((const __bf16*)q, (const __bf16*)k, (const __bf16*)v, (const __bf16*)out, lse, (const __bf16*)dout, segs, sh,
             (__bf16*)dq, dq_row, (__bf16*)dk, dk_row, (__bf16*)dv, dv_row, delta, lse2, stream, sentinel);
}

}  // namespace vfm
