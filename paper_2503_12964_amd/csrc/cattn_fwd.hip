// Causal packed attention forward with grouped heads for gfx950 (bf16 MFMA, fp32 accumulate).
//
//     S_ij = scale q_i . k_j  (j <= i + off),   out_i = sum_j softmax_j(S_ij) v_j,   lse_i = ln sum_j exp(S_ij)
//
// One workgroup owns a tile of rows (query token x head of the group, see cattn_common.h) of one (sequence, K/V head), 32 rows
// per wavefront, and streams the keys that its last row sees through LDS in units of 32.  The loop is that of the
// bidirectional forward (attn_fwd.hip): S^T = K Q^T so that a lane holds 16 keys of one row, P^T is the B operand of
// O^T += V^T P^T as it stands, S(u+1) and O += V(u-1) P(u-1) run under the softmax of unit u, the softmax reference moves only when
// a unit's exponentials would grow too large, K and V in rings of four LDS slots.  What the causal order adds: a wavefront masks only the
// units that reach past its first row's limit, computes none past its last row's (it keeps fetching its share and
// meeting the barriers for the wavefronts behind it), and a sequence's row tiles are handed out longest first, the sequence with the
// most keys first (the tiles of all sequences together are in no order).
// Bound by the matrix pipe with the exponentials beside it: 12,007 tokens x 32/8 heads x 128 in 1,045 us, 1.13 PFLOP/s of the pairs that
// are seen (a large library product on the same card: 1.33).
#include "cattn_careful.h"
#include "cattn_common.h"
#include "cattn_plan.h"

namespace vfm {

constexpr int kCRing = 4;               // LDS ring slots for K and for V
constexpr float kCLn2 = 0.6931471805599453f;
constexpr float kCUnset = -3.0e38f;      // reference of a row that has seen no key
constexpr float kCSafeSum = 256.0f;     // a unit's exponentials may sum to this before the reference moves

template <int D, int W>
struct CFwdCfg {
  static constexpr int kRows = W * 32;
  static constexpr int kUnitBytes = kCU * D * 2;
  static constexpr int kQBase = (2 * kCRing - 2) * kUnitBytes;     // Q rows: over the V ring's last two slots and behind
  static constexpr int kLdsBytes = kQBase + (kRows * D * 2 > 2 * kUnitBytes ? kRows * D * 2 : 2 * kUnitBytes);
  static_assert(kLdsBytes <= 160 * 1024, "LDS of one CU");
  static constexpr int kChunksPerRow = D / 8;
  static constexpr int kLoadsPerWave = kCU * kChunksPerRow / (W * 64);
};

constexpr int kSgcValu = 0x002, kSgcMfma = 0x008, kSgcDsRead = 0x100;

// Wavefronts per SIMD
constexpr int fwd_waves(int D, int W) { return W == 1 ? 1 : W == 2 ? (D == 64 ? 2 : 1) : D == 64 ? 3 : 2; }
// In a cut call, which has a workgroup per CU: room for what the loop over tiles keeps (spilled otherwise: 2,000 tokens x 8/2 heads x 64
// took 27 us, not 22).  Eight wavefronts are two per SIMD in any case: 24 registers of the loop over tiles are spilled there.
constexpr int split_waves(int D, int W) { return W == 4 ? (D == 64 ? 2 : 1) : fwd_waves(D, W); }

// A wavefront's sums over keys [j0, j1) hold a NaN: they are formed again over the keys that each row sees, if those that
// it does not see may have made one.
template <int D>
__device__ __forceinline__ void fwd_checked(f32x16 (&acc)[D / 32], const __bf16* q, const __bf16* k, const __bf16* v,
                                            const CausalSeq& cs, const CausalShape& sh, int kvh, int row_w, int j0, int j1, float m) {
  constexpr int RB = D * 2;
  const char* kbase = (const char*)k + (size_t)cs.ks * sh.k_row + (size_t)kvh * RB;
  const char* vbase = (const char*)v + (size_t)cs.ks * sh.v_row + (size_t)kvh * RB;
  const int row = min(row_w + (lane_anew() & 31), cs.rows - 1), tok = row / sh.group;
  const char* q_row = (const char*)q + (size_t)(cs.qs + tok) * sh.q_row + (size_t)(kvh * sh.group + row - tok * sh.group) * RB;
  fwd_again<D>(acc, q_row, kbase, sh.k_row, vbase, sh.v_row, j0, min(j1, cs.kl), j1, tok + cs.off, min(row_w, cs.rows - 1) / sh.group + cs.off, m,
               sh.scale_log2);
}

// What a workgroup does of one tile: the units [u0, u1) of the keys that the tile's last row sees.  slot: null, or where the
// unfinished results of a tile go that other workgroups share: per wavefront its accumulators as they lie (16 bytes a
// lane), then the reference and the sum of its 32 rows.
template <int D, int W>
constexpr size_t slot_floats() { return (size_t)W * (32 * D + 64); }

template <int D, int W, class Segs>
__device__ __forceinline__
void fwd_segment(const __bf16* __restrict__ q, const __bf16* __restrict__ k, const __bf16* __restrict__ v,
                 __bf16* __restrict__ out, float* __restrict__ lse, const Segs& segs, const CausalShape& sh, int kvh, int seq,
                 int tq, int u0, int u1, float* __restrict__ slot) {
  using Cfg = CFwdCfg<D, W>;
  constexpr int KS = D / 16, DB = D / 32;
  constexpr int LPW = Cfg::kLoadsPerWave;
  constexpr int UB = Cfg::kUnitBytes;
  constexpr int RB = D * 2;
  constexpr int kInFlight = 2 * 2 * LPW;

  extern __shared__ __attribute__((aligned(16))) char smem[];
  const CausalSeq cs = causal_seq(segs, seq, sh.group);
  const int r0 = tq * Cfg::kRows;                               // first row of the tile

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = lane_anew();         // (what hangs on it is not carried from one segment to the next)
  const int c = lane & 31;
  const int g = lane >> 5;

  const int row_w = r0 + wave * 32;                             // the wavefront's first row
  const int rows_valid = cs.rows - row_w;                       // may be <= 0, or more than 32
  auto row_tok = [&](int r) { return r / sh.group; };
  const int lim_g = row_tok(min(row_w + c, cs.rows - 1)) + cs.off - 4 * g;   // this lane's row sees keys <= lim_g + 4 g
  // units that the workgroup, and this wavefront, look at, counted from u0
  const int n_units = u1 - u0;
  const int wave_min = __builtin_amdgcn_readfirstlane(row_tok(min(row_w, cs.rows - 1)) + cs.off);   // its first row's limit
  const int wave_last = row_tok(min(row_w + 32, cs.rows) - 1) + cs.off;
  const int wave_units = __builtin_amdgcn_readfirstlane(
      rows_valid <= 0 || wave_last < u0 * kCU ? 0 : min(wave_last / kCU + 1 - u0, n_units));

  // address of row r of the wavefront's tile in out
  auto out_row = [&](int r) {
    const int row = row_w + r, tok = row_tok(row);
    return out + ((size_t)(cs.qs + tok) * sh.n_heads + kvh * sh.group + (row - tok * sh.group)) * D;
  };
  auto lse_at = [&](int row) {
    const int tok = row_tok(row);
    return (size_t)(kvh * sh.group + (row - tok * sh.group)) * sh.total_q + cs.qs + tok;
  };
  float* const wave_slot = slot + wave * (32 * D + 64);
  auto write_empty = [&]() {                                    // rows that see no key of these
    if (slot) {
      if (rows_valid <= 0) return;
      if (lane < 32) {
        wave_slot[32 * D + 2 * lane] = kCUnset;
        wave_slot[32 * D + 2 * lane + 1] = 0.f;
      }
      for (int i = lane; i < 8 * D; i += 64) reinterpret_cast<f32x4*>(wave_slot)[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      return;
    }
    if (row_w + c < cs.rows && g == 0) lse[lse_at(row_w + c)] = -INFINITY;
    const u32x4 z = {0u, 0u, 0u, 0u};
    for (int i = lane; i < 32 * Cfg::kChunksPerRow; i += 64) {
      const int r = i / Cfg::kChunksPerRow;
      if (r < rows_valid) *reinterpret_cast<u32x4*>(out_row(r) + (i % Cfg::kChunksPerRow) * 8) = z;
    }
  };
  if (n_units == 0) { write_empty(); return; }

  // ---- K/V staging with direct global->LDS loads (as in attn_fwd.hip); byte offsets count from the sequence's first
  // key; keys past the last one clamp to it (no row sees them)
  const char* kbase = uniform_ptr(reinterpret_cast<const char*>(k) + (size_t)cs.ks * sh.k_row + (size_t)kvh * RB);
  const char* vbase = uniform_ptr(reinterpret_cast<const char*>(v) + (size_t)cs.ks * sh.v_row + (size_t)kvh * RB);
  const uint32_t k_last = (uint32_t)(cs.kl - 1) * sh.k_row, v_last = (uint32_t)(cs.kl - 1) * sh.v_row;
  uint32_t st_colb[LPW], k_rowoff[LPW], v_rowoff[LPW];
#pragma unroll
  for (int x = 0; x < LPW; ++x) {
    const int p = (x * W + wave) * 64 + lane;
    const int r = p / Cfg::kChunksPerRow;
    k_rowoff[x] = (uint32_t)(u0 * kCU + r) * sh.k_row;
    v_rowoff[x] = (uint32_t)(u0 * kCU + r) * sh.v_row;
    st_colb[x] = (uint32_t)(((p % Cfg::kChunksPerRow) ^ swz<D>(r)) * 16);
  }
  const uint32_t wave_lds = __builtin_amdgcn_readfirstlane(lds_addr_of(smem) + wave * 1024);
  auto issue_k = [&](int slot) {
#pragma unroll
    for (int x = 0; x < LPW; ++x) {
      lds_dma16(kbase, min(k_rowoff[x], k_last) + st_colb[x], wave_lds + slot * UB + x * W * 1024);
      k_rowoff[x] += kCU * sh.k_row;
    }
  };
  auto issue_v = [&](int slot) {
#pragma unroll
    for (int x = 0; x < LPW; ++x) {
      lds_dma16(vbase, min(v_rowoff[x], v_last) + st_colb[x], wave_lds + (kCRing + slot) * UB + x * W * 1024);
      v_rowoff[x] += kCU * sh.v_row;
    }
  };
  // units that this wavefront does not compute: its share of the requests, the wait, the barrier
  auto idle_unit = [&](int u) {
    issue_k((u + 1) % kCRing);
    issue_v((u + 2) % kCRing);
    wait_vmcnt<kInFlight>();
    __syncthreads();
  };

  if (wave_units == 0) {
    issue_k(0); issue_k(1); issue_k(2); issue_k(3);
    issue_v(0); issue_v(1);
    wait_vmcnt<0>();
    __syncthreads();
    __syncthreads();
    issue_k(0);
    for (int u = 0; u < n_units; ++u) idle_unit(u);
    wait_vmcnt<0>();
    __syncthreads();
    write_empty();
    return;
  }

  const int kbase_off = tile_off<D>(c, 8 * g);
  int vbase_off[2];
#pragma unroll
  for (int t = 0; t < 2; ++t)
    vbase_off[t] = tile_off<D>(8 * t + 4 * g + ((lane & 15) >> 2), 16 * ((lane >> 4) & 1) + 4 * (lane & 3));

  const f32x16 zero16 = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  f32x16 oacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) oacc[db] = zero16;

  auto read_k = [&](int slot, bf16x8 (&ka)[KS]) {
    const char* kt = smem + slot * UB;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) ka[ks] = lds_read_b128(kt, kbase_off ^ (ks << 5));
  };
  auto mask = [&](int u, f32x16& s) {    // keys that the lane's row does not see
    const int j0 = (u0 + u) * kCU;
    if (j0 + kCU - 1 > wave_min) {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (j0 + 8 * (r >> 2) + (r & 3) > lim_g) s[r] = -INFINITY;
    }
  };

  // ---- prologue: Q rows, K units 0..3 and V units 0..1; S(0); operands of K(1)
  const uint32_t q_lds = lds_addr_of(smem) + Cfg::kQBase + wave * (32 * RB);
  {
    const char* qbase = uniform_ptr(reinterpret_cast<const char*>(q) + (size_t)cs.qs * sh.q_row + (size_t)kvh * sh.group * RB);
    const uint32_t q_s = __builtin_amdgcn_readfirstlane(q_lds);
#pragma unroll
    for (int x = 0; x < 32 * RB / 1024; ++x) {
      const int p = x * 64 + lane, r = p / Cfg::kChunksPerRow;
      const int row = min(row_w + r, cs.rows - 1), tok = row_tok(row);
      lds_dma16(qbase, (uint32_t)tok * sh.q_row + (uint32_t)(row - tok * sh.group) * RB +
                           (uint32_t)(((p % Cfg::kChunksPerRow) ^ swz<D>(r)) * 16), q_s + x * 1024);
    }
  }
  issue_k(0); issue_k(1); issue_k(2); issue_k(3);
  issue_v(0); issue_v(1);
  wait_vmcnt<0>();
  bf16x8 qreg[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    qreg[ks] = lds_read_b128_at(q_lds + (kbase_off ^ (ks << 5)));
    settle(qreg[ks]);
  }
  __syncthreads();

  bf16x8 ka[KS];
  f32x16 s_cur;
  {
    bf16x8 k0[KS];
    read_k(0, k0);
    read_k(1, ka);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) s_cur = mfma32(k0[ks], qreg[ks], ks == 0 ? zero16 : s_cur);
    mask(0, s_cur);
  }
  // first reference point: the row maximum of the first unit (a row that sees any of these keys sees the first); a row that sees
  // none keeps a finite one, far below all others
  float m_run, l_run = 0.f;
  {
    float mx = s_cur[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s_cur[r]);
    m_run = pair_max(mx) * sh.scale_log2;
    if (m_run == -INFINITY) m_run = kCUnset;
  }
  __syncthreads();            // every wave holds K(0), K(1) in registers: slots 0, 1 are free
  issue_k(0);                 // K unit 4

  bf16x8 pb_prev[2];
  pb_prev[0] = pb_prev[1] = bf16x8{};

  auto iteration = [&](auto slot_c, auto pv_c, int u) {
    constexpr int SLOT = decltype(slot_c)::value;
    constexpr bool PV = decltype(pv_c)::value != 0;
    issue_k((SLOT + 1) % kCRing);     // K(u+5)
    issue_v((SLOT + 2) % kCRing);     // V(u+2)

    // ---- region 1: S(u+1) MFMAs | V(u-1) operand reads | first half of softmax(u)
    s16x4 vlo[2][DB], vhi[2][DB];
    if constexpr (PV) {
      const char* vt = smem + (kCRing + (SLOT + 3) % kCRing) * UB;
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          vlo[s2][db] = lds_read_tr(vt, (vbase_off[0] ^ (db << 6)) + 16 * s2 * RB);
          vhi[s2][db] = lds_read_tr(vt, (vbase_off[1] ^ (db << 6)) + 16 * s2 * RB);
        }
    }
    f32x16 s_next, s_odd;     // two accumulation chains: a single one cannot issue back to back
#pragma unroll
    for (int ks = 0; ks < KS; ks += 2) {
      s_next = mfma32(ka[ks], qreg[ks], ks == 0 ? zero16 : s_next);
      s_odd = mfma32(ka[ks + 1], qreg[ks + 1], ks == 0 ? zero16 : s_odd);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) s_next[r] += s_odd[r];

    f32x8 p0, p1;
#pragma unroll
    for (int r = 0; r < 8; ++r) p0[r] = fast_exp2(s_cur[r] * sh.scale_log2 - m_run);
    bf16x8 pb_cur[2];
    pb_cur[0] = to_bf16x8(p0);
    float lsum = 0.f;
#pragma unroll
    for (int r = 0; r < 8; ++r) lsum += p0[r];
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      __builtin_amdgcn_sched_group_barrier(kSgcMfma, 1, 0);
      __builtin_amdgcn_sched_group_barrier(kSgcDsRead, PV ? 2 : 0, 0);
      __builtin_amdgcn_sched_group_barrier(kSgcValu, 5, 0);
    }
    __builtin_amdgcn_sched_barrier(0);

    // ---- region 2: O += V(u-1) P(u-1) MFMAs | K(u+2) operand reads | second half of softmax(u)
    if constexpr (PV) {
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
        for (int db = 0; db < DB; ++db)
          oacc[db] = mfma32(join_tr(vlo[s2][db], vhi[s2][db]), pb_prev[s2], oacc[db]);
    }
    bf16x8 ka_next[KS];
    read_k((SLOT + 2) % kCRing, ka_next);
#pragma unroll
    for (int r = 0; r < 8; ++r) p1[r] = fast_exp2(s_cur[8 + r] * sh.scale_log2 - m_run);
    pb_cur[1] = to_bf16x8(p1);
#pragma unroll
    for (int r = 0; r < 8; ++r) lsum += p1[r];
    const bool redo = __builtin_amdgcn_ballot_w64(!(lsum <= kCSafeSum)) != 0;
#pragma unroll
    for (int i = 0; i < 2 * DB; ++i) {
      __builtin_amdgcn_sched_group_barrier(kSgcMfma, PV ? 1 : 0, 0);
      __builtin_amdgcn_sched_group_barrier(kSgcDsRead, 1, 0);
      __builtin_amdgcn_sched_group_barrier(kSgcValu, 4, 0);
    }
    asm volatile("" : "+v"(pb_cur[0]), "+v"(pb_cur[1]), "+v"(lsum));
    __builtin_amdgcn_sched_barrier(0);

    // rare (wave-uniform): move the reference to the true running maximum and bring everything to it
    if (redo) {
      float mx = s_cur[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s_cur[r]);
      const float m_new = fmaxf(m_run, pair_max(mx) * sh.scale_log2);
      const float alpha = fast_exp2(m_run - m_new);
      m_run = m_new;
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        p0[r] = fast_exp2(s_cur[r] * sh.scale_log2 - m_new);
        p1[r] = fast_exp2(s_cur[8 + r] * sh.scale_log2 - m_new);
      }
      pb_cur[0] = to_bf16x8(p0);
      pb_cur[1] = to_bf16x8(p1);
      lsum = 0.f;
#pragma unroll
      for (int r = 0; r < 8; ++r) lsum += p0[r] + p1[r];
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[db][r] *= alpha;
    }
    l_run += lsum;

    mask(u + 1, s_next);
    s_cur = s_next;
    pb_prev[0] = pb_cur[0];
    pb_prev[1] = pb_cur[1];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) ka[ks] = ka_next[ks];

    wait_vmcnt<kInFlight>();   // everything but the two youngest batches has landed ...
    __syncthreads();           // ... for every wave, and every wave is done with this unit's slots
  };

  iteration(IntC<0>{}, IntC<0>{}, 0);
  for (int u = 1; u < wave_units; u += 4) {
    iteration(IntC<1>{}, IntC<1>{}, u);
    if (u + 1 < wave_units) iteration(IntC<2>{}, IntC<1>{}, u + 1);
    if (u + 2 < wave_units) iteration(IntC<3>{}, IntC<1>{}, u + 2);
    if (u + 3 < wave_units) iteration(IntC<0>{}, IntC<1>{}, u + 3);
  }
  // ---- drain: accumulate the wavefront's last unit (its slot is taken again two units on, a barrier away)
  {
    const char* vt = smem + (kCRing + (wave_units - 1) % kCRing) * UB;
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const bf16x8 va = join_tr(lds_read_tr(vt, (vbase_off[0] ^ (db << 6)) + 16 * s2 * RB),
                                  lds_read_tr(vt, (vbase_off[1] ^ (db << 6)) + 16 * s2 * RB));
        oacc[db] = mfma32(va, pb_prev[s2], oacc[db]);
      }
  }
  for (int u = wave_units; u < n_units; ++u) idle_unit(u);
  wait_vmcnt<0>();   // no load may still be writing LDS when the workgroup ends

  if (any_nan(oacc))     // (rare)
    fwd_checked<D>(oacc, q, k, v, cs, shape_anew(sh), kvh, row_w, u0 * kCU, (u0 + wave_units) * kCU, m_run);

  if (slot) {
    float* o = slot + wave * (32 * D + 64);
    const int ln = lane_anew();
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4)
        reinterpret_cast<f32x4*>(o)[(db * 4 + q4) * 64 + ln] =
            f32x4{oacc[db][q4 * 4], oacc[db][q4 * 4 + 1], oacc[db][q4 * 4 + 2], oacc[db][q4 * 4 + 3]};
    const float l_part = pair_sum(l_run);
    if (ln < 32) {
      o[32 * D + 2 * ln] = m_run;
      o[32 * D + 2 * ln + 1] = l_part;
    }
    __syncthreads();
    return;
  }

  // ---- epilogue: normalise, write out (bf16) and lse (natural log); a row without keys: 0 and -inf
  const float l_tot = pair_sum(l_run);
  const float inv = l_tot == 0.f ? 0.f : 1.0f / l_tot;
  const int row = row_w + (lane_anew() & 31);
  if (row < cs.rows && lane_anew() < 32) lse[lse_at(row)] = l_tot == 0.f ? -INFINITY : (m_run + __log2f(l_tot)) * kCLn2;
  __syncthreads();   // the rings are free: each wavefront turns its tile through a piece of them
  store_tile_rows_at<D>(smem + wave * (32 * RB), oacc, inv, rows_valid, out_row);
}

// One workgroup per (K/V head, tile): all K/V heads of one tile before the next (heads on consecutive XCDs: an XCD keeps to
// its heads), a sequence's last tile, which sees most, first.
template <int D, int W>
__global__ __launch_bounds__(W * 64, fwd_waves(D, W))
void cattn_fwd_kernel(const __bf16* __restrict__ q, const __bf16* __restrict__ k, const __bf16* __restrict__ v,
                      __bf16* __restrict__ out, float* __restrict__ lse, const XSegTable segs, const TileIndex ti,
                      const CausalShape sh) {
  constexpr int kRows = W * 32;
  const int kvh = blockIdx.x % sh.n_kv_heads;
  int seq, t;
  locate_tile_wave<VFM_MAX_XSEQS>(ti.cu, segs.n, blockIdx.x / sh.n_kv_heads, seq, t);
  const CausalSeq cs = causal_seq(segs, seq, sh.group);
  const int tq = (cs.rows + kRows - 1) / kRows - 1 - t;
  fwd_segment<D, W>(q, k, v, out, lse, segs, sh, kvh, seq, tq, 0, tile_units(cs.rows, cs.off, sh.group, kRows, tq), nullptr);
}

// ---------------------------------------------------------------- few tiles, many keys
// The line of units that a piece is cut from: see make_split in cattn_plan.h.
__device__ __forceinline__ void split_tile(const SplitPlan& plan, const CausalShape& sh, int rows_per_tile, int tile, int& seq, int& tq, int& units) {
  int t;
  locate_tile_wave<kSplitSeqs>(plan.cu, plan.n, tile, seq, t);
  const CausalSeq cs = causal_seq(plan, seq, sh.group);
  tq = (cs.rows + rows_per_tile - 1) / rows_per_tile - 1 - t;
  units = tile_units(cs.rows, cs.off, sh.group, rows_per_tile, tq);
}

template <int D, int W>
__global__ __launch_bounds__(W * 64, split_waves(D, W))
void cattn_fwd_split_kernel(const __bf16* __restrict__ q, const __bf16* __restrict__ k, const __bf16* __restrict__ v,
                            __bf16* __restrict__ out, float* __restrict__ lse, const SplitPlan plan, const CausalShape sh,
                            float* __restrict__ slots) {
  const int kvh = blockIdx.x % sh.n_kv_heads, piece = blockIdx.x / sh.n_kv_heads;
  const uint32_t from = plan.start[piece], to = plan.start[piece + 1];
  int tile = from >> 16, u = from & 0xffff;
  for (bool first = true; (((uint32_t)tile << 16) | (uint32_t)u) < to; first = false) {
    int seq, tq, units;
    split_tile(plan, sh, W * 32, tile, seq, tq, units);
    const int end = tile < (int)(to >> 16) ? units : (int)(to & 0xffff);
    float* slot = u == 0 && end == units ? nullptr : slots + (size_t)(2 * blockIdx.x + (first ? 0 : 1)) * slot_floats<D, W>();
    if (!first) __syncthreads();
    fwd_segment<D, W>(q, k, v, out, lse, plan, sh, kvh, seq, tq, u, end, slot);
    ++tile;
    u = 0;
  }
}

// Joins the parts of the tile that piece boundary blockIdx.x + 1 cuts, if no earlier boundary cuts it.  Workgroup y of a tile
// takes 32 of its rows, a wavefront 32 columns of them and every fourth part, four of those at a time; the four shares
// are then summed in order.
constexpr int kJoinShares = 4;
template <int D, int W>
__global__ __launch_bounds__(D * 2 * kJoinShares)
void cattn_fwd_join_kernel(__bf16* __restrict__ out, float* __restrict__ lse, const SplitPlan plan, const CausalShape sh,
                           const float* __restrict__ slots) {
  const int kvh = blockIdx.x % sh.n_kv_heads, p = blockIdx.x / sh.n_kv_heads + 1;
  const uint32_t at = plan.start[p], prev = plan.start[p - 1];
  const int tile = at >> 16;
  if ((at & 0xffff) == 0 || at == prev) return;
  if ((int)(prev >> 16) == tile && (prev & 0xffff) != 0) return;
  int seq, tq, units;
  split_tile(plan, sh, W * 32, tile, seq, tq, units);
  const CausalSeq cs = causal_seq(plan, seq, sh.group);
  __shared__ __attribute__((aligned(16))) float shares[(kJoinShares - 1) * (D / 32)][18][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), db = wave % (D / 32), share = wave / (D / 32);
  const int lane = threadIdx.x & 63, c = lane & 31, g = lane >> 5;
  const int row_w = tq * W * 32 + blockIdx.y * 32;
  if (row_w >= cs.rows) return;
  // the tile's parts: pieces p - 1 .. last (empty pieces among them have none)
  int last = p;
  while (last + 1 < plan.pieces && (int)(plan.start[last + 1] >> 16) == tile) ++last;
  auto part = [&](int x) {
    // the tile is the first segment of every piece but the one that it begins within
    const bool later = x == p - 1 && prev < ((uint32_t)tile << 16);
    return slots + (size_t)(2 * (x * sh.n_kv_heads + kvh) + (later ? 1 : 0)) * slot_floats<D, W>() + blockIdx.y * (32 * D + 64);
  };
  float o[16], m = kCUnset, l = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) o[i] = 0.f;
  constexpr int kAtOnce = 4;
  for (int x0 = p - 1 + share; x0 <= last; x0 += kAtOnce * kJoinShares) {
    float pm[kAtOnce], pl[kAtOnce];
    f32x4 v[kAtOnce][4];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int x = x0 + i * kJoinShares;
      const bool there = x <= last && plan.start[x < plan.pieces ? x : 0] != plan.start[x < plan.pieces ? x + 1 : 0];
      pm[i] = kCUnset;
      pl[i] = 0.f;
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) v[i][q4] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (there) {
        const float* s = part(x);
        pm[i] = s[32 * D + 2 * c];
        pl[i] = s[32 * D + 2 * c + 1];
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) v[i][q4] = reinterpret_cast<const f32x4*>(s)[(db * 4 + q4) * 64 + lane];
      }
    }
    float mn = m;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) mn = fmaxf(mn, pm[i]);
    const float a = fast_exp2(m - mn);
    m = mn;
    l *= a;
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i] *= a;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const float b = fast_exp2(pm[i] - mn);
      l += pl[i] * b;
#pragma unroll
      for (int e = 0; e < 16; ++e) o[e] += v[i][e >> 2][e & 3] * b;
    }
  }
  if (share > 0) {
    float (*mine)[64] = shares[(share - 1) * (D / 32) + db];
#pragma unroll
    for (int i = 0; i < 16; ++i) mine[i][lane] = o[i];
    mine[16][lane] = m;
    mine[17][lane] = l;
  }
  __syncthreads();
  if (share > 0 || row_w + c >= cs.rows) return;
#pragma unroll
  for (int x = 0; x < kJoinShares - 1; ++x) {
    const float (*other)[64] = shares[x * (D / 32) + db];
    const float mn = fmaxf(m, other[16][lane]), a = fast_exp2(m - mn), b = fast_exp2(other[16][lane] - mn);
    m = mn;
    l = l * a + other[17][lane] * b;
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i] = o[i] * a + other[i][lane] * b;
  }
  const int row = row_w + c, tok = row / sh.group, head = kvh * sh.group + row - tok * sh.group;
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  if (db == 0 && g == 0) lse[(size_t)head * sh.total_q + cs.qs + tok] = l == 0.f ? -INFINITY : (m + __log2f(l)) * kCLn2;
  __bf16* dst = out + ((size_t)(cs.qs + tok) * sh.n_heads + head) * D + db * 32 + 4 * g;
#pragma unroll
  for (int q4 = 0; q4 < 4; ++q4)
    *reinterpret_cast<bf16x4*>(dst + 8 * q4) = to_bf16x4(f32x4{o[4 * q4], o[4 * q4 + 1], o[4 * q4 + 2], o[4 * q4 + 3]} * inv);
}

size_t cattn_fwd_workspace(const XSegTable& segs, const CausalShape& sh, int head_dim) {
  SplitPlan plan;
  const int rows = causal_rows(segs, sh, head_dim);
  if (!make_split(segs, sh, rows, head_dim, causal_slots(rows), &plan)) return 0;
  return (size_t)2 * plan.pieces * sh.n_kv_heads * (rows / 32) * (32 * head_dim + 64) * sizeof(float);
}

template <int D, int W>
static hipError_t launch_cfg(const __bf16* q, const __bf16* k, const __bf16* v, const XSegTable& segs, const CausalShape& sh,
                             __bf16* out, float* lse, float* workspace, hipStream_t stream) {
  using Cfg = CFwdCfg<D, W>;
  SplitPlan plan;
  if (make_split(segs, sh, Cfg::kRows, D, causal_slots(Cfg::kRows), &plan)) {
    auto kern = cattn_fwd_split_kernel<D, W>;
    hipError_t e = allow_lds(kern, Cfg::kLdsBytes);
    if (e != hipSuccess) return e;
    e = launch(kern, dim3(plan.pieces * sh.n_kv_heads), dim3(W * 64), Cfg::kLdsBytes, stream, q, k, v, out, lse, plan, sh, workspace);
    if (e != hipSuccess) return e;
    return launch(cattn_fwd_join_kernel<D, W>, dim3((plan.pieces - 1) * sh.n_kv_heads, W), dim3(D * 2 * kJoinShares), 0, stream, out, lse, plan, sh,
                  (const float*)workspace);
  }
  const TileIndex ti = make_causal_index<false>(segs, sh.group, Cfg::kRows);
  const int tiles = count_tiles(ti);
  if (tiles == 0) return hipSuccess;
  auto kern = cattn_fwd_kernel<D, W>;
  hipError_t e = allow_lds(kern, Cfg::kLdsBytes);
  if (e != hipSuccess) return e;
  return launch(kern, dim3((unsigned)tiles * sh.n_kv_heads), dim3(W * 64), Cfg::kLdsBytes, stream, q, k, v, out, lse, segs, ti, sh);
}

hipError_t launch_cattn_fwd(const void* q, const void* k, const void* v, const XSegTable& segs, const CausalShape& sh,
                            int head_dim, void* out, float* lse, void* workspace, hipStream_t stream) {
  const int rows = causal_rows(segs, sh, head_dim);
  auto run = head_dim == 64 ? (rows == 32 ? launch_cfg<64, 1> : rows == 64 ? launch_cfg<64, 2> : launch_cfg<64, 4>)
             : rows == 32   ? launch_cfg<128, 1>
             : rows == 64   ? launch_cfg<128, 2>
             : rows == 128  ? launch_cfg<128, 4>
                            : launch_cfg<128, 8>;
  return run((const __bf16*)q, (const __bf16*)k, (const __bf16*)v, segs, sh, (__bf16*)out, lse, (float*)workspace, stream);
}

}  // namespace vfm
