// Attention of the newest tokens over the paged 4-bit cache (gfx950): grouped heads, causal among the new tokens.
//
//     out_i = sum_j softmax_j(scale q_i . k_j) v_j,   j <= lens + t_i   (k_j, v_j: the values that the cache holds)
//
// Few rows against many keys: the cache is read once per row block and nothing else is big, so HBM bounds it (72 bytes of
// K and of V per token and head at head_dim 128 against 4 * 128 operations a row).  What follows from that:
//  - The cache's rows are read as they lie, 16 bytes of codes (32 elements) and their factor byte per lane.  The contraction of
//    the score product may run in any order, so a lane's 32 consecutive elements of K are its operand of four
//    16x16x32 MFMAs as they come, with Q held in the same order; one conversion instruction makes two bf16 and applies the factor.
//  - V is needed with keys along the contraction: its rows go through LDS (a wavefront's own 32 keys, no barrier) and come
//    back by transposing reads, the key order of the score MFMA's accumulators, so that P is an operand as it stands.
//  - The next 32 keys of a wavefront are in flight while the present ones are computed.
//  - The lengths are only known on the device (a captured step serves any), so the key blocks of all (sequence, K/V head, row
//    block) units form one line that every workgroup takes an equal piece of.  A unit that lies within one piece is
//    finished there; the others leave (maximum, sum, unnormalised output) per piece in the workspace, joined by a second
//    launch in the order of the pieces: no atomics, the same bits every time.
#include "kv4_common.h"

namespace vfm {

constexpr int kKvWaves = 4;
constexpr int kKvStep = 32;                          // keys per wavefront and step
constexpr int kKvBlockKeys = kKvWaves * kKvStep;     // a workgroup's step
constexpr int kKvThreads = kKvWaves * 64;
constexpr float kKvLog2e = 1.4426950408889634f;
constexpr float kKvLn2 = 0.6931471805599453f;
constexpr float kKvSafeSum = 256.f;
constexpr float kKvUnset = -3.0e38f;                 // reference of a row that has seen no key: every difference is finite or -inf

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

struct Kv4Shape {
  int n_heads, group, total, rb_rows;   // rb_rows: rows of a row block
  uint32_t q_row;                       // bytes between consecutive tokens of q
  float scale_log2;
};

// The line of key blocks.  Every workgroup works it out for itself from the lengths: before[s] = blocks of the sequences
// before s.
struct Kv4Line {
  int rb, nb;            // of the sequence: row blocks, key blocks
  int kvh, rblk;         // the unit: K/V head, row block
  long long at;          // first block of the unit
};
__device__ __forceinline__ int kv4_keys(const Kv4Cache& c, int len, int nq) {   // keys of a sequence
  if (len < 0 || nq == 0) return 0;
  const long long have = (long long)len + nq, room = (long long)c.max_pages << c.shift;
  const long long keys = have < room ? have : room;
  return (int)(keys < 0x7fffff00 ? keys : 0x7fffff00);
}
__device__ __forceinline__ int kv4_row_blocks(int nq, const Kv4Shape& sh) { return (nq * sh.group + sh.rb_rows - 1) / sh.rb_rows; }

// Fills before[0 .. 256] (LDS) for this run; returns the total.  All kKvThreads threads take part.
__device__ __forceinline__ long long kv4_scan(const Kv4Table& t, const Kv4Cache& c, const Kv4Shape& sh, long long* before, long long* part) {
  static_assert(kKvThreads == VFM_MAX_SEQS, "one sequence per thread");
  const int s = threadIdx.x, lane = s & 63, wave = s >> 6;
  long long mine = 0;
  if (s < t.n) {
    const int nq = t.cu[s + 1] - t.cu[s];
    const int keys = kv4_keys(c, c.lens[s], nq);
    mine = (long long)((keys + kKvBlockKeys - 1) / kKvBlockKeys) * kv4_row_blocks(nq, sh) * c.n_kv_heads;
  }
  long long sum = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const long long up = __shfl_up(sum, o);
    if (lane >= o) sum += up;
  }
  if (lane == 63) part[wave] = sum;
  __syncthreads();
  long long base = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kKvWaves; ++w) {
    if (w < wave) base += part[w];
    total += part[w];
  }
  before[s] = base + sum - mine;
  if (s == kKvThreads - 1) before[kKvThreads] = total;
  __syncthreads();
  return total;
}
// Sequence of block x: the last one that begins at or before it and has blocks
__device__ __forceinline__ int kv4_find(const long long* before, long long x) {
  int lo = 0, hi = VFM_MAX_SEQS;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (before[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

// A piece's results: per slot rb_rows rows of (reference, sum), then rb_rows rows of D values.
template <int D>
__device__ __forceinline__ size_t kv4_slot_floats(int rb_rows) { return (size_t)rb_rows * (D + 2); }

// Workgroups of a CU: what the registers allow
constexpr int kv4_per_cu(int D, int R) { return D == 128 ? (R == 1 ? 3 : R == 2 ? 2 : 1) : (R == 1 ? 4 : R == 2 ? 3 : 2); }

template <int D, int R>
__global__ __launch_bounds__(kKvThreads, kv4_per_cu(D, R))
void kv4_attn_kernel(const char* __restrict__ q, const Kv4Table t, const Kv4Cache c, const Kv4Shape sh,
                     __bf16* __restrict__ out, float* __restrict__ lse, float* __restrict__ slots) {
  constexpr int KS = D / 32;          // MFMAs of a 16-key score tile
  constexpr int DT = D / 16;          // 16-wide tiles of the head vector
  constexpr int LB = D / 8;           // bytes of codes per lane and key (a lane holds D/4 elements)
  constexpr int LW = LB / 4;
  constexpr int RB = D * 2;
  constexpr int kVBytes = kKvStep * RB;              // a wavefront's V tile
  constexpr int kORow = D + 4;                       // padded row of the join, floats
  constexpr int kJoin = kKvWaves * 16 * kORow * 4;
  __shared__ __attribute__((aligned(16))) char smem[kKvWaves * kVBytes > kJoin ? kKvWaves * kVBytes : kJoin];
  __shared__ long long before[VFM_MAX_SEQS + 1], part[kKvWaves];
  __shared__ float stat[2][kKvWaves][16];

  const long long total = kv4_scan(t, c, sh, before, part);
  const long long per = (total + gridDim.x - 1) / gridDim.x;
  long long x = (long long)blockIdx.x * per;
  const long long x_first = x, x_end = x + per < total ? x + per : total;
  if (x >= x_end) return;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int li = lane & 15, g = lane >> 4;           // key or row of a 16-tile; group of the contraction
  char* vt = smem + wave * kVBytes;

  while (x < x_end) {
    // ---- the unit that block x lies in
    const int s = __builtin_amdgcn_readfirstlane(kv4_find(before, x));
    const int q0 = t.cu[s], nq = t.cu[s + 1] - q0;
    const int len = c.lens[s];
    const int keys = kv4_keys(c, len, nq);
    const int nb = (keys + kKvBlockKeys - 1) / kKvBlockKeys;
    const int n_rb = kv4_row_blocks(nq, sh);
    const int unit = __builtin_amdgcn_readfirstlane((int)((x - before[s]) / nb));
    const long long u0 = before[s] + (long long)unit * nb;
    const int kvh = unit / n_rb, rblk = unit - kvh * n_rb;
    const int b0 = __builtin_amdgcn_readfirstlane((int)(x - u0));
    const int b1 = __builtin_amdgcn_readfirstlane((int)((u0 + nb < x_end ? u0 + nb : x_end) - u0));
    const bool whole = b0 == 0 && b1 == nb;
    const int rows = nq * sh.group, r0 = rblk * (16 * R);

    // ---- Q rows (B operand: lane row li, elements g*D/4 ..) and the last key each sees
    bf16x8 qreg[R][KS];
    int lim[R];
#pragma unroll
    for (int rt = 0; rt < R; ++rt) {
      const int row = min(r0 + rt * 16 + li, rows - 1), tok = row / sh.group;
      const char* qp = q + (size_t)(q0 + tok) * sh.q_row + (size_t)(kvh * sh.group + row - tok * sh.group) * RB + g * (D / 2);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) qreg[rt][ks] = *reinterpret_cast<const bf16x8*>(qp + ks * 16);
      lim[rt] = min(len + tok, keys - 1);
    }
    const int lim_min = min(len + min(r0, rows - 1) / sh.group, keys - 1);   // (rows of a block: the first sees least)

    f32x4 o[R][DT];
    float m_run[R], l_run[R];
#pragma unroll
    for (int rt = 0; rt < R; ++rt) {
      m_run[rt] = kKvUnset;
      l_run[rt] = 0.f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[rt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // ---- 32 keys of the cache on their way
    struct Fetch { uint32_t k[2][LW], v[2][LW], kf[2], vf[2]; };
    auto fetch = [&](int blk, Fetch& f) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int j0 = blk * kKvBlockKeys + wave * kKvStep + 16 * h;    // (16 keys lie in one page)
        const int page = j0 < keys ? kv4_page(c, s, j0) : -1;
        const bool there = page >= 0 && j0 + li < keys;
        if (there) {
          const size_t row = kv4_row(c, page, kvh, j0) + li;
          const uint32_t* kp = reinterpret_cast<const uint32_t*>(c.k4 + row * (D / 2) + g * LB);
          const uint32_t* vp = reinterpret_cast<const uint32_t*>(c.v4 + row * (D / 2) + g * LB);
          if constexpr (LW == 4) {
            const u32x4 a = *reinterpret_cast<const u32x4*>(kp), b = *reinterpret_cast<const u32x4*>(vp);
#pragma unroll
            for (int i = 0; i < LW; ++i) { f.k[h][i] = a[i]; f.v[h][i] = b[i]; }
          } else {
            const u32x2 a = *reinterpret_cast<const u32x2*>(kp), b = *reinterpret_cast<const u32x2*>(vp);
#pragma unroll
            for (int i = 0; i < LW; ++i) { f.k[h][i] = a[i]; f.v[h][i] = b[i]; }
          }
          f.kf[h] = c.ks[row * (D / kKv4Block) + g * D / 128];
          f.vf[h] = c.vs[row * (D / kKv4Block) + g * D / 128];
        } else {       // past the end, or no such page: nothing that any row sees, and zeros where P = 0 meets V
#pragma unroll
          for (int i = 0; i < LW; ++i) f.k[h][i] = f.v[h][i] = 0;
          f.kf[h] = page < 0 ? 256u : 127u;
          f.vf[h] = 127u;
        }
      }
    };

    Fetch cur, nxt;
    fetch(b0, cur);
    for (int blk = b0; blk < b1; ++blk) {
      if (blk + 1 < b1) fetch(blk + 1, nxt);
      const int j0 = blk * kKvBlockKeys + wave * kKvStep;
      // blocks that held a NaN or an infinity make the scores of their keys NaN and weigh nothing themselves
      uint32_t poison = 0, gone = 0;     // bits: keys of the 32
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint64_t bad = __builtin_amdgcn_ballot_w64(cur.kf[h] == kKv4Nan || cur.vf[h] == kKv4Nan);
        if (bad) {
          bad |= bad >> 32;
          bad |= bad >> 16;
          poison |= (uint32_t)(bad & 0xffff) << (16 * h);
          if (cur.kf[h] == kKv4Nan) cur.kf[h] = 127;
          if (cur.vf[h] == kKv4Nan) cur.vf[h] = 127;
        }
        if (__builtin_amdgcn_ballot_w64(cur.kf[h] == 256u) != 0) gone |= 0xffffu << (16 * h);
      }
      // ---- V: to bf16, through LDS
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < LW; ++i)
          *reinterpret_cast<bf16x8*>(vt + tile_off<D>(16 * h + li, g * (D / 4) + 8 * i)) = kv4_values(cur.v[h][i], kv4_factor(cur.vf[h]));
      // ---- S^T = K Q^T: lane holds row li of the queries, keys 4g .. 4g+3 of each 16
      f32x4 sc[R][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const bf16x8 ka = kv4_values(cur.k[h][ks], kv4_factor(cur.kf[h] & 255u));
#pragma unroll
          for (int rt = 0; rt < R; ++rt)
            sc[rt][h] = mfma16(ka, qreg[rt][ks], ks == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : sc[rt][h]);
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      bf16x8 pb[R];
#pragma unroll
      for (int rt = 0; rt < R; ++rt) {
        if (poison | gone) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t bit = 1u << (16 * h + 4 * g + e);
              if (poison & bit) sc[rt][h][e] = __builtin_nanf("");
              if (gone & bit) sc[rt][h][e] = -INFINITY;
            }
        }
        if (j0 + kKvStep - 1 > lim_min) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (j0 + 16 * h + 4 * g + e > lim[rt]) sc[rt][h][e] = -INFINITY;
        }
        f32x8 p;
        float lsum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = fast_exp2(sc[rt][e >> 2][e & 3] * sh.scale_log2 - m_run[rt]);
          lsum += p[e];
        }
        // the reference moves only when the exponentials would grow too large (or are the row's first)
        if (__builtin_amdgcn_ballot_w64(!(lsum <= kKvSafeSum)) != 0) {
          float mx = sc[rt][0][0];
#pragma unroll
          for (int e = 1; e < 8; ++e) mx = fmaxf(mx, sc[rt][e >> 2][e & 3]);
          mx = fmaxf(mx, __shfl_xor(mx, 16));
          mx = pair_max(mx);
          const float m_new = fmaxf(m_run[rt], mx * sh.scale_log2);
          const float alpha = fast_exp2(m_run[rt] - m_new);
          m_run[rt] = m_new;
          lsum = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            p[e] = fast_exp2(sc[rt][e >> 2][e & 3] * sh.scale_log2 - m_new);
            lsum += p[e];
          }
          l_run[rt] *= alpha;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) o[rt][dt] *= alpha;
        }
        l_run[rt] += lsum;
        pb[rt] = to_bf16x8(p);
      }
      // ---- O^T += V^T P^T, contraction slots 8g + e: keys 4g + e (e < 4) and 16 + 4g + e - 4
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const int col = dt * 16 + 4 * (lane & 3), r = 4 * g + ((lane & 15) >> 2);
        const bf16x8 va = join_tr(lds_read_tr(vt, tile_off<D>(r, col)), lds_read_tr(vt, tile_off<D>(16 + r, col)));
#pragma unroll
        for (int rt = 0; rt < R; ++rt) o[rt][dt] = mfma16(va, pb[rt], o[rt][dt]);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      cur = nxt;
    }

    // ---- join the four wavefronts, one row tile at a time
#pragma unroll
    for (int rt = 0; rt < R; ++rt) {
      if (r0 + rt * 16 >= rows) break;
      float l = l_run[rt];
      l += __shfl_xor(l, 16);
      l = pair_sum(l);
      __syncthreads();       // everyone is done with the V tiles, and with the row tile before
      if (g == 0) { stat[0][wave][li] = m_run[rt]; stat[1][wave][li] = l; }
      float* ow = reinterpret_cast<float*>(smem) + (wave * 16 + li) * kORow + 4 * g;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4*>(ow + dt * 16) = o[rt][dt];
      __syncthreads();
      constexpr int TPR = kKvThreads / 16, CPT = D / TPR;    // threads per row, columns per thread
      const int row = tid / TPR, col = (tid % TPR) * CPT;
      const int at = r0 + rt * 16 + row;
      float m = stat[0][0][row];
#pragma unroll
      for (int w = 1; w < kKvWaves; ++w) m = fmaxf(m, stat[0][w][row]);
      float sum = 0.f, acc[CPT];
#pragma unroll
      for (int i = 0; i < CPT; ++i) acc[i] = 0.f;
#pragma unroll
      for (int w = 0; w < kKvWaves; ++w) {
        const float f = fast_exp2(stat[0][w][row] - m);
        sum += stat[1][w][row] * f;
#pragma unroll
        for (int i = 0; i < CPT; ++i) acc[i] += reinterpret_cast<const float*>(smem)[(w * 16 + row) * kORow + col + i] * f;
      }
      if (at < rows) {
        if (whole) {
          const int tok = at / sh.group, head = kvh * sh.group + at - tok * sh.group;
          const float inv = sum == 0.f ? 0.f : 1.f / sum;
          __bf16* op = out + ((size_t)(q0 + tok) * sh.n_heads + head) * D + col;
#pragma unroll
          for (int i = 0; i < CPT; ++i) op[i] = (__bf16)(acc[i] * inv);
          if (col == 0) lse[(size_t)head * sh.total + q0 + tok] = sum == 0.f ? -INFINITY : (m + __log2f(sum)) * kKvLn2;
        } else {
          float* sp = slots + (size_t)(2 * blockIdx.x + (x > x_first ? 1 : 0)) * kv4_slot_floats<D>(sh.rb_rows);
          const int rr = rt * 16 + row;
          if (col == 0) { sp[2 * rr] = m; sp[2 * rr + 1] = sum; }
#pragma unroll
          for (int i = 0; i < CPT; ++i) sp[2 * sh.rb_rows + rr * D + col + i] = acc[i];
        }
      }
    }
    x = u0 + b1;
    __syncthreads();         // the join's LDS is the next unit's
  }
}

// Joins the pieces of every unit that more than one workgroup worked on, and writes the rows of sequences that have nothing
// to look at.  blockIdx.x: (unit, row of its row block); units as in the line: sequence, K/V head, row block.
template <int D>
__global__ __launch_bounds__(kKvThreads) void kv4_join_kernel(const Kv4Table t, const Kv4Cache c, const Kv4Shape sh, int pieces,
                                                              __bf16* __restrict__ out, float* __restrict__ lse,
                                                              const float* __restrict__ slots) {
  constexpr int TPP = D / 4, PAR = kKvThreads / TPP;     // threads per piece, pieces at a time
  __shared__ long long before[VFM_MAX_SEQS + 1], part[kKvWaves];
  __shared__ float red[PAR][D + 1], redm[PAR];
  const long long total = kv4_scan(t, c, sh, before, part);
  const long long per = (total + pieces - 1) / pieces;

  // output row blockIdx.x: token-major, head-minor
  const int tok_all = t.cu[0] + blockIdx.x / sh.n_heads, head = blockIdx.x % sh.n_heads;
  const int s = kv4_seq_of(t, tok_all);
  const int q0 = t.cu[s], nq = t.cu[s + 1] - q0, tok = tok_all - q0;
  const int keys = kv4_keys(c, c.lens[s], nq);
  const int kvh = head / sh.group, row = tok * sh.group + head - kvh * sh.group;
  __bf16* op = out + ((size_t)tok_all * sh.n_heads + head) * D;
  float* lp = lse + (size_t)head * sh.total + tok_all;
  const int tid = threadIdx.x;
  if (keys == 0) {
    if (tid < D) op[tid] = (__bf16)0.f;
    if (tid == 0) *lp = -INFINITY;
    return;
  }
  const int nb = (keys + kKvBlockKeys - 1) / kKvBlockKeys;
  const int n_rb = kv4_row_blocks(nq, sh), rblk = row / sh.rb_rows, rr = row - rblk * sh.rb_rows;
  const long long u0 = before[s] + (long long)(kvh * n_rb + rblk) * nb, u1 = u0 + nb;
  const int p0 = (int)(u0 / per), p1 = (int)((u1 - 1) / per);
  if (p0 == p1) return;                                  // one workgroup had all of it
  auto slot = [&](int p) {                               // the unit is the piece's second, last one where it begins inside the piece
    const bool inside = p == p0 && u0 > (long long)p * per;
    return slots + (size_t)(2 * p + (inside ? 1 : 0)) * kv4_slot_floats<D>(sh.rb_rows);
  };
  const int sub = tid / TPP, col = (tid % TPP) * 4;
  float m = kKvUnset, l = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int p = p0 + sub; p <= p1; p += PAR) {
    const float* sp = slot(p);
    const float pm = sp[2 * rr], pl = sp[2 * rr + 1];
    const f32x4 v = *reinterpret_cast<const f32x4*>(sp + 2 * sh.rb_rows + rr * D + col);
    const float mn = fmaxf(m, pm), a = fast_exp2(m - mn), b = fast_exp2(pm - mn);
    m = mn;
    l = l * a + pl * b;
    acc = acc * a + v * b;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) red[sub][col + i] = acc[i];
  if (col == 0) { red[sub][D] = l; redm[sub] = m; }
  __syncthreads();
  if (tid < D) {
    float mm = redm[0];
#pragma unroll
    for (int i = 1; i < PAR; ++i) mm = fmaxf(mm, redm[i]);
    float sum = 0.f, v = 0.f;
#pragma unroll
    for (int i = 0; i < PAR; ++i) {
      const float f = fast_exp2(redm[i] - mm);
      sum += red[i][D] * f;
      v += red[i][tid] * f;
    }
    op[tid] = (__bf16)(sum == 0.f ? 0.f : v / sum);
    if (tid == 0) *lp = sum == 0.f ? -INFINITY : (mm + __log2f(sum)) * kKvLn2;
  }
}

// Row tiles of 16 that a workgroup takes at once: the rows of the call's longest sequence, up to 64.  More share each key that
// is fetched and converted; fewer leave more workgroups and registers to fetches.
static int row_tiles(const int32_t* cu, int n, int group) {
  int most = 0;
  for (int s = 0; s < n; ++s) most = most > cu[s + 1] - cu[s] ? most : cu[s + 1] - cu[s];
  const long long rows = (long long)most * group;
  return rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
}
// Workgroups that share the line: as many as the chip holds at once.
static int pieces_of(int head_dim, int r) { return compute_unit_count() * kv4_per_cu(head_dim, r); }

size_t kv4_attn_workspace(const int32_t* cu, int n_seqs, int n_heads, int n_kv_heads, int head_dim) {
  size_t most = 0;
  for (int s0 = 0; s0 < n_seqs; s0 += VFM_MAX_SEQS) {
    const int r = row_tiles(cu + s0, n_seqs - s0 < VFM_MAX_SEQS ? n_seqs - s0 : VFM_MAX_SEQS, n_heads / n_kv_heads);
    const size_t need = (size_t)2 * pieces_of(head_dim, r) * 16 * r * (head_dim + 2) * sizeof(float);
    most = need > most ? need : most;
  }
  return most;
}

hipError_t launch_kv4_attn(const void* q, uint32_t q_row, const Kv4Table& t, const Kv4Cache& c, int n_heads, int total,
                           int head_dim, float scale, void* out, float* lse, void* workspace, hipStream_t stream) {
  const int rows_out = (t.cu[t.n] - t.cu[0]) * n_heads;
  if (rows_out == 0) return hipSuccess;
  const int group = n_heads / c.n_kv_heads;
  const int r = row_tiles(t.cu, t.n, group);
  const Kv4Shape sh{n_heads, group, total, 16 * r, q_row, scale * kKvLog2e};
  const int pieces = pieces_of(head_dim, r);
  auto pick = [&](auto d_c) {
    constexpr int D = decltype(d_c)::value;
    return r == 1 ? kv4_attn_kernel<D, 1> : r == 2 ? kv4_attn_kernel<D, 2> : kv4_attn_kernel<D, 4>;
  };
  auto kern = head_dim == 128 ? pick(IntC<128>{}) : pick(IntC<64>{});
  hipError_t e = launch(kern, dim3(pieces), dim3(kKvThreads), 0, stream, (const char*)q, t, c, sh, (__bf16*)out, lse, (float*)workspace);
  if (e != hipSuccess) return e;
  auto join = head_dim == 128 ? kv4_join_kernel<128> : kv4_join_kernel<64>;
  return launch(join, dim3(rows_out), dim3(kKvThreads), 0, stream, t, c, sh, pieces, (__bf16*)out, lse, (const float*)workspace);
}

}  // namespace vfm
