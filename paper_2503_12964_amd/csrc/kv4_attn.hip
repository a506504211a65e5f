// Attention of the newest tokens over the paged 4-bit cache (gfx950): grouped heads, causal among the new tokens.
//
//     out_i = sum_j softmax_j(scale q_i . k_j) v_j,   j <= lens + t_i   (k_j, v_j: the values that the cache holds)
//
// Few rows against many keys: the cache is read once per row block and nothing else is big, so HBM bounds it (68 bytes of
// K and of V per token and head at head_dim 128 against 4 * 128 operations a row).  What follows from that:
//  - The cache's rows are read as they lie, 16 bytes of codes (32 elements) and their factor byte per lane.  The contraction of
//    the score product may run in any order, so a lane's 32 consecutive elements of K are its operand of four
//    16x16x32 MFMAs as they come, with Q held in the same order; one conversion instruction makes two bf16 and applies the factor.
//  - V is needed with keys along the contraction: its rows go through LDS (a wavefront's own 32 keys, no barrier) and come
//    back by transposing reads, the key order of the score MFMA's accumulators, so that P is an operand as it stands.
//  - The next 32 keys of a wavefront are in flight while the present ones are computed; the pages of its next 32 steps sit in
//    one register, a lane each, so that no fetch waits for a page number.
//  - The lengths are only known on the device (a captured step serves any), so the key blocks of all (sequence, K/V head, row
//    block) units form one line that every workgroup takes an equal piece of.  A unit that lies within one piece is
//    finished there; the others leave (maximum, sum, unnormalised output) per piece in the workspace, joined by a second
//    launch in the order of the pieces: no atomics, the same bits every time.
// Measured in a captured graph, both launches: 64 sequences of 4000 keys, 32/8 heads, 55 us at head_dim 128 (279 MB, 5.1 TB/s;
// the fetches alone, nothing computed: 54), 36 us at 64; one sequence of 100000 keys, 16/1 heads: 31 us, 9 of them the join and its
// launch.
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

// The line of key blocks.  Every workgroup works it out for itself from the lengths.
__device__ __forceinline__ int kv4_keys(const Kv4Cache& c, int len, int nq) {   // keys of a sequence
  if (len < 0 || nq == 0) return 0;
  const long long have = (long long)len + nq, room = (long long)c.max_pages << c.shift;
  const long long keys = have < room ? have : room;
  return (int)(keys < 0x7fffff00 ? keys : 0x7fffff00);
}
__device__ __forceinline__ int kv4_last(int len, int tok, int keys) {   // the last key that new token tok sees
  const long long last = (long long)len + tok;                          // (a length may lie far past the table)
  return last < keys ? (int)last : keys - 1;
}
__device__ __forceinline__ int kv4_row_blocks(int nq, const Kv4Shape& sh) { return (nq * sh.group + sh.rb_rows - 1) / sh.rb_rows; }

// Fills before[] (blocks of the sequences before each) and lens for this run; returns the total.  All kKvThreads threads take part.
struct Kv4Scan {
  long long before[VFM_MAX_SEQS + 1], part[kKvWaves];
  int lens[VFM_MAX_SEQS];
};
__device__ __forceinline__ long long kv4_scan(const Kv4Table& t, const Kv4Cache& c, const Kv4Shape& sh, Kv4Scan& m) {
  static_assert(kKvThreads == VFM_MAX_SEQS, "one sequence per thread");
  const int s = threadIdx.x, lane = s & 63, wave = s >> 6;
  long long mine = 0;
  if (s < t.n) {
    const int nq = t.cu[s + 1] - t.cu[s], len = c.lens[s];
    const int keys = kv4_keys(c, len, nq);
    m.lens[s] = len;
    mine = (long long)((keys + kKvBlockKeys - 1) / kKvBlockKeys) * kv4_row_blocks(nq, sh) * c.n_kv_heads;
  }
  long long sum = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const long long up = __shfl_up(sum, o);
    if (lane >= o) sum += up;
  }
  if (lane == 63) m.part[wave] = sum;
  __syncthreads();
  long long base = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kKvWaves; ++w) {
    if (w < wave) base += m.part[w];
    total += m.part[w];
  }
  m.before[s] = base + sum - mine;
  if (s == kKvThreads - 1) m.before[kKvThreads] = total;
  __syncthreads();
  return total;
}
// Sequence of block x: the last one that begins at or before it (of several that begin there the last, the others are empty)
__device__ __forceinline__ int kv4_find(const long long* before, long long x) {
  const int lane = threadIdx.x & 63;
  int n = 0;
#pragma unroll
  for (int i = 0; i < VFM_MAX_SEQS; i += 64) n += __builtin_popcountll(__builtin_amdgcn_ballot_w64(before[i + lane] <= x));
  return __builtin_amdgcn_readfirstlane(n - 1);
}

// The workspace: the line's before[] for the join, then slots.  A piece's results: per slot rb_rows rows of (reference, sum), then
// rb_rows rows of D values.
constexpr size_t kKvHead = (VFM_MAX_SEQS + 1 + 7) / 8 * 8 * sizeof(long long);
template <int D>
__device__ __forceinline__ size_t kv4_slot_floats(int rb_rows) { return (size_t)rb_rows * (D + 2); }

// Workgroups of a CU: what the registers allow.  (At head_dim 128 and one row tile three would fit: 62 us instead of 55 at 64
// sequences of 4000 keys, the line cut into more pieces than the fetches of two leave room for.)
constexpr int kv4_per_cu(int D, int R) { return D == 128 ? (R <= 2 ? 2 : 1) : (R == 1 ? 4 : 2); }

template <int D, int R>
__global__ __launch_bounds__(kKvThreads, kv4_per_cu(D, R))
void kv4_attn_kernel(const char* __restrict__ q, const Kv4Table t, const Kv4Cache c, const Kv4Shape sh,
                     __bf16* __restrict__ out, float* __restrict__ lse, char* __restrict__ workspace) {
  constexpr int KS = D / 32;          // MFMAs of a 16-key score tile
  constexpr int DT = D / 16;          // 16-wide tiles of the head vector
  constexpr int LB = D / 8;           // bytes of codes per lane and key (a lane holds D/4 elements)
  constexpr int LW = LB / 4;
  constexpr int RB = D * 2;
  constexpr int kVBytes = kKvStep * RB;              // a wavefront's V tile
  constexpr int kORow = D + 4;                       // padded row of the join, floats
  constexpr int kJoin = kKvWaves * 16 * kORow * 4;
  __shared__ __attribute__((aligned(16))) char smem[kKvWaves * kVBytes > kJoin ? kKvWaves * kVBytes : kJoin];
  __shared__ Kv4Scan scan;
  __shared__ float stat[2][kKvWaves][16];
  float* const slots = reinterpret_cast<float*>(workspace + kKvHead);
  const long long* before = scan.before;

  const long long total = kv4_scan(t, c, sh, scan);
  if (blockIdx.x == 0) {
    reinterpret_cast<long long*>(workspace)[threadIdx.x] = before[threadIdx.x];
    if (threadIdx.x == 0) reinterpret_cast<long long*>(workspace)[VFM_MAX_SEQS] = total;
  }
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
    const int s = kv4_find(before, x);
    const int q0 = t.cu[s], nq = t.cu[s + 1] - q0;
    const int len = __builtin_amdgcn_readfirstlane(scan.lens[s]);
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
      lim[rt] = kv4_last(len, tok, keys);
    }
    const int lim_min = kv4_last(len, min(r0, rows - 1) / sh.group, keys);   // (rows of a block: the first sees least)

    f32x4 o[R][DT];
    float m_run[R], l_run[R];
#pragma unroll
    for (int rt = 0; rt < R; ++rt) {
      m_run[rt] = kKvUnset;
      l_run[rt] = 0.f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[rt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // ---- pages of 32 steps: lane l holds that of step l / 2, 16-key half l % 2 (which lies in one page), -1 where there is none
    int pages, pages_at;
    auto take_pages = [&](int blk) {
      const long long j = ((long long)blk + (lane >> 1)) * kKvBlockKeys + wave * kKvStep + 16 * (lane & 1);
      pages = j < keys ? kv4_page(c, s, j) : -1;
      pages_at = blk;
    };
    // ---- 32 keys of the cache on their way.  No lane is masked out: places of the last page past the sequence's end are read like
    // the others (and given the factor 1 below), a half without a page reads page 0 in its place.
    struct Fetch { uint32_t k[2][LW], v[2][LW], factors, gone; };   // factors: see unpack; gone: bit h: half h has no page
    auto fetch = [&](int blk, Fetch& f) {
      const int j0 = blk * kKvBlockKeys + wave * kKvStep, at = 2 * (blk - pages_at);
      const int page[2] = {__builtin_amdgcn_readlane(pages, at), __builtin_amdgcn_readlane(pages, at + 1)};
      f.gone = (page[0] < 0 ? 1u : 0u) | (page[1] < 0 ? 2u : 0u);
      uint64_t row[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        row[h] = kv4_row(c, max(page[h], 0), kvh, j0 + 16 * h);
        const uint8_t* kp = c.k4 + row[h] * (D / 2) + (uint32_t)(li * (D / 2) + g * LB);
        const uint8_t* vp = c.v4 + row[h] * (D / 2) + (uint32_t)(li * (D / 2) + g * LB);
        if constexpr (LW == 4) {
          const u32x4 a = *reinterpret_cast<const u32x4*>(kp), b = *reinterpret_cast<const u32x4*>(vp);
#pragma unroll
          for (int i = 0; i < LW; ++i) { f.k[h][i] = a[i]; f.v[h][i] = b[i]; }
        } else {
          const u32x2 a = *reinterpret_cast<const u32x2*>(kp), b = *reinterpret_cast<const u32x2*>(vp);
#pragma unroll
          for (int i = 0; i < LW; ++i) { f.k[h][i] = a[i]; f.v[h][i] = b[i]; }
        }
      }
      // the factor bytes of all 32 keys' K and V rows in one load: 16 lanes each for K keys 0.., 16.., V keys 0.., 16..
      // (addresses chosen as integers: a select of pointers would be a load of unknown address space, which the LDS
      // counter waits for too)
      const uint64_t addr = (lane & 32 ? (uint64_t)c.vs : (uint64_t)c.ks) + ((lane & 16) ? row[1] : row[0]) * (D / kKv4Block) +
                            (uint32_t)(li * (D / kKv4Block));
      if constexpr (D == 128) f.factors = *reinterpret_cast<const __attribute__((address_space(1))) uint32_t*>(addr);
      else f.factors = *reinterpret_cast<const __attribute__((address_space(1))) uint16_t*>(addr);
    };
    // The factor byte of this lane's block of K and of V, for both halves: each row of 16 lanes to all rows, then the block's byte
    auto unpack = [&](uint32_t w, uint32_t (&kf)[2], uint32_t (&vf)[2]) {
      const auto x = __builtin_amdgcn_permlane32_swap(w, w, false, false);      // rows {0, 1, 0, 1}, {2, 3, 2, 3}
      const auto k2 = __builtin_amdgcn_permlane16_swap(x[0], x[0], false, false);
      const auto v2 = __builtin_amdgcn_permlane16_swap(x[1], x[1], false, false);
      const int shift = 8 * (g * D / 128);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        kf[h] = (k2[h] >> shift) & 255u;
        vf[h] = (v2[h] >> shift) & 255u;
      }
    };

    auto step = [&](int blk, const Fetch& cur) {
      const int j0 = blk * kKvBlockKeys + wave * kKvStep;
      uint32_t kf[2], vf[2];
      unpack(cur.factors, kf, vf);
      // what no row sees has finite values (its weight is 0): places past the end, halves without a page
      if (j0 + kKvStep > keys || cur.gone) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (j0 + 16 * h + li >= keys || ((cur.gone >> h) & 1)) kf[h] = vf[h] = 127;
      }
      // blocks that held a NaN or an infinity make the scores of their keys NaN and weigh nothing themselves
      uint32_t poison = 0, gone = 0;     // bits: keys of the 32
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint64_t bad = __builtin_amdgcn_ballot_w64(kf[h] == kKv4Nan || vf[h] == kKv4Nan);
        if (bad) {
          bad |= bad >> 32;
          bad |= bad >> 16;
          poison |= (uint32_t)(bad & 0xffff) << (16 * h);
          if (kf[h] == kKv4Nan) kf[h] = 127;
          if (vf[h] == kKv4Nan) vf[h] = 127;
        }
        if ((cur.gone >> h) & 1) gone |= 0xffffu << (16 * h);
      }
      // ---- V: to bf16, through LDS
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < LW; ++i)
          *reinterpret_cast<bf16x8*>(vt + tile_off<D>(16 * h + li, g * (D / 4) + 8 * i)) = kv4_values(cur.v[h][i], kv4_factor(vf[h]));
      // ---- S^T = K Q^T: lane holds row li of the queries, keys 4g .. 4g+3 of each 16
      f32x4 sc[R][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const bf16x8 ka = kv4_values(cur.k[h][ks], kv4_factor(kf[h]));
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
    };
    // Two sets of registers in turn (copied from one to the other, a fetch would be waited for at the copy), and a fetch on every
    // path (at the end of the last block again), so that what is waited for is the older one only.
    auto ask = [&](int blk, Fetch& f) {
      blk = min(blk, b1 - 1);
      if (blk - pages_at == 32) take_pages(blk);
      fetch(blk, f);
    };
    if (c.n_pages > 0) {       // (a cache without pages has no memory at all)
      Fetch even, odd;
      take_pages(b0);
      fetch(b0, even);
      for (int blk = b0; blk < b1; blk += 2) {
        ask(blk + 1, odd);
        step(blk, even);
        if (blk + 1 >= b1) break;
        ask(blk + 2, even);
        step(blk + 1, odd);
      }
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
// to look at.  blockIdx.x: output row, token-major, head-minor.  D / 4 threads share a piece, four pieces each at a time.
template <int D>
__global__ __launch_bounds__(kKvThreads) void kv4_join_kernel(const Kv4Table t, const Kv4Cache c, const Kv4Shape sh, int pieces,
                                                              __bf16* __restrict__ out, float* __restrict__ lse,
                                                              const char* __restrict__ workspace) {
  constexpr int TPP = D / 4, PAR = kKvThreads / TPP;     // threads per piece, pieces at a time
  constexpr int kAtOnce = 4;
  __shared__ float red[PAR][D + 1], redm[PAR];
  const float* slots = reinterpret_cast<const float*>(workspace + kKvHead);
  const long long* before = reinterpret_cast<const long long*>(workspace);
  const int tok_all = t.cu[0] + blockIdx.x / sh.n_heads, head = blockIdx.x % sh.n_heads;
  const int tid = threadIdx.x, lane = tid & 63;
  int s = -1;                                            // the last sequence that begins at or before the token
#pragma unroll
  for (int i = 0; i < VFM_MAX_SEQS; i += 64) s += __builtin_popcountll(__builtin_amdgcn_ballot_w64(i + lane < t.n && t.cu[i + lane] <= tok_all));
  s = __builtin_amdgcn_readfirstlane(s);
  const int q0 = t.cu[s], nq = t.cu[s + 1] - q0, tok = tok_all - q0;
  const int keys = kv4_keys(c, c.lens[s], nq);
  const long long total = before[VFM_MAX_SEQS], first = before[s];
  const long long per = (total + pieces - 1) / pieces;
  const int kvh = head / sh.group, row = tok * sh.group + head - kvh * sh.group;
  __bf16* op = out + ((size_t)tok_all * sh.n_heads + head) * D;
  float* lp = lse + (size_t)head * sh.total + tok_all;
  if (keys == 0) {
    if (tid < D) op[tid] = (__bf16)0.f;
    if (tid == 0) *lp = -INFINITY;
    return;
  }
  const int nb = (keys + kKvBlockKeys - 1) / kKvBlockKeys;
  const int n_rb = kv4_row_blocks(nq, sh), rblk = row / sh.rb_rows, rr = row - rblk * sh.rb_rows;
  const long long u0 = first + (long long)(kvh * n_rb + rblk) * nb, u1 = u0 + nb;
  const int p0 = (int)(u0 / per), p1 = (int)((u1 - 1) / per);
  if (p0 == p1) return;                                  // one workgroup had all of it
  const int sub = tid / TPP, col = (tid % TPP) * 4;
  float m = kKvUnset, l = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int p = p0 + sub; p <= p1; p += PAR * kAtOnce) {
    float pm[kAtOnce], pl[kAtOnce];
    f32x4 v[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int x = p + i * PAR;
      pm[i] = kKvUnset;
      pl[i] = 0.f;
      v[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (x <= p1) {
        // the unit is the piece's second, last one where it begins inside the piece
        const bool inside = x == p0 && u0 > (long long)x * per;
        const float* sp = slots + (size_t)(2 * x + (inside ? 1 : 0)) * kv4_slot_floats<D>(sh.rb_rows);
        pm[i] = sp[2 * rr];
        pl[i] = sp[2 * rr + 1];
        v[i] = *reinterpret_cast<const f32x4*>(sp + 2 * sh.rb_rows + rr * D + col);
      }
    }
    float mn = m;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) mn = fmaxf(mn, pm[i]);
    const float a = fast_exp2(m - mn);
    m = mn;
    l *= a;
    acc *= a;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const float b = fast_exp2(pm[i] - mn);
      l += pl[i] * b;
      acc += v[i] * b;
    }
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
  return most == 0 ? 0 : kKvHead + most;
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
  hipError_t e = launch(kern, dim3(pieces), dim3(kKvThreads), 0, stream, (const char*)q, t, c, sh, (__bf16*)out, lse, (char*)workspace);
  if (e != hipSuccess) return e;
  auto join = head_dim == 128 ? kv4_join_kernel<128> : kv4_join_kernel<64>;
  return launch(join, dim3(rows_out), dim3(kKvThreads), 0, stream, t, c, sh, pieces, (__bf16*)out, lse, (const char*)workspace);
}

}  // namespace vfm
