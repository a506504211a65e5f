// How the calls of causal attention are cut: host code, from the sizes alone.
#pragma once

#include <math.h>

#include "cattn_common.h"

namespace vfm {

// ---------------------------------------------------------------- forward
constexpr int kCU = 32;                 // keys per pipeline unit

// Units of the keys that the last row of tile tq sees
__host__ __device__ inline int tile_units(int rows, int off, int group, int rows_per_tile, int tq) {
  const int last = ((tq + 1) * rows_per_tile < rows ? (tq + 1) * rows_per_tile : rows) - 1;
  const int keys = last / group + off + 1;
  return keys > 0 ? (keys + kCU - 1) / kCU : 0;
}

// A chunk of a prompt against a long past is fewer tiles than the chip has CUs, and each takes as long as the past is long.
// Then every K/V head's line of units (tile after tile) is cut into equal pieces, one workgroup each.  A tile within a piece
// is finished there; a cut tile's parts go to the workspace, and a second launch joins them in order.
constexpr int kSplitSeqs = 32;          // the plan travels in 4 KB of kernel arguments
constexpr int kSplitPieces = 768;
constexpr int kSplitTile = 5;           // a tile's prologue and epilogue, as units
constexpr int kSplitJoin = 10;          // the second launch, as units

struct SplitPlan {
  int n, pieces;
  int qs[kSplitSeqs], ql[kSplitSeqs], ks[kSplitSeqs], kl[kSplitSeqs];
  int cu[kSplitSeqs + 1];               // tiles of the sequences before
  uint32_t start[kSplitPieces + 1];     // (tile << 16 | unit) where a piece begins; the last: where all end
  __device__ __host__ int q_start(int s) const { return qs[s]; }
  __device__ __host__ int q_len(int s) const { return ql[s]; }
  __device__ __host__ int kv_start(int s) const { return ks[s]; }
  __device__ __host__ int kv_len(int s) const { return kl[s]; }
};

// Cuts a run into pieces if that pays; false: it does not (or the plan cannot hold it).  In units (0.45 us with 128 rows, which
// one workgroup per CU does at the chip's full rate): without, the run takes as long as its longest tile.  In pieces it takes work
// / pieces and the traffic of the cuts, rows * head_dim * 8 bytes each out and back, which all pieces make at once: with as many
// pieces as there is room (rows * head_dim / 2048 + 2) units per end of a piece.
inline bool make_split(const XSegTable& segs, const CausalShape& sh, int rows_per_tile, int head_dim, int slots, SplitPlan* plan) {
  if (segs.n > kSplitSeqs || segs.n == 0) return false;
  long long cost = 0;
  int tiles = 0, longest = 0;
  for (int s = 0; s < segs.n; ++s) {
    const long long rows = (long long)segs.ql[s] * sh.group, n = (rows + rows_per_tile - 1) / rows_per_tile;
    if (tiles + n > 0xffff || (tiles + n) * sh.n_kv_heads > 2LL * slots) return false;   // (enough of them)
    for (int t = 0; t < n; ++t) {
      const int u = tile_units((int)rows, segs.kl[s] - segs.ql[s], sh.group, rows_per_tile, t);
      if (u > longest) longest = u;
      cost += u + kSplitTile;
    }
    tiles += (int)n;
  }
  const int room = slots / sh.n_kv_heads < kSplitPieces ? slots / sh.n_kv_heads : kSplitPieces;
  if (room < 2 || longest > 0xffff) return false;
  const float ends = 2.f * (rows_per_tile * head_dim / 2048 + 2);
  int pieces = (int)sqrtf((float)cost * room / ends);          // where work / pieces + ends * pieces / room is least
  if (pieces > room) pieces = room;
  if (pieces < 2 || (float)cost / pieces + ends * pieces / room + kSplitJoin > 0.8f * (longest + kSplitTile)) return false;
  plan->n = segs.n;
  int at = 0;
  for (int s = 0; s <= kSplitSeqs; ++s) {
    plan->cu[s] = at;
    if (s == kSplitSeqs) break;
    const bool live = s < segs.n;
    plan->qs[s] = live ? segs.qs[s] : 0;
    plan->ql[s] = live ? segs.ql[s] : 0;
    plan->ks[s] = live ? segs.ks[s] : 0;
    plan->kl[s] = live ? segs.kl[s] : 0;
    if (live) at += (int)(((long long)segs.ql[s] * sh.group + rows_per_tile - 1) / rows_per_tile);
  }
  int p = 0;
  long long before = 0;
  plan->start[p++] = 0;
  for (int s = 0, tile = 0; s < segs.n; ++s) {
    const int rows = segs.ql[s] * sh.group, n = (rows + rows_per_tile - 1) / rows_per_tile;
    for (int t = 0; t < n; ++t, ++tile) {
      const int u = tile_units(rows, segs.kl[s] - segs.ql[s], sh.group, rows_per_tile, n - 1 - t);
      for (; p < pieces; ++p) {
        long long cut = cost * p / pieces - before - kSplitTile;   // in units of this tile
        if (cut >= u - 2) break;                                   // (a part of one or two units is not worth its slot)
        if (cut < 2) cut = 0;
        const uint32_t at = (uint32_t)tile << 16 | (uint32_t)cut;
        if (at <= plan->start[p - 1]) { plan->start[p] = plan->start[p - 1]; continue; }   // an empty piece
        plan->start[p] = at;
      }
      before += u + kSplitTile;
    }
  }
  for (; p <= pieces; ++p) plan->start[p] = (uint32_t)tiles << 16;
  plan->pieces = pieces;
  return true;
}

// Rows of a workgroup's tile.  256 where keys are many, for half the K/V traffic per product, if the chip is full of such
// tiles or of long pieces of them; else 128, whose units take half as long.  No more than the longest sequence has, down to 32 (a
// token or two against many keys: a wavefront without rows only takes LDS).  Measured at head_dim 128, 256 and 128 rows: 2,000 tokens x
// 16/4 heads 50 and 37 us, 4,000 98 and 83, 6,000 x 32/8 284 with 256; in pieces 512 + 130 queries x 18,432 + 7,001 keys x 32/8
// 179 and 225, 8,000 tokens x 2/1 69 and 89, 64 queries x 30,000 keys x 32/8 57 and 52.
inline int causal_rows(const XSegTable& segs, const CausalShape& sh, int head_dim) {
  int longest = 0;
  long long rows = 0, tiles = 0, units = 0;
  for (int s = 0; s < segs.n; ++s) {
    const long long r = (long long)segs.ql[s] * sh.group, n = (r + 255) / 256;
    longest = longest > segs.kl[s] ? longest : segs.kl[s];
    rows = rows > r ? rows : r;
    tiles += n;
    units += n * (segs.kl[s] - segs.ql[s] / 2) / kCU;
  }
  if (rows <= 64) return rows <= 32 ? 32 : 64;
  const int cus = compute_unit_count();
  if (head_dim == 64 || longest <= 1024) return 128;
  const long long share = units * sh.n_kv_heads / cus;   // units per CU, were they dealt evenly; split if the longest tile has many more
  return tiles * sh.n_kv_heads >= cus || (share >= 30 && longest / kCU * 2 >= 5 * share) ? 256 : 128;
}
// Workgroups that a split call is cut for
inline int causal_slots(int rows) { return compute_unit_count() * (rows <= 64 ? 2 : 1); }

// ---------------------------------------------------------------- backward
constexpr int kCBwdBC = 128;   // keys per workgroup (RG = 1)

// How the dK/dV pass is cut.  rg: wavefronts that share the keys of a workgroup (RG of cattn_dkdv_kernel): 1 where the workgroups of
// 128 keys keep the chip busy; more where the longest of them, which walks all of its sequence's rows, takes longer than an
// even share of the work.  splits: workgroups that share a key tile's rows, where that leaves the longest far longer still.
// (Whole backward with rg = 1, 2, 4: head_dim 64: 2,146 and shorter x 12/4 heads 134, 101, 86 us; 6,000 x 16/4 463, 353, 370; 6,000 x
// 32/8 609, 540, 659.  head_dim 128, rg = 1, 2: 2,000 x 16/4 227, 174; 3,000 + 2,500 x 24/8 357, 361; 6,000 x 32/8 956, 985.
// Uncut and cut by share: head_dim 128: 1,000 x 8/2 75, 57; 2,000 x 16/4 158, 113; 4,000 x 16/4 327, 268; 8,000 x 16/1 1,918, 839;
// 5,000 x 7/1 568, 235; 500 in two x 16/1 78, 47; head_dim 64, rg = 4
// uncut and rg = 2 cut: 4,000 x 8/2 138, 101; 1,500 in three x 12/4 29, 34; in twice as many pieces 4,000 x 16/4 278,
// 8,000 x 16/1 873.)
struct KeysPlan { int rg, splits; };
inline KeysPlan keys_plan(const XSegTable& segs, const CausalShape& sh, int head_dim, int cus) {
  long long longest = 0, work = 0, tiles_k = 0;    // in 64-row tiles of 128 keys
  for (int s = 0; s < segs.n; ++s) {
    const long long tiles = ((long long)segs.ql[s] * sh.group + 63) / 64, n = (segs.kl[s] + kCBwdBC - 1) / kCBwdBC;
    // keys before the first query are seen by all rows, the others by half of them on average
    const long long before = segs.kl[s] > segs.ql[s] ? (segs.kl[s] - segs.ql[s]) / kCBwdBC : 0;
    longest = longest > tiles ? longest : tiles;
    work += before * tiles + (n - before) * (tiles + 1) / 2;
    tiles_k += n;
  }
  const long long share = work * sh.n_kv_heads / cus;
  if (longest <= (head_dim == 64 ? share : share + share / 2) + 4) return {1, 1};
  // about an even share of the work per piece, no shorter than kLeast tiles; at most eight workgroups per CU.  rg = 4 where a walk
  // is too short to be cut
  constexpr int kLeast = 14;
  if (head_dim == 64 && longest > 3 * share && longest <= 4 * kLeast) return {4, 1};
  const int rg = 2;
  const long long piece = share > kLeast ? share : kLeast;
  long long splits = (longest / rg + piece * 2 / 3) / piece;
  const long long room = 8LL * cus / (tiles_k * rg * sh.n_kv_heads + 1);
  splits = splits < room ? splits : room;
  return {rg, (int)(splits < 2 ? 1 : splits > 16 ? 16 : splits)};
}

// Wavefronts that share the rows of a dQ workgroup (KG of cattn_dq_kernel).  A workgroup takes some us for its rows and results and
// then its time per 64-key tile; the call takes as long as the longest of them or as all of them on the chip's CUs.  In us, as measured
// at head_dim 128 with 256 rows (KG = 1), 64 and 32, and at 64 with 128, 64 and 32.  (Whole backward, KG = 1, 2, 4: head_dim 128:
// 1,000 tokens x 8/2 heads 95, 84, 77; 2,000 x 16/4 174, 162, 184; 4,000 x 16/4 340, 384, 432; 256 queries x 4,096 keys x 16/4 138,
// 101, 71; head_dim 64: 1,000 x 8/2 47, 44, 41; 4,000 x 8/2 154, 143, 168; 6,000 x 16/4 351, 359, 502.)
inline int dq_shares(const XSegTable& segs, const CausalShape& sh, int head_dim, int cus) {
  struct Cost { int rows; float each, tile, busy, at_once; };   // per workgroup, per tile alone, per tile on a busy CU, on a CU at once
  static const Cost costs[2][3] = {{{256, 6.f, 1.28f, 1.28f, 1.f}, {64, 6.7f, 0.64f, 0.64f, 1.f}, {32, 7.5f, 0.35f, 0.35f, 1.f}},
                                   {{128, 6.f, 1.15f, 0.72f, 3.f}, {64, 6.7f, 0.6f, 0.4f, 2.f}, {32, 7.5f, 0.33f, 0.47f, 1.f}}};
  int best = 0;
  float least = 0.f;
  for (int x = 0; x < 3; ++x) {
    const Cost& c = costs[head_dim == 64][x];
    long long longest = 0, groups = 0;
    double work = 0.;
    for (int s = 0; s < segs.n; ++s) {
      const long long tiles = (segs.kl[s] + 63) / 64, n = ((long long)segs.ql[s] * sh.group + c.rows - 1) / c.rows;
      const long long before = segs.kl[s] > segs.ql[s] ? (segs.kl[s] - segs.ql[s]) / 64 : 0;
      if (n > 0) longest = longest > tiles ? longest : tiles;
      groups += n;
      work += (double)n * (before + (tiles - before + 1) / 2);
    }
    const float alone = c.each + longest * c.tile;
    const float all = (float)((groups * (c.each / c.at_once) + work * c.busy) * sh.n_kv_heads / cus);
    const float t = alone > all ? alone : all;
    if (x == 0 || t < least) { least = t; best = x; }
  }
  return 1 << best;
}

}  // namespace vfm
