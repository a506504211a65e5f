// Host-only exercise of the C entry points of causal attention and of the 4-bit cache, and of the plans that their calls are cut by,
// under AddressSanitizer and UndefinedBehaviorSanitizer (no GPU, nothing launched).  Built by
// tests/test_host_sanitizers_causal.py from csrc/causal_api.hip plus the launcher stubs below, which stand in for the kernels'
// launchers and check what the tables and plans they are handed contain.
#include <stdio.h>
#include <stdlib.h>

#include <algorithm>
#include <random>
#include <vector>

#include "cattn_plan.h"
#include "kv4_common.h"

static long g_launches = 0, g_splits = 0, g_cuts = 0;
static int g_failures = 0, g_cus = 256;
#define EXPECT(cond)                                                              \
  do {                                                                            \
    if (!(cond)) { ++g_failures; fprintf(stderr, "FAILED %s:%d: %s\n", __FILE__, __LINE__, #cond); } \
  } while (0)

namespace vfm {

int launch_status(hipError_t) { return VFM_ERR_LAUNCH; }
int compute_unit_count() { return g_cus; }

// A run's table: sequences with anything in them, most keys first, inside the call.
static void check_segs(const XSegTable& segs, const CausalShape& sh) {
  EXPECT(segs.n >= 0 && segs.n <= VFM_MAX_XSEQS);
  for (int s = 0; s < segs.n; ++s) {
    EXPECT(segs.ql[s] >= 0 && segs.kl[s] >= 0 && segs.ql[s] + segs.kl[s] > 0 && segs.qs[s] >= 0 && segs.ks[s] >= 0);
    EXPECT(segs.qs[s] + segs.ql[s] <= sh.total_q);
    if (s > 0) EXPECT(segs.kl[s - 1] >= segs.kl[s]);
  }
}

// A cut of the forward: pieces follow one another, begin inside a tile's units or with a tile, and end with the last one.
static void check_split(const XSegTable& segs, const CausalShape& sh, int rows, int head_dim) {
  SplitPlan plan;
  const int slots = causal_slots(rows);
  if (!make_split(segs, sh, rows, head_dim, slots, &plan)) return;
  ++g_splits;
  EXPECT(plan.n == segs.n && plan.pieces >= 2 && plan.pieces <= kSplitPieces && plan.pieces * sh.n_kv_heads <= slots);
  std::vector<int> units;
  for (int s = 0; s < plan.n; ++s) {
    EXPECT(plan.cu[s] == (int)units.size());
    const int r = segs.ql[s] * sh.group, n = (r + rows - 1) / rows;
    for (int t = 0; t < n; ++t) units.push_back(tile_units(r, segs.kl[s] - segs.ql[s], sh.group, rows, n - 1 - t));
  }
  for (int s = plan.n; s <= kSplitSeqs; ++s) EXPECT(plan.cu[s] == (int)units.size());
  EXPECT(plan.start[0] == 0 && plan.start[plan.pieces] == (uint32_t)units.size() << 16);
  for (int p = 0; p < plan.pieces; ++p) {
    EXPECT(plan.start[p] <= plan.start[p + 1]);
    const uint32_t tile = plan.start[p] >> 16, u = plan.start[p] & 0xffff;
    if (plan.start[p] == plan.start[plan.pieces]) continue;           // (an empty one at the end)
    EXPECT(tile < units.size() && (u == 0 || (int)u < units[tile]));
    // a piece's unfinished tiles are its first and its last: two slots
    int unfinished = 0;
    for (uint32_t t = tile, at = u; (t << 16 | at) < plan.start[p + 1]; ++t, at = 0) {
      const int end = t < plan.start[p + 1] >> 16 ? units[t] : (int)(plan.start[p + 1] & 0xffff);
      if (at != 0 || end != units[t]) ++unfinished;
      EXPECT((int)at <= end);
    }
    EXPECT(unfinished <= 2);
  }
}

size_t cattn_fwd_workspace(const XSegTable& segs, const CausalShape& sh, int head_dim) {
  SplitPlan plan;
  const int rows = causal_rows(segs, sh, head_dim);
  EXPECT(rows == 32 || rows == 64 || rows == 128 || (rows == 256 && head_dim == 128));
  return make_split(segs, sh, rows, head_dim, causal_slots(rows), &plan) ? (size_t)plan.pieces * sh.n_kv_heads : 0;
}
size_t cattn_bwd_parts(const XSegTable& segs, const CausalShape& sh, int head_dim) {
  const KeysPlan plan = keys_plan(segs, sh, head_dim, compute_unit_count());
  EXPECT((plan.rg == 1 || plan.rg == 2 || (plan.rg == 4 && head_dim == 64)) && plan.splits >= 1 && plan.splits <= 16);
  EXPECT(plan.rg != 1 || plan.splits == 1);
  g_cuts += plan.rg > 1;
  return plan.splits > 1 ? 256 * plan.splits : 0;
}
hipError_t launch_cattn_fwd(const void*, const void*, const void*, const XSegTable& segs, const CausalShape& sh, int head_dim,
                            void*, float*, void* workspace, hipStream_t) {
  ++g_launches;
  check_segs(segs, sh);
  EXPECT(workspace != nullptr || cattn_fwd_workspace(segs, sh, head_dim) == 0);
  for (int rows : {32, 64, 128, 256}) {
    check_split(segs, sh, rows, head_dim);
    const TileIndex ti = make_causal_index<false>(segs, sh.group, rows);
    int tiles = 0;
    for (int s = 0; s < segs.n; ++s) {
      EXPECT(ti.cu[s] == tiles);
      tiles += (segs.ql[s] * sh.group + rows - 1) / rows;
    }
    EXPECT(count_tiles(ti) == tiles);
  }
  return hipSuccess;
}
hipError_t launch_cattn_bwd(const void*, const void*, const void*, const void*, const float*, const void*, const XSegTable& segs,
                            const CausalShape& sh, int head_dim, void*, uint32_t, void*, uint32_t, void*, uint32_t, float* delta,
                            float* lse2, float* sentinel, float* parts, hipStream_t) {
  ++g_launches;
  check_segs(segs, sh);
  const int kg = dq_shares(segs, sh, head_dim, compute_unit_count());
  EXPECT(kg == 1 || kg == 2 || kg == 4);
  cattn_bwd_parts(segs, sh, head_dim);
  EXPECT(lse2 - delta >= (long)sh.total_q * sh.n_heads && sentinel - lse2 >= (long)sh.total_q * sh.n_heads && parts - sentinel >= 2);
  return hipSuccess;
}

static void check_run(const Kv4Table& t, const Kv4Cache& c) {
  ++g_launches;
  EXPECT(t.n >= 0 && t.n <= VFM_MAX_SEQS && c.shift >= 4 && c.shift <= 20);
  for (int s = 0; s < VFM_MAX_SEQS; ++s) EXPECT(t.cu[s] <= t.cu[s + 1]);
}
hipError_t launch_kv4_append(const void*, uint32_t, const void*, uint32_t, const Kv4Table& t, const Kv4Cache& c, int, hipStream_t) {
  check_run(t, c);
  return hipSuccess;
}
hipError_t launch_kv4_gather(const Kv4Table& t, const Kv4Cache& c, int, void*, void*, hipStream_t) {
  check_run(t, c);
  return hipSuccess;
}
hipError_t launch_kv4_attn(const void*, uint32_t, const Kv4Table& t, const Kv4Cache& c, int, int, int, float, void*, float*, void*, hipStream_t) {
  check_run(t, c);
  return hipSuccess;
}
size_t kv4_attn_workspace(const int32_t* cu, int n, int, int, int) { return n > 0 && cu[n] > 0 ? 1000 : 0; }

}  // namespace vfm

int main() {
  std::mt19937 rng(7);
  char* const P = reinterpret_cast<char*>(0x100000);                  // never dereferenced
  float* const F = reinterpret_cast<float*>(0x100000);
  const int32_t* const I = reinterpret_cast<const int32_t*>(0x100000);
  const size_t big = (size_t)1 << 60;
  for (int trial = 0; trial < 1500; ++trial) {
    const int n = trial % 7 == 0 ? (int)(rng() % 300) : (int)(rng() % 6);
    const int hd = rng() % 2 ? 64 : 128, kvh = 1 + rng() % 8, heads = kvh * (1 + rng() % 16);
    g_cus = trial % 11 == 0 ? 1 + rng() % 300 : 256;
    std::vector<int32_t> cq(1, 0), ck(1, 0);
    const int most = 1 << (rng() % 13);
    for (int s = 0; s < n; ++s) {
      const int q = rng() % 5 == 0 ? 0 : rng() % most;
      cq.push_back(cq.back() + q);
      ck.push_back(ck.back() + (rng() % 3 == 0 ? q : rng() % 4 == 0 ? 0 : (int)(rng() % (4 * most)) + (rng() % 40 == 0 ? 60000 : 0)));
    }
    const int tq = cq.back(), tk = ck.back(), qs = heads * hd + 8 * (rng() % 3), ks = kvh * hd + 8 * (rng() % 3);
    const size_t fw = vfm_cattn_fwd_workspace_size(cq.data(), ck.data(), n, tq, tk, heads, kvh, hd);
    const size_t bw = vfm_cattn_bwd_workspace_size(cq.data(), ck.data(), n, tq, tk, heads, kvh, hd);
    EXPECT(fw % 256 == 0 && bw % 256 == 0 && bw >= (size_t)8 * tq * heads);
    EXPECT(vfm_cattn_fwd(P, qs, P, ks, P, ks, cq.data(), ck.data(), n, tq, tk, heads, kvh, hd, 0.1f, P, F, fw ? P : nullptr, fw, VFM_BF16, nullptr) == VFM_OK);
    if (fw) {
      EXPECT(vfm_cattn_fwd(P, qs, P, ks, P, ks, cq.data(), ck.data(), n, tq, tk, heads, kvh, hd, 0.1f, P, F, P, fw - 1, VFM_BF16, nullptr) == VFM_ERR_WORKSPACE);
      EXPECT(vfm_cattn_fwd(P, qs, P, ks, P, ks, cq.data(), ck.data(), n, tq, tk, heads, kvh, hd, 0.1f, P, F, nullptr, big, VFM_BF16, nullptr) == VFM_ERR_WORKSPACE);
      EXPECT(vfm_cattn_fwd(P, qs, P, ks, P, ks, cq.data(), ck.data(), n, tq, tk, heads, kvh, hd, 0.1f, P, F, P + 128, big, VFM_BF16, nullptr) == VFM_ERR_WORKSPACE);
    }
    if (tq + tk > 0) {
      EXPECT(vfm_cattn_bwd(P, qs, P, ks, P, ks, P, F, P, cq.data(), ck.data(), n, tq, tk, heads, kvh, hd, 0.1f, P, qs, P, ks, P, ks, P, bw, VFM_BF16,
                           nullptr) == VFM_OK);
      EXPECT(vfm_cattn_bwd(P, qs, P, ks, P, ks, P, F, P, cq.data(), ck.data(), n, tq, tk, heads, kvh, hd, 0.1f, P, qs, P, ks, P, ks, P, bw - 1, VFM_BF16,
                           nullptr) == VFM_ERR_WORKSPACE);
    }
    const int pages = rng() % 9, page = 16 << (rng() % 8);
    EXPECT(vfm_kv4_append(P, ks, P, ks, cq.data(), n, tq, I, I, pages, P, P, P, P, 40, page, kvh, hd, VFM_BF16, nullptr) == VFM_OK);
    EXPECT(vfm_kv4_gather(P, P, P, P, 40, page, I, pages, ck.data(), n, tk, kvh, hd, P, P, VFM_BF16, nullptr) == VFM_OK);
    EXPECT(vfm_kv4_attn(P, qs, P, P, P, P, 40, page, I, pages, I, cq.data(), n, tq, heads, kvh, hd, 0.1f, P, F, P, big, VFM_BF16, nullptr) ==
           ((long long)tq * heads > 1 << 22 ? VFM_ERR_SHAPE : VFM_OK));
    if (n >= 2) {                                                       // malformed boundaries: refused before any table is built
      std::vector<int32_t> bad(cq);
      bad[n / 2] = bad[n] + 1;
      const long before = g_launches;
      EXPECT(vfm_cattn_fwd(P, qs, P, ks, P, ks, bad.data(), ck.data(), n, tq, tk, heads, kvh, hd, 0.1f, P, F, P, big, VFM_BF16, nullptr) == VFM_ERR_CU_SEQLENS);
      EXPECT(vfm_kv4_append(P, ks, P, ks, bad.data(), n, tq, I, I, pages, P, P, P, P, 40, page, kvh, hd, VFM_BF16, nullptr) == VFM_ERR_CU_SEQLENS);
      EXPECT(g_launches == before);
    }
  }
  EXPECT(g_splits > 100 && g_cuts > 100);
  // the largest calls: 2^27 query rows, 2^28 key rows, as one sequence and in a launch's most
  for (int n : {1, VFM_MAX_XSEQS}) {
    std::vector<int32_t> cq(1, 0), ck(1, 0);
    for (int s = 1; s <= n; ++s) {
      cq.push_back((int32_t)((1LL << 24) * s / n));
      ck.push_back((int32_t)((1LL << 24) * s / n));
    }
    const int st = vfm_cattn_fwd(P, 512, P, 128, P, 128, cq.data(), ck.data(), n, 1 << 24, 1 << 24, 8, 2, 64, 0.1f, P, F, P, big, VFM_BF16, nullptr);
    EXPECT(st == (n == 1 ? VFM_ERR_SHAPE : VFM_OK));                  // (one sequence: more than 4 GiB)
    EXPECT(vfm_cattn_fwd(P, 64, P, 64, P, 64, cq.data(), ck.data(), n, 1 << 24, 1 << 24, 1, 1, 64, 0.1f, P, F, P, big, VFM_BF16, nullptr) == VFM_OK);
  }
  const int32_t one[2] = {0, 1}, many[2] = {0, 1 << 22};
  EXPECT(vfm_cattn_fwd(P, 65535 * 64, P, 65535 * 64, P, 65535 * 64, one, many, 1, 1, 1 << 22, 65535, 65535, 64, 0.1f, P, F, P, big, VFM_BF16, nullptr) ==
         VFM_ERR_SHAPE);
  printf("%s: %ld stub launches, %ld split plans, %ld cut backwards, %d failures\n", g_failures ? "FAILED" : "ok", g_launches, g_splits, g_cuts, g_failures);
  return g_failures ? 1 : 0;
}
