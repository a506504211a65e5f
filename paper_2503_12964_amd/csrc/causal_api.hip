// C ABI of causal attention with grouped heads and of the 4-bit key/value cache: argument validation, sequence tables,
// launches.  No allocation, no sync.
#include <math.h>

#include <algorithm>

#include "cattn_common.h"
#include "kv4_common.h"

namespace {

using vfm::CausalShape;
using vfm::Kv4Cache;
using vfm::Kv4Table;
using vfm::XSegTable;

constexpr long long kMaxRows = 1LL << 27;      // (token, head) rows: fewer than 2^32 threads in every launch, 32-bit byte offsets into lse
constexpr long long kMaxFewRows = 1LL << 22;   // the same of vfm_kv4_attn, whose join takes 256 threads a row
constexpr long long kMaxKeyRows = 1LL << 28;   // (key, K/V head) rows, likewise
constexpr long long kMaxSpan = 0xffffffffLL;   // bytes of one sequence's rows of a tensor, for 32-bit offsets
constexpr long long kSlack = 512;              // rows that a kernel's running offset goes past a sequence's end

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

int check_heads(int n_seqs, int total, int n_heads, int n_kv_heads, int head_dim) {
  if (n_seqs < 0 || total < 0 || n_heads < 1 || n_heads > 65535 || n_kv_heads < 1 || n_heads % n_kv_heads != 0) return VFM_ERR_SHAPE;
  if (head_dim != 64 && head_dim != 128) return VFM_ERR_SHAPE;
  if ((long long)total * n_heads > kMaxRows) return VFM_ERR_SHAPE;
  return VFM_OK;
}

int check_cu(const int32_t* cu, int n_seqs, int total) {
  if (cu[0] != 0) return VFM_ERR_CU_SEQLENS;
  for (int s = 0; s < n_seqs; ++s)
    if (cu[s + 1] < cu[s]) return VFM_ERR_CU_SEQLENS;
  return cu[n_seqs] == total ? VFM_OK : VFM_ERR_CU_SEQLENS;
}

int check_stride(int64_t stride, int heads, int head_dim) {
  return stride % 8 == 0 && stride >= (int64_t)heads * head_dim && stride <= 0x7fffffff / 2 ? VFM_OK : VFM_ERR_STRIDE;
}

int check_span(const int32_t* cu, int n_seqs, int64_t stride) {
  int longest = 0;
  for (int s = 0; s < n_seqs; ++s) longest = std::max(longest, cu[s + 1] - cu[s]);
  return ((long long)longest + kSlack) * stride * 2 > kMaxSpan && longest > 0 ? VFM_ERR_SHAPE : VFM_OK;
}

// Sizes and tables of a causal call.
int check_causal(const int32_t* cu_q, const int32_t* cu_kv, int n_seqs, int total_q, int total_kv, int n_heads,
                 int n_kv_heads, int head_dim) {
  int st = check_heads(n_seqs, total_q, n_heads, n_kv_heads, head_dim);
  if (!st && (total_kv < 0 || (long long)total_kv * n_kv_heads > kMaxKeyRows)) st = VFM_ERR_SHAPE;
  if (!st) st = check_cu(cu_q, n_seqs, total_q);
  if (!st) st = check_cu(cu_kv, n_seqs, total_kv);
  return st;
}

// Sequences of one run, longest key range first; a sequence's costliest tiles come first within it.  (Its short ones still come before
// the next sequence's long ones: all tiles of a call in order of length would need a table of tiles.)  Sequences with neither
// queries nor keys are dropped.
void build_table(const int32_t* cu_q, const int32_t* cu_kv, int n_seqs, XSegTable* t) {
  int order[VFM_MAX_XSEQS];
  int n = 0;
  for (int s = 0; s < n_seqs; ++s)
    if (cu_q[s + 1] > cu_q[s] || cu_kv[s + 1] > cu_kv[s]) order[n++] = s;
  std::stable_sort(order, order + n, [&](int a, int b) { return cu_kv[a + 1] - cu_kv[a] > cu_kv[b + 1] - cu_kv[b]; });
  t->n = n;
  for (int i = 0; i < VFM_MAX_XSEQS; ++i) {
    const bool live = i < n;
    t->qs[i] = live ? cu_q[order[i]] : 0;
    t->ql[i] = live ? cu_q[order[i] + 1] - cu_q[order[i]] : 0;
    t->ks[i] = live ? cu_kv[order[i]] : 0;
    t->kl[i] = live ? cu_kv[order[i] + 1] - cu_kv[order[i]] : 0;
  }
}

CausalShape make_shape(int total_q, int n_heads, int n_kv_heads, int64_t q_stride, int64_t k_stride, int64_t v_stride, float scale) {
  return {total_q, n_heads, n_kv_heads, n_heads / n_kv_heads, (uint32_t)(2 * q_stride), (uint32_t)(2 * k_stride),
          (uint32_t)(2 * v_stride), scale, scale * 1.4426950408889634f};
}

bool good_scale(float scale) { return scale > 0.f && isfinite(scale) && isfinite(scale * 1.4426950408889634f); }

size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// Workspace of a causal forward: the runs follow one another on the stream and share it.
size_t fwd_workspace(const int32_t* cu_q, const int32_t* cu_kv, int n_seqs, const CausalShape& sh, int head_dim) {
  size_t most = 0;
  for (int s0 = 0; s0 < n_seqs; s0 += VFM_MAX_XSEQS) {
    XSegTable segs;
    build_table(cu_q + s0, cu_kv + s0, std::min(VFM_MAX_XSEQS, n_seqs - s0), &segs);
    most = std::max(most, vfm::cattn_fwd_workspace(segs, sh, head_dim));
  }
  return align_up(most, 256);
}

// Workspace of a causal backward: the statistics of all rows, and what the runs share for split dK/dV passes.
size_t stats_bytes(int total_q, int n_heads) { return 2 * align_up((size_t)total_q * n_heads * sizeof(float), 256) + 256; }
size_t bwd_parts(const int32_t* cu_q, const int32_t* cu_kv, int n_seqs, const CausalShape& sh, int head_dim) {
  size_t most = 0;
  for (int s0 = 0; s0 < n_seqs; s0 += VFM_MAX_XSEQS) {
    XSegTable segs;
    build_table(cu_q + s0, cu_kv + s0, std::min(VFM_MAX_XSEQS, n_seqs - s0), &segs);
    most = std::max(most, vfm::cattn_bwd_parts(segs, sh, head_dim));
  }
  return align_up(most, 256);
}

int check_pages(int n_pages, int max_pages, int page_size) {
  if (n_pages < 0 || max_pages < 0 || page_size < 16 || page_size > (1 << 20) || (page_size & (page_size - 1))) return VFM_ERR_PAGE;
  return VFM_OK;
}

Kv4Cache make_cache(const void* k4, const void* v4, const void* ks, const void* vs, const int32_t* pages, const int32_t* lens,
                    int n_pages, int max_pages, int page_size, int n_kv_heads) {
  auto p = [](const void* x) { return static_cast<uint8_t*>(const_cast<void*>(x)); };
  return {p(k4), p(v4), p(ks), p(vs), pages, lens, n_pages, max_pages, __builtin_ctz(page_size), n_kv_heads};
}

// The run of sequences [s0, s0 + VFM_MAX_SEQS) of a call.
Kv4Table make_run(const int32_t* cu, int n_seqs, int s0, Kv4Cache* c) {
  Kv4Table t;
  t.n = std::min(VFM_MAX_SEQS, n_seqs - s0);
  for (int s = 0; s <= VFM_MAX_SEQS; ++s) t.cu[s] = cu[s0 + std::min(s, t.n)];
  if (c->lens) c->lens += s0 == 0 ? 0 : VFM_MAX_SEQS;
  c->pages += s0 == 0 ? 0 : (size_t)VFM_MAX_SEQS * c->max_pages;
  return t;
}

bool cache_null(const void* k4, const void* v4, const void* ks, const void* vs, int n_pages) {
  return n_pages > 0 && (!k4 || !v4 || !ks || !vs);
}
bool cache_aligned(const void* k4, const void* v4, const void* ks, const void* vs, const int32_t* pages, const int32_t* lens) {
  return aligned(k4, 16) && aligned(v4, 16) && aligned(ks, 16) && aligned(vs, 16) && aligned(pages, 4) && aligned(lens, 4);
}

}  // namespace

extern "C" {

size_t vfm_cattn_fwd_workspace_size(const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_kv, int n_seqs, int total_q,
                                    int total_kv, int n_heads, int n_kv_heads, int head_dim) {
  if (!cu_seqlens_q || !cu_seqlens_kv ||
      check_causal(cu_seqlens_q, cu_seqlens_kv, n_seqs, total_q, total_kv, n_heads, n_kv_heads, head_dim))
    return 0;
  return fwd_workspace(cu_seqlens_q, cu_seqlens_kv, n_seqs, make_shape(total_q, n_heads, n_kv_heads, 0, 0, 0, 1.f), head_dim);
}

int vfm_cattn_fwd(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                  const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_kv, int n_seqs, int total_q, int total_kv,
                  int n_heads, int n_kv_heads, int head_dim, float scale, void* out, float* lse, void* workspace,
                  size_t workspace_bytes, vfm_dtype dt, void* hip_stream) {
  if (!cu_seqlens_q || !cu_seqlens_kv || (total_q > 0 && (!q || !out || !lse)) || (total_kv > 0 && (!k || !v))) return VFM_ERR_NULL;
  if (dt != VFM_BF16) return VFM_ERR_DTYPE;
  int st = check_causal(cu_seqlens_q, cu_seqlens_kv, n_seqs, total_q, total_kv, n_heads, n_kv_heads, head_dim);
  if (st) return st;
  if (!good_scale(scale)) return VFM_ERR_SHAPE;
  st = check_stride(q_stride, n_heads, head_dim);
  if (!st) st = check_stride(k_stride, n_kv_heads, head_dim);
  if (!st) st = check_stride(v_stride, n_kv_heads, head_dim);
  if (!st) st = check_span(cu_seqlens_q, n_seqs, q_stride);
  if (!st) st = check_span(cu_seqlens_kv, n_seqs, std::max(k_stride, v_stride));
  if (st) return st;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16) || !aligned(lse, 16)) return VFM_ERR_ALIGN;
  const CausalShape sh = make_shape(total_q, n_heads, n_kv_heads, q_stride, k_stride, v_stride, scale);
  const size_t need = fwd_workspace(cu_seqlens_q, cu_seqlens_kv, n_seqs, sh, head_dim);
  if (need > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < need)) return VFM_ERR_WORKSPACE;
  for (int s0 = 0; s0 < n_seqs; s0 += VFM_MAX_XSEQS) {
    XSegTable segs;
    build_table(cu_seqlens_q + s0, cu_seqlens_kv + s0, std::min(VFM_MAX_XSEQS, n_seqs - s0), &segs);
    hipError_t e = vfm::launch_cattn_fwd(q, k, v, segs, sh, head_dim, out, lse, workspace, static_cast<hipStream_t>(hip_stream));
    if (e != hipSuccess) return vfm::launch_status(e);
  }
  return VFM_OK;
}

// Delta and lse in log2 units (fp32 [n_heads, total_q] each, padded to 256 bytes), 256 bytes of constants, shares of dK and dV.
size_t vfm_cattn_bwd_workspace_size(const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_kv, int n_seqs, int total_q,
                                    int total_kv, int n_heads, int n_kv_heads, int head_dim) {
  if (!cu_seqlens_q || !cu_seqlens_kv ||
      check_causal(cu_seqlens_q, cu_seqlens_kv, n_seqs, total_q, total_kv, n_heads, n_kv_heads, head_dim))
    return 0;
  return stats_bytes(total_q, n_heads) +
         bwd_parts(cu_seqlens_q, cu_seqlens_kv, n_seqs, make_shape(total_q, n_heads, n_kv_heads, 0, 0, 0, 1.f), head_dim);
}

int vfm_cattn_bwd(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                  const void* out, const float* lse, const void* dout, const int32_t* cu_seqlens_q,
                  const int32_t* cu_seqlens_kv, int n_seqs, int total_q, int total_kv, int n_heads, int n_kv_heads,
                  int head_dim, float scale, void* dq, int64_t dq_stride, void* dk, int64_t dk_stride, void* dv,
                  int64_t dv_stride, void* workspace, size_t workspace_bytes, vfm_dtype dt, void* hip_stream) {
  if (!cu_seqlens_q || !cu_seqlens_kv || (total_q > 0 && (!q || !out || !lse || !dout || !dq)) ||
      (total_kv > 0 && (!k || !v || !dk || !dv)))
    return VFM_ERR_NULL;
  if (dt != VFM_BF16) return VFM_ERR_DTYPE;
  int st = check_causal(cu_seqlens_q, cu_seqlens_kv, n_seqs, total_q, total_kv, n_heads, n_kv_heads, head_dim);
  if (st) return st;
  if (!good_scale(scale)) return VFM_ERR_SHAPE;
  for (int64_t x : {q_stride, dq_stride})
    if (!st) st = check_stride(x, n_heads, head_dim);
  for (int64_t x : {k_stride, v_stride, dk_stride, dv_stride})
    if (!st) st = check_stride(x, n_kv_heads, head_dim);
  if (!st) st = check_span(cu_seqlens_q, n_seqs, q_stride);   // (dout's stride is n_heads * head_dim, no more than q's)
  if (!st) st = check_span(cu_seqlens_kv, n_seqs, std::max(k_stride, v_stride));
  if (st) return st;
  for (const void* p : {q, k, v, out, (const void*)lse, dout, (const void*)dq, (const void*)dk, (const void*)dv})
    if (!aligned(p, 16)) return VFM_ERR_ALIGN;
  if (total_q == 0 && total_kv == 0) return VFM_OK;
  const size_t need = vfm_cattn_bwd_workspace_size(cu_seqlens_q, cu_seqlens_kv, n_seqs, total_q, total_kv, n_heads, n_kv_heads, head_dim);
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < need) return VFM_ERR_WORKSPACE;
  const size_t stats = stats_bytes(total_q, n_heads), part = (stats - 256) / 2;
  float* delta = static_cast<float*>(workspace);
  float* lse2 = reinterpret_cast<float*>(static_cast<char*>(workspace) + part);
  float* sentinel = reinterpret_cast<float*>(static_cast<char*>(workspace) + 2 * part);
  float* parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + stats);
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const CausalShape sh = make_shape(total_q, n_heads, n_kv_heads, q_stride, k_stride, v_stride, scale);
  for (int s0 = 0; s0 < n_seqs; s0 += VFM_MAX_XSEQS) {
    XSegTable segs;
    build_table(cu_seqlens_q + s0, cu_seqlens_kv + s0, std::min(VFM_MAX_XSEQS, n_seqs - s0), &segs);
    hipError_t e = vfm::launch_cattn_bwd(q, k, v, out, lse, dout, segs, sh, head_dim, dq, (uint32_t)(2 * dq_stride), dk,
                                         (uint32_t)(2 * dk_stride), dv, (uint32_t)(2 * dv_stride), delta, lse2, sentinel, parts, stream);
    if (e != hipSuccess) return vfm::launch_status(e);
  }
  return VFM_OK;
}

int vfm_kv4_append(const void* k, int64_t k_stride, const void* v, int64_t v_stride, const int32_t* cu_seqlens, int n_seqs,
                   int total_tokens, const int32_t* lens, const int32_t* pages, int max_pages, void* k4, void* v4,
                   void* k_scales, void* v_scales, int n_pages, int page_size, int n_kv_heads, int head_dim, vfm_dtype dt,
                   void* hip_stream) {
  if (!cu_seqlens || (total_tokens > 0 && (!k || !v || !lens || (max_pages > 0 && !pages))) || cache_null(k4, v4, k_scales, v_scales, n_pages))
    return VFM_ERR_NULL;
  if (dt != VFM_BF16) return VFM_ERR_DTYPE;
  int st = check_heads(n_seqs, total_tokens, n_kv_heads, n_kv_heads, head_dim);
  if (!st) st = check_pages(n_pages, max_pages, page_size);
  if (!st) st = check_stride(k_stride, n_kv_heads, head_dim);
  if (!st) st = check_stride(v_stride, n_kv_heads, head_dim);
  if (!st) st = check_cu(cu_seqlens, n_seqs, total_tokens);
  if (st) return st;
  if (!aligned(k, 16) || !aligned(v, 16) || !cache_aligned(k4, v4, k_scales, v_scales, pages, lens)) return VFM_ERR_ALIGN;
  Kv4Cache c = make_cache(k4, v4, k_scales, v_scales, pages, lens, n_pages, max_pages, page_size, n_kv_heads);
  for (int s0 = 0; s0 < n_seqs; s0 += VFM_MAX_SEQS) {
    const Kv4Table t = make_run(cu_seqlens, n_seqs, s0, &c);
    hipError_t e = vfm::launch_kv4_append(k, (uint32_t)(2 * k_stride), v, (uint32_t)(2 * v_stride), t, c, head_dim, static_cast<hipStream_t>(hip_stream));
    if (e != hipSuccess) return vfm::launch_status(e);
  }
  return VFM_OK;
}

int vfm_kv4_gather(const void* k4, const void* v4, const void* k_scales, const void* v_scales, int n_pages, int page_size,
                   const int32_t* pages, int max_pages, const int32_t* cu_seqlens, int n_seqs, int total_tokens,
                   int n_kv_heads, int head_dim, void* k, void* v, vfm_dtype dt, void* hip_stream) {
  if (!cu_seqlens || (total_tokens > 0 && (!k || !v || (max_pages > 0 && !pages))) || cache_null(k4, v4, k_scales, v_scales, n_pages))
    return VFM_ERR_NULL;
  if (dt != VFM_BF16) return VFM_ERR_DTYPE;
  int st = check_heads(n_seqs, total_tokens, n_kv_heads, n_kv_heads, head_dim);
  if (!st) st = check_pages(n_pages, max_pages, page_size);
  if (!st) st = check_cu(cu_seqlens, n_seqs, total_tokens);
  if (st) return st;
  if (!aligned(k, 16) || !aligned(v, 16) || !cache_aligned(k4, v4, k_scales, v_scales, pages, nullptr)) return VFM_ERR_ALIGN;
  Kv4Cache c = make_cache(k4, v4, k_scales, v_scales, pages, nullptr, n_pages, max_pages, page_size, n_kv_heads);
  for (int s0 = 0; s0 < n_seqs; s0 += VFM_MAX_SEQS) {
    const Kv4Table t = make_run(cu_seqlens, n_seqs, s0, &c);
    hipError_t e = vfm::launch_kv4_gather(t, c, head_dim, k, v, static_cast<hipStream_t>(hip_stream));
    if (e != hipSuccess) return vfm::launch_status(e);
  }
  return VFM_OK;
}

size_t vfm_kv4_attn_workspace_size(const int32_t* cu_seqlens, int n_seqs, int total_tokens, int n_heads, int n_kv_heads, int head_dim) {
  if (!cu_seqlens || check_heads(n_seqs, total_tokens, n_heads, n_kv_heads, head_dim) || check_cu(cu_seqlens, n_seqs, total_tokens)) return 0;
  if (total_tokens == 0) return 0;
  return align_up(vfm::kv4_attn_workspace(cu_seqlens, n_seqs, n_heads, n_kv_heads, head_dim), 256);
}

int vfm_kv4_attn(const void* q, int64_t q_stride, const void* k4, const void* v4, const void* k_scales, const void* v_scales,
                 int n_pages, int page_size, const int32_t* pages, int max_pages, const int32_t* lens,
                 const int32_t* cu_seqlens, int n_seqs, int total_tokens, int n_heads, int n_kv_heads, int head_dim,
                 float scale, void* out, float* lse, void* workspace, size_t workspace_bytes, vfm_dtype dt, void* hip_stream) {
  if (!cu_seqlens || (total_tokens > 0 && (!q || !out || !lse || !lens || (max_pages > 0 && !pages))) ||
      cache_null(k4, v4, k_scales, v_scales, n_pages))
    return VFM_ERR_NULL;
  if (dt != VFM_BF16) return VFM_ERR_DTYPE;
  int st = check_heads(n_seqs, total_tokens, n_heads, n_kv_heads, head_dim);
  if (!st && ((long long)total_tokens * n_heads > kMaxFewRows || !good_scale(scale))) st = VFM_ERR_SHAPE;
  if (!st) st = check_pages(n_pages, max_pages, page_size);
  if (!st) st = check_stride(q_stride, n_heads, head_dim);
  if (!st) st = check_cu(cu_seqlens, n_seqs, total_tokens);
  if (st) return st;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(lse, 16) || !cache_aligned(k4, v4, k_scales, v_scales, pages, lens)) return VFM_ERR_ALIGN;
  if (total_tokens == 0) return VFM_OK;
  const size_t need = vfm_kv4_attn_workspace_size(cu_seqlens, n_seqs, total_tokens, n_heads, n_kv_heads, head_dim);
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < need) return VFM_ERR_WORKSPACE;
  Kv4Cache c = make_cache(k4, v4, k_scales, v_scales, pages, lens, n_pages, max_pages, page_size, n_kv_heads);
  for (int s0 = 0; s0 < n_seqs; s0 += VFM_MAX_SEQS) {
    const Kv4Table t = make_run(cu_seqlens, n_seqs, s0, &c);
    hipError_t e = vfm::launch_kv4_attn(q, (uint32_t)(2 * q_stride), t, c, n_heads, total_tokens, head_dim, scale, out, lse,
                                        workspace, static_cast<hipStream_t>(hip_stream));
    if (e != hipSuccess) return vfm::launch_status(e);
  }
  return VFM_OK;
}

}  // extern "C"
