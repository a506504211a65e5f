// Writing rows into the 4-bit key/value cache and reading them back (gfx950).  Both are bound by HBM: 2 D + D/2 + D/32 bytes a row
// and tensor, whichever way.
//
// head_dim / 8 lanes share a row, 8 elements (16 bytes of bf16, 4 bytes of codes) a lane, so that a wavefront's
// loads and stores are whole rows on both sides; the four lanes of a block find its maximum by two lane
// exchanges.  A workgroup takes consecutive rows (token-major, head-minor) of K and of V.
// Measured, 8 K/V heads x 128: 12,087 tokens written in 16 us (63 MB, 3.9 TB/s), 23,809 read back in 27 us (123 MB, 4.5 TB/s; a large
// copy reaches 4.6).  Requesting a row before its place is looked up: 18 us.
#include "kv4_common.h"

namespace vfm {

constexpr int kKv4Threads = 256;

// Factor byte of a block whose largest magnitude is `top` (fp32 of a bf16): 127 - e for the largest e with top 2^e <= 6, e in
// [-125, 120]; 127 for an all-zero block.  top = f 2^E, f in [1, 2): e = 2 - E where f <= 1.5, else 1 - E.
__device__ __forceinline__ uint32_t kv4_byte_of(float top) {
  const uint32_t u = __builtin_bit_cast(uint32_t, top);
  const int E = (int)(u >> 23) - 127;                       // (a subnormal top: -127, e is cut to 120)
  int e = (u & 0x7fffffu) <= 0x400000u ? 2 - E : 1 - E;
  e = min(max(e, -125), 120);
  return u == 0 ? 127u : u >= 0x7f800000u ? kKv4Nan : (uint32_t)(127 - e);
}

template <int D>
__global__ __launch_bounds__(kKv4Threads) void kv4_append_kernel(const char* __restrict__ k, const char* __restrict__ v,
                                                                 uint32_t k_row, uint32_t v_row, const Kv4Table t,
                                                                 const Kv4Cache c) {
  constexpr int kLanes = D / 8;
  const long long row = (long long)blockIdx.x * (kKv4Threads / kLanes) + threadIdx.x / kLanes;
  const int chunk = threadIdx.x % kLanes;
  const int rel = (int)(row / c.n_kv_heads), kvh = (int)(row - (long long)rel * c.n_kv_heads);
  const int tok = t.cu[0] + rel;
  if (tok >= t.cu[t.n]) return;                             // (whole rows: no lane of an exchange is missing)
  const int s = kv4_seq_of(t, tok);
  const int len = c.lens[s];
  const long long pos = (long long)len + (tok - t.cu[s]);
  const int page = len < 0 ? -1 : kv4_page(c, s, pos);
  if (page < 0) return;
  const size_t at = kv4_row(c, page, kvh, pos);
  const u32x4 kw = *reinterpret_cast<const u32x4*>(k + (size_t)tok * k_row + (size_t)kvh * (D * 2) + chunk * 16);
  const u32x4 vw = *reinterpret_cast<const u32x4*>(v + (size_t)tok * v_row + (size_t)kvh * (D * 2) + chunk * 16);
  auto put = [&](const u32x4& w, uint8_t* codes, uint8_t* factors) {
    float x[8];
    uint32_t top = 0;                                       // magnitudes compare as integers; NaN and infinity come out on top
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __builtin_bit_cast(float, w[i] << 16);
      x[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u);
      top = max(top, max((w[i] << 16) & 0x7fffffffu, w[i] & 0x7fff0000u));
    }
    top = max(top, (uint32_t)__shfl_xor((int)top, 1));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2));
    const uint32_t b = kv4_byte_of(__builtin_bit_cast(float, top));
    uint32_t word = 0;
    if (b != kKv4Nan) {
      const float f = kv4_factor(b), most = 6.f * f;        // (more than 6 f only where e was cut to -125)
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = fminf(fmaxf(x[i], -most), most);
      word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[0], x[1], f, 0);
      word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[2], x[3], f, 1);
      word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[4], x[5], f, 2);
      word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[6], x[7], f, 3);
    }
    *reinterpret_cast<uint32_t*>(codes + at * (D / 2) + chunk * 4) = word;
    if ((chunk & 3) == 0) factors[at * (D / kKv4Block) + chunk / 4] = (uint8_t)b;
  };
  put(kw, c.k4, c.ks);
  put(vw, c.v4, c.vs);
}

// Rows 0 .. of every sequence; a row whose page is not there comes out as zeros.
template <int D>
__global__ __launch_bounds__(kKv4Threads) void kv4_gather_kernel(const Kv4Table t, const Kv4Cache c, __bf16* __restrict__ k,
                                                                 __bf16* __restrict__ v) {
  constexpr int kLanes = D / 8;
  const long long row = (long long)blockIdx.x * (kKv4Threads / kLanes) + threadIdx.x / kLanes;
  const int chunk = threadIdx.x % kLanes;
  const int rel = (int)(row / c.n_kv_heads), kvh = (int)(row - (long long)rel * c.n_kv_heads);
  const int tok = t.cu[0] + rel;
  if (tok >= t.cu[t.n]) return;
  const int s = kv4_seq_of(t, tok);
  const int pos = tok - t.cu[s];
  const int page = kv4_page(c, s, pos);
  const size_t to = ((size_t)tok * c.n_kv_heads + kvh) * D + chunk * 8;
  auto get = [&](const uint8_t* codes, const uint8_t* factors, __bf16* dst) {
    u32x4 w = {0u, 0u, 0u, 0u};
    if (page >= 0) {
      const size_t at = kv4_row(c, page, kvh, pos);
      const uint32_t b = factors[at * (D / kKv4Block) + chunk / 4];
      const uint32_t x = *reinterpret_cast<const uint32_t*>(codes + at * (D / 2) + chunk * 4);
      w = b == kKv4Nan ? u32x4{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u}
                       : __builtin_bit_cast(u32x4, kv4_values(x, kv4_factor(b)));
    }
    *reinterpret_cast<u32x4*>(dst + to) = w;
  };
  get(c.k4, c.ks, k);
  get(c.v4, c.vs, v);
}

static unsigned row_blocks(const Kv4Table& t, int n_kv_heads, int head_dim) {
  const long long rows = (long long)(t.cu[t.n] - t.cu[0]) * n_kv_heads, per = kKv4Threads / (head_dim / 8);
  return (unsigned)((rows + per - 1) / per);
}

hipError_t launch_kv4_append(const void* k, uint32_t k_row, const void* v, uint32_t v_row, const Kv4Table& t,
                             const Kv4Cache& c, int head_dim, hipStream_t stream) {
  const unsigned blocks = row_blocks(t, c.n_kv_heads, head_dim);
  if (blocks == 0) return hipSuccess;
  auto kern = head_dim == 128 ? kv4_append_kernel<128> : kv4_append_kernel<64>;
  return launch(kern, dim3(blocks), dim3(kKv4Threads), 0, stream, (const char*)k, (const char*)v, k_row, v_row, t, c);
}

hipError_t launch_kv4_gather(const Kv4Table& t, const Kv4Cache& c, int head_dim, void* k, void* v, hipStream_t stream) {
  const unsigned blocks = row_blocks(t, c.n_kv_heads, head_dim);
  if (blocks == 0) return hipSuccess;
  auto kern = head_dim == 128 ? kv4_gather_kernel<128> : kv4_gather_kernel<64>;
  return launch(kern, dim3(blocks), dim3(kKv4Threads), 0, stream, t, c, (__bf16*)k, (__bf16*)v);
}

}  // namespace vfm
