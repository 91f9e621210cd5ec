// New keys and values into 8 bits, and rows of such a cache back into 16.
#include "paged/coded.cuh"
#include "paged/entries.h"

namespace gorio {
namespace paged {

namespace {

constexpr int kThreads = 256;

struct RowsArgs {
  gorio_quantized_rows_desc d;
  u32 columns;                 // 2 * heads: keys' and values' rows of a token
};

// One (token, key or value, head) of a thread group's: where its 16-bit numbers, its codes and its scale are.
struct Side {
  u16 *wide;
  u8 *codes;
  float *scale;
  i64 wide_t, codes_p, codes_t, scale_p, scale_t;
};
__device__ __forceinline__ Side side_of(const gorio_quantized_rows_desc &d, u32 column) {
  const u32 v = column >= d.n_heads, h = column - v * d.n_heads;
  Side s;
  s.wide = (u16 *)(v ? d.values : d.keys) + (i64)h * (v ? d.v_head_stride : d.k_head_stride);
  s.codes = (u8 *)(v ? d.value_pages : d.key_pages) + (i64)h * (v ? d.vp_head_stride : d.kp_head_stride);
  s.scale = (v ? d.value_scales : d.key_scales) + (i64)h * (v ? d.vs_head_stride : d.ks_head_stride);
  s.wide_t = v ? d.v_token_stride : d.k_token_stride;
  s.codes_p = v ? d.vp_page_stride : d.kp_page_stride;
  s.codes_t = v ? d.vp_token_stride : d.kp_token_stride;
  s.scale_p = v ? d.vs_page_stride : d.ks_page_stride;
  s.scale_t = v ? d.vs_token_stride : d.ks_token_stride;
  return s;
}

// The largest magnitude of eight 16-bit numbers, as bits: of numbers without their sign the order is that of their bits.
__device__ __forceinline__ u32 largest8(uint4 x) {
  constexpr u32 k = 0x7fff7fffu;
  return __vmaxu2(__vmaxu2(x.x & k, x.y & k), __vmaxu2(x.z & k, x.w & k));
}

template <Format F>
__device__ __forceinline__ u32 encode4(float2 a, float2 b, float inverse) {
  // products are rounded to 32 bits before the codes are, as the format has it
  const float x0 = __fmul_rn(a.x, inverse), x1 = __fmul_rn(a.y, inverse), x2 = __fmul_rn(b.x, inverse), x3 = __fmul_rn(b.y, inverse);
  if (F == kE4m3) {
    u16 lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(x1), "f"(x0));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(x3), "f"(x2));
    return (u32)lo | ((u32)hi << 16);
  }
  // 1.5 * 2^23 more: the nearest whole number, ties to even, stands in the low bits
  constexpr float k = 12582912.0f;
  const u32 b0 = __float_as_uint(__fadd_rn(x0, k)), b1 = __float_as_uint(__fadd_rn(x1, k)), b2 = __float_as_uint(__fadd_rn(x2, k)),
            b3 = __float_as_uint(__fadd_rn(x3, k));
  return __byte_perm(__byte_perm(b0, b1, 0x0040), __byte_perm(b2, b3, 0x0040), 0x5410);
}

// A row of d numbers: M = max |x|, scale = M / L, codes = x * (L / M) rounded (L = 448 or 127).  LANES lanes a row, two pieces of 16 bytes each, one
// LANES pieces behind the other; all loads of EACH tokens are in flight at once; M is a maximum over bits and over the lanes.  Read once, written
// once: 3 bytes and a bit a number.  What is left beside that are instructions, and of those the ones that a row has whatever its length (slots,
// the maximum over lanes, two divisions): a piece a lane, with twice the lanes, took 34 us for 16383 tokens of 8 heads of 128 (float16 to int8) where this takes 25.
// Below M = 2^-100 (bfloat16 only) L / M would leave the range of 32 bits: such a row is stored as zeros.
constexpr int kPieces = 2;

template <typename T, Format F, int LANES, int EACH>
__global__ void __launch_bounds__(kThreads, 4) store_kernel(const RowsArgs a) {
  const u32 group = blockIdx.x * (kThreads / LANES) + threadIdx.x / LANES, lane = threadIdx.x % LANES;
  const u32 step = group / a.columns;
  const i64 first = (i64)step * EACH;
  if (first >= a.d.n_tokens) return;             // all lanes of a row together
  const u32 row_lanes = ((1u << LANES) - 1) << ((threadIdx.x & 31) / LANES * LANES);
  const Side s = side_of(a.d, group - step * a.columns);
  const u32 places = a.d.n_pages * a.d.page_size;
  uint4 x[EACH][kPieces];
  i64 slot[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    slot[i] = first + i < a.d.n_tokens ? a.d.slots[first + i] : -1;
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const u32 at = (lane + j * LANES) * 8;
      x[i][j] = make_uint4(0, 0, 0, 0);
      if (first + i < a.d.n_tokens && at < a.d.dim) x[i][j] = __ldcs((const uint4 *)(s.wide + (first + i) * s.wide_t + at));
    }
  }
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    if ((u64)slot[i] >= (u64)places) continue;   // negative ones too; the same for all lanes of a row
    u32 m = __vmaxu2(largest8(x[i][0]), largest8(x[i][1]));
#pragma unroll
    for (int k = LANES / 2; k; k >>= 1) m = __vmaxu2(m, __shfl_xor_sync(row_lanes, m, k));
    m = max(m & 0xffffu, m >> 16);
    const bool finite = (m & ExponentBits<T>::mask) != ExponentBits<T>::mask;
    const float top = unpack2<T>(m).x;
    const bool some = finite && top >= 0x1p-100f;
    const float scale = finite ? (some ? top / kLargest<F> : 0.0f) : __int_as_float(0x7fffffff), inverse = some ? kLargest<F> / top : 0.0f;
    const u32 page = (u32)slot[i] / a.d.page_size, in = (u32)slot[i] - page * a.d.page_size;
    u8 *const to = s.codes + (i64)page * s.codes_p + (i64)in * s.codes_t;
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const u32 at = (lane + j * LANES) * 8;
      const uint4 w = x[i][j];
      uint2 codes = make_uint2(encode4<F>(unpack2<T>(w.x), unpack2<T>(w.y), inverse), encode4<F>(unpack2<T>(w.z), unpack2<T>(w.w), inverse));
      if (!some) codes = make_uint2(0, 0);
      if (at < a.d.dim) *(uint2 *)(to + at) = codes;
    }
    if (lane == 0) s.scale[(i64)page * s.scale_p + (i64)in * s.scale_t] = scale;
  }
}

// Code times scale, rounded to 32 bits and to the type.
template <typename T, Format F, int LANES, int EACH>
__global__ void __launch_bounds__(kThreads) load_kernel(const RowsArgs a) {
  const u32 group = blockIdx.x * (kThreads / LANES) + threadIdx.x / LANES, lane = threadIdx.x % LANES;
  const u32 step = group / a.columns;
  const i64 first = (i64)step * EACH;
  if (first >= a.d.n_tokens) return;
  const Side s = side_of(a.d, group - step * a.columns);
  const u32 places = a.d.n_pages * a.d.page_size;
  i64 slot[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) slot[i] = first + i < a.d.n_tokens ? a.d.slots[first + i] : -1;
  uint2 codes[EACH][kPieces];
  float scale[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    scale[i] = 0.0f;
#pragma unroll
    for (int j = 0; j < kPieces; ++j) codes[i][j] = make_uint2(0, 0);
    if ((u64)slot[i] < (u64)places) {
      const u32 page = (u32)slot[i] / a.d.page_size, in = (u32)slot[i] - page * a.d.page_size;
      const u8 *const from = s.codes + (i64)page * s.codes_p + (i64)in * s.codes_t;
#pragma unroll
      for (int j = 0; j < kPieces; ++j) {
        const u32 at = (lane + j * LANES) * 8;
        if (at < a.d.dim) codes[i][j] = *(const uint2 *)(from + at);
      }
      scale[i] = s.scale[(i64)page * s.scale_p + (i64)in * s.scale_t];
    }
  }
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    if (first + i >= a.d.n_tokens) break;
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const u32 at = (lane + j * LANES) * 8;
      u32 h[4];
      decode_along<F>(codes[i][j].x, h[0], h[1]);
      decode_along<F>(codes[i][j].y, h[2], h[3]);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float2 v = unpack2<__half>(h[k]);
        h[k] = pack2<T>(v.x * scale[i], v.y * scale[i]);
      }
      if (at < a.d.dim) __stcs((uint4 *)(s.wide + (first + i) * s.wide_t + at), make_uint4(h[0], h[1], h[2], h[3]));
    }
  }
}

// Four tokens a thread where that still fills the GPU, one where it does not: more threads then have their loads in flight at once.
constexpr u32 kEach = 4;
constexpr u64 kFewThreads = 148 * 2048;

template <typename T, Format F, int LANES>
cudaError_t launch_lanes(const RowsArgs &a, bool store, cudaStream_t s) {
  const u64 each = (u64)a.d.n_tokens * a.columns * LANES >= kFewThreads * kEach ? kEach : 1;
  const u64 groups = (a.d.n_tokens + each - 1) / each * a.columns, blocks = (groups + kThreads / LANES - 1) / (kThreads / LANES);
  if (groups >= (1ull << 32) - kThreads || blocks >= (1ull << 31)) return cudaErrorInvalidConfiguration;
  if (store) {
    if (each == 1) store_kernel<T, F, LANES, 1><<<(u32)blocks, kThreads, 0, s>>>(a);
    else store_kernel<T, F, LANES, kEach><<<(u32)blocks, kThreads, 0, s>>>(a);
  } else {
    if (each == 1) load_kernel<T, F, LANES, 1><<<(u32)blocks, kThreads, 0, s>>>(a);
    else load_kernel<T, F, LANES, kEach><<<(u32)blocks, kThreads, 0, s>>>(a);
  }
  return cudaGetLastError();
}

template <typename T, Format F>
cudaError_t pick_lanes(const RowsArgs &a, bool store, cudaStream_t s) {
  if (a.d.dim <= 64) return launch_lanes<T, F, 4>(a, store, s);
  if (a.d.dim <= 128) return launch_lanes<T, F, 8>(a, store, s);
  return launch_lanes<T, F, 16>(a, store, s);
}

template <typename T>
cudaError_t pick_format(const RowsArgs &a, bool store, cudaStream_t s) {
  return a.d.format == GORIO_CODES_E4M3 ? pick_lanes<T, kE4m3>(a, store, s) : pick_lanes<T, kInt8>(a, store, s);
}

}  // namespace

cudaError_t launch_quantized_rows(const gorio_quantized_rows_desc &d, bool store, cudaStream_t s) {
  const RowsArgs a{d, 2 * d.n_heads};
  return d.dtype == GORIO_KV_BF16 ? pick_format<__nv_bfloat16>(a, store, s) : pick_format<__half>(a, store, s);
}

}  // namespace paged
}  // namespace gorio
