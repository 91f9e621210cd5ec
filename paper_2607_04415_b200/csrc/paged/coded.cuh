// Keys and values held in 8 bits: what the kernels of a quantised cache share.
//
// A row (a token's numbers of one key head) is 8-bit codes and a scale of 32 bits; code times scale is the value.  Codes are
// e4m3 (4 bits of exponent, 3 of mantissa) or whole numbers.  Both become 16-bit floating-point numbers exactly: e4m3 by the conversion
// instruction, two codes in one cycle (by shifts and masks, 14 cycles for four codes where this takes 2); a whole number's byte
// under the exponent of 1024 is 1024 more than itself (4 cycles).
#pragma once
#include "common.cuh"
#include "mma.cuh"

namespace gorio {
namespace paged {

struct CodedAttn : Attn {
  const float *ks, *vs;        // [page][key head][place], strides in elements
  i64 ks_p, ks_h, ks_t, vs_p, vs_h, vs_t;
};

enum Format { kE4m3 = 0, kInt8 = 1 };
template <Format F>
constexpr float kLargest = F == kE4m3 ? 448.0f : 127.0f;

// the two e4m3 codes in a half of w
__device__ __forceinline__ void decode_e4m3(u32 w, u32 &lo, u32 &hi) {
  asm("{ .reg .b16 x, y; mov.b32 {x, y}, %2; cvt.rn.f16x2.e4m3x2 %0, x; cvt.rn.f16x2.e4m3x2 %1, y; }" : "=r"(lo), "=r"(hi) : "r"(w));
}
// two bytes of w ^ 0x80.., chosen by `which`
__device__ __forceinline__ u32 decode_int8(u32 w, u32 which) {
  const u32 x = __byte_perm(w, 0x64646464u, which);
  u32 r;
  asm("add.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(0xe480e480u));      // - (1024 + 128)
  return r;
}

// Four codes in their order; bytes 0 and 2, bytes 1 and 3.
template <Format F>
__device__ __forceinline__ void decode_along(u32 w, u32 &lo, u32 &hi) {
  if (F == kE4m3) {
    decode_e4m3(w, lo, hi);
  } else {
    w ^= 0x80808080u;
    lo = decode_int8(w, 0x4140);
    hi = decode_int8(w, 0x4342);
  }
}
template <Format F>
__device__ __forceinline__ void decode_across(u32 w, u32 &even, u32 &odd) {
  if (F == kE4m3) {
    decode_e4m3(__byte_perm(w, 0, 0x3120), even, odd);
  } else {
    w ^= 0x80808080u;
    even = decode_int8(w, 0x4240);
    odd = decode_int8(w, 0x4341);
  }
}
// 480 in the place of e4m3 codes that are no numbers: the store writes none, but what no query sees may hold any
template <Format F>
__device__ __forceinline__ u32 finite_codes(u32 h) {
  if (F == kE4m3) asm("min.f16x2 %0, %0, %1;" : "+r"(h) : "r"(0x5f805f80u));
  return h;
}

// log2 of a value's scale, cut to what running maxima count.  A weight is 2^(x - m + 15) at most, m >= x + log2(scale): with a scale of 0 it is 2^95, which sums
// of 2^32 keys hold; with the largest scale it is some 2^-90, and still above what is flushed to 0 for keys that weigh 2^-30 of it.
__device__ __forceinline__ float scale_log2(float scale) {
  float e;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(fabsf(scale)));
  return fminf(fmaxf(e, -80.0f), 100.0f);                     // also of a scale that is not a number
}

// 4 bytes, or zeros
__device__ __forceinline__ void cp_async4(void *to, const void *from, u32 bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_addr(to)), "l"(from), "r"(bytes) : "memory");
}

// Queries become float16 too, each row times a power of two that brings its largest number to 2^14 or more: nothing is lost but
// what lies below 2^-38 of that.  `largest` is a magnitude's bits; returns the factor.
__device__ __forceinline__ float query_factor(float largest) {
  const int e = (int)(__float_as_uint(largest) >> 23);
  return largest == 0.0f || e == 255 ? 1.0f : __uint_as_float((u32)min(127 + 14 + 127 - e, 127 + 100) << 23);
}

// launchers, one for each format
cudaError_t launch_coded_rows_e4m3(const CodedAttn &a, int dtype, int dim, bool few, u32 sms, cudaStream_t s);
cudaError_t launch_coded_rows_int8(const CodedAttn &a, int dtype, int dim, bool few, u32 sms, cudaStream_t s);
bool launch_coded_chunk_e4m3(const CodedAttn &a, int dtype, int dim, u32 sms, cudaStream_t s, cudaError_t *e);
bool launch_coded_chunk_int8(const CodedAttn &a, int dtype, int dim, u32 sms, cudaStream_t s, cudaError_t *e);

}  // namespace paged
}  // namespace gorio
