// Keys and values held in 8 bits: what the kernels of a quantised cache share.
//
// A row (a token's numbers of one key head) is 8-bit codes and a scale of 32 bits; code times scale is the value.  Codes are
// e4m3 (4 bits of exponent, 3 of mantissa) or whole numbers.  Both become 16-bit floating-point numbers exactly: an e4m3 code, with
// its 7 low bits 7 places up, is the number times 2^-8 in float16, below its normal numbers too; a whole number's byte under
// the exponent of 1024 is 1024 more than itself.  That is 2 to 4 operations for two codes, where the conversion instruction would also make
// numbers that are not finite of e4m3's two codes for them.  The store never writes those; here they read as +-480.
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
// what a decoded code has to be multiplied by
template <Format F>
constexpr float kUnit = F == kE4m3 ? 256.0f : 1.0f;
template <Format F>
constexpr float kLargest = F == kE4m3 ? 448.0f : 127.0f;

// two e4m3 codes in the high bytes of the halves of t
__device__ __forceinline__ u32 decode_e4m3(u32 t) { return (t & 0x80008000u) | ((t >> 1) & 0x3f803f80u); }
// two bytes of w ^ 0x80.., chosen by `which`
__device__ __forceinline__ u32 decode_int8(u32 w, u32 which) {
  const u32 x = __byte_perm(w, 0x64646464u, which);
  u32 r;
  asm("add.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(0xe480e480u));      // - (1024 + 128)
  return r;
}

// Four codes: bytes 0 and 2, bytes 1 and 3.
template <Format F>
__device__ __forceinline__ void decode_across(u32 w, u32 &even, u32 &odd) {
  if (F == kE4m3) {
    even = decode_e4m3(w << 8);
    odd = decode_e4m3(w);
  } else {
    w ^= 0x80808080u;
    even = decode_int8(w, 0x4240);
    odd = decode_int8(w, 0x4341);
  }
}
// Four codes in their order.
template <Format F>
__device__ __forceinline__ void decode_along(u32 w, u32 &lo, u32 &hi) {
  if (F == kE4m3) {
    lo = decode_e4m3(__byte_perm(w, 0, 0x1404));
    hi = decode_e4m3(__byte_perm(w, 0, 0x3424));
  } else {
    w ^= 0x80808080u;
    lo = decode_int8(w, 0x4140);
    hi = decode_int8(w, 0x4342);
  }
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
cudaError_t launch_coded_rows_e4m3(const CodedAttn &a, int dtype, int dim, u32 sms, cudaStream_t s);
cudaError_t launch_coded_rows_int8(const CodedAttn &a, int dtype, int dim, u32 sms, cudaStream_t s);
bool launch_coded_chunk_e4m3(const CodedAttn &a, int dtype, int dim, u32 sms, cudaStream_t s, cudaError_t *e);
bool launch_coded_chunk_int8(const CodedAttn &a, int dtype, int dim, u32 sms, cudaStream_t s, cudaError_t *e);

}  // namespace paged
}  // namespace gorio
