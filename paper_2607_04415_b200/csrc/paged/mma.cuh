// Warp-level pieces of the attention kernels: asynchronous copies, matrix fragments, the weights'
// arithmetic, and the end of a row.
#pragma once
#include "common.cuh"

namespace gorio {
namespace paged {

__device__ __forceinline__ u32 smem_addr(const void *p) { return (u32)__cvta_generic_to_shared(p); }

// 16 bytes, of which `bytes` (16 or 0) are read and the rest are zeros
__device__ __forceinline__ void cp_async16(void *to, const void *from, u32 bytes) {
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(smem_addr(to)), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void ldmatrix4(u32 (&r)[4], const void *p) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(smem_addr(p)) : "memory");
}
__device__ __forceinline__ void ldmatrix4t(u32 (&r)[4], const void *p) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(smem_addr(p)) : "memory");
}

template <typename T>
__device__ __forceinline__ void mma16816(float (&c)[4], const u32 (&a)[4], u32 b0, u32 b1);
template <>
__device__ __forceinline__ void mma16816<__nv_bfloat16>(float (&c)[4], const u32 (&a)[4], u32 b0, u32 b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16816<__half>(float (&c)[4], const u32 (&a)[4], u32 b0, u32 b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <typename T>
__device__ __forceinline__ u32 pack2(float lo, float hi);
template <>
__device__ __forceinline__ u32 pack2<__nv_bfloat16>(float lo, float hi) {
  u32 r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <>
__device__ __forceinline__ u32 pack2<__half>(float lo, float hi) {
  u32 r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

template <typename T>
__device__ __forceinline__ float2 unpack2(u32 v);
template <>
__device__ __forceinline__ float2 unpack2<__nv_bfloat16>(u32 v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
template <>
__device__ __forceinline__ float2 unpack2<__half>(u32 v) { return __half22float2(*reinterpret_cast<const __half2 *>(&v)); }

// whether one of two (eight) 16-bit numbers is an infinity or not a number: its exponent bits are all ones
template <typename T>
struct ExponentBits { static constexpr u32 mask = 0x7f80u; };
template <>
struct ExponentBits<__half> { static constexpr u32 mask = 0x7c00u; };
template <typename T>
__device__ __forceinline__ bool not_finite2(u32 v) {
  constexpr u32 lo = ExponentBits<T>::mask, hi = lo << 16;
  return (v & lo) == lo || (v & hi) == hi;
}
template <typename T>
__device__ __forceinline__ bool not_finite8(uint4 v) {
  return not_finite2<T>(v.x) || not_finite2<T>(v.y) || not_finite2<T>(v.z) || not_finite2<T>(v.w);
}

// The weights' exponents are counted from the running maximum minus `to - MAX`: the largest weight is 2^to, where MAX is the power by
// which weights may pass the one of the running maximum.  A float16 holds 2^15, and nothing below 2^-25: with the largest
// weight at 1, 40000 keys of 2^-25.6 each were lost beside one of 1 (out by 8e-4 of the values, where a float16 shows 5e-4).
// The sums carry the same factor, so that the results do not.  A bfloat16 has the range of the 32-bit sums.
template <typename T, int MAX>
struct WeightLift { static constexpr float value = 0.0f; };
template <int MAX>
struct WeightLift<__half, MAX> { static constexpr float value = 15.0f - MAX; };

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A sum that counted from 2^(m + d), d <= 0, now that it counts from 2^m.  WIDE: over codes a maximum holds the logarithm of a scale and may move by 180 octaves, while
// the sum's weights are as far above 1: 2^d alone would be 0 and the sum lost.
template <bool WIDE>
__device__ __forceinline__ float moved_sum(float sum, float d) {
  if (!WIDE) return exp2_approx(d) * sum;
  const float h = exp2_approx(0.5f * d);
  return sum * h * h;
}

__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// cap * tanh(u), u = x / cap, good to some 2^-20 of x however large the cap is.  From |u| = 1/4 on it is cap * (1 - 2 / (1 + e^2u)), whose
// error is some 2^-22 of the cap (the hardware's tanh is good to 2^-11 of it only, which would show in the weights).  Below,
// that would be any part of x, up to all of it; there it is x * (1 - u^2/3 + 2u^4/15 - 17u^6/315), whose next term is below
// 2^-21.  In units of log2, and of w = 2u log2(e), the exponent.
constexpr float kCapSeries = 0.25f * 2.0f * kLog2e;                      // |w| below: the series
constexpr float kCapUnit = (kLn2 / 2.0f) * (kLn2 / 2.0f);                // u^2 = kCapUnit * w^2
constexpr float kCap1 = -kCapUnit / 3.0f, kCap2 = 2.0f * kCapUnit * kCapUnit / 15.0f, kCap3 = -17.0f * kCapUnit * kCapUnit * kCapUnit / 315.0f;

// w of a dot product of 1; finite, so that a dot product of 0 stays 0 under the smallest caps
__device__ __forceinline__ float cap_in(const Attn &a) { return fminf(a.scale * (2.0f * kLog2e) / a.softcap, 1e38f); }

// `in` as above, `out` is cap * log2(e), `linear` is scale * log2(e)
__device__ __forceinline__ float capped_log2(float dot, float in, float out, float linear) {
  const float w = dot * in, q = w * w;
  const float small = dot * linear * fmaf(q, fmaf(q, fmaf(q, kCap3, kCap2), kCap1), 1.0f);
  const float large = fmaf(-2.0f * out, rcp_approx(1.0f + exp2_approx(w)), out);
  return fabsf(w) < kCapSeries ? small : large;
}

// How a row ends.  `m` (in units of log2) and `l` are its maximum and sum: weights count from 2^m.  Alone a row is divided by its sum; of
// the shared keys it is left as it is; of a request's own keys it is first joined to what was left of the shared ones.
struct RowEnd {
  float f;
  __device__ __forceinline__ RowEnd(const Attn &a, const NoRows &, i64 tok, int head, int, float m, float l, bool first) {
    f = l == 0.0f ? 0.0f : 1.0f / l;
    if (first && a.lse) a.lse[tok * a.hq + head] = l == 0.0f ? -INFINITY : m * kLn2 + logf(l);
  }
  template <typename T>
  __device__ __forceinline__ void write4(const Attn &a, i64 tok, int head, int col, float4 o) const {
    *(uint2 *)((u16 *)a.out + tok * a.o_t + (i64)head * a.o_h + col) = make_uint2(pack2<T>(o.x * f, o.y * f), pack2<T>(o.z * f, o.w * f));
  }
  template <typename T>
  __device__ __forceinline__ void write32(const Attn &a, i64 tok, int head, int col, const float *o) const {
    uint4 *to = (uint4 *)((u16 *)a.out + tok * a.o_t + (i64)head * a.o_h + col);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      to[k] = make_uint4(pack2<T>(o[8 * k] * f, o[8 * k + 1] * f), pack2<T>(o[8 * k + 2] * f, o[8 * k + 3] * f), pack2<T>(o[8 * k + 4] * f, o[8 * k + 5] * f),
                         pack2<T>(o[8 * k + 6] * f, o[8 * k + 7] * f));
  }
};

struct PrefixRowEnd {
  float *to;
  __device__ __forceinline__ PrefixRowEnd(const PrefixAttn &a, const NoRows &, i64 tok, int head, int dim, float m, float l, bool first) {
    to = a.mid_o + (tok * a.hq + head) * dim;
    if (first) {
      a.mid_ml[tok * a.hq + head] = make_float2(m, l);
      a.mid_at[tok * a.hq + head] = make_int4(0, -1, 0, 0);
    }
  }
  template <typename T>
  __device__ __forceinline__ void write4(const PrefixAttn &, i64, int, int col, float4 o) const { *(float4 *)(to + col) = o; }
  template <typename T>
  __device__ __forceinline__ void write32(const PrefixAttn &, i64, int, int col, const float *o) const {
#pragma unroll
    for (int k = 0; k < 8; ++k) *(float4 *)(to + col + 4 * k) = make_float4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
  }
};

struct OwnRowEnd {
  float f, g;                  // of its own sums, and of those over the shared keys
  const float *from;           // NULL: none
  __device__ __forceinline__ OwnRowEnd(const OwnAttn &a, const CoveredRows &rows, i64 tok, int head, int dim, float m, float l, bool first) {
    wait_for_first(a);
    from = nullptr;
    float2 mid = make_float2(-INFINITY, 0.0f);
    if (tok >= rows.from && tok < rows.to) {
      mid = __ldcg(a.mid_ml + tok * a.hq + head);
      from = a.mid_o + (tok * a.hq + head) * dim;
    }
    const float top = fmaxf(m, mid.x), base = top == -INFINITY ? 0.0f : top;
    f = exp2_approx(m - base);
    g = exp2_approx(mid.x - base);
    const float sum = f * l + g * mid.y, inverse = sum == 0.0f ? 0.0f : 1.0f / sum;
    if (first && a.lse) a.lse[tok * a.hq + head] = sum == 0.0f ? -INFINITY : top * kLn2 + logf(sum);
    f *= inverse;
    g *= inverse;
  }
  __device__ __forceinline__ float4 joined(float4 o, int col) const {
    const float4 x = from ? __ldcg((const float4 *)(from + col)) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    return make_float4(o.x * f + x.x * g, o.y * f + x.y * g, o.z * f + x.z * g, o.w * f + x.w * g);
  }
  template <typename T>
  __device__ __forceinline__ void write4(const OwnAttn &a, i64 tok, int head, int col, float4 o) const {
    o = joined(o, col);
    *(uint2 *)((u16 *)a.out + tok * a.o_t + (i64)head * a.o_h + col) = make_uint2(pack2<T>(o.x, o.y), pack2<T>(o.z, o.w));
  }
  template <typename T>
  __device__ __forceinline__ void write32(const OwnAttn &a, i64 tok, int head, int col, const float *o) const {
    uint4 *to = (uint4 *)((u16 *)a.out + tok * a.o_t + (i64)head * a.o_h + col);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float4 x = joined(make_float4(o[8 * k], o[8 * k + 1], o[8 * k + 2], o[8 * k + 3]), col + 8 * k);
      const float4 y = joined(make_float4(o[8 * k + 4], o[8 * k + 5], o[8 * k + 6], o[8 * k + 7]), col + 8 * k + 4);
      to[k] = make_uint4(pack2<T>(x.x, x.y), pack2<T>(x.z, x.w), pack2<T>(y.x, y.y), pack2<T>(y.z, y.w));
    }
  }
};

template <typename A>
struct EndOf { typedef RowEnd type; };
template <>
struct EndOf<PrefixAttn> { typedef PrefixRowEnd type; };
template <>
struct EndOf<OwnAttn> { typedef OwnRowEnd type; };

// Writes four columns of a finished row, rounded once.  A row that sees no key has sum 0 and gives 0 and
// -inf.  `row` counts (token, head of the group) pairs of the request, `top` is in units of log2.
template <typename T, int D, typename A, typename Rows>
__device__ __forceinline__ void finish_row(const A &a, const Rows &rows, int q0, i64 row, u32 h, int col, float4 acc, float top, float sum) {
  const int tok = (int)(row / a.group), head = (int)(row - (i64)tok * a.group) + (int)(h * a.group);
  const typename EndOf<A>::type end(a, rows, q0 + tok, head, D, top, sum, col == 0);
  end.template write4<T>(a, q0 + tok, head, col, acc);
}

// Joins the parts of a unit that blocks i0..i1 left, in the order of the key axis.  Block-collective.  What it costs
// is waiting for loads, 0.7 us a time, so a thread keeps those of AHEAD parts in flight: the 33 parts of one token over
// 4097 keys take 22 us in all with 2, 16 with 4, 14 with 8, no less with 16.
template <typename T, int D, int ROWS, int NT, int ITEMS, int AHEAD, bool WIDE, typename A, typename Rows>
__device__ __forceinline__ void join_parts(const A &a, const Rows &covered, const Cursor &c, i64 row0, int rows, u32 i0, u32 i1) {
  const int items = rows * (D / 4);
  for (int x0 = (int)threadIdx.x; x0 < items; x0 += NT * ITEMS) {
    float top[ITEMS], sum[ITEMS];
    float4 acc[ITEMS];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) { top[k] = -INFINITY; sum[k] = 0.0f; acc[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f); }
    for (u32 i = i0; i <= i1; i += AHEAD) {
      float2 ml[ITEMS][AHEAD];
      float4 v[ITEMS][AHEAD];
#pragma unroll
      for (int k = 0; k < ITEMS; ++k)
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
          ml[k][j] = make_float2(-INFINITY, 0.0f);
          v[k][j] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          const int x = x0 + k * NT, row = x / (D / 4);
          if (x < items && i + j <= i1) {
            const i64 at = (i64)(2 * (i + j) + (i + j == i0 ? 1 : 0)) * ROWS + row;
            ml[k][j] = __ldcg((const float2 *)(a.part_ml + at * 2));
            v[k][j] = __ldcg((const float4 *)(a.part_o + at * D + (x - row * (D / 4)) * 4));
          }
        }
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        float now = top[k];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) now = fmaxf(now, ml[k][j].x);
        const float base = now == -INFINITY ? 0.0f : now, f = exp2_approx(top[k] - base);
        sum[k] = moved_sum<WIDE>(sum[k], top[k] - base);
        top[k] = now;
        acc[k].x *= f; acc[k].y *= f; acc[k].z *= f; acc[k].w *= f;
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
          const float g = exp2_approx(ml[k][j].x - base);
          sum[k] += WIDE ? moved_sum<WIDE>(ml[k][j].y, ml[k][j].x - base) : g * ml[k][j].y;
          acc[k].x += g * v[k][j].x; acc[k].y += g * v[k][j].y; acc[k].z += g * v[k][j].z; acc[k].w += g * v[k][j].w;
        }
      }
    }
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const int x = x0 + k * NT, row = x / (D / 4);
      if (x < items) finish_row<T, D>(a, covered, c.req.q0, row0 + row, c.h, (x - row * (D / 4)) * 4, acc[k], top[k], sum[k]);
    }
  }
}

}  // namespace paged
}  // namespace gorio
