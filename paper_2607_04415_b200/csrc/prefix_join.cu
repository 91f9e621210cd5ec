// Joins the parts of rows over shared keys.
#include "paged/common.cuh"
#include "paged/mma.cuh"

namespace gorio {
namespace paged {

namespace {

constexpr int kThreads = 256;

// A warp a row: its parts' maxima and sums, a lane each, and their columns, four a lane, 8 parts' loads in flight with the maxima's.  In the order of
// the key axis, so that results do not depend on timing.  What it costs is three trips to L2, one after the other.
template <int D>
__global__ void __launch_bounds__(kThreads, 4) prefix_join_kernel(const PrefixAttn a, const u32 part_rows) {
  let_next_begin();
  wait_for_kernel();
  constexpr int kAhead = 8;
  const int lane = threadIdx.x & 31;
  const i64 row = (i64)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  if (row >= (i64)a.n_tok * a.hq) return;
  // Whole.  Or: rows of no group, and all rows of a first kernel that gave up, have anything here; it must not lead out of the parts.
  const int4 at = __ldcg(a.mid_at + row);
  if (at.y < at.x || at.x < 0 || at.z < 0 || at.z >= at.w || at.w > 256 || (u64)(2 * (i64)at.y + 2) * (u32)at.w > part_rows) return;
  const int parts = at.y - at.x + 1;
  const i64 start = (i64)(2 * at.x + 1) * at.w + at.z;             // the first part is in its block's second place, the others in their first
  auto place = [&](int k) { return start + (k == 0 ? 0 : (2 * k - 1) * (i64)at.w); };
  const bool mine = lane < D / 4;
  float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  float top = -INFINITY, sum = 0.0f;
  for (int k0 = 0; k0 < parts; k0 += 32) {                         // 32 parts, a lane's maximum and sum each
    float2 x = make_float2(-INFINITY, 0.0f);
    if (k0 + lane < parts) x = __ldcg((const float2 *)a.part_ml + place(k0 + lane));
    const int some = min(32, parts - k0);
    float base = 0.0f;
    for (int k1 = 0; k1 < some; k1 += kAhead) {
      float4 v[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        v[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (k1 + i < some && mine) v[i] = __ldcg((const float4 *)(a.part_o + place(k0 + k1 + i) * D) + lane);
      }
      if (k1 == 0) {
        float now = x.x;
#pragma unroll
        for (int d = 16; d; d >>= 1) now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, d));
        now = fmaxf(now, top);
        base = now == -INFINITY ? 0.0f : now;
        const float f = exp2_approx(top - base);
        top = now;
        x.x = exp2_approx(x.x - base);                             // the part's weight from here on
        x.y *= x.x;
        float part_sums = x.y;
#pragma unroll
        for (int d = 16; d; d >>= 1) part_sums += __shfl_xor_sync(0xffffffffu, part_sums, d);
        sum = sum * f + part_sums;
        acc.x *= f; acc.y *= f; acc.z *= f; acc.w *= f;
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const float g = __shfl_sync(0xffffffffu, x.x, (k1 + i) & 31);
        acc.x += g * v[i].x; acc.y += g * v[i].y; acc.z += g * v[i].z; acc.w += g * v[i].w;
      }
    }
  }
  if (mine) *(float4 *)(a.mid_o + row * D + lane * 4) = acc;
  if (lane == 0) a.mid_ml[row] = make_float2(top, sum);
}

}  // namespace

cudaError_t launch_prefix_join(const PrefixAttn &a, int dim, u32 sms, cudaStream_t s) {
  const u64 rows = (u64)a.n_tok * a.hq;                            // below 2^31
  const u32 blocks = (u32)((rows + kThreads / 32 - 1) / (kThreads / 32)), part_rows = sms * kPartRowsPerSm;
  auto *const kernel = dim == 64 ? prefix_join_kernel<64> : dim == 96 ? prefix_join_kernel<96> : prefix_join_kernel<128>;
  return launch_kernel<Joining>(kernel, blocks, kThreads, 0, s, a, part_rows);
}

}  // namespace paged
}  // namespace gorio
