// Attention of few rows over a paged cache: the single-token form.
//
// One unit is up to 16 rows ((token, query head) pairs that share a key head).  For 16 rows a key costs
// 4 * 16 * D operations for its 4 * D bytes, far below what the matrix pipe does in the time the bytes
// take, so the kernel is bound by the cache's bytes and everything in it serves one end: loads in
// flight at all times.  A block is four warps; of a tile of 64 keys each warp takes 16, loads them itself
// into a ring of its own (cp.async, three tiles deep, 16 bytes a lane) and keeps its own running
// maximum, sum and output, so that no barrier stands in the loop.  The warps' four partial results
// are joined at the end of a unit, in the ring slot that each warp has just used up.
// Blocks take equal shares of all keys of the call (the plan); a unit that is cut between blocks
// leaves parts in the workspace that its last block joins.
// 64 ragged requests over up to 8192 keys (32 heads of 128, 8 key heads, 1.06 GB) take 168 us in a burst, 176 sustained:
// 6.0 to 6.3 TB/s, where a copy reaches 6.55.
//
// Scores: s = q.k (16-bit operands, 32-bit sums), then in 32 bits the scale, cap, bias and mask, the running
// maximum m and sum l of 2^(x - m), x in units of log2.  The weights 2^(x - m) <= 1 (float16: <= 2^15, see WeightLift) are rounded to the
// cache's type for the second product, whose error that doubles at most; l sums them unrounded.
#pragma once
#include "common.cuh"
#include "mma.cuh"

namespace gorio {
namespace paged {

namespace {

constexpr int kRows = 16;
constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kWarpKeys = 16;
constexpr int kTile = kWarps * kWarpKeys;
constexpr int kStages = 3;
constexpr int kOver = 1;            // a unit's start and end cost about what a tile does
// Behind shared keys, requests' own are few: with more places without work between units fewer of them are cut, which there costs more than uneven
// shares do (64 requests of up to 1024 own keys behind 16391 shared ones: 102 us with 1, 96 with 3 and with 6, 100 with 12).
template <typename A>
constexpr int kOverOf = kOver;
template <>
constexpr int kOverOf<OwnAttn> = 4;
constexpr float kSpread = 0.25f;    // joining 16 parts takes about what a tile does
// As many as shared memory (24 KB a warp at head size 128) and registers hold: at head size 64, 64 ragged single-token requests take
// 96 us with four blocks, 101 with three, 122 with two; more stages instead did nothing.
template <int D>
constexpr int kBlocksPerSm = D == 64 ? 4 : D == 96 ? 3 : 2;

template <int D>
struct RowsShared {
  // per warp and stage: 16 keys, then 16 values; the same bytes hold the warp's 16 x D output at a unit's end
  u16 ring[kWarps][kStages][2][kWarpKeys * D];
  float m[kWarps][kRows], l[kWarps][kRows];
  PlanShared plan;
  u32 last;
};

// Rows of D elements in shared memory: 16-byte pieces, xor-ed with the row so that eight consecutive rows'
// pieces of one column lie in different banks (D = 96: rows are 12 pieces, odd rows lie half of the banks on
// already, and the xor stays within the low two bits and so inside the row).
template <int D>
__device__ __forceinline__ int piece_at(int row, int piece) {
  constexpr int P = D / 8;
  if (P % 8 == 0) return row * P + (piece ^ (row & 7));
  return row * P + (piece ^ ((row >> 1) & 3));
}

template <typename T, int D, bool SCORED, typename A>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm<D>) attention_rows_kernel(const A a) {
  extern __shared__ __align__(128) unsigned char raw[];
  RowsShared<D> &sh = *(RowsShared<D> *)raw;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  let_second_begin(a);
  const Plan plan = block_plan<kRows, kTile, kOverOf<A>, kThreads>(a, sh.plan, kSpread);
  if (plan.begin >= plan.end) {
    wait_for_first(a);                           // so that this kernel never ends before the first
    return;
  }
  const auto covered = covered_rows(a);

  constexpr int P = D / 8;                       // 16-byte pieces of a row
  constexpr int kLoads = kWarpKeys * P / 32;     // cp.async a lane for 16 rows
  constexpr float kLift = WeightLift<T, 0>::value;
  const float to_log2 = a.scale * kLog2e, to_cap = SCORED && a.softcap > 0.0f ? cap_in(a) : 0.0f;

  // --- the loading side: a cursor that runs ahead, and the cache row of the next tile's key that this lane looks up.
  // Where pages are multiples of a warp's 16 keys, those keys follow each other in one page: one address a lane and steps
  // from there, instead of two shuffles and four products in 64 bits for each of its rows.
  const bool in_line = 32 % P == 0 && a.page % kWarpKeys == 0;
  Cursor ld = plan.first;
  u32 ld_left = plan.end - plan.begin;
  settle<kRows, kTile, kOverOf<A>>(a, ld, ld_left, plan.fill);
  int key_page = -1, key_in = 0;                 // of key (lane & 15) of the tile at ld; -1: zeros
  auto look_up = [&]() {
    if (ld_left == 0) return;
    const int key0 = (ld.span.first + ld.at) * kTile + warp * kWarpKeys, key = in_line ? key0 : key0 + (lane & 15);
    key_page = -1;
    if (in_line ? key0 + kWarpKeys > ld.span.lo && key0 < ld.span.hi : key >= ld.span.lo && key < ld.span.hi) {
      const u32 at = (u32)key / a.page;
      key_in = (int)((u32)key - at * a.page);
      const int pg = __ldg(a.tables + (i64)ld.r * a.tab_r + at);
      if ((u32)pg < a.n_pages) key_page = pg;
    }
  };
  auto issue = [&](int stage) {
    if (ld_left) {
      const u16 *kh = (const u16 *)a.kp + (i64)ld.h * a.k_h, *vh = (const u16 *)a.vp + (i64)ld.h * a.v_h;
      u16 *ks = sh.ring[warp][stage][0], *vs = sh.ring[warp][stage][1];
      if (in_line) {
        const int key0 = (ld.span.first + ld.at) * kTile + warp * kWarpKeys, row0 = lane / P, piece = lane % P;
        const int from = key_page >= 0 ? ld.span.lo - key0 : kWarpKeys, to = ld.span.hi - key0;      // rows to read
        const i64 page = key_page >= 0 ? key_page : 0, tok = key_page >= 0 ? key_in + row0 : 0;
        const u16 *k_at = kh + page * a.k_p + tok * a.k_t + piece * 8, *v_at = vh + page * a.v_p + tok * a.v_t + piece * 8;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const int row = i * (32 / P) + row0;
          const u32 bytes = row >= from && row < to ? 16u : 0u;       // 0: the piece is filled with zeros
          cp_async16(ks + piece_at<D>(row, piece) * 8, k_at, bytes);
          cp_async16(vs + piece_at<D>(row, piece) * 8, v_at, bytes);
          k_at += (32 / P) * a.k_t;
          v_at += (32 / P) * a.v_t;
        }
      } else
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int x = i * 32 + lane, row = x / P, piece = x - row * P;
        const int pg = __shfl_sync(0xffffffffu, key_page, row), in = __shfl_sync(0xffffffffu, key_in, row);
        const u32 bytes = pg >= 0 ? 16u : 0u;
        const i64 page = pg >= 0 ? pg : 0, tok = pg >= 0 ? in : 0;
        cp_async16(ks + piece_at<D>(row, piece) * 8, kh + page * a.k_p + tok * a.k_t + piece * 8, bytes);
        cp_async16(vs + piece_at<D>(row, piece) * 8, vh + page * a.v_p + tok * a.v_t + piece * 8, bytes);
      }
      --ld_left;
      ++ld.at;
      settle<kRows, kTile, kOverOf<A>>(a, ld, ld_left, plan.fill);
      look_up();
    }
    cp_async_commit();
  };
  look_up();
#pragma unroll 1
  for (int s = 0; s < kStages - 1; ++s) issue(s);

  // --- the computing side
  Cursor c = plan.first;
  int stage = 0;
  const int g = lane >> 2, t4 = lane & 3;
  u32 left = plan.end - plan.begin;
  for (settle<kRows, kTile, kOverOf<A>>(a, c, left, plan.fill); left; settle<kRows, kTile, kOverOf<A>>(a, c, left, plan.fill)) {
    const int from = c.at;
    const int to = (int)min((u32)c.span.tiles, (u32)from + left);
    const i64 row0 = (i64)c.m * kRows;
    const int rows = (int)min((i64)kRows, (i64)c.req.n * a.group - row0);
    // this lane's two rows: g and g + 8
    u32 qf[D / 16][4];
    int lo_key[2], hi_key[2];                     // visible keys of the row
    float slope[2];
    int pos[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = g + 8 * i;
      const int tok = row < rows ? (int)((row0 + row) / a.group) : 0;
      const int head = row < rows ? (int)((row0 + row) - (i64)tok * a.group) + (int)(c.h * a.group) : 0;
      pos[i] = position_of(a, c.req, tok);
      hi_key[i] = a.causal ? min(c.req.len, pos[i] + 1) : c.req.len;
      lo_key[i] = a.window ? (int)max((i64)0, (i64)pos[i] - a.window + 1) : 0;
      slope[i] = SCORED && a.slopes ? a.slopes[head] * kLog2e : 0.0f;
      const u16 *src = (const u16 *)a.q + (i64)(c.req.q0 + tok) * a.q_t + (i64)head * a.q_h + t4 * 2;
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        qf[k][i] = row < rows ? *(const u32 *)(src + k * 16) : 0u;
        qf[k][2 + i] = row < rows ? *(const u32 *)(src + k * 16 + 8) : 0u;
      }
    }
    float o[D / 8][4];
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};
#pragma unroll
    for (int n = 0; n < D / 8; ++n)
#pragma unroll
      for (int x = 0; x < 4; ++x) o[n][x] = 0.0f;

    for (int at = from; at < to; ++at) {
      issue(stage == 0 ? kStages - 1 : stage - 1);          // the slot that the tile before has left
      cp_async_wait<kStages - 1>();
      __syncwarp();
      const u16 *ks = sh.ring[warp][stage][0], *vs = sh.ring[warp][stage][1];
      const int key0 = (c.span.first + at) * kTile + warp * kWarpKeys;
      float s[2][4];
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int x = 0; x < 4; ++x) s[n][x] = 0.0f;
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        u32 b[4];
        const int row = (lane & 7) + ((lane >> 4) << 3), piece = 2 * k + ((lane >> 3) & 1);
        ldmatrix4(b, ks + piece_at<D>(row, piece) * 8);
        mma16816<T>(s[0], qf[k], b[0], b[1]);
        mma16816<T>(s[1], qf[k], b[2], b[3]);
      }
      // scores in units of log2, masked
      const bool all_seen = __all_sync(0xffffffffu, key0 >= lo_key[0] && key0 >= lo_key[1] && key0 + kWarpKeys <= hi_key[0] &&
                                                        key0 + kWarpKeys <= hi_key[1]);
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int i = x >> 1, key = key0 + n * 8 + t4 * 2 + (x & 1);
          if (SCORED) {
            const float v = a.softcap > 0.0f ? capped_log2(s[n][x], to_cap, a.softcap * kLog2e, to_log2) : s[n][x] * to_log2;
            s[n][x] = v + slope[i] * (float)(key - pos[i]);
          } else {
            s[n][x] *= to_log2;
          }
          if (!all_seen && (key < lo_key[i] || key >= hi_key[i])) s[n][x] = -INFINITY;
        }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float top = fmaxf(fmaxf(s[0][2 * i], s[0][2 * i + 1]), fmaxf(s[1][2 * i], s[1][2 * i + 1]));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const float was = m[i];
        m[i] = fmaxf(was, top);
        const float most = m[i] == -INFINITY ? 0.0f : m[i], base = most - kLift;   // nothing seen yet: every weight is 2^-inf = 0
        if (__any_sync(0xffffffffu, m[i] != was)) {
          const float f = exp2_approx(was - most);
          l[i] *= f;
#pragma unroll
          for (int n = 0; n < D / 8; ++n) { o[n][2 * i] *= f; o[n][2 * i + 1] *= f; }
        }
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const float w = exp2_approx(s[n][2 * i + x] - base);
            s[n][2 * i + x] = w;
            l[i] += w;
          }
      }
      // A weight of 0 does not hide a value that is not finite from the matrix product (0 * inf), so where some rows do
      // not see some keys of the tile and a value there is not finite, the sum over values is made without it.
      bool odd = false;
      if (!all_seen) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const int x = i * 32 + lane, row = x / P;
          odd |= not_finite8<T>(*(const uint4 *)(vs + piece_at<D>(row, x - row * P) * 8));
        }
        odd = __any_sync(0xffffffffu, odd);
      }
      if (!odd) {
        const u32 pf[4] = {pack2<T>(s[0][0], s[0][1]), pack2<T>(s[0][2], s[0][3]), pack2<T>(s[1][0], s[1][1]), pack2<T>(s[1][2], s[1][3])};
#pragma unroll
        for (int n = 0; n < D / 16; ++n) {
          u32 b[4];
          const int row = (lane & 7) + (((lane >> 3) & 1) << 3), piece = 2 * n + (lane >> 4);
          ldmatrix4t(b, vs + piece_at<D>(row, piece) * 8);
          mma16816<T>(o[2 * n], pf, b[0], b[1]);
          mma16816<T>(o[2 * n + 1], pf, b[2], b[3]);
        }
      } else {
        for (int j = 0; j < kWarpKeys; ++j) {
          const int src = (lane & ~3) | ((j & 7) >> 1), key = key0 + j;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float s0 = j & 1 ? s[0][2 * i + 1] : s[0][2 * i], s1 = j & 1 ? s[1][2 * i + 1] : s[1][2 * i];
            const float w = __shfl_sync(0xffffffffu, j & 8 ? s1 : s0, src);
            if (key < lo_key[i] || key >= hi_key[i]) continue;
#pragma unroll
            for (int n = 0; n < D / 8; ++n) {
              const float2 v = unpack2<T>(*(const u32 *)(vs + piece_at<D>(j, n) * 8 + t4 * 2));
              o[n][2 * i] += w * v.x;
              o[n][2 * i + 1] += w * v.y;
            }
          }
        }
      }
      __syncwarp();
      if (at + 1 < to) stage = stage + 1 == kStages ? 0 : stage + 1;     // at the unit's end the slot is needed below
    }
    left -= (u32)(to - from);
    c.at = to;

    // --- join the four warps
    float *mine = (float *)sh.ring[warp][stage];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
      const int row = g + 8 * i;
      if (t4 == 0) { sh.m[warp][row] = m[i] - kLift; sh.l[warp][row] = l[i]; }
      if (row < rows) {
#pragma unroll
        for (int n = 0; n < D / 8; ++n) *(float2 *)(mine + row * D + (n ^ (row & 3)) * 8 + t4 * 2) = make_float2(o[n][2 * i], o[n][2 * i + 1]);
      }
    }
    __syncthreads();
    const bool whole = from == 0 && to == c.span.tiles;
    const u32 unit0 = plan.end - left - (u32)to;   // the unit's place on the line
    const u32 i0 = whole ? 0 : plan.shares.owner(unit0);
    const u32 slot = 2 * blockIdx.x + (blockIdx.x == i0 ? 1 : 0);
    for (int x = tid; x < rows * (D / 4); x += kThreads) {
      const int row = x / (D / 4), col = (x - row * (D / 4)) * 4;
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) top = fmaxf(top, sh.m[w][row]);
      const float base = top == -INFINITY ? 0.0f : top;
      float sum = 0.0f;
      float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float f = exp2_approx(sh.m[w][row] - base);
        const float4 v = *(const float4 *)((const float *)sh.ring[w][stage] + row * D + ((col >> 3) ^ (row & 3)) * 8 + (col & 7));
        sum += f * sh.l[w][row];
        acc.x += f * v.x; acc.y += f * v.y; acc.z += f * v.z; acc.w += f * v.w;
      }
      if (whole) {
        finish_row<T, D>(a, covered, c.req.q0, row0 + row, c.h, col, acc, top, sum);
      } else {
        *(float4 *)(a.part_o + ((i64)slot * kRows + row) * D + col) = acc;
        if (col == 0) *(float2 *)(a.part_ml + ((i64)slot * kRows + row) * 2) = make_float2(top, sum);
        if (leaves_parts(a) && col == 0 && blockIdx.x == i0) {
          const int tok = (int)((row0 + row) / a.group), head = (int)((row0 + row) - (i64)tok * a.group) + (int)(c.h * a.group);
          tell_parts(a, (i64)(c.req.q0 + tok) * a.hq + head, i0, plan.shares.owner(unit0 + (u32)c.span.tiles - 1), row, kRows);
        }
      }
    }
    if (!whole && !leaves_parts(a)) {
      const u32 i1 = plan.shares.owner(unit0 + (u32)c.span.tiles - 1);
      __threadfence();
      __syncthreads();
      if (tid == 0) {
        const u32 before = atomicAdd(a.arrived + i0, 1u);
        sh.last = before == i1 - i0;
        if (sh.last) a.arrived[i0] = 0;            // ready for the next call
        __threadfence();
      }
      __syncthreads();
      if (sh.last) join_parts<T, D, kRows, kThreads, 1, 8, false>(a, covered, c, row0, rows, i0, i1);
    }
    __syncthreads();
    stage = stage + 1 == kStages ? 0 : stage + 1;
  }
  cp_async_wait<0>();
  wait_for_first(a);
}

template <typename T, int D, bool SCORED, typename A>
cudaError_t launch(const A &a, u32 sms, cudaStream_t s) {
  static bool ready[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 64 && !ready[dev]) {
    e = cudaFuncSetAttribute(attention_rows_kernel<T, D, SCORED, A>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(RowsShared<D>));
    if (e != cudaSuccess) return e;
    ready[dev] = true;
  }
  return launch_kernel<A>(attention_rows_kernel<T, D, SCORED, A>, sms * kBlocksPerSm<D>, kThreads, sizeof(RowsShared<D>), s, a);
}

template <typename T, int D, typename A>
cudaError_t pick_scored(const A &a, u32 sms, cudaStream_t s) {
  return a.softcap > 0.0f || a.slopes ? launch<T, D, true>(a, sms, s) : launch<T, D, false>(a, sms, s);
}

template <typename T, typename A>
cudaError_t pick_dim(const A &a, int dim, u32 sms, cudaStream_t s) {
  if (dim == 64) return pick_scored<T, 64>(a, sms, s);
  if (dim == 96) return pick_scored<T, 96>(a, sms, s);
  return pick_scored<T, 128>(a, sms, s);
}

template <typename A>
cudaError_t launch_rows_of(const A &a, int dtype, int dim, u32 sms, cudaStream_t s) {
  return dtype == 0 ? pick_dim<__nv_bfloat16>(a, dim, sms, s) : pick_dim<__half>(a, dim, sms, s);
}

}  // namespace
}  // namespace paged
}  // namespace gorio
