// Attention of few rows over a quantised paged cache: the single-token form.
//
// The plan, the units of 16 rows and the four warps with a ring each are those of the 16-bit cache's kernel (rows.cuh).  What is
// different comes from the 8 bits.  The same bytes in flight are twice as many keys, so a warp's tile is 32 keys.  Codes
// become float16 in registers, exactly, in the lanes and the order in which the matrix instructions want them:
//   keys     a 16-byte piece of a row is what one product over 16 elements takes.  A lane gets four neighbouring codes of a
//            key, and its queries are loaded in the same order, so that nothing is moved.
//   values   read transposed by pairs of codes, a lane gets two neighbouring columns of two neighbouring keys; taken apart they are
//            the operand of one product for the even columns and of one for the odd ones.
// Products of queries (float16, a power of two a row) and codes are summed in 32 bits; the key's scale comes after.  The value's scale
// goes to the weight before that is rounded to float16: 2^(x - base) * scale.  So that the largest such weight is 2^15 whatever the scales are,
// a row's running maximum is that of x + log2(scale).
#pragma once
#include "coded.cuh"
#include "rows.cuh"

namespace gorio {
namespace paged {

namespace {

constexpr int kCodedKeys = 32;                   // of a warp's tile
constexpr int kCodedTile = kWarps * kCodedKeys;
constexpr int kCodedStages = 3;
template <int D>
constexpr int kCodedBlocks = D == 64 ? 4 : D == 96 ? 3 : 2;
constexpr float kScaleRange = 80.0f;             // a scale's power of two that the maximum counts, at most

template <int D>
struct CodedShared {
  // per warp and stage: the codes of 32 keys, then of 32 values; the same bytes hold the warp's 16 x D output at a unit's end
  u8 ring[kWarps][kCodedStages][2][kCodedKeys * D];
  float scales[kWarps][kCodedStages][2][kCodedKeys];
  float m[kWarps][kRows], l[kWarps][kRows];
  PlanShared plan;
  u32 last;
};

// Rows of D bytes in 16-byte pieces, xor-ed so that eight consecutive rows' pieces of one column lie in different banks.
template <int D>
__device__ __forceinline__ int code_piece(int row, int piece) {
  constexpr int P = D / 16;
  if (P == 8) return row * P + (piece ^ (row & 7));
  if (P == 4) return row * P + (piece ^ ((row >> 1) & 3));
  return row * P + (piece ^ ((row >> 2) & 1));   // 96 bytes: four rows lie apart by themselves, the next four one piece on
}

// log2 of a value's scale, cut to what the running maximum counts
__device__ __forceinline__ float scale_log2(float scale) {
  float e;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(fabsf(scale)));
  return fminf(fmaxf(e, -kScaleRange), kScaleRange);          // also of a scale that is not a number
}

// q.k of one 16 x 8 tile and 16 elements, of one 16 x 8 output tile and 16 keys
__device__ __forceinline__ void mma_half(float (&c)[4], const u32 (&a)[4], u32 b0, u32 b1) { mma16816<__half>(c, a, b0, b1); }

template <typename T, Format F, int D, bool SCORED>
__global__ void __launch_bounds__(kThreads, kCodedBlocks<D>) coded_rows_kernel(const CodedAttn a) {
  extern __shared__ __align__(128) unsigned char raw[];
  CodedShared<D> &sh = *(CodedShared<D> *)raw;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const Plan plan = block_plan<kRows, kCodedTile, kOver, kThreads>(a, sh.plan, kSpread);
  if (plan.begin >= plan.end) return;

  constexpr int P = D / 16;                      // 16-byte pieces of a row
  constexpr int kLoads = kCodedKeys * P / 32;    // cp.async a lane for 32 rows
  constexpr float kLift = 15.0f;
  const float to_log2 = a.scale * kLog2e, to_cap = SCORED && a.softcap > 0.0f ? cap_in(a) : 0.0f;

  // --- the loading side: a cursor that runs ahead; lane i looks up the cache row of the next tile's key i.  Where pages are
  // multiples of 16 keys, a half of the tile follows on in one page: one address for each half, and steps from there.
  const bool in_line = 32 % P == 0 && a.page % 16 == 0;
  Cursor ld = plan.first;
  u32 ld_left = plan.end - plan.begin;
  settle<kRows, kCodedTile, kOver>(a, ld, ld_left, plan.fill);
  int key_page = -1, key_in = 0;                 // of key `lane` of the warp's tile at ld; -1: zeros
  auto look_up = [&]() {
    if (ld_left == 0) return;
    const int key = (ld.span.first + ld.at) * kCodedTile + warp * kCodedKeys + lane;
    key_page = -1;
    if (key >= ld.span.lo && key < ld.span.hi) {
      const u32 at = (u32)key / a.page;
      key_in = (int)((u32)key - at * a.page);
      const int pg = __ldg(a.tables + (i64)ld.r * a.tab_r + at);
      if ((u32)pg < a.n_pages) key_page = pg;
    }
  };
  auto issue = [&](int stage) {
    if (ld_left) {
      const u8 *kh = (const u8 *)a.kp + (i64)ld.h * a.k_h, *vh = (const u8 *)a.vp + (i64)ld.h * a.v_h;
      u8 *ks = sh.ring[warp][stage][0], *vs = sh.ring[warp][stage][1];
      const u32 there = __ballot_sync(0xffffffffu, key_page >= 0);
      if (in_line) {
        const int row0 = lane / P, piece = lane % P;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          // any key of the half that is there gives the half's page
          const u32 some = there >> (16 * half) & 0xffffu;
          const int from = some ? __ffs(some) - 1 : 0, src = 16 * half + from;
          const i64 page = some ? __shfl_sync(0xffffffffu, key_page, src) : 0;
          const i64 tok = some ? __shfl_sync(0xffffffffu, key_in, src) - from + row0 : 0;
          const u8 *k_at = kh + page * a.k_p + tok * a.k_t + piece * 16, *v_at = vh + page * a.v_p + tok * a.v_t + piece * 16;
#pragma unroll
          for (int i = 0; i < kLoads / 2; ++i) {
            const int row = i * (32 / P) + row0, at = 16 * half + row;
            const u32 bytes = some >> row & 1 ? 16u : 0u;             // 0: the piece is filled with zeros
            cp_async16(ks + code_piece<D>(at, piece) * 16, k_at, bytes);
            cp_async16(vs + code_piece<D>(at, piece) * 16, v_at, bytes);
            if (some) { k_at += (32 / P) * a.k_t; v_at += (32 / P) * a.v_t; }
          }
        }
      } else
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int x = i * 32 + lane, row = x / P, piece = x - row * P;
        const int pg = __shfl_sync(0xffffffffu, key_page, row), in = __shfl_sync(0xffffffffu, key_in, row);
        const u32 bytes = pg >= 0 ? 16u : 0u;
        const i64 page = pg >= 0 ? pg : 0, tok = pg >= 0 ? in : 0;
        cp_async16(ks + code_piece<D>(row, piece) * 16, kh + page * a.k_p + tok * a.k_t + piece * 16, bytes);
        cp_async16(vs + code_piece<D>(row, piece) * 16, vh + page * a.v_p + tok * a.v_t + piece * 16, bytes);
      }
      const i64 page = key_page >= 0 ? key_page : 0, tok = key_page >= 0 ? key_in : 0;
      const u32 bytes = key_page >= 0 ? 4u : 0u;
      cp_async4(&sh.scales[warp][stage][0][lane], a.ks + (i64)ld.h * a.ks_h + page * a.ks_p + tok * a.ks_t, bytes);
      cp_async4(&sh.scales[warp][stage][1][lane], a.vs + (i64)ld.h * a.vs_h + page * a.vs_p + tok * a.vs_t, bytes);
      --ld_left;
      ++ld.at;
      settle<kRows, kCodedTile, kOver>(a, ld, ld_left, plan.fill);
      look_up();
    }
    cp_async_commit();
  };
  look_up();
#pragma unroll 1
  for (int s = 0; s < kCodedStages - 1; ++s) issue(s);

  // --- the computing side
  Cursor c = plan.first;
  int stage = 0;
  const int g = lane >> 2, t4 = lane & 3;
  u32 left = plan.end - plan.begin;
  for (settle<kRows, kCodedTile, kOver>(a, c, left, plan.fill); left; settle<kRows, kCodedTile, kOver>(a, c, left, plan.fill)) {
    const int from = c.at;
    const int to = (int)min((u32)c.span.tiles, (u32)from + left);
    const i64 row0 = (i64)c.m * kRows;
    const int rows = (int)min((i64)kRows, (i64)c.req.n * a.group - row0);
    // this lane's two rows: g and g + 8
    u32 qf[P][4];
    int lo_key[2], hi_key[2];                     // visible keys of the row
    float slope[2], to_dot[2];
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
      const u16 *src = (const u16 *)a.q + (i64)(c.req.q0 + tok) * a.q_t + (i64)head * a.q_h + t4 * 4;
      uint2 x[P];
      float top = 0.0f;
#pragma unroll
      for (int k = 0; k < P; ++k) {
        x[k] = row < rows ? *(const uint2 *)(src + k * 16) : make_uint2(0, 0);
        const float2 lo = unpack2<T>(x[k].x), hi = unpack2<T>(x[k].y);
        top = fmaxf(top, fmaxf(fmaxf(fabsf(lo.x), fabsf(lo.y)), fmaxf(fabsf(hi.x), fabsf(hi.y))));
      }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const float f = query_factor(top);
      to_dot[i] = 1.0f / f;                       // powers of two
#pragma unroll
      for (int k = 0; k < P; ++k) {
        const float2 lo = unpack2<T>(x[k].x), hi = unpack2<T>(x[k].y);
        qf[k][i] = pack2<__half>(lo.x * f, lo.y * f);
        qf[k][2 + i] = pack2<__half>(hi.x * f, hi.y * f);
      }
    }
    float o[P][2][4];                             // even and odd columns of 16
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};
#pragma unroll
    for (int n = 0; n < P; ++n)
#pragma unroll
      for (int x = 0; x < 4; ++x) o[n][0][x] = o[n][1][x] = 0.0f;

    for (int at = from; at < to; ++at) {
      issue(stage == 0 ? kCodedStages - 1 : stage - 1);      // the slot that the tile before has left
      cp_async_wait<kCodedStages - 1>();
      __syncwarp();
      const u8 *ks = sh.ring[warp][stage][0], *vs = sh.ring[warp][stage][1];
      const int key0 = (c.span.first + at) * kCodedTile + warp * kCodedKeys;
      float s[4][4];
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int x = 0; x < 4; ++x) s[n][x] = 0.0f;
#pragma unroll
      for (int k = 0; k < P; ++k) {
        u32 w[4];
        ldmatrix4(w, ks + code_piece<D>(lane, k) * 16);
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          u32 b0, b1;
          decode_along<F>(w[n], b0, b1);
          mma_half(s[n], qf[k], b0, b1);
        }
      }
      // scores in units of log2, masked; v_scale: of the values, 0 where no lane's row may take them
      const bool all_seen = __all_sync(0xffffffffu, key0 >= lo_key[0] && key0 >= lo_key[1] && key0 + kCodedKeys <= hi_key[0] &&
                                                        key0 + kCodedKeys <= hi_key[1]);
      float2 v_scale[4], v_log2[4];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const float2 k_scale = *(const float2 *)&sh.scales[warp][stage][0][n * 8 + t4 * 2];
        v_scale[n] = *(const float2 *)&sh.scales[warp][stage][1][n * 8 + t4 * 2];
        v_log2[n] = make_float2(scale_log2(v_scale[n].x), scale_log2(v_scale[n].y));
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int i = x >> 1, key = key0 + n * 8 + t4 * 2 + (x & 1);
          const float dot = s[n][x] * (x & 1 ? k_scale.y : k_scale.x) * to_dot[i];
          if (SCORED) {
            const float v = a.softcap > 0.0f ? capped_log2(dot, to_cap, a.softcap * kLog2e, to_log2) : dot * to_log2;
            s[n][x] = v + slope[i] * (float)(key - pos[i]);
          } else {
            s[n][x] = dot * to_log2;
          }
          if (!all_seen && (key < lo_key[i] || key >= hi_key[i])) s[n][x] = -INFINITY;
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float top = -INFINITY;
#pragma unroll
        for (int n = 0; n < 4; ++n) top = fmaxf(top, fmaxf(s[n][2 * i] + v_log2[n].x, s[n][2 * i + 1] + v_log2[n].y));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const float was = m[i];
        m[i] = fmaxf(was, top);
        const float most = m[i] == -INFINITY ? 0.0f : m[i], base = most - kLift;   // nothing seen yet: every weight is 2^-inf = 0
        if (__any_sync(0xffffffffu, m[i] != was)) {
          const float f = exp2_approx(was - most);
          l[i] *= f;
#pragma unroll
          for (int n = 0; n < P; ++n)
#pragma unroll
            for (int y = 0; y < 2; ++y) { o[n][y][2 * i] *= f; o[n][y][2 * i + 1] *= f; }
        }
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const float w = exp2_approx(s[n][2 * i + x] - base), scale = x ? v_scale[n].y : v_scale[n].x;
            l[i] += w;
            // a key that the row does not see has weight 0 whatever its value's scale is
            s[n][2 * i + x] = !all_seen && s[n][2 * i + x] == -INFINITY ? 0.0f : w * scale;
          }
      }
#pragma unroll
      for (int n = 0; n < P; ++n) {
        u32 w[4], even[4], odd[4];
        ldmatrix4t(w, vs + code_piece<D>(lane, n) * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) decode_across<F>(w[j], even[j], odd[j]);
        if (F == kE4m3 && !all_seen) {
#pragma unroll
          for (int j = 0; j < 4; ++j) { even[j] = finite_codes<F>(even[j]); odd[j] = finite_codes<F>(odd[j]); }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const u32 pf[4] = {pack2<__half>(s[2 * j][0], s[2 * j][1]), pack2<__half>(s[2 * j][2], s[2 * j][3]), pack2<__half>(s[2 * j + 1][0], s[2 * j + 1][1]),
                             pack2<__half>(s[2 * j + 1][2], s[2 * j + 1][3])};
          mma_half(o[n][0], pf, even[2 * j], even[2 * j + 1]);
          mma_half(o[n][1], pf, odd[2 * j], odd[2 * j + 1]);
        }
      }
      __syncwarp();
      if (at + 1 < to) stage = stage + 1 == kCodedStages ? 0 : stage + 1;     // at the unit's end the slot is needed below
    }
    left -= (u32)(to - from);
    c.at = to;

    // --- join the four warps
    float *mine = (float *)sh.ring[warp][stage][0];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
      const int row = g + 8 * i;
      if (t4 == 0) { sh.m[warp][row] = m[i] - kLift; sh.l[warp][row] = l[i]; }
      if (row < rows) {
#pragma unroll
        for (int n = 0; n < P; ++n)
          *(float4 *)(mine + row * D + (n ^ (row & 1)) * 16 + t4 * 4) = make_float4(o[n][0][2 * i], o[n][1][2 * i], o[n][0][2 * i + 1], o[n][1][2 * i + 1]);
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
        const float4 v = *(const float4 *)((const float *)sh.ring[w][stage][0] + row * D + ((col >> 4) ^ (row & 1)) * 16 + (col & 15));
        sum += f * sh.l[w][row];
        acc.x += f * v.x; acc.y += f * v.y; acc.z += f * v.z; acc.w += f * v.w;
      }
      if (whole) {
        finish_row<T, D>((const Attn &)a, NoRows{}, c.req.q0, row0 + row, c.h, col, acc, top, sum);
      } else {
        *(float4 *)(a.part_o + ((i64)slot * kRows + row) * D + col) = acc;
        if (col == 0) *(float2 *)(a.part_ml + ((i64)slot * kRows + row) * 2) = make_float2(top, sum);
      }
    }
    if (!whole) {
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
      if (sh.last) join_parts<T, D, kRows, kThreads, 1, 8>((const Attn &)a, NoRows{}, c, row0, rows, i0, i1);
    }
    __syncthreads();
    stage = stage + 1 == kCodedStages ? 0 : stage + 1;
  }
  cp_async_wait<0>();
}

template <typename T, Format F, int D, bool SCORED>
cudaError_t launch_coded(const CodedAttn &a, u32 sms, cudaStream_t s) {
  static bool ready[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 64 && !ready[dev]) {
    e = cudaFuncSetAttribute(coded_rows_kernel<T, F, D, SCORED>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(CodedShared<D>));
    if (e != cudaSuccess) return e;
    ready[dev] = true;
  }
  return launch_kernel<Attn>(coded_rows_kernel<T, F, D, SCORED>, sms * kCodedBlocks<D>, kThreads, sizeof(CodedShared<D>), s, a);
}

template <typename T, Format F, int D>
cudaError_t pick_coded_scored(const CodedAttn &a, u32 sms, cudaStream_t s) {
  return a.softcap > 0.0f || a.slopes ? launch_coded<T, F, D, true>(a, sms, s) : launch_coded<T, F, D, false>(a, sms, s);
}

template <typename T, Format F>
cudaError_t pick_coded_dim(const CodedAttn &a, int dim, u32 sms, cudaStream_t s) {
  if (dim == 64) return pick_coded_scored<T, F, 64>(a, sms, s);
  if (dim == 96) return pick_coded_scored<T, F, 96>(a, sms, s);
  return pick_coded_scored<T, F, 128>(a, sms, s);
}

template <Format F>
cudaError_t launch_coded_rows_of(const CodedAttn &a, int dtype, int dim, u32 sms, cudaStream_t s) {
  return dtype == 0 ? pick_coded_dim<__nv_bfloat16, F>(a, dim, sms, s) : pick_coded_dim<__half, F>(a, dim, sms, s);
}

}  // namespace
}  // namespace paged
}  // namespace gorio
