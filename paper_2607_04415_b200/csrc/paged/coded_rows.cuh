// Attention of few rows over a quantised paged cache: the single-token form.
//
// The plan and the four warps with a ring each are those of the 16-bit cache's kernel (rows.cuh).  What is different comes from the
// 8 bits.  The same bytes in flight are twice as many keys, and what is computed for a key has half the time: with the 16-bit kernel's products,
// 16 rows by 8 keys, 64 requests over up to 16384 keys took 254 us, waiting for one operation after the other.  So keys are
// the products' first operand here, 16 by 8 rows, which up to 8 rows (heads that share a key head) halves products, scores and registers, and
// so leaves room for more warps; more rows take two of them.  A warp's tile is 32 keys.
// Codes become float16 in registers, exactly, in the lanes and the order in which the matrix instructions want them:
//   keys     a 16-byte piece of a row is what one product over 16 elements takes.  A lane gets four neighbouring codes of a
//            key, and its queries are loaded in the same order, so that nothing is moved.
//   values   read transposed by pairs of codes, a lane gets two neighbouring columns of two neighbouring keys; taken apart the even columns are
//            the first eight rows of a product's operand, the odd ones the other eight.
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
constexpr int kCodedStages = 2;
// Blocks of an SM for heads of D and 8 * NT rows: what shared memory (17 KB a warp at head size 128) and registers hold.
template <int D, int NT>
constexpr int kCodedBlocks = D == 64 ? 4 : NT == 1 ? 3 : 2;

template <int D>
struct CodedShared {
  // per warp and stage: the codes of 32 keys, then of 32 values; the same bytes hold the warp's output, up to 16 x D, at a unit's end
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

// The transpose of an 8 x 8 matrix of 16-bit numbers, two neighbouring columns of a row to a lane.
__device__ __forceinline__ u32 transpose8(u32 v) {
  u32 r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}

template <typename T, Format F, int D, bool SCORED, int NT>
__global__ void __launch_bounds__(kThreads, (kCodedBlocks<D, NT>)) coded_rows_kernel(const CodedAttn a) {
  extern __shared__ __align__(128) unsigned char raw[];
  CodedShared<D> &sh = *(CodedShared<D> *)raw;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  constexpr int kUnitRows = 8 * NT;
  const Plan plan = block_plan<kUnitRows, kCodedTile, kOver, kThreads>(a, sh.plan, kSpread);
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
  settle<kUnitRows, kCodedTile, kOver>(a, ld, ld_left, plan.fill);
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
      settle<kUnitRows, kCodedTile, kOver>(a, ld, ld_left, plan.fill);
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
  for (settle<kUnitRows, kCodedTile, kOver>(a, c, left, plan.fill); left; settle<kUnitRows, kCodedTile, kOver>(a, c, left, plan.fill)) {
    const int from = c.at;
    const int to = (int)min((u32)c.span.tiles, (u32)from + left);
    const i64 row0 = (i64)c.m * kUnitRows;
    const int rows = (int)min((i64)kUnitRows, (i64)c.req.n * a.group - row0);
    // queries: this lane's row of each eight is g
    u32 qf[P][NT][2];
    float inverse[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const int row = 8 * i + g;
      const int tok = row < rows ? (int)((row0 + row) / a.group) : 0;
      const int head = row < rows ? (int)((row0 + row) - (i64)tok * a.group) + (int)(c.h * a.group) : 0;
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
      inverse[i] = 1.0f / f;                      // powers of two
#pragma unroll
      for (int k = 0; k < P; ++k) {
        const float2 lo = unpack2<T>(x[k].x), hi = unpack2<T>(x[k].y);
        qf[k][i][0] = pack2<__half>(lo.x * f, lo.y * f);
        qf[k][i][1] = pack2<__half>(hi.x * f, hi.y * f);
      }
    }
    // scores and outputs: this lane's rows of each eight are 2 * t4 and the next
    int lo_key[2 * NT], hi_key[2 * NT];           // visible keys of the row
    float slope[2 * NT], to_dot[2 * NT];
    int pos[2 * NT];
    bool sees_all = true;
#pragma unroll
    for (int i = 0; i < 2 * NT; ++i) {
      const int row = (i >> 1) * 8 + t4 * 2 + (i & 1);
      const int tok = row < rows ? (int)((row0 + row) / a.group) : 0;
      const int head = row < rows ? (int)((row0 + row) - (i64)tok * a.group) + (int)(c.h * a.group) : 0;
      pos[i] = position_of(a, c.req, tok);
      hi_key[i] = a.causal ? min(c.req.len, pos[i] + 1) : c.req.len;
      lo_key[i] = a.window ? (int)max((i64)0, (i64)pos[i] - a.window + 1) : 0;
      slope[i] = SCORED && a.slopes ? a.slopes[head] * kLog2e : 0.0f;
      to_dot[i] = __shfl_sync(0xffffffffu, inverse[i >> 1], (t4 * 2 + (i & 1)) * 4);
    }
    float o[P][NT][4];                            // column 2g of 16: rows 2 * t4 and the next; column 2g + 1: the same
    float m[2 * NT], l[2 * NT];
#pragma unroll
    for (int i = 0; i < 2 * NT; ++i) { m[i] = -INFINITY; l[i] = 0.0f; }
#pragma unroll
    for (int n = 0; n < P; ++n)
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int x = 0; x < 4; ++x) o[n][i][x] = 0.0f;

    for (int at = from; at < to; ++at) {
      issue(stage == 0 ? kCodedStages - 1 : stage - 1);      // the slot that the tile before has left
      cp_async_wait<kCodedStages - 1>();
      __syncwarp();
      const u8 *ks = sh.ring[warp][stage][0], *vs = sh.ring[warp][stage][1];
      const int key0 = (c.span.first + at) * kCodedTile + warp * kCodedKeys;
      float s[2][NT][4];                          // of 16 keys: g, rows 2 * t4 and the next; g + 8, the same
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int x = 0; x < 4; ++x) s[n][i][x] = 0.0f;
#pragma unroll
      for (int k = 0; k < P; ++k) {
        u32 w[4];
        ldmatrix4(w, ks + code_piece<D>(lane, k) * 16);
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          u32 b[4];
          decode_along<F>(w[2 * n], b[0], b[2]);
          decode_along<F>(w[2 * n + 1], b[1], b[3]);
#pragma unroll
          for (int i = 0; i < NT; ++i) mma16816<__half>(s[n][i], b, qf[k][i][0], qf[k][i][1]);
        }
      }
      // scores in units of log2, masked
      sees_all = true;
#pragma unroll
      for (int i = 0; i < 2 * NT; ++i) sees_all = sees_all && key0 >= lo_key[i] && key0 + kCodedKeys <= hi_key[i];
      const bool all_seen = __all_sync(0xffffffffu, sees_all);
      float v_scale[4], v_log2[4];                // of keys g, g + 8 ...
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float k_scale = sh.scales[warp][stage][0][8 * j + g];
        v_scale[j] = sh.scales[warp][stage][1][8 * j + g];
        v_log2[j] = scale_log2(v_scale[j]);
        const int key = key0 + 8 * j + g;
#pragma unroll
        for (int i = 0; i < 2 * NT; ++i) {
          float &x = s[j >> 1][i >> 1][2 * (j & 1) + (i & 1)];
          const float dot = x * k_scale * to_dot[i];
          if (SCORED) {
            const float v = a.softcap > 0.0f ? capped_log2(dot, to_cap, a.softcap * kLog2e, to_log2) : dot * to_log2;
            x = v + slope[i] * (float)(key - pos[i]);
          } else {
            x = dot * to_log2;
          }
          if (!all_seen && (key < lo_key[i] || key >= hi_key[i])) x = -INFINITY;
        }
      }
      bool moved = false;
      float down[2 * NT], base[2 * NT];
#pragma unroll
      for (int i = 0; i < 2 * NT; ++i) {
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j) top = fmaxf(top, s[j >> 1][i >> 1][2 * (j & 1) + (i & 1)] + v_log2[j]);
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
        const float was = m[i];
        m[i] = fmaxf(was, top);
        const float most = m[i] == -INFINITY ? 0.0f : m[i];
        base[i] = most - kLift;                   // nothing seen yet: every weight is 2^-inf = 0
        down[i] = was - most;
        moved = moved || m[i] != was;
      }
      if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
        for (int i = 0; i < 2 * NT; ++i) {
          const float half = exp2_approx(0.5f * down[i]), f = half * half;
          l[i] = l[i] * half * half;             // see moved_sum
#pragma unroll
          for (int n = 0; n < P; ++n) { o[n][i >> 1][i & 1] *= f; o[n][i >> 1][2 + (i & 1)] *= f; }
        }
      }
      u32 weights[4][NT];                         // of 8 keys, then of their transposes
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float u[2];
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const float score = s[j >> 1][n][2 * (j & 1) + x], w = exp2_approx(score - base[2 * n + x]);
            l[2 * n + x] += w;
            // a key that the row does not see has weight 0 whatever its value's scale is
            u[x] = !all_seen && score == -INFINITY ? 0.0f : w * v_scale[j];
          }
          weights[j][n] = transpose8(pack2<__half>(u[0], u[1]));
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
          const u32 b[4] = {even[2 * j], odd[2 * j], even[2 * j + 1], odd[2 * j + 1]};
#pragma unroll
          for (int i = 0; i < NT; ++i) mma16816<__half>(o[n][i], b, weights[2 * j][i], weights[2 * j + 1][i]);
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
    for (int i = 0; i < 2 * NT; ++i) {
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 4);
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 8);
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 16);
      const int row = (i >> 1) * 8 + t4 * 2 + (i & 1);
      if (g == 0) { sh.m[warp][row] = m[i] - kLift; sh.l[warp][row] = l[i]; }
      if (row < rows) {
#pragma unroll
        for (int n = 0; n < P; ++n)
          *(float2 *)(mine + row * D + (n ^ (t4 & 1)) * 16 + g * 2) = make_float2(o[n][i >> 1][i & 1], o[n][i >> 1][2 + (i & 1)]);
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
        const float4 v = *(const float4 *)((const float *)sh.ring[w][stage][0] + row * D + ((col >> 4) ^ (row >> 1 & 1)) * 16 + (col & 15));
        sum += moved_sum<true>(sh.l[w][row], sh.m[w][row] - base);
        acc.x += f * v.x; acc.y += f * v.y; acc.z += f * v.z; acc.w += f * v.w;
      }
      if (whole) {
        finish_row<T, D>((const Attn &)a, NoRows{}, c.req.q0, row0 + row, c.h, col, acc, top, sum);
      } else {
        *(float4 *)(a.part_o + ((i64)slot * kUnitRows + row) * D + col) = acc;
        if (col == 0) *(float2 *)(a.part_ml + ((i64)slot * kUnitRows + row) * 2) = make_float2(top, sum);
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
      if (sh.last) join_parts<T, D, kUnitRows, kThreads, 1, 8, true>((const Attn &)a, NoRows{}, c, row0, rows, i0, i1);
    }
    __syncthreads();
    stage = stage + 1 == kCodedStages ? 0 : stage + 1;
  }
  cp_async_wait<0>();
}

template <typename T, Format F, int D, bool SCORED, int NT>
cudaError_t launch_coded(const CodedAttn &a, u32 sms, cudaStream_t s) {
  static bool ready[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 64 && !ready[dev]) {
    e = cudaFuncSetAttribute(coded_rows_kernel<T, F, D, SCORED, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(CodedShared<D>));
    if (e != cudaSuccess) return e;
    ready[dev] = true;
  }
  return launch_kernel<Attn>(coded_rows_kernel<T, F, D, SCORED, NT>, sms * kCodedBlocks<D, NT>, kThreads, sizeof(CodedShared<D>), s, a);
}

template <typename T, Format F, int D>
cudaError_t pick_coded_scored(const CodedAttn &a, bool few, u32 sms, cudaStream_t s) {
  if (a.softcap > 0.0f || a.slopes) return few ? launch_coded<T, F, D, true, 1>(a, sms, s) : launch_coded<T, F, D, true, 2>(a, sms, s);
  return few ? launch_coded<T, F, D, false, 1>(a, sms, s) : launch_coded<T, F, D, false, 2>(a, sms, s);
}

template <typename T, Format F>
cudaError_t pick_coded_dim(const CodedAttn &a, int dim, bool few, u32 sms, cudaStream_t s) {
  if (dim == 64) return pick_coded_scored<T, F, 64>(a, few, sms, s);
  if (dim == 96) return pick_coded_scored<T, F, 96>(a, few, sms, s);
  return pick_coded_scored<T, F, 128>(a, few, sms, s);
}

// few: no request has more than 8 rows.
template <Format F>
cudaError_t launch_coded_rows_of(const CodedAttn &a, int dtype, int dim, bool few, u32 sms, cudaStream_t s) {
  return dtype == 0 ? pick_coded_dim<__nv_bfloat16, F>(a, dim, few, sms, s) : pick_coded_dim<__half, F>(a, dim, few, sms, s);
}

}  // namespace
}  // namespace paged
}  // namespace gorio
