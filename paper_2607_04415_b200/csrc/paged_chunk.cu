// Attention of many rows over a paged cache: the chunk form, on the fifth-generation tensor cores.
//
// A unit is up to 256 rows ((token, query head) pairs that share a key head) in two tiles of 128, so that each
// tile of 128 keys that a block copies in serves 256 rows.  Per 128 x 128 scores both products take 2 * 2^21
// multiply-adds, 1024 cycles of the matrix unit at head size 128, and the softmax takes 2^14 exponentials, 1024
// cycles of the special function units: the two row tiles take turns, one in the matrix unit while the other is
// in the softmax.  One block an SM, twelve warps:
//   0-3, 4-7  the softmax of row tile 0 and 1: a thread a row.  Scores come from tensor memory, weights go back to
//             it over the scores (16 bits each), where the second product reads them as its first operand.
//   8         issues both products (one thread); zeros value rows that no query sees before they are used.
//   9         copies key and value tiles, page by page (tensor copies, zeros for pages outside the cache), into a
//             ring of stages with the 128-byte swizzle.
//   10        looks for values that are not finite in tiles that some rows see and others do not.
// Tensor memory, 512 columns: scores of tile 0 and 1 (128 each), outputs of tile 0 and 1 (head size each).
//
// Running maximum: a row's reference only moves when its maximum passes it by more than 2^8, since moving it
// costs a pass over the output in tensor memory; weights are then at most 2^8, far inside both types.
// The sum of the weights is held unrounded in 32 bits, the weights are rounded once to the cache's type.
//
// Blocks take equal shares of all key tiles of the call (make_plan), cut units are joined by their last block.
// Values that are not finite (and masked for some rows) would reach rows that do not see them, as 0 * inf in the
// product: a unit that meets one is computed again row by row from the cache, slowly, in plain_columns.
#include "paged/common.cuh"
#include "paged/tensor.cuh"

namespace gorio {
namespace paged {

namespace {

constexpr int kRows = 256;
constexpr int kTileRows = 128;
constexpr int kTileKeys = 128;
constexpr int kThreads = 384;
constexpr int kSoftmaxRegs = 224, kOtherRegs = 56;   // a thread, of 168 * 3 = 224 * 2 + 56 at launch
constexpr u32 kScores = 0, kOutputs = 256;       // columns of tensor memory
constexpr int kScans = 8;                         // more parts than the ring of stages lets warp 10 run ahead

template <int D>
struct Shape {
  static constexpr int chunks = (D + 63) / 64;                            // of 64 elements, 128 bytes
  static constexpr int tile_bytes = chunks * kTileKeys * 128;
  static constexpr int stages = chunks == 1 ? 8 : 5;
};

template <int D>
struct ChunkShared {
  unsigned char q[2][Shape<D>::tile_bytes];
  unsigned char kv[Shape<D>::stages][Shape<D>::tile_bytes];
  u64 kv_full[Shape<D>::stages], kv_empty[Shape<D>::stages];
  u64 q_full[2], s_full[2], p_full[2], o_full[2], scanned[kScans];
  u32 odd[kScans];
  u32 tmem, failed, last;
  PlanShared plan;
};

// One part of a unit: its tiles [from, to) of this block's share.
struct Part {
  int from, to;
  i64 row0;
  int rows;
};

__device__ __forceinline__ Part part_of(const Attn &a, const Cursor &c, u64 left) {
  Part p;
  p.from = c.at;
  p.to = (int)min((u64)c.span.tiles, (u64)c.at + left);
  p.row0 = (i64)c.m * kRows;
  p.rows = (int)min((i64)kRows, (i64)c.req.n * a.group - p.row0);
  return p;
}

// What one row sees.
struct Row {
  int pos, lo, hi;
  int head;          // query head
  i64 tok;           // row of q and out
};

__device__ __forceinline__ Row row_of(const Attn &a, const Cursor &c, i64 row) {
  Row r;
  const int tok = (int)((u32)row / a.group);
  r.head = (int)((u32)row - (u32)tok * a.group + c.h * a.group);
  r.tok = c.req.q0 + tok;
  r.pos = c.req.len - c.req.n + tok;
  r.hi = a.causal ? min(c.req.len, r.pos + 1) : c.req.len;
  r.lo = a.window ? (int)max((i64)0, (i64)r.pos - a.window + 1) : 0;
  return r;
}

// Whether every row of the unit sees every key of [lo, hi) that lies in the tile.
__device__ __forceinline__ bool seen_by_all(const Attn &a, const Cursor &c, const Part &p, int key0) {
  const int t0 = (int)((u32)p.row0 / a.group), t1 = (int)((u32)(p.row0 + p.rows - 1) / a.group);
  const int first = c.req.len - c.req.n + t0, last = c.req.len - c.req.n + t1;
  if (a.causal && min(key0 + kTileKeys, c.span.hi) > first + 1) return false;
  if (a.window && (i64)max(key0, c.span.lo) < (i64)last - a.window + 1) return false;
  return true;
}

// Score of one row and key in units of log2, and 32 columns of the weighted sum, straight from the cache: for units with
// values that are not finite.  Keys [k0, k1) of the row's own [lo, hi); `top` is the reference of the weights, taken
// from the row's maximum where `fresh`.
template <typename T, int D>
__device__ __noinline__ void plain_columns(const Attn &a, u32 req, u32 h, const Row &r, int k0, int k1, int col, float *acc, float &top, float &sum) {
  const u16 *q = (const u16 *)a.q + r.tok * a.q_t + (i64)r.head * a.q_h;
  const float slope = a.slopes ? a.slopes[r.head] * kLog2e : 0.0f;
  for (int pass = col == 0 ? 0 : 1; pass < 2; ++pass) {
    if (pass == 0) top = -INFINITY; else sum = col == 0 ? 0.0f : sum;
    for (int key = max(k0, r.lo); key < min(k1, r.hi); ++key) {
      const u32 at = (u32)key / a.page;
      const int pg = a.tables[(i64)req * a.tab_r + at];
      const i64 in = (i64)((u32)key - at * a.page);
      const bool there = (u32)pg < a.n_pages;
      const u16 *k = (const u16 *)a.kp + (i64)pg * a.k_p + (i64)h * a.k_h + in * a.k_t;
      float x = 0.0f;
      for (int d = 0; d < D; d += 2) {
        const float2 u = unpack2<T>(*(const u32 *)(q + d)), v = there ? unpack2<T>(*(const u32 *)(k + d)) : make_float2(0.0f, 0.0f);
        x += u.x * v.x;
        x += u.y * v.y;
      }
      x *= a.scale;
      if (a.softcap > 0.0f) x = capped(x, a.softcap);
      x = x * kLog2e + slope * (float)(key - r.pos);
      if (pass == 0) { top = fmaxf(top, x); continue; }
      const float w = exp2_approx(x - (top == -INFINITY ? 0.0f : top));
      if (col == 0) sum += w;
      if (!there) continue;
      const u16 *v = (const u16 *)a.vp + (i64)pg * a.v_p + (i64)h * a.v_h + in * a.v_t + col;
#pragma unroll
      for (int d = 0; d < 32; d += 2) {
        const float2 u = unpack2<T>(*(const u32 *)(v + d));
        acc[d] += w * u.x;
        acc[d + 1] += w * u.y;
      }
    }
  }
}

template <typename T, int D, bool SCORED>
__global__ void __launch_bounds__(kThreads, 1) attention_chunk_kernel(const Attn a, const __grid_constant__ CUtensorMap keys,
                                                                      const __grid_constant__ CUtensorMap values, const u32 box_rows) {
  extern __shared__ unsigned char raw[];
  ChunkShared<D> &sh = *(ChunkShared<D> *)(raw + ((1024 - (smem_addr(raw) & 1023)) & 1023));
  typedef Shape<D> S;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) {
    for (int i = 0; i < S::stages; ++i) { bar_init(&sh.kv_full[i], 1); bar_init(&sh.kv_empty[i], 2); }
    for (int t = 0; t < 2; ++t) { bar_init(&sh.q_full[t], kTileRows); bar_init(&sh.s_full[t], 1); bar_init(&sh.p_full[t], kTileRows); bar_init(&sh.o_full[t], 1); }
    for (int i = 0; i < kScans; ++i) { bar_init(&sh.scanned[i], 1); sh.odd[i] = 0; }
    sh.failed = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async();
  }
  if (warp == 8) tmem_alloc(&sh.tmem, 512);
  const Plan plan = make_plan<kRows, kTileKeys, kThreads>(a, sh.plan, 1);
  mma_fence_before();
  __syncthreads();
  mma_fence_after();
  const u32 tmem = sh.tmem;
  volatile u32 *failed = &sh.failed;
  Cursor c = plan.first;
  u64 left = plan.end - plan.begin;

  if (warp < 8) {
    // ------------------------------------------------------------------ softmax of row tile t
    more_registers<kSoftmaxRegs>();
    const int t = warp >> 2, row = tid & (kTileRows - 1);
    const u32 lanes = (u32)(warp & 3) << 21;                 // this warp's 32 lanes of tensor memory
    const u32 scores = tmem + kScores + t * 128 + lanes, outputs = tmem + kOutputs + t * D + lanes;
    u32 s_phase = 0, o_phase = 0, part_no = 0;
    auto put_q = [&](const Cursor &at, const Part &p) {      // the tile's queries, swizzled; zeros past the last row
      constexpr int P = D / 8;
#pragma unroll 4
      for (int x = row; x < kTileRows * P; x += kTileRows) {
        const int r = x / P, piece = x - r * P;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (t * kTileRows + r < p.rows) {
          const u32 flat = (u32)(p.row0 + t * kTileRows + r), tok = flat / a.group, head = flat - tok * a.group + at.h * a.group;
          v = *(const uint4 *)((const u16 *)a.q + (i64)(at.req.q0 + (int)tok) * a.q_t + (i64)head * a.q_h + piece * 8);
        }
        *(uint4 *)(sh.q[t] + (piece >> 3) * (kTileRows * 128) + r * 128 + (((piece & 7) ^ (r & 7)) << 4)) = v;
      }
      fence_async();
      bar_arrive(&sh.q_full[t]);
    };
    const float to_log2 = a.scale * kLog2e;
    Part p{};
    if (left) {
      p = part_of(a, c, left);
      if (t == 0 || p.rows > kTileRows) put_q(c, p);
    }
    while (left) {
      const bool mine = t == 0 || p.rows > kTileRows;        // does the unit have this row tile at all
      const bool valid = t * kTileRows + row < p.rows;
      const Row r = row_of(a, c, valid ? p.row0 + t * kTileRows + row : p.row0);
      const float slope = SCORED && a.slopes ? a.slopes[r.head] * kLog2e : 0.0f;
      float m = -INFINITY, l = 0.0f;
      if (mine) {
        for (int at = p.from; at < p.to; ++at) {
          if (!bar_wait(&sh.s_full[t], s_phase, failed)) break;
          s_phase ^= 1;
          mma_fence_after();
          float s[128];
#pragma unroll
          for (int i = 0; i < 4; ++i) tmem_ld32(s + 32 * i, scores + 32 * i);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < 4; ++i) keep(s + 32 * i);
          const int key0 = (c.span.first + at) * kTileKeys;
          float mul = to_log2;
          if (SCORED) {
            mul = 1.0f;
#pragma unroll
            for (int i = 0; i < 128; ++i) {
              float x = s[i] * a.scale;
              if (a.softcap > 0.0f) x = capped(x, a.softcap);
              s[i] = x * kLog2e + slope * (float)(key0 + i - r.pos);
            }
          }
          if (__any_sync(0xffffffffu, key0 < r.lo || key0 + kTileKeys > r.hi)) {
#pragma unroll
            for (int i = 0; i < 128; ++i)
              if (key0 + i < r.lo || key0 + i >= r.hi) s[i] = -INFINITY;
          }
          float top = s[0];
#pragma unroll
          for (int i = 1; i < 128; ++i) top = fmaxf(top, s[i]);
          top *= mul;
          const bool moves = top > m + 8.0f || (m == -INFINITY && top > -INFINITY);
          if (__any_sync(0xffffffffu, moves)) {
            const float to = moves ? top : m;
            const float f = m == -INFINITY ? 0.0f : exp2_approx(m - to);
            m = to;
            l *= f;
            if (at > p.from) {                               // the scores' arrival says that the product before is done
#pragma unroll
              for (int i = 0; i < D / 32; ++i) {
                float o[32];
                tmem_ld32(o, outputs + 32 * i);
                tmem_wait_ld();
                keep(o);
                u32 w[32];
#pragma unroll
                for (int k = 0; k < 32; ++k) w[k] = __float_as_uint(o[k] * f);
                tmem_st32(outputs + 32 * i, w);
              }
            }
          }
          const float base = m == -INFINITY ? 0.0f : m;
          float l0 = 0.0f, l1 = 0.0f, l2 = 0.0f, l3 = 0.0f;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            u32 w[32];
#pragma unroll
            for (int k = 0; k < 32; k += 2) {
              const float w0 = exp2_approx(fmaf(s[64 * i + 2 * k], mul, -base)), w1 = exp2_approx(fmaf(s[64 * i + 2 * k + 1], mul, -base));
              const float w2 = exp2_approx(fmaf(s[64 * i + 2 * k + 2], mul, -base)), w3 = exp2_approx(fmaf(s[64 * i + 2 * k + 3], mul, -base));
              l0 += w0; l1 += w1; l2 += w2; l3 += w3;
              w[k] = pack2<T>(w0, w1);
              w[k + 1] = pack2<T>(w2, w3);
            }
            tmem_st32(scores + 32 * i, w);
          }
          l += (l0 + l1) + (l2 + l3);
          tmem_wait_st();
          mma_fence_before();
          bar_arrive(&sh.p_full[t]);
        }
      }
      left -= (u64)(p.to - p.from);
      // the next unit's queries go in before this unit's output is read: its first product runs meanwhile
      Cursor next = c;
      Part np{};
      if (left) {
        next_unit<kRows, kTileKeys>(a, next);
        np = part_of(a, next, left);
        if ((t == 0 || np.rows > kTileRows) && !*failed) put_q(next, np);
      }
      const bool whole = p.from == 0 && p.to == c.span.tiles;
      const u64 unit0 = plan.end - left - (u64)p.to;
      const u32 i0 = whole ? 0 : part_owner(plan.total, unit0, plan.parts);
      bool fine = true;
      if (mine) {
        fine = bar_wait(&sh.scanned[part_no % kScans], (part_no / kScans) & 1, failed) && bar_wait(&sh.o_full[t], o_phase, failed);
        o_phase ^= 1;
        mma_fence_after();
        if (fine) {
          const bool odd = sh.odd[part_no % kScans] != 0;
          const int k0 = (c.span.first + p.from) * kTileKeys, k1 = (c.span.first + p.to) * kTileKeys;
          const i64 slot_row = (i64)(2 * blockIdx.x + (blockIdx.x == i0 ? 1 : 0)) * kRows + t * kTileRows + row;
#pragma unroll 1
          for (int i = 0; i < D / 32; ++i) {
            float o[32];
            if (!odd) {
              tmem_ld32(o, outputs + 32 * i);
              tmem_wait_ld();
              keep(o);
            } else {
              float x[32], top = m, sum = l;                 // not o itself, which stays in registers
#pragma unroll
              for (int k = 0; k < 32; ++k) x[k] = 0.0f;
              plain_columns<T, D>(a, c.r, c.h, r, k0, k1, 32 * i, x, top, sum);
              m = top;
              l = sum;
#pragma unroll
              for (int k = 0; k < 32; ++k) o[k] = x[k];
            }
            if (!valid) continue;
            if (whole) {
              const float f = l == 0.0f ? 0.0f : 1.0f / l;
              uint4 *to = (uint4 *)((u16 *)a.out + r.tok * a.o_t + (i64)r.head * a.o_h + 32 * i);
#pragma unroll
              for (int k = 0; k < 4; ++k)
                to[k] = make_uint4(pack2<T>(o[8 * k] * f, o[8 * k + 1] * f), pack2<T>(o[8 * k + 2] * f, o[8 * k + 3] * f), pack2<T>(o[8 * k + 4] * f, o[8 * k + 5] * f),
                                   pack2<T>(o[8 * k + 6] * f, o[8 * k + 7] * f));
              if (i == 0 && a.lse) a.lse[r.tok * a.hq + r.head] = l == 0.0f ? -INFINITY : m * kLn2 + logf(l);
            } else {
              float4 *to = (float4 *)(a.part_o + slot_row * D + 32 * i);
#pragma unroll
              for (int k = 0; k < 8; ++k) to[k] = make_float4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
              if (i == 0) *(float2 *)(a.part_ml + slot_row * 2) = make_float2(m, l);
            }
          }
        }
      }
      ++part_no;
      mma_fence_before();
      if (!whole) {
        const u32 i1 = part_owner(plan.total, unit0 + (u64)c.span.tiles - 1, plan.parts);
        __threadfence();
        some_barrier(1, 256);
        if (tid == 0) {
          const u32 before = atomicAdd(a.arrived + i0, 1u);
          sh.last = before == i1 - i0;
          if (sh.last) a.arrived[i0] = 0;
          __threadfence();
        }
        some_barrier(1, 256);
        if (sh.last) join_parts<T, D, kRows, 256>(a, c, p.row0, p.rows, i0, i1);
        some_barrier(1, 256);
      }
      c = next;                                              // after a failed wait the rest is walked through, not computed
      p = np;
    }
  } else {
    fewer_registers<kOtherRegs>();
    if (warp == 8) {
      // ---------------------------------------------------------------- the products
      constexpr u32 kScoreShape = mma_shape<T>(kTileKeys, false), kOutShape = mma_shape<T>(D, true);
      int stage = 0;
      u32 kv_phase = 0, q_phase[2] = {0, 0}, p_phase[2] = {0, 0};
      bool fine = true;
      auto scores_of = [&](int t, int k_stage) {
        if (lane == 0) {
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const int at = (k >> 2) * (kTileKeys * 128) + (k & 3) * 32;
            mma_ss(tmem + kScores + t * 128, operand(sh.q[t] + at, 16), operand(sh.kv[k_stage] + at, 16), kScoreShape, k > 0);
          }
          mma_commit(&sh.s_full[t]);
        }
      };
      auto step = [&]() { if (++stage == S::stages) { stage = 0; kv_phase ^= 1; } };
      while (left && fine) {
        const Part p = part_of(a, c, left);
        const int tiles = p.rows > kTileRows ? 2 : 1;
        for (int t = 0; t < tiles; ++t) {
          fine = fine && bar_wait(&sh.q_full[t], q_phase[t], failed);
          q_phase[t] ^= 1;
        }
        fine = fine && bar_wait(&sh.kv_full[stage], kv_phase, failed);
        if (!fine) break;
        mma_fence_after();
        for (int t = 0; t < tiles; ++t) scores_of(t, stage);
        if (lane == 0) mma_commit(&sh.kv_empty[stage]);
        step();
        for (int at = p.from; at < p.to && fine; ++at) {
          const int v_stage = stage;
          const bool more = at + 1 < p.to;
          fine = bar_wait(&sh.kv_full[v_stage], kv_phase, failed);
          if (!fine) break;
          step();
          // rows of the tile that lie outside [lo, hi) in pages that were read: zero, whatever the pages hold there
          const int key0 = (c.span.first + at) * kTileKeys;
          if (key0 < c.span.lo || key0 + kTileKeys > c.span.hi) {
            const int z0 = max(0, min(kTileKeys, c.span.lo - key0)), z1 = max(0, min(kTileKeys, c.span.hi - key0));
            for (int x = lane; x < S::chunks * kTileKeys * 8; x += 32) {
              const int k = (x >> 3) & (kTileKeys - 1);
              if (k < z0 || k >= z1) *(uint4 *)(sh.kv[v_stage] + x * 16) = make_uint4(0, 0, 0, 0);
            }
            fence_async();
            __syncwarp();
          }
          for (int t = 0; t < tiles && fine; ++t) {
            fine = bar_wait(&sh.p_full[t], p_phase[t], failed);
            p_phase[t] ^= 1;
            if (!fine) break;
            mma_fence_after();
            if (lane == 0) {
#pragma unroll
              for (int k = 0; k < kTileKeys / 16; ++k)
                mma_ts(tmem + kOutputs + t * D, tmem + kScores + t * 128 + k * 8, operand(sh.kv[v_stage] + k * 2048, kTileKeys * 128), kOutShape, at > p.from || k > 0);
              if (!more) mma_commit(&sh.o_full[t]);
            }
            if (more) {
              if (t == 0) {
                fine = bar_wait(&sh.kv_full[stage], kv_phase, failed);
                if (!fine) break;
                mma_fence_after();
              }
              scores_of(t, stage);
            }
          }
          if (lane == 0) mma_commit(&sh.kv_empty[v_stage]);
          if (more) {
            if (lane == 0) mma_commit(&sh.kv_empty[stage]);
            step();
          }
        }
        left -= (u64)(p.to - p.from);
        if (left) next_unit<kRows, kTileKeys>(a, c);
      }
    } else if (warp == 9) {
      // ---------------------------------------------------------------- the copies
      const int boxes = kTileKeys / (int)box_rows * S::chunks;       // at most 32: a lane each
      const int g = lane / S::chunks, chunk = lane - g * S::chunks;
      int stage = 0;
      u32 phase = 1;                                                  // the first round finds the stages free
      bool fine = true;
      while (left && fine) {
        const Part p = part_of(a, c, left);
        for (int at = p.from; at < p.to && fine; ++at) {
          const int key = (c.span.first + at) * kTileKeys + g * (int)box_rows;
          int page = (int)a.n_pages, in = 0;                          // past the last page: zeros
          if (lane < boxes && key < c.span.hi && key + (int)box_rows > c.span.lo) {
            const u32 pi = (u32)key / a.page;
            const int pg = __ldg(a.tables + (i64)c.r * a.tab_r + pi);
            if ((u32)pg < a.n_pages) { page = pg; in = (int)((u32)key - pi * a.page); }
          }
#pragma unroll
          for (int kv = 0; kv < 2; ++kv) {
            fine = fine && bar_wait(&sh.kv_empty[stage], phase, failed);
            if (!fine) break;
            if (lane == 0) bar_expect(&sh.kv_full[stage], (u32)S::tile_bytes);
            __syncwarp();
            if (lane < boxes)
              copy_box(sh.kv[stage] + chunk * (kTileKeys * 128) + g * (int)box_rows * 128, kv ? &values : &keys, chunk * 64, in, (int)c.h, page, &sh.kv_full[stage]);
            if (++stage == S::stages) { stage = 0; phase ^= 1; }
          }
        }
        left -= (u64)(p.to - p.from);
        if (left) next_unit<kRows, kTileKeys>(a, c);
      }
      if (!fine) {                                                    // leave no copy in flight behind: each stage's last one
        const u64 t0 = now_ns();
        for (int i = 0; i < S::stages; ++i) {
          const u32 ph = (u32)(i < stage ? phase ^ 1 : phase);        // phase of the stage's last fill, as kv_full counts it
          while (!bar_try(&sh.kv_full[i], ph ^ 0) && now_ns() - t0 < kWaitLimitNs) {}
        }
      }
    } else if (warp == 10) {
      // ---------------------------------------------------------------- values that are not finite
      int stage = 0;
      u32 phase = 0, part_no = 0;
      bool fine = true;
      while (left && fine) {
        const Part p = part_of(a, c, left);
        u32 odd = 0;
        for (int at = p.from; at < p.to && fine; ++at) {
          const int key0 = (c.span.first + at) * kTileKeys;
          const bool look = !seen_by_all(a, c, p, key0);
#pragma unroll
          for (int kv = 0; kv < 2; ++kv) {
            fine = fine && bar_wait(&sh.kv_full[stage], phase, failed);
            if (!fine) break;
            if (kv && look) {
              const int z0 = max(0, c.span.lo - key0), z1 = min(kTileKeys, c.span.hi - key0);
              for (int x = lane; x < S::chunks * kTileKeys * 8; x += 32) {
                const int k = (x >> 3) & (kTileKeys - 1);
                if (k >= z0 && k < z1 && not_finite8<T>(*(const uint4 *)(sh.kv[stage] + x * 16))) odd = 1;
              }
            }
            __syncwarp();
            if (lane == 0) bar_arrive(&sh.kv_empty[stage]);
            if (++stage == S::stages) { stage = 0; phase ^= 1; }
          }
        }
        odd = __any_sync(0xffffffffu, odd);
        if (lane == 0) {
          sh.odd[part_no % kScans] = odd;
          bar_arrive(&sh.scanned[part_no % kScans]);
        }
        ++part_no;
        left -= (u64)(p.to - p.from);
        if (left) next_unit<kRows, kTileKeys>(a, c);
      }
    }
  }
  mma_fence_before();
  __syncthreads();
  mma_fence_after();
  if (warp == 8) tmem_free(tmem, 512);
  if (tid == 0 && sh.failed) a.arrived[kErrorWord] = 1;
}

}  // namespace

namespace {

typedef CUresult (*EncodeFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                             const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeFn encoder() {
  static EncodeFn fn = [] {
    void *p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess)
      p = nullptr;
    return (EncodeFn)p;
  }();
  return fn;
}

bool page_map(CUtensorMap *map, const Attn &a, const void *base, i64 st, i64 sh, i64 sp, int dtype, int dim, u32 box_rows) {
  const cuuint64_t dims[4] = {(cuuint64_t)dim, a.page, a.hkv, a.n_pages};
  const cuuint64_t strides[3] = {(cuuint64_t)st * 2, (cuuint64_t)sh * 2, (cuuint64_t)sp * 2};
  const cuuint32_t box[4] = {64, box_rows, 1, 1}, step[4] = {1, 1, 1, 1};
  return encoder()(map, dtype == 0 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<void *>(base), dims, strides, box, step,
                   CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int D, bool SCORED>
cudaError_t launch(const Attn &a, const CUtensorMap &k, const CUtensorMap &v, u32 box_rows, u32 sms, cudaStream_t s) {
  static bool ready[64] = {};
  constexpr size_t bytes = sizeof(ChunkShared<D>) + 1024;
  static_assert(bytes <= 227 * 1024, "shared memory of one block");
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 64) return cudaErrorInvalidDevice;
  if (!ready[dev]) {
    e = cudaFuncSetAttribute(attention_chunk_kernel<T, D, SCORED>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e != cudaSuccess) return e;
    // the warps' register shares come out of what the block is launched with: with fewer they would wait for ever
    cudaFuncAttributes f;
    e = cudaFuncGetAttributes(&f, attention_chunk_kernel<T, D, SCORED>);
    if (e != cudaSuccess) return e;
    if (f.numRegs * kThreads < kSoftmaxRegs * 256 + kOtherRegs * 128) return cudaErrorInvalidKernelImage;
    ready[dev] = true;
  }
  attention_chunk_kernel<T, D, SCORED><<<sms, kThreads, bytes, s>>>(a, k, v, box_rows);
  return cudaGetLastError();
}

template <typename T, int D>
cudaError_t pick_scored(const Attn &a, const CUtensorMap &k, const CUtensorMap &v, u32 box_rows, u32 sms, cudaStream_t s) {
  return a.softcap > 0.0f || a.slopes ? launch<T, D, true>(a, k, v, box_rows, sms, s) : launch<T, D, false>(a, k, v, box_rows, sms, s);
}

template <typename T>
cudaError_t pick_dim(const Attn &a, const CUtensorMap &k, const CUtensorMap &v, u32 box_rows, int dim, u32 sms, cudaStream_t s) {
  if (dim == 64) return pick_scored<T, 64>(a, k, v, box_rows, sms, s);
  if (dim == 96) return pick_scored<T, 96>(a, k, v, box_rows, sms, s);
  return pick_scored<T, 128>(a, k, v, box_rows, sms, s);
}

}  // namespace

bool launch_chunk(const Attn &a, int dtype, int dim, u32 sms, cudaStream_t s, cudaError_t *e) {
  if (!encoder() || a.n_pages == 0) return false;
  u32 box_rows = a.page & (0u - a.page);               // the largest power of two in the page size, so that a box stays in its page
  if (box_rows > (u32)kTileKeys) box_rows = kTileKeys;
  CUtensorMap k, v;
  if (!page_map(&k, a, a.kp, a.k_t, a.k_h, a.k_p, dtype, dim, box_rows) || !page_map(&v, a, a.vp, a.v_t, a.v_h, a.v_p, dtype, dim, box_rows)) return false;
  *e = dtype == 0 ? pick_dim<__nv_bfloat16>(a, k, v, box_rows, dim, sms, s) : pick_dim<__half>(a, k, v, box_rows, dim, sms, s);
  return true;
}

}  // namespace paged
}  // namespace gorio
