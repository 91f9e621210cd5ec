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
//   10        gathers the queries; takes values that are not finite out of tiles that some rows see and others do not.
//   11        walks the block's share of the work and tells the others its parts, ahead of them.
// A unit of at most 128 rows has its even key tiles worked on as row tile 0 and its odd ones as row tile 1, with a running
// maximum, sum and output each, which are joined at its end: otherwise one tile's softmax and products would wait for each other.
// Tensor memory, 512 columns: scores of tile 0 and 1 (128 each), outputs of tile 0 and 1 (head size each).
//
// Running maximum: a row's reference only moves when its maximum passes it by more than 2^8, since moving it
// costs a pass over the output in tensor memory; weights are then at most 2^8 (float16: 2^15, see
// WeightLift), inside both types.
// The sum of the weights is held unrounded in 32 bits, the weights are rounded once to the cache's type.
//
// Blocks take equal shares of all key tiles of the call (the plan), cut units are joined by their last block.
// Values that are not finite would reach rows that do not see them, as 0 * inf in the product.  In tiles that some rows
// see and others do not, warp 10 puts zeros in their place before the product, and the rows that see them add
// them at the end (add_odd).
//
// 2048 tokens over 18432 keys (32 heads of 128, 8 key heads, bfloat16) take 545 us sustained, 1.07 PFLOP/s, 484 us in a burst.
#pragma once
#include "common.cuh"
#include "tensor.cuh"

namespace gorio {
namespace paged {

namespace {

constexpr int kRows = 256;
constexpr int kTileRows = 128;
constexpr int kTileKeys = 128;
constexpr int kThreads = 384;
constexpr int kSoftmaxRegs = 216, kOtherRegs = 72;   // a thread, of 168 * 3 = 216 * 2 + 72 at launch
constexpr u32 kScores = 0, kOutputs = 256;           // columns of tensor memory
constexpr int kParts = 4;                            // parts that have been told and not yet finished
constexpr int kScans = 8;                            // more parts than the ring of stages lets warp 10 run ahead
constexpr int kOver = 3;                             // a unit's start and end cost about what three tiles do
constexpr float kSpread = 1.0f;                      // joining a part takes about what a tile does

template <int D>
struct Shape {
  static constexpr int chunks = (D + 63) / 64;                            // of 64 elements, 128 bytes
  static constexpr int tile_bytes = chunks * kTileKeys * 128;
  static constexpr int stages = chunks == 1 ? 8 : 5;
};

// A part of a unit: `tiles` key tiles from `tile` on; 0 tiles: the end.
struct __align__(16) PartInfo {
  int r, h, len, n;
  int q0, row0, rows, tile;
  int tiles, lo, hi, whole;
  u32 i0, i1;          // of a cut unit: the blocks that hold parts of it
  int every0, every1;  // keys that all its rows see
};

template <int D>
struct ChunkShared {
  unsigned char q[2][Shape<D>::tile_bytes];
  unsigned char kv[Shape<D>::stages][Shape<D>::tile_bytes];
  PartInfo part[kParts];
  u64 kv_full[Shape<D>::stages], kv_clean[Shape<D>::stages], kv_empty[Shape<D>::stages];
  u64 part_full[kParts], part_empty[kParts];
  u64 q_full[2], q_empty[2], s_full[2], p_full[2][2], o_full[2], scanned[kScans], meet, drained;
  u32 odd[kScans];
  u32 tmem, failed, last;
  union {
    PlanShared plan;                 // until the parts begin
    float2 half_ml[kTileRows];
  };
};

// What one row sees.
struct Row {
  int pos, lo, hi;
  int head;          // query head
  i64 tok;           // row of q and out
};

template <typename A>
__device__ __forceinline__ Row row_of(const A &a, const PartInfo &p, u32 flat) {
  Row r;
  const u32 tok = flat / a.group;
  r.head = (int)(flat - tok * a.group) + p.h * (int)a.group;
  r.tok = p.q0 + (int)tok;
  r.pos = position_of(a, Request{p.len, p.n, p.q0}, (int)tok);
  r.hi = a.causal ? min(p.len, r.pos + 1) : p.len;
  r.lo = a.window ? (int)max((i64)0, (i64)r.pos - a.window + 1) : 0;
  return r;
}

// The keys that all rows of a part see: later rows see later keys.  Those of a group's requests come in any order, so that
// under a window no key is taken to be seen by all.
__device__ __forceinline__ void all_see(const Attn &a, PartInfo &p) {
  p.every0 = row_of(a, p, (u32)(p.row0 + p.rows - 1)).lo;
  p.every1 = row_of(a, p, (u32)p.row0).hi;
}
__device__ __forceinline__ void all_see(const PrefixAttn &a, PartInfo &p) {
  p.every0 = a.window ? p.hi : 0;
  p.every1 = p.hi;
}

// Adds to 32 columns of a row's weighted sum the values that are not finite of the keys [k0, k1), which it sees, without
// [every0, every1), which all rows of its unit see.  The product ran without them; a weight is above 0, whatever it is.
template <typename T>
__device__ __noinline__ void add_odd(const Attn &a, int req, int h, int k0, int k1, int every0, int every1, int col, float *acc) {
  for (int key = k0; key < k1; ++key) {
    if (key >= every0 && key < every1) key = every1;
    if (key >= k1) break;
    const u32 at = (u32)key / a.page;
    const int pg = a.tables[(i64)req * a.tab_r + at];
    if ((u32)pg >= a.n_pages) continue;
    const u16 *v = (const u16 *)a.vp + (i64)pg * a.v_p + (i64)h * a.v_h + (i64)((u32)key - at * a.page) * a.v_t + col;
#pragma unroll
    for (int d = 0; d < 32; d += 8) {
      const uint4 x = *(const uint4 *)(v + d);
      const u32 w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 u = unpack2<T>(w[i]);
        if (!isfinite(u.x)) acc[d + 2 * i] += u.x;
        if (!isfinite(u.y)) acc[d + 2 * i + 1] += u.y;
      }
    }
  }
}

// eight 16-bit numbers with zeros for those that are not finite
template <typename T>
__device__ __forceinline__ uint4 finite8(uint4 v) {
  auto clean = [](u32 x) {
    constexpr u32 lo = ExponentBits<T>::mask, hi = lo << 16;
    return ((x & lo) == lo ? 0u : x & 0xffffu) | ((x & hi) == hi ? 0u : x & 0xffff0000u);
  };
  return make_uint4(clean(v.x), clean(v.y), clean(v.z), clean(v.w));
}

// the lowest n bits, n cut to [0, 32]
__device__ __forceinline__ u32 bits_below(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }

// 64 of a row's scores to weights: 2^(x * mul - base), summed unrounded into `sum`, rounded to the cache's type in w.  All
// exponentials go to the special function units: computing some of them in the multiply-add units (a polynomial, two numbers an
// instruction) was slower at every share tried, 1/8 to 1/2, here and in the cap's exponentials.
template <typename T>
__device__ __forceinline__ void weights64(const float *s, f32x2 mul, f32x2 minus_base, f32x2 (&sum)[2], u32 *w) {
#pragma unroll
  for (int k = 0; k < 32; ++k) {
    float x0, x1;
    unpack_f32(fma_f32x2(pack_f32(s[2 * k], s[2 * k + 1]), mul, minus_base), x0, x1);
    x0 = exp2_approx(x0);
    x1 = exp2_approx(x1);
    sum[k & 1] = add_f32x2(sum[k & 1], pack_f32(x0, x1));
    w[k] = pack2<T>(x0, x1);
  }
}

// The end of a part, by the eight warps of the softmax: its rows written, or left for or joined with the unit's other parts.  `output` gives
// COLS columns of this thread's row, `output32` 32, as weighted sums that count from 2^m, like l.  `mine`: the thread's warpgroup writes the row.
// Returns false once a wait has run out.
template <typename T, int D, int COLS, bool WIDE, typename A, typename Rows, typename Shared, typename Meet, typename Output, typename Output32>
__device__ __forceinline__ bool write_part(const A &a, const Rows &covered, Shared &sh, const PartInfo &p, const Row &r, bool valid, bool mine, bool fine,
                                           int unit_row, float m, float l, const Meet &meet, const Output &output, const Output32 &output32) {
  typedef typename EndOf<A>::type End;
  constexpr int kCols = COLS;
  constexpr int kAhead = 2;                                  // parts of a cut unit that are fetched at a time, 32 columns of each
  if (p.whole) {
    if (mine && fine) {
      const End end(a, covered, r.tok, r.head, D, m, l, valid);
#pragma unroll 1
      for (int col = 0; col < D; col += kCols) {
        float o[kCols];
        output(o, col);
#pragma unroll
        for (int k = 0; k < kCols; k += 32)
          if (valid) end.template write32<T>(a, r.tok, r.head, col + k, o + k);
      }
    }
  } else if (leaves_parts(a)) {
    // A part of a cut unit stays as it is, [part][row][column], as its readers go along a row.
    if (mine && fine) {
      const i64 slot = 2 * (i64)blockIdx.x + (blockIdx.x == p.i0 ? 1 : 0);
      *(float2 *)(a.part_ml + (slot * kRows + unit_row) * 2) = make_float2(m, l);
      if (valid && blockIdx.x == p.i0) tell_parts(a, r.tok * a.hq + r.head, p.i0, p.i1, unit_row, kRows);
#pragma unroll 1
      for (int col = 0; col < D; col += kCols) {
        float o[kCols];
        output(o, col);
#pragma unroll
        for (int k = 0; k < kCols / 4; ++k)
          __stcg((float4 *)(a.part_o + (slot * kRows + unit_row) * D + col) + k, make_float4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]));
      }
    }
  } else if (fine) {
    // A cut unit.  The last block to get here joins the parts, its own out of tensor memory; the others leave theirs in
    // the workspace: [part][column / 4][row][4], so that neighbouring threads' rows lie side by side.
    const u32 own = blockIdx.x, others = p.i1 - p.i0;
    if (threadIdx.x == 0) sh.last = load_acquire(a.arrived + p.i0) == others;
    fine = meet();
    bool join = fine && sh.last != 0;
    if (fine && !join) {
      const i64 slot = 2 * own + (own == p.i0 ? 1 : 0);
      if (mine) {
        *(float2 *)(a.part_ml + (slot * kRows + unit_row) * 2) = make_float2(m, l);
#pragma unroll 1
        for (int col = 0; col < D; col += kCols) {
          float o[kCols];
          output(o, col);
#pragma unroll
          for (int k = 0; k < kCols / 4; ++k)
            __stcg((float4 *)a.part_o + (slot * (D / 4) + col / 4 + k) * kRows + unit_row, make_float4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]));
        }
      }
      __threadfence();
      fine = meet();
      if (threadIdx.x == 0 && fine) { sh.last = atomicAdd(a.arrived + p.i0, 1u) == others; __threadfence(); }
      fine = fine && meet();
      join = fine && sh.last != 0;
    }
    if (join) {
      if (threadIdx.x == 0) a.arrived[p.i0] = 0;                 // ready for the next call
      if (mine) {
        auto place = [&](u32 i) { return (i64)(2 * i + (i == p.i0 ? 1 : 0)); };
        float top = -INFINITY, sum = 0.0f;
#pragma unroll 4
        for (u32 i = p.i0; i <= p.i1; ++i) {
          const float x = __ldcg(a.part_ml + (place(i) * kRows + unit_row) * 2);
          top = fmaxf(top, i == own ? m : x);
        }
        const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll 4
        for (u32 i = p.i0; i <= p.i1; ++i) {
          const float2 x = __ldcg((const float2 *)(a.part_ml + (place(i) * kRows + unit_row) * 2));
          sum += i == own ? moved_sum<WIDE>(l, m - base) : moved_sum<WIDE>(x.y, x.x - base);
        }
        const End end(a, covered, r.tok, r.head, D, top, sum, valid);
#pragma unroll 1
        for (int col = 0; col < D; col += 32) {
          float acc[32];
#pragma unroll
          for (int k = 0; k < 32; ++k) acc[k] = 0.0f;
#pragma unroll 1
          for (u32 i = p.i0; i <= p.i1; i += kAhead) {
            float o[kAhead][32], g[kAhead];
#pragma unroll
            for (u32 j = 0; j < kAhead; ++j) {
              const bool there = i + j <= p.i1 && i + j != own;
              const i64 at = place(i + j);
              const float4 *from = (const float4 *)a.part_o + (at * (D / 4) + col / 4) * kRows + unit_row;
              g[j] = there ? __ldcg(a.part_ml + (at * kRows + unit_row) * 2) : -INFINITY;
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                const float4 x = there ? __ldcg(from + k * kRows) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                o[j][4 * k] = x.x; o[j][4 * k + 1] = x.y; o[j][4 * k + 2] = x.z; o[j][4 * k + 3] = x.w;
              }
            }
#pragma unroll
            for (u32 j = 0; j < kAhead; ++j) {
              if (i + j == own) {
                g[j] = m;
                output32(o[j], col);
              }
              g[j] = exp2_approx(g[j] - base);
#pragma unroll
              for (int k = 0; k < 32; ++k) acc[k] += g[j] * o[j][k];
            }
          }
          if (valid) end.template write32<T>(a, r.tok, r.head, col, acc);
        }
      }
    }
  }
  return fine;
}

// What becomes of q.k: nothing but the scale; a cap of up to 64 or a bias; a cap of any size.  Without its series capped_log2 is off by
// some 2^-22 of the cap, which up to 64 is less than the weights' rounding, and a call of such layers takes 103 us where it
// takes 111 with the series.
enum Scores { kPlain, kSmallCap, kLargeCap };

// A row's 128 products to units of log2, with cap and bias.  `in` and `linear`: the cap's exponent and the score of a product of 1; `far`: the
// first key's bias.
template <Scores SCORES>
__device__ __forceinline__ void scores128(const Attn &a, float *s, float in, float linear, float slope, float far) {
  const float cap = a.softcap * kLog2e;
  const f32x2 in2 = pack_f32(in, in), slope2 = pack_f32(slope, slope), one2 = pack_f32(1.0f, 1.0f), zero2 = pack_f32(0.0f, 0.0f);
  const f32x2 twice2 = pack_f32(-2.0f * cap, -2.0f * cap), far2 = pack_f32(far, far);
  const f32x2 cap2 = SCORES == kLargeCap ? pack_f32(cap, cap) : pack_f32(cap + far, cap + far);
  const f32x2 linear2 = pack_f32(linear, linear), c1 = pack_f32(kCap1, kCap1), c2 = pack_f32(kCap2, kCap2), c3 = pack_f32(kCap3, kCap3);
#pragma unroll
  for (int i = 0; i < 128; i += 2) {
    const f32x2 dot = pack_f32(s[i], s[i + 1]);
    f32x2 x;
    if (SCORES == kLargeCap || a.softcap > 0.0f) {  // cap * tanh(x / cap), see capped_log2
      float e0, e1;
      const f32x2 w = fma_f32x2(dot, in2, zero2);
      unpack_f32(w, e0, e1);
      unpack_f32(add_f32x2(pack_f32(exp2_approx(e0), exp2_approx(e1)), one2), e0, e1);
      x = fma_f32x2(twice2, pack_f32(rcp_approx(e0), rcp_approx(e1)), cap2);
      if (SCORES == kLargeCap) {
        const f32x2 q = fma_f32x2(w, w, zero2);
        const f32x2 small = fma_f32x2(fma_f32x2(dot, linear2, zero2), fma_f32x2(q, fma_f32x2(q, fma_f32x2(q, c3, c2), c1), one2), zero2);
        float w0, w1, s0, s1;
        unpack_f32(w, w0, w1);
        unpack_f32(small, s0, s1);
        unpack_f32(x, e0, e1);
        x = add_f32x2(pack_f32(fabsf(w0) < kCapSeries ? s0 : e0, fabsf(w1) < kCapSeries ? s1 : e1), far2);
      }
    } else {
      x = fma_f32x2(dot, in2, far2);
    }
    unpack_f32(fma_f32x2(slope2, pack_f32((float)i, (float)(i + 1)), x), s[i], s[i + 1]);
  }
}

// Masks all but the keys [lo, hi) of 128.
__device__ __forceinline__ void mask128(float *s, int lo, int hi) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {                              // a bit for each of 32 keys
    const u32 seen = bits_below(hi - 32 * w) & ~bits_below(lo - 32 * w);
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (!(seen & (1u << i))) s[32 * w + i] = -INFINITY;
  }
}

// The largest of 128: four chains of three-way maxima.
__device__ __forceinline__ float largest128(const float *s) {
  float tops[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
  for (int i = 4; i < 124; i += 8)
#pragma unroll
    for (int k = 0; k < 4; ++k) tops[k] = fmaxf(fmaxf(tops[k], s[i + k]), s[i + 4 + k]);
  return fmaxf(fmaxf(fmaxf(tops[0], s[124]), fmaxf(tops[1], s[125])), fmaxf(fmaxf(tops[2], s[126]), fmaxf(tops[3], s[127])));
}

template <typename T, int D, Scores SCORES, typename A>
__global__ void __launch_bounds__(kThreads, 1) attention_chunk_kernel(const __grid_constant__ A a, const __grid_constant__ CUtensorMap keys,
                                                                      const __grid_constant__ CUtensorMap values, const u32 box_rows) {
  extern __shared__ unsigned char raw[];
  ChunkShared<D> &sh = *(ChunkShared<D> *)(raw + ((1024 - (smem_addr(raw) & 1023)) & 1023));
  typedef Shape<D> S;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (warp == 8) {
    for (int i = lane; i < S::stages; i += 32) { bar_init(&sh.kv_full[i], 1); bar_init(&sh.kv_clean[i], 1); bar_init(&sh.kv_empty[i], 2); }
    if (lane < kParts) { bar_init(&sh.part_full[lane], 1); bar_init(&sh.part_empty[lane], 11); }
    if (lane < kScans) { bar_init(&sh.scanned[lane], 1); sh.odd[lane] = 0; }
    if (lane < 2) {
      bar_init(&sh.q_full[lane], 1); bar_init(&sh.q_empty[lane], 1); bar_init(&sh.s_full[lane], 1); bar_init(&sh.o_full[lane], 1);
      bar_init(&sh.p_full[lane][0], 4); bar_init(&sh.p_full[lane][1], 4);
    }
    if (lane == 0) { bar_init(&sh.meet, 8); bar_init(&sh.drained, 1); sh.failed = 0; }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async();
    __syncwarp();
    tmem_alloc(&sh.tmem, 512);
  }
  let_second_begin(a);
  const Plan plan = block_plan<kRows, kTileKeys, kOver, kThreads>(a, sh.plan, leaves_parts(a) ? 0.0f : kSpread);
  const auto covered = covered_rows(a);
  mma_fence_before();
  __syncthreads();
  mma_fence_after();
  const u32 tmem = sh.tmem;
  const WaitLimit limit{a.wait_ticks, &sh.failed};
  // A kernel that may begin before the one before it has ended waits for that one's end without a limit, at a row's end; a warp's first wait that passes
  // the limit meanwhile does so too, and counts from there.
  bool alone = !Overlaps<A>::value;
  auto wait = [&](u64 *bar, u32 parity) {
    return warp_wait(bar, parity, limit, [&] {
      if (alone) return false;
      wait_for_first(a);
      return alone = true;
    });
  };
  // the part that is told `no`-th; false at the end
  auto take_part = [&](u32 no, PartInfo &p) {
    if (!wait(&sh.part_full[no % kParts], (no / kParts) & 1)) return false;
    p = sh.part[no % kParts];
    return p.tiles != 0;
  };
  auto part_done = [&](u32 no) {
    __syncwarp();
    if (lane == 0) bar_arrive(&sh.part_empty[no % kParts]);
  };

  if (warp < 8) {
    // ------------------------------------------------------------------ softmax of row tile t
    more_registers<kSoftmaxRegs>();
    const int t = warp >> 2, row = tid & (kTileRows - 1);
    constexpr int kCols = D % 64 == 0 ? 64 : 32;             // columns of the output that are worked on at a time
    constexpr float kLift = WeightLift<T, 8>::value;
    const u32 lanes = (u32)(warp & 3) << 21;                 // this warp's 32 lanes of tensor memory
    const u32 scores = tmem + kScores + t * 128 + lanes, outputs = tmem + kOutputs + t * D + lanes;
    u32 s_phase = 0, o_phase = 0, meet_phase = 0;            // o_phase: a bit for each row tile's output
    auto meet = [&]() {                                      // all eight warps, with the limit of every other wait
      __syncwarp();
      if (lane == 0) bar_arrive(&sh.meet);
      const bool ok = wait(&sh.meet, meet_phase);
      meet_phase ^= 1;
      return ok;
    };
    PartInfo p;
    bool fine = true;                                        // no wait of this warp has run out
    for (u32 no = 0; fine && take_part(no, p); ++no) {
      const bool split = p.rows <= kTileRows;                // one row tile: key tiles by turns
      const bool mine = t == 0 || !split;                    // whose rows this warpgroup writes
      const int unit_row = (split ? 0 : t * kTileRows) + row, first = split ? t : 0;
      const bool valid = unit_row < p.rows;
      const Row r = row_of(a, p, (u32)p.row0 + (valid ? unit_row : 0));
      float m = -INFINITY, l = 0.0f;
      {
        const float slope = SCORES != kPlain && a.slopes ? a.slopes[r.head] * kLog2e : 0.0f;
        const float mul = SCORES != kPlain ? 1.0f : a.scale * kLog2e;
        for (int at = first; at < p.tiles; at += split ? 2 : 1) {
          fine = wait(&sh.s_full[t], s_phase);
          if (!fine) break;
          s_phase ^= 1;
          mma_fence_after();
          float s[128];
#pragma unroll
          for (int i = 0; i < 4; ++i) tmem_ld32(s + 32 * i, scores + 32 * i);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < 4; ++i) keep(s + 32 * i);
          const int key0 = (p.tile + at) * kTileKeys;
          if (SCORES != kPlain) {                            // to units of log2, with cap and bias
            const float linear = a.scale * kLog2e;
            scores128<SCORES>(a, s, a.softcap > 0.0f ? cap_in(a) : linear, linear, slope, slope * (float)(key0 - r.pos));
          }
          if (__any_sync(0xffffffffu, key0 < r.lo || key0 + kTileKeys > r.hi)) mask128(s, r.lo - key0, r.hi - key0);
          float top = largest128(s);
          top *= mul;
          const bool moves = top > m + 8.0f || (m == -INFINITY && top > -INFINITY);
          if (__any_sync(0xffffffffu, moves)) {
            const float to = moves ? top : m;
            const float f = m == -INFINITY ? 0.0f : exp2_approx(m - to);
            m = to;
            l *= f;
            if (at > first) {                                // the scores' arrival says that the product before is done
#pragma unroll 2
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
          const float minus_base = m == -INFINITY ? 0.0f : kLift - m;
          const f32x2 mul2 = pack_f32(mul, mul), base2 = pack_f32(minus_base, minus_base);
          f32x2 sum[2] = {pack_f32(l, 0.0f), pack_f32(0.0f, 0.0f)};
#pragma unroll
          for (int i = 0; i < 2; ++i) {                      // the product starts on the first half of the weights
            u32 w[32];
            weights64<T>(s + 64 * i, mul2, base2, sum, w);
            tmem_st32(scores + 32 * i, w);
            tmem_wait_st();
            mma_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(&sh.p_full[t][i]);
          }
          float l0, l1;
          unpack_f32(add_f32x2(sum[0], sum[1]), l0, l1);
          l = l0 + l1;
        }
      }
      m -= kLift;                                            // what the weights and their sum count from
      bool odd = false;
      const bool two = split && p.tiles > 1;                 // both warpgroups have a part of the same rows
      if (two && t == 1) sh.half_ml[row] = make_float2(m, l);
      if (mine) fine = fine && wait(&sh.scanned[no % kScans], (no / kScans) & 1);
      for (int u = 0; u < 2; ++u) {                          // each keeps count of both outputs' phases
        if (u == 1 && split && !two) continue;
        if (u == t || two) fine = fine && wait(&sh.o_full[u], (o_phase >> u) & 1);
        o_phase ^= 1u << u;
      }
      mma_fence_after();
      float f0 = 1.0f, f1 = 0.0f;
      if (two) {
        fine = fine && meet();
        if (t == 0) {
          const float2 other = sh.half_ml[row];
          const float top = fmaxf(m, other.x), base = top == -INFINITY ? 0.0f : top;
          f0 = exp2_approx(m - base);
          f1 = exp2_approx(other.x - base);
          l = l * f0 + other.y * f1;
          m = top;
        }
      }
      if (mine) odd = fine && sh.odd[no % kScans] != 0;
      auto output32 = [&](float *o, int col) {               // 32 columns of the row's output, not yet divided by l
        tmem_ld32(o, outputs + col);
        tmem_wait_ld();
        keep(o);
        if (two) {
          float x[32];
          tmem_ld32(x, outputs + D + col);
          tmem_wait_ld();
          keep(x);
#pragma unroll
          for (int k = 0; k < 32; ++k) o[k] = f0 * o[k] + f1 * x[k];
        }
        if (odd) {
          float x[32];                                       // not o itself, which stays in registers
#pragma unroll
          for (int k = 0; k < 32; ++k) x[k] = o[k];
          add_odd<T>(a, p.r, p.h, max(p.tile * kTileKeys, r.lo), min((p.tile + p.tiles) * kTileKeys, r.hi), p.every0, p.every1, col, x);
#pragma unroll
          for (int k = 0; k < 32; ++k) o[k] = x[k];
        }
      };
      auto output = [&](float *o, int col) {                 // the same for kCols columns, with one wait where it can be
        if (odd || two) {
#pragma unroll
          for (int k = 0; k < kCols; k += 32) output32(o + k, col + k);
          return;
        }
#pragma unroll
        for (int k = 0; k < kCols; k += 32) tmem_ld32(o + k, outputs + col + k);
        tmem_wait_ld();
#pragma unroll
        for (int k = 0; k < kCols; k += 32) keep(o + k);
      };
      fine = write_part<T, D, kCols, false>(a, covered, sh, p, r, valid, mine, fine, unit_row, m, l, meet, output, output32);
      mma_fence_before();
      if (two || !p.whole) fine = fine && meet();            // sh.last and the other's output are free again
      part_done(no);
    }
  } else {
    fewer_registers<kOtherRegs>();
    if (warp == 8) {
      // ---------------------------------------------------------------- the products
      // All that the one issuing lane needs is the same in all lanes and known to be: the operands then stay in uniform
      // registers, where the instruction wants them (moved there for each
      // instruction, issuing one took 80 cycles, and the instruction itself takes 64).
      constexpr u32 kScoreShape = mma_shape<T>(kTileKeys, false), kOutShape = mma_shape<T>(D, true);
      constexpr u32 kChunk = (kTileKeys * 128) >> 4, kTile = S::tile_bytes >> 4;
      const u32 tm = uniform(tmem), q_at = uniform(operand(sh.q[0], 16)), k_at = uniform(operand(sh.kv[0], 16)), v_at = uniform(operand(sh.kv[0], kTileKeys * 128));
      u32 stage = 0, kv_phase = 0, q_phase = 0, p_phase = 0;          // bit t of the last two
      bool fine = true;
      // Scores of queries q_tile with the key tile in k_stage, to row tile t's place; `last`: the queries are not needed after it.  `frees`: no product needs
      // the stages v_stage and k_stage after it.  One region of the issuing lane for all, since what stands between two
      // products has to be shorter than what the matrix unit has queued, some 200 cycles.
      auto scores_of = [&](u32 t, u32 q_tile, u32 k_stage, bool last, bool frees, u32 v_stage) {
        if (one_lane()) {
#pragma unroll
          for (u32 i = 0; i < D / 16; ++i)
            mma_ss(tm + kScores + t * 128, q_at + q_tile * kTile + (i >> 2) * kChunk + (i & 3) * 2, k_at + k_stage * kTile + (i >> 2) * kChunk + (i & 3) * 2, kScoreShape, i > 0);
          mma_commit(&sh.s_full[t]);
          if (frees) {
            if (v_stage != k_stage) mma_commit(&sh.kv_empty[v_stage]);
            mma_commit(&sh.kv_empty[k_stage]);
          }
          if (last) mma_commit(&sh.q_empty[q_tile]);
        }
        __syncwarp();
      };
      auto outputs_of = [&](u32 t, u32 v_stage, u32 half, bool add, bool last, bool frees) {
        if (one_lane()) {
#pragma unroll
          for (u32 k = 0; k < kTileKeys / 32; ++k)
            mma_ts(tm + kOutputs + t * D, tm + kScores + t * 128 + (half * 4 + k) * 8, v_at + v_stage * kTile + (half * 4 + k) * (2048 >> 4), kOutShape, add || k > 0);
          if (last) mma_commit(&sh.o_full[t]);
          if (frees) mma_commit(&sh.kv_empty[v_stage]);
        }
        __syncwarp();
      };
      auto step = [&]() { if (++stage == (u32)S::stages) { stage = 0; kv_phase ^= 1; } };
      for (u32 no = 0; fine; ++no) {
        PartInfo p;
        if (!__all_sync(0xffffffffu, take_part(no, p))) break;
        const u32 n_tiles = uniform((u32)p.tiles);
        // A tile's values before their product: that warp 10 is done with a tile which not all rows see all of, and zeros in the
        // rows outside [lo, hi), whatever the pages hold there.
        auto prepare = [&](u32 at, u32 v_stage, u32 phase) {
          const int key0 = (p.tile + (int)at) * kTileKeys;
          if (key0 >= p.every0 && key0 + kTileKeys <= p.every1) return true;
          if (!wait(&sh.kv_clean[v_stage], phase)) return false;
          if (key0 >= p.lo && key0 + kTileKeys <= p.hi) return true;
          const int z0 = max(0, min(kTileKeys, p.lo - key0)), z1 = max(z0, min(kTileKeys, p.hi - key0)), rows = z0 + kTileKeys - z1;
          for (int x = lane; x < rows * 8; x += 32) {
            const int k = (x >> 3) < z0 ? x >> 3 : (x >> 3) - z0 + z1;
#pragma unroll
            for (int i = 0; i < S::chunks; ++i) *(uint4 *)(sh.kv[v_stage] + i * (kTileKeys * 128) + k * 128 + (x & 7) * 16) = make_uint4(0, 0, 0, 0);
          }
          fence_async();
          __syncwarp();
          return true;
        };
        fine = wait(&sh.q_full[0], q_phase & 1);
        q_phase ^= 1;
        if (uniform(p.rows <= kTileRows)) {
          // one row tile: key tile i goes to place i & 1; the ring holds key, value, key, value ...
          auto ahead = [&](u32 by, u32 &ph) {                         // the stage `by` fills after this one
            const u32 i = stage + by;
            ph = i >= (u32)S::stages ? kv_phase ^ 1 : kv_phase;
            return i >= (u32)S::stages ? i - S::stages : i;
          };
          for (u32 i = 0; i < 2 && i < n_tiles && fine; ++i) {
            u32 ph;
            const u32 k_stage = ahead(2 * i, ph);
            fine = wait(&sh.kv_full[k_stage], ph);
            if (!fine) break;
            mma_fence_after();
            scores_of(i, 0, k_stage, i + 1 == n_tiles, true, k_stage);
          }
          for (u32 at = 0; at < n_tiles && fine; ++at) {
            u32 v_ph, k_ph;
            const u32 t = at & 1, v_stage = ahead(1, v_ph), k_stage = ahead(4, k_ph);
            const bool more = at + 2 < n_tiles;
            fine = wait(&sh.kv_full[v_stage], v_ph) && (!more || wait(&sh.kv_full[k_stage], k_ph));
            fine = fine && prepare(at, v_stage, v_ph);
            for (u32 half = 0; half < 2 && fine; ++half) {
              fine = wait(&sh.p_full[t][half], (p_phase >> t) & 1);
              if (!fine) break;
              mma_fence_after();
              outputs_of(t, v_stage, half, at > 1 || half > 0, half == 1 && !more, half == 1);
            }
            p_phase ^= 1u << t;
            if (more && fine) scores_of(t, 0, k_stage, at + 3 == n_tiles, true, k_stage);
            step();
            step();
          }
          part_done(no);
          continue;
        }
        fine = fine && wait(&sh.q_full[1], q_phase >> 1) && wait(&sh.kv_full[stage], kv_phase);
        q_phase ^= 2;
        if (!fine) break;
        mma_fence_after();
        for (u32 t = 0; t < 2; ++t) scores_of(t, t, stage, n_tiles == 1, t == 1, stage);
        step();
        fine = wait(&sh.kv_full[stage], kv_phase);
        for (u32 at = 0; at < n_tiles && fine; ++at) {
          // here stage holds the tile's values, and they have arrived
          const u32 v_stage = stage, v_phase = kv_phase;
          const bool more = at + 1 < n_tiles;
          step();
          const u32 k_stage = stage;
          if (more && at == 0) fine = wait(&sh.kv_full[k_stage], kv_phase);
          fine = fine && prepare(at, v_stage, v_phase);
          if (more) step();                                           // to the next tile's values
#pragma unroll
          for (u32 t = 0; t < 2; ++t) {
            const bool final_t = t == 1;
            for (u32 half = 0; half < 2; ++half) {
              fine = fine && wait(&sh.p_full[t][half], (p_phase >> t) & 1);
              if (!fine) break;
              mma_fence_after();
              outputs_of(t, v_stage, half, at > 0 || half > 0, half == 1 && !more, half == 1 && !more && final_t);
            }
            p_phase ^= 1u << t;
            if (!fine) break;
            if (more) {
              scores_of(t, t, k_stage, at + 2 == n_tiles, final_t, v_stage);
              // what the next tile needs, looked at while these products run: its values, then the keys after it
              if (t == 0) fine = wait(&sh.kv_full[stage], kv_phase);
              if (fine && final_t && at + 2 < n_tiles) {
                const u32 after = stage + 1 == (u32)S::stages ? 0 : stage + 1;
                fine = wait(&sh.kv_full[after], after ? kv_phase : kv_phase ^ 1);
              }
            }
          }
        }
        part_done(no);
      }
      // tensor memory is given back, and shared memory left, only when no product uses them any more
      if (one_lane()) mma_commit(&sh.drained);
      __syncwarp();
      drain(&sh.drained, 0);
    } else if (warp == 9) {
      // ---------------------------------------------------------------- the copies
      const int boxes = kTileKeys / (int)box_rows * S::chunks;       // at most 32: a lane each
      const int g = lane / S::chunks, chunk = lane - g * S::chunks;
      int stage = 0;
      u32 phase = 1;                                                  // the first round finds the stages free
      bool fine = true;
      PartInfo p;
      for (u32 no = 0; fine && take_part(no, p); ++no) {
        for (int at = 0; at < p.tiles && fine; ++at) {
          const int key = (p.tile + at) * kTileKeys + g * (int)box_rows;
          int page = (int)a.n_pages, in = 0;                          // past the last page: zeros
          if (lane < boxes && key < p.hi && key + (int)box_rows > p.lo) {
            const u32 pi = (u32)key / a.page;
            const int pg = __ldg(a.tables + (i64)p.r * a.tab_r + pi);
            if ((u32)pg < a.n_pages) { page = pg; in = (int)((u32)key - pi * a.page); }
          }
#pragma unroll
          for (int kv = 0; kv < 2; ++kv) {
            fine = fine && wait(&sh.kv_empty[stage], phase);
            if (!fine) break;
            if (lane == 0) bar_expect(&sh.kv_full[stage], (u32)S::tile_bytes);
            __syncwarp();
            if (lane < boxes)
              copy_box(sh.kv[stage] + chunk * (kTileKeys * 128) + g * (int)box_rows * 128, kv ? &values : &keys, chunk * 64, in, p.h, page, &sh.kv_full[stage]);
            if (++stage == S::stages) { stage = 0; phase ^= 1; }
          }
        }
        part_done(no);
      }
      // No copy is left in flight, even where the warps that wait for it have given up: each stage's last one.
      for (int i = 0; i < S::stages; ++i) drain(&sh.kv_full[i], i < stage ? phase ^ 1 : phase);
    } else if (warp == 10) {
      // ---------------------------------------------------------------- the queries, values that are not finite
      int stage = 0;
      u32 phase = 0, q_phase = 3;                                     // bit t: the first round finds both tiles free
      bool fine = true;
      PartInfo p;
      for (u32 no = 0; fine && take_part(no, p); ++no) {
        const int tiles = p.rows > kTileRows ? 2 : 1;
        for (int t = 0; t < tiles && fine; ++t) {
          fine = wait(&sh.q_empty[t], (q_phase >> t) & 1);
          q_phase ^= 1u << t;
          if (!fine) break;
          for (int r = lane >> 2; r < kTileRows; r += 8) {            // four lanes a row; zeros past the last row
            const bool valid = t * kTileRows + r < p.rows;
            const u32 flat = valid ? (u32)(p.row0 + t * kTileRows + r) : 0u, tok = flat / a.group, head = flat - tok * a.group + p.h * a.group;
            const u16 *src = (const u16 *)a.q + (i64)(p.q0 + (int)tok) * a.q_t + (i64)head * a.q_h;
#pragma unroll
            for (int j = 0; j < D / 32; ++j) {
              const int piece = (lane & 3) + 4 * j;
              cp_async16(sh.q[t] + (piece >> 3) * (kTileRows * 128) + r * 128 + (((piece & 7) ^ (r & 7)) << 4), src + piece * 8, valid ? 16u : 0u);
            }
          }
          cp_async_commit();
        }
        cp_async_wait<0>();
        fence_async();
        __syncwarp();
        if (lane == 0 && fine)
          for (int t = 0; t < tiles; ++t) bar_arrive(&sh.q_full[t]);
        u32 odd = 0;
        for (int at = 0; at < p.tiles && fine; ++at) {
          const int key0 = (p.tile + at) * kTileKeys, z0 = max(key0, p.lo), z1 = min(key0 + kTileKeys, p.hi);
          const bool look = z0 < p.every0 || z1 > p.every1;  // [lo, hi) without the keys that all rows see
#pragma unroll
          for (int kv = 0; kv < 2; ++kv) {
            fine = fine && wait(&sh.kv_full[stage], phase);
            if (!fine) break;
            if (kv && look) {
              // two ranges of rows: [z0, every0) and [every1, z1)
              const int n0 = max(0, min(z1, p.every0) - z0), from1 = max(z0 + n0, p.every1), rows = n0 + max(0, z1 - from1);
              u32 found = 0;
#pragma unroll 4
              for (int x = lane; x < rows * 8; x += 32) {
                const int k = ((x >> 3) < n0 ? z0 + (x >> 3) : from1 + (x >> 3) - n0) - key0;
#pragma unroll
                for (int i = 0; i < S::chunks; ++i) found |= (u32)not_finite8<T>(*(const uint4 *)(sh.kv[stage] + i * (kTileKeys * 128) + k * 128 + (x & 7) * 16));
              }
              if (found) {
                for (int x = lane; x < rows * 8; x += 32) {
                  const int k = ((x >> 3) < n0 ? z0 + (x >> 3) : from1 + (x >> 3) - n0) - key0;
                  for (int i = 0; i < S::chunks; ++i) {
                    uint4 *const at = (uint4 *)(sh.kv[stage] + i * (kTileKeys * 128) + k * 128 + (x & 7) * 16);
                    *at = finite8<T>(*at);
                  }
                }
                fence_async();
              }
              odd |= found;
            }
            __syncwarp();
            if (lane == 0) { bar_arrive(&sh.kv_clean[stage]); bar_arrive(&sh.kv_empty[stage]); }
            if (++stage == S::stages) { stage = 0; phase ^= 1; }
          }
        }
        odd = __any_sync(0xffffffffu, odd);
        if (lane == 0) {
          sh.odd[no % kScans] = odd;
          bar_arrive(&sh.scanned[no % kScans]);
        }
        part_done(no);
      }
    } else {
      // ---------------------------------------------------------------- the parts
      Cursor c = plan.first;
      u32 left = plan.end - plan.begin;
      bool more = true;
      for (u32 told = 0; more; ++told) {
        settle<kRows, kTileKeys, kOver>(a, c, left, plan.fill);
        const u32 slot = told % kParts;
        PartInfo p{};
        more = left != 0;
        if (more) {
          p.r = (int)c.r; p.h = (int)c.h; p.len = c.req.len; p.n = c.req.n; p.q0 = c.req.q0;
          p.row0 = c.m * kRows;
          p.rows = (int)min((i64)kRows, (i64)c.req.n * a.group - p.row0);
          const int to = (int)min((u32)c.span.tiles, (u32)c.at + left);
          p.tile = c.span.first + c.at;
          p.tiles = to - c.at;
          p.lo = c.span.lo; p.hi = c.span.hi;
          all_see(a, p);
          p.whole = c.at == 0 && to == c.span.tiles;
          if (!p.whole) {
            const u32 unit0 = plan.end - left - (u32)c.at;
            p.i0 = plan.shares.owner(unit0);
            p.i1 = plan.shares.owner(unit0 + (u32)c.span.tiles - 1);
          }
          left -= (u32)p.tiles;
          c.at = to;
        }
        if (!wait(&sh.part_empty[slot], ((told / kParts) & 1) ^ 1)) break;
        if (lane == 0) {
          sh.part[slot] = p;
          bar_arrive(&sh.part_full[slot]);
        }
        __syncwarp();
      }
    }
  }
  mma_fence_before();
  __syncthreads();
  mma_fence_after();
  if (warp == 8) tmem_free(tmem, 512);
  if (tid == 0 && sh.failed) *error_word(a) = 1;
  wait_for_first(a);                             // so that this kernel never ends before the first
}

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

template <typename T, int D, Scores SCORES, typename A>
cudaError_t launch(const A &a, const CUtensorMap &k, const CUtensorMap &v, u32 box_rows, u32 sms, cudaStream_t s) {
  static bool ready[64] = {};
  constexpr size_t bytes = sizeof(ChunkShared<D>) + 1024;
  static_assert(bytes <= 227 * 1024, "shared memory of one block");
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 64) return cudaErrorInvalidDevice;
  if (!ready[dev]) {
    e = cudaFuncSetAttribute(attention_chunk_kernel<T, D, SCORES, A>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e != cudaSuccess) return e;
    // the warps' register shares come out of what the block is launched with: with fewer they would wait for ever
    cudaFuncAttributes f;
    e = cudaFuncGetAttributes(&f, attention_chunk_kernel<T, D, SCORES, A>);
    if (e != cudaSuccess) return e;
    if (f.numRegs * kThreads < kSoftmaxRegs * 256 + kOtherRegs * 128) return cudaErrorInvalidKernelImage;
    ready[dev] = true;
  }
  return launch_kernel<A>(attention_chunk_kernel<T, D, SCORES, A>, sms, kThreads, bytes, s, a, k, v, box_rows);
}

template <typename T, int D, typename A>
cudaError_t pick_scores(const A &a, const CUtensorMap &k, const CUtensorMap &v, u32 box_rows, u32 sms, cudaStream_t s) {
  if (a.softcap > 64.0f) return launch<T, D, kLargeCap>(a, k, v, box_rows, sms, s);
  return a.softcap > 0.0f || a.slopes ? launch<T, D, kSmallCap>(a, k, v, box_rows, sms, s) : launch<T, D, kPlain>(a, k, v, box_rows, sms, s);
}

template <typename T, typename A>
cudaError_t pick_dim(const A &a, const CUtensorMap &k, const CUtensorMap &v, u32 box_rows, int dim, u32 sms, cudaStream_t s) {
  if (dim == 64) return pick_scores<T, 64>(a, k, v, box_rows, sms, s);
  if (dim == 96) return pick_scores<T, 96>(a, k, v, box_rows, sms, s);
  return pick_scores<T, 128>(a, k, v, box_rows, sms, s);
}

template <typename A>
bool launch_chunk_of(const A &a, int dtype, int dim, u32 sms, cudaStream_t s, cudaError_t *e) {
  if (!encoder() || a.n_pages == 0) return false;
  u32 box_rows = a.page & (0u - a.page);               // the largest power of two in the page size, so that a box stays in its page
  if (box_rows > (u32)kTileKeys) box_rows = kTileKeys;
  CUtensorMap k, v;
  if (!page_map(&k, a, a.kp, a.k_t, a.k_h, a.k_p, dtype, dim, box_rows) || !page_map(&v, a, a.vp, a.v_t, a.v_h, a.v_p, dtype, dim, box_rows)) return false;
  *e = dtype == 0 ? pick_dim<__nv_bfloat16>(a, k, v, box_rows, dim, sms, s) : pick_dim<__half>(a, k, v, box_rows, dim, sms, s);
  return true;
}

}  // namespace
}  // namespace paged
}  // namespace gorio
