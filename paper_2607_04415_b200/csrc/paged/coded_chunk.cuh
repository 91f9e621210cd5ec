// Attention of many rows over a quantised paged cache: the chunk form, on the fifth-generation tensor cores.
//
// Units, parts, products, softmax and joins are those of the 16-bit cache's kernel (chunk.cuh); what is new stands between the copies and
// the products.  Sixteen warps:
//   0-3, 4-7  the softmax of row tile 0 and 1: a thread a row.  At a part's start each thread brings its own row of queries, as float16 times a
//             power of two.
//   8         issues both products (one thread).
//   9         copies codes of keys and values, and their scales, into the stages that they are taken apart in.
//   10        finds the logarithms of the scales of a tile's values, and their range.
//   11        walks the block's share of the work and tells the others its parts.
//   12-15     take codes apart, in place, into the 16-bit tiles that the products read.  (With a ring of their own for codes three pieces of 64 keys
//             were all that shared memory held beside them, too few on their way: 972 us where this takes 671 for 2048 tokens over 18432 keys.)
// Keys and values become their codes, exactly.  A score is multiplied by its key's scale in 32 bits, and a weight by its value's before it is rounded, once, to
// float16: 2^(x - m) * scale.  So that weights use that type's range whatever the scales are, m follows the maximum of x + log2(scale), as in the kernel of few rows.
// Where a row sees all of a tile and the tile's scales lie within 2^4 of each other, the largest x and the largest scale stand for it, at most 4 more; elsewhere it is found
// key by key, where it may move m.  So a row's weights are the same whatever scales the keys have that it does not see.  (Key by key in every tile is 128 numbers more
// from shared memory for each row: 771 us where this takes 671 for 2048 tokens over 18432 keys; scales within the exponent, 2^(x + log2(scale) - m), which the
// sum then takes back by a product, 861.  The largest scale in every tile loses the weights of rows whose own scales lie far below it.  With values
// multiplied by their scales as they become float16, two roundings more, float16 results were 3.7e-4 off where this is 2.9e-4 off and a rounding is 2.1e-4.)
//
// A value's scale that is not finite counts as 0 there, and stands in the key's place instead: scores of rows that see the key are then not a number,
// others do not notice.  With it all operands are finite, so that tiles that some rows see and others do not need no care beyond the mask.
#pragma once
#include "chunk.cuh"
#include "coded.cuh"

#include <type_traits>

namespace gorio {
namespace paged {

namespace {

constexpr int kCodedThreads = 512;
constexpr int kCodedSoftmaxRegs = 200, kCodedOtherRegs = 64, kDecodeRegs = 48;   // a thread, of 128 * 4 = 200 * 2 + 64 + 48 at launch
// Tiles whose scales are there.  The second softmax warpgroup has nothing to wait for in a part of one row tile and one key tile, and so may come to a tile that is
// as many behind the first one's as parts are told ahead.  Parity says whether a slot has been filled for it only while that slot cannot be the first one's.
constexpr int kScaleSlots = 8;
static_assert(kScaleSlots > kParts, "a wait for scales would pass on those of an earlier tile");

template <int D>
struct CodedShape {
  static constexpr int chunks = Shape<D>::chunks, tile_bytes = Shape<D>::tile_bytes;
  static constexpr int stages = chunks == 1 ? 8 : 4;
};

template <int D>
struct CodedChunkShared {
  unsigned char q[2][CodedShape<D>::tile_bytes];
  unsigned char kv[CodedShape<D>::stages][CodedShape<D>::tile_bytes];
  __align__(128) float k_scale[kScaleSlots][kTileKeys];
  float v_scale[kScaleSlots][kTileKeys];
  float v_log2[kScaleSlots][kTileKeys];
  float2 v_range[kScaleSlots];                   // the largest and the smallest of them
  u32 scales_boxes[kScaleSlots];                 // which boxes of them were copied
  float q_to_dot[kTileRows];                     // of the rows of a unit of one row tile
  PartInfo part[kParts];
  u64 codes_full[CodedShape<D>::stages], kv_full[CodedShape<D>::stages], kv_empty[CodedShape<D>::stages];
  u64 scales_there[kScaleSlots], scales_full[kScaleSlots], scales_empty[kScaleSlots];
  u64 part_full[kParts], part_empty[kParts];
  u64 q_full[2], q_empty[2], s_full[2], p_full[2][2], o_full[2], meet, drained;
  u32 tmem, failed, last;
  union {
    PlanShared plan;                 // until the parts begin
    float2 half_ml[kTileRows];
  };
};

__device__ __forceinline__ f32x2 mul_f32x2(f32x2 a, f32x2 b) {
  f32x2 v;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
  return v;
}
// weights64 for values with scales of their own: the sum is that of the weights alone.
__device__ __forceinline__ void scaled_weights64(const float *s, const float *scale, f32x2 mul, f32x2 minus_base, f32x2 (&sum)[2], u32 *w) {
#pragma unroll
  for (int k = 0; k < 32; k += 2) {
    const float4 v = *(const float4 *)(scale + 2 * k);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float x0, x1;
      unpack_f32(fma_f32x2(pack_f32(s[2 * (k + i)], s[2 * (k + i) + 1]), mul, minus_base), x0, x1);
      const f32x2 x = pack_f32(exp2_approx(x0), exp2_approx(x1));
      sum[i] = add_f32x2(sum[i], x);
      unpack_f32(mul_f32x2(x, i ? pack_f32(v.z, v.w) : pack_f32(v.x, v.y)), x0, x1);
      w[k + i] = pack2<__half>(x0, x1);
    }
  }
}
__device__ __forceinline__ void bar_arrive_n(u64 *bar, u32 n) {
  asm volatile("mbarrier.arrive.shared.b64 _, [%0], %1;" ::"r"(smem_addr(bar)), "r"(n) : "memory");
}
// The scales of some rows of a page into shared memory: both addresses are multiples of 16 bytes, and so is the size.  (A tensor copy would want
// 128 bytes of the second, which a page of 8 or 16 rows does not give.)
__device__ __forceinline__ void copy_scales(void *to, const float *from, u32 bytes, u64 *bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_addr(to)), "l"(from), "r"(bytes),
               "r"(smem_addr(bar))
               : "memory");
}
// The largest of 128 scores * mul + logarithms of their values' scales.  Few registers, one load after the other: where this stands nearly all are taken, and what
// the compiler would load ahead it spills for in every tile (757 us where this way takes 694 for 2048 tokens over 18432 keys, before the part was read anew).
__device__ __forceinline__ float largest_scaled128(const float *s, float mul, const float *log2s) {
  float top = -INFINITY;
  const u32 at = smem_addr(log2s);
#pragma unroll
  for (int i = 0; i < 128; i += 2) {
    float a, b;
    asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(a), "=f"(b) : "r"(at + i * 4));
    top = fmaxf(fmaxf(top, fmaf(s[i], mul, a)), fmaf(s[i + 1], mul, b));
  }
  return top;
}

template <typename T, Format F, int D, Scores SCORES>
__global__ void __launch_bounds__(kCodedThreads, 1) coded_chunk_kernel(const __grid_constant__ CodedAttn a, const __grid_constant__ CUtensorMap keys,
                                                                       const __grid_constant__ CUtensorMap values, const u32 box_rows) {
  extern __shared__ unsigned char raw[];
  typedef CodedChunkShared<D> Shared;
  Shared &sh = *(Shared *)(raw + ((1024 - (smem_addr(raw) & 1023)) & 1023));
  typedef CodedShape<D> S;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (warp == 8) {
    if (lane < S::stages) { bar_init(&sh.codes_full[lane], 1); bar_init(&sh.kv_full[lane], 4); bar_init(&sh.kv_empty[lane], 1); }
    if (lane < kScaleSlots) { bar_init(&sh.scales_there[lane], 1); bar_init(&sh.scales_full[lane], 1); bar_init(&sh.scales_empty[lane], 8); }
    if (lane < kParts) { bar_init(&sh.part_full[lane], 1); bar_init(&sh.part_empty[lane], 15); }
    if (lane < 2) {
      bar_init(&sh.q_full[lane], 4); bar_init(&sh.q_empty[lane], 1); bar_init(&sh.s_full[lane], 1); bar_init(&sh.o_full[lane], 1);
      bar_init(&sh.p_full[lane][0], 4); bar_init(&sh.p_full[lane][1], 4);
    }
    if (lane == 0) { bar_init(&sh.meet, 8); bar_init(&sh.drained, 1); sh.failed = 0; }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async();
    __syncwarp();
    tmem_alloc(&sh.tmem, 512);
  }
  const Plan plan = block_plan<kRows, kTileKeys, kOver, kCodedThreads>(a, sh.plan, kSpread);
  mma_fence_before();
  __syncthreads();
  mma_fence_after();
  const u32 tmem = sh.tmem;
  const WaitLimit limit{a.wait_ticks, &sh.failed};
  auto wait = [&](u64 *bar, u32 parity) { return warp_wait(bar, parity, limit); };
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
    more_registers<kCodedSoftmaxRegs>();
    const int t = warp >> 2, row = tid & (kTileRows - 1);
    constexpr int kCols = D % 64 == 0 ? 64 : 32;             // columns of the output that are worked on at a time
    constexpr float kLift = WeightLift<__half, 8>::value;
    const u32 lanes = (u32)(warp & 3) << 21;                 // this warp's 32 lanes of tensor memory
    const u32 scores = tmem + kScores + t * 128 + lanes, outputs = scores + (kOutputs - kScores) + t * (D - 128);
    u32 s_phase = 0, o_phase = 0, meet_phase = 0, q_phase = 1;   // o_phase: a bit for each row tile's output
    u32 tile_no = 0;                                         // tiles of the parts before
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
      float m = -INFINITY, l = 0.0f;
      {
        const bool split = p.rows <= kTileRows;                // one row tile: key tiles by turns
        const int unit_row = (split ? 0 : t * kTileRows) + row, first = split ? t : 0;
        const bool valid = unit_row < p.rows;
        const Row r = row_of(a, p, (u32)p.row0 + (valid ? unit_row : 0));
        float to_dot = 1.0f;
        if (t == 0 || !split) {
          // this thread's row of queries: float16, times a power of two
          fine = wait(&sh.q_empty[t], q_phase);
          q_phase ^= 1;
          const u16 *src = (const u16 *)a.q + r.tok * a.q_t + (i64)r.head * a.q_h;
          uint4 x[D / 8];
          float top = 0.0f;
#pragma unroll
          for (int k = 0; k < D / 8; ++k) x[k] = valid ? *(const uint4 *)(src + 8 * k) : make_uint4(0, 0, 0, 0);
#pragma unroll
          for (int k = 0; k < D / 8; ++k) {
            const u32 w[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float2 v = unpack2<T>(w[i]);
              top = fmaxf(top, fmaxf(fabsf(v.x), fabsf(v.y)));
            }
          }
          const float f = query_factor(top);
          to_dot = 1.0f / f;                                   // powers of two
#pragma unroll
          for (int k = 0; k < D / 8; ++k) {
            u32 w[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float2 v = unpack2<T>(w[i]);
              w[i] = pack2<__half>(v.x * f, v.y * f);
            }
            if (fine) *(uint4 *)(sh.q[t] + (k >> 3) * (kTileRows * 128) + row * 128 + (((k & 7) ^ (row & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
          }
          if (split && fine) sh.q_to_dot[row] = to_dot;
          fence_async();
          __syncwarp();
          if (lane == 0 && fine) bar_arrive(&sh.q_full[t]);
        }
        const float slope = SCORES != kPlain && a.slopes ? a.slopes[r.head] * kLog2e : 0.0f;
        for (int at = first; at < p.tiles && fine; at += split ? 2 : 1) {
          const u32 slot = (tile_no + (u32)at) % kScaleSlots;
          fine = wait(&sh.scales_full[slot], ((tile_no + (u32)at) / kScaleSlots) & 1) && wait(&sh.s_full[t], s_phase);
          if (!fine) break;
          s_phase ^= 1;
          mma_fence_after();
          if (split && t == 1 && at == 1) to_dot = sh.q_to_dot[row];     // the queries came before the scores
          const float mul = SCORES != kPlain ? 1.0f : a.scale * kLog2e * to_dot;
          float s[128];
#pragma unroll
          for (int i = 0; i < 4; ++i) tmem_ld32(s + 32 * i, scores + 32 * i);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < 4; ++i) keep(s + 32 * i);
#pragma unroll
          for (int i = 0; i < 128; i += 4) {
            const float4 k = *(const float4 *)&sh.k_scale[slot][i];
            unpack_f32(mul_f32x2(pack_f32(s[i], s[i + 1]), pack_f32(k.x, k.y)), s[i], s[i + 1]);
            unpack_f32(mul_f32x2(pack_f32(s[i + 2], s[i + 3]), pack_f32(k.z, k.w)), s[i + 2], s[i + 3]);
          }
          const int key0 = (p.tile + at) * kTileKeys;
          if (SCORES != kPlain) {                            // to units of log2, with cap and bias
            const float linear = a.scale * kLog2e * to_dot;
            scores128<SCORES>(a, s, a.softcap > 0.0f ? cap_in(a) * to_dot : linear, linear, slope, slope * (float)(key0 - r.pos));
          }
          if (__any_sync(0xffffffffu, key0 < r.lo || key0 + kTileKeys > r.hi)) mask128(s, r.lo - key0, r.hi - key0);
          const f32x2 mul2 = pack_f32(mul, mul);
          const float2 range = sh.v_range[slot];
          float top = largest128(s) * mul + range.x;
          const bool by_key = key0 < r.lo || key0 + kTileKeys > r.hi || range.x - range.y > 4.0f;
          // half an octave less than what moves m, for the roundings of what stands for the maximum
          if (__any_sync(0xffffffffu, by_key && (top > m + 7.5f || (m == -INFINITY && top > -INFINITY)))) {
            const float found = largest_scaled128(s, mul, sh.v_log2[slot]);
            if (by_key) top = found;
          }
          const bool moves = top > m + 8.0f || (m == -INFINITY && top > -INFINITY);
          if (__any_sync(0xffffffffu, moves)) {
            const float to = moves ? top : m;
            const float half = m == -INFINITY ? 0.0f : exp2_approx(0.5f * (m - to)), f = half * half;
            m = to;
            l = l * half * half;                             // see moved_sum
            if (at > first) {                                // the scores' arrival says that the product before is done
              // 16 columns at a time: with 32, beside the 128 scores, what every tile needs was spilled
#pragma unroll 1
              for (int i = 0; i < D / 16; ++i) {
                float o[16];
                tmem_ld16(o, outputs + 16 * i);
                tmem_wait_ld();
                keep16(o);
#pragma unroll
                for (int k = 0; k < 16; ++k) o[k] *= f;
                tmem_st16(outputs + 16 * i, o);
              }
            }
          }
          const float minus_base = m == -INFINITY ? 0.0f : kLift - m;
          const f32x2 base2 = pack_f32(minus_base, minus_base);
          f32x2 sum[2] = {pack_f32(l, 0.0f), pack_f32(0.0f, 0.0f)};
#pragma unroll
          for (int i = 0; i < 2; ++i) {                      // the product starts on the first half of the weights
            u32 w[32];
            scaled_weights64(s + 64 * i, sh.v_scale[slot] + 64 * i, mul2, base2, sum, w);
            tmem_st32(scores + 32 * i, w);
            tmem_wait_st();
            mma_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(&sh.p_full[t][i]);
          }
          if (lane == 0) bar_arrive_n(&sh.scales_empty[slot], split ? 2 : 1);      // all lanes have read them before they told of their weights
          float l0, l1;
          unpack_f32(add_f32x2(sum[0], sum[1]), l0, l1);
          l = l0 + l1;
        }
      }
      // Anew: kept through the tiles, these would take the registers that those are short of.
      p = sh.part[no % kParts];
      const bool split = p.rows <= kTileRows, mine = t == 0 || !split;   // mine: whose rows this warpgroup writes
      const int unit_row = (split ? 0 : t * kTileRows) + row;
      const bool valid = unit_row < p.rows;
      tile_no += (u32)p.tiles;
      m -= kLift;                                            // what the weights and their sum count from
      const bool two = split && p.tiles > 1;                 // both warpgroups have a part of the same rows
      if (two && t == 1) sh.half_ml[row] = make_float2(m, l);
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
          l = moved_sum<true>(l, m - base) + moved_sum<true>(other.y, other.x - base);
          m = top;
        }
      }
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
      };
      auto output = [&](float *o, int col) {                 // the same for kCols columns, with one wait where it can be
        if (two) {
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
      fine = write_part<T, D, kCols, true>((const Attn &)a, NoRows{}, sh, p, row_of(a, p, (u32)p.row0 + (valid ? unit_row : 0)), valid, mine, fine, unit_row, m, l, meet,
                                     output, output32);
      mma_fence_before();
      if (two || !p.whole) fine = fine && meet();            // sh.last and the other's output are free again
      part_done(no);
    }
  } else if (warp >= 12) {
    fewer_registers<kDecodeRegs>();
    // ---------------------------------------------------------------- codes to float16
    // A row's codes lie 128 bytes apart where its first 64 numbers will stand: a warp that has read some rows may write them.  Pieces of 16 codes go
    // to lanes so that eight lanes write even places of one row and odd ones of the next, or the other way round, which lie in different banks:
    // four neighbouring lanes have four pieces of a row, the rest of the row comes in another step (of 96 numbers: two pieces of twice as many rows).
    constexpr int kGroup = D == 64 ? 32 : 16, kEach = D == 96 ? 3 : 4;      // rows that are read before they are written; a lane's pieces of them
    auto row_at = [&](int i) { return D == 128 ? (i >> 1) * 8 + (lane >> 2) : D == 96 && i == 2 ? lane >> 1 : i * 8 + (lane >> 2); };
    auto piece_at = [&](int i) { return D == 128 ? (i & 1) * 4 + (lane & 3) : D == 96 && i == 2 ? 4 + (lane & 1) : lane & 3; };
    // This warp's 32 rows of a tile.
    auto decode_rows = [&](unsigned char *tile, auto clean) {
#pragma unroll 1
      for (int row0 = (warp - 12) * 32; row0 < (warp - 11) * 32; row0 += kGroup) {
        uint4 w[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) w[i] = *(const uint4 *)(tile + (row0 + row_at(i)) * 128 + piece_at(i) * 16);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
          const int row = row0 + row_at(i), piece = piece_at(i) * 2;
          u32 h[8];
          decode_along<F>(w[i].x, h[0], h[1]);
          decode_along<F>(w[i].y, h[2], h[3]);
          decode_along<F>(w[i].z, h[4], h[5]);
          decode_along<F>(w[i].w, h[6], h[7]);
          if (decltype(clean)::value) {
#pragma unroll
            for (int k = 0; k < 8; ++k) h[k] = finite_codes<F>(h[k]);
          }
          unsigned char *const at = tile + (piece >> 3) * (kTileKeys * 128) + row * 128;
          *(uint4 *)(at + (((piece & 7) ^ (row & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
          *(uint4 *)(at + (((piece + 1) & 7 ^ (row & 7)) << 4)) = make_uint4(h[4], h[5], h[6], h[7]);
        }
      }
      fence_async();
      __syncwarp();
    };
    int stage = 0;
    u32 phase = 0;
    bool fine = true;
    PartInfo p;
    for (u32 no = 0; fine && take_part(no, p); ++no) {
      for (int at = 0; at < p.tiles && fine; ++at) {
        const int key0 = (p.tile + at) * kTileKeys;
        const bool every = key0 >= p.every0 && key0 + kTileKeys <= p.every1;      // all rows see all keys of the tile
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          fine = fine && wait(&sh.codes_full[stage], phase);
          if (!fine) break;
          if (F != kE4m3 || !kv || every) decode_rows(sh.kv[stage], std::false_type{});
          else decode_rows(sh.kv[stage], std::true_type{});
          if (lane == 0) bar_arrive(&sh.kv_full[stage]);
          if (++stage == S::stages) { stage = 0; phase ^= 1; }
        }
      }
      part_done(no);
    }
  } else {
    fewer_registers<kCodedOtherRegs>();
    if (warp == 8) {
      // ---------------------------------------------------------------- the products, as in the 16-bit cache's kernel
      constexpr u32 kScoreShape = mma_shape<__half>(kTileKeys, false), kOutShape = mma_shape<__half>(D, true);
      constexpr u32 kChunk = (kTileKeys * 128) >> 4, kTile = S::tile_bytes >> 4;
      const u32 tm = uniform(tmem), q_at = uniform(operand(sh.q[0], 16)), k_at = uniform(operand(sh.kv[0], 16)), v_at = uniform(operand(sh.kv[0], kTileKeys * 128));
      u32 stage = 0, kv_phase = 0, q_phase = 0, p_phase = 0;          // bit t of the last two
      bool fine = true;
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
          const u32 v_stage = stage;
          const bool more = at + 1 < n_tiles;
          step();
          const u32 k_stage = stage;
          if (more && at == 0) fine = wait(&sh.kv_full[k_stage], kv_phase);
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
      // ---------------------------------------------------------------- the copies of codes and scales
      const int boxes = kTileKeys / (int)box_rows;                    // at most 16: a lane each
      int stage = 0;
      u32 phase = 1, tile_no = 0;                                     // the first round finds the stages free
      bool fine = true;
      PartInfo p{};
      // Page and place of this lane's box in each half of a tile, looked up a tile ahead: the entry of a table is far away.
      int page, in;
      auto look_up = [&](int tile) {
        const int key = tile * kTileKeys + lane * (int)box_rows;
        page = (int)a.n_pages;                                        // past the last page: zeros
        in = 0;
        if (lane < boxes && key < p.hi && key + (int)box_rows > p.lo) {
          const u32 pi = (u32)key / a.page;
          const int pg = __ldg(a.tables + (i64)p.r * a.tab_r + pi);
          if ((u32)pg < a.n_pages) { page = pg; in = (int)((u32)key - pi * a.page); }
        }
      };
      for (u32 no = 0; fine && take_part(no, p); ++no) {
        look_up(p.tile);
        for (int at = 0; at < p.tiles && fine; ++at, ++tile_no) {
          const int page_now = page, in_now = in;
          if (at + 1 < p.tiles) look_up(p.tile + at + 1);
          const u32 slot = tile_no % kScaleSlots;
          fine = wait(&sh.scales_empty[slot], ((tile_no / kScaleSlots) & 1) ^ 1);
          if (!fine) break;
          const bool there = lane < boxes && page_now < (int)a.n_pages;
          const u32 all = __ballot_sync(0xffffffffu, there);          // a bit for each box
          if (lane == 0) {
            sh.scales_boxes[slot] = all;
            bar_expect(&sh.scales_there[slot], (u32)__popc(all) * 2 * box_rows * 4);
          }
          __syncwarp();
          if (there) {
            const int to = lane * (int)box_rows;
            copy_scales(&sh.k_scale[slot][to], a.ks + (i64)p.h * a.ks_h + (i64)page_now * a.ks_p + in_now, box_rows * 4, &sh.scales_there[slot]);
            copy_scales(&sh.v_scale[slot][to], a.vs + (i64)p.h * a.vs_h + (i64)page_now * a.vs_p + in_now, box_rows * 4, &sh.scales_there[slot]);
          }
#pragma unroll
          for (int kv = 0; kv < 2; ++kv) {
            fine = fine && wait(&sh.kv_empty[stage], phase);
            if (!fine) break;
            if (lane == 0) bar_expect(&sh.codes_full[stage], (u32)(kTileKeys * 128));
            __syncwarp();
            if (lane < boxes) copy_box(sh.kv[stage] + lane * (int)box_rows * 128, kv ? &values : &keys, 0, in_now, p.h, page_now, &sh.codes_full[stage]);
            if (++stage == S::stages) { stage = 0; phase ^= 1; }
          }
        }
        part_done(no);
      }
      // No copy is left in flight, even where the warps that wait for it have given up: each stage's last one.
      for (int i = 0; i < S::stages; ++i) drain(&sh.codes_full[i], i < stage ? phase ^ 1 : phase);
      for (u32 i = 0; i < kScaleSlots; ++i) drain(&sh.scales_there[i], i < tile_no % kScaleSlots ? (tile_no / kScaleSlots) & 1 : ((tile_no / kScaleSlots) & 1) ^ 1);
    } else if (warp == 10) {
      // ---------------------------------------------------------------- the scales
      // A lane has keys lane, lane + 32 ... of a tile.  Keys outside the unit's have scale 0, whatever is there.
      u32 tile_no = 0;
      bool fine = true;
      PartInfo p;
      for (u32 no = 0; fine && take_part(no, p); ++no) {
        for (int at = 0; at < p.tiles && fine; ++at, ++tile_no) {
          const u32 slot = tile_no % kScaleSlots;
          fine = wait(&sh.scales_there[slot], (tile_no / kScaleSlots) & 1);
          if (!fine) break;
          const u32 all = sh.scales_boxes[slot];
          float most = -INFINITY, least = INFINITY;
#pragma unroll
          for (int j = 0; j < kTileKeys / 32; ++j) {
            const int at_key = j * 32 + lane, key = (p.tile + at) * kTileKeys + at_key;
            float v = sh.v_scale[slot][at_key];
            if (!(all >> ((u32)at_key / box_rows) & 1)) {             // outside the cache: zeros
              v = 0.0f;
              sh.k_scale[slot][at_key] = 0.0f;
            }
            if (key < p.lo || key >= p.hi) v = 0.0f;
            if (!isfinite(v)) {
              sh.k_scale[slot][at_key] = __int_as_float(0x7fffffff);
              v = 0.0f;
            }
            const float e = scale_log2(v);
            sh.v_scale[slot][at_key] = v;
            sh.v_log2[slot][at_key] = e;
            most = fmaxf(most, e);
            least = fminf(least, e);
          }
#pragma unroll
          for (int d = 16; d; d >>= 1) {
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
            least = fminf(least, __shfl_xor_sync(0xffffffffu, least, d));
          }
          if (lane == 0) sh.v_range[slot] = make_float2(most, least);
          fence_async();                                              // the next copy to this slot comes after these accesses
          __syncwarp();
          if (lane == 0) bar_arrive(&sh.scales_full[slot]);
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
}

// Rows come 128 bytes apart, the last of them zeros where a head is shorter.
bool codes_map(CUtensorMap *map, const CodedAttn &a, const void *base, i64 st, i64 sh, i64 sp, int dim, u32 box_rows) {
  const cuuint64_t dims[4] = {(cuuint64_t)dim, a.page, a.hkv, a.n_pages};
  const cuuint64_t strides[3] = {(cuuint64_t)st, (cuuint64_t)sh, (cuuint64_t)sp};
  const cuuint32_t box[4] = {128, box_rows, 1, 1}, step[4] = {1, 1, 1, 1};
  return encoder()(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void *>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                   CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// What copy_scales wants of a tensor of scales.
bool scales_in_line(const float *base, i64 st, i64 sh, i64 sp) { return st == 1 && sh % 4 == 0 && sp % 4 == 0 && ((uintptr_t)base & 15) == 0; }

struct CodedMaps {
  CUtensorMap k, v;
  u32 box_rows;
};

template <typename T, Format F, int D, Scores SCORES>
cudaError_t launch_coded_chunk(const CodedAttn &a, const CodedMaps &m, u32 sms, cudaStream_t s) {
  static bool ready[64] = {};
  constexpr size_t bytes = sizeof(CodedChunkShared<D>) + 1024;
  static_assert(bytes <= 227 * 1024, "shared memory of one block");
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 64) return cudaErrorInvalidDevice;
  if (!ready[dev]) {
    e = cudaFuncSetAttribute(coded_chunk_kernel<T, F, D, SCORES>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e != cudaSuccess) return e;
    // the warps' register shares come out of what the block is launched with: with fewer they would wait for ever
    cudaFuncAttributes f;
    e = cudaFuncGetAttributes(&f, coded_chunk_kernel<T, F, D, SCORES>);
    if (e != cudaSuccess) return e;
    if (f.numRegs * kCodedThreads < kCodedSoftmaxRegs * 256 + (kCodedOtherRegs + kDecodeRegs) * 128) return cudaErrorInvalidKernelImage;
    ready[dev] = true;
  }
  return launch_kernel<Attn>(coded_chunk_kernel<T, F, D, SCORES>, sms, kCodedThreads, bytes, s, a, m.k, m.v, m.box_rows);
}

template <typename T, Format F, int D>
cudaError_t pick_coded_scores(const CodedAttn &a, const CodedMaps &m, u32 sms, cudaStream_t s) {
  if (a.softcap > 64.0f) return launch_coded_chunk<T, F, D, kLargeCap>(a, m, sms, s);
  return a.softcap > 0.0f || a.slopes ? launch_coded_chunk<T, F, D, kSmallCap>(a, m, sms, s)
                                      : launch_coded_chunk<T, F, D, kPlain>(a, m, sms, s);
}

template <typename T, Format F>
cudaError_t pick_coded_chunk_dim(const CodedAttn &a, const CodedMaps &m, int dim, u32 sms, cudaStream_t s) {
  if (dim == 64) return pick_coded_scores<T, F, 64>(a, m, sms, s);
  if (dim == 96) return pick_coded_scores<T, F, 96>(a, m, sms, s);
  return pick_coded_scores<T, F, 128>(a, m, sms, s);
}

// False where no tensor map of the pages can be made, or where scales do not follow each other along a page: nothing ran.
template <Format F>
bool launch_coded_chunk_of(const CodedAttn &a, int dtype, int dim, u32 sms, cudaStream_t s, cudaError_t *e) {
  if (!encoder() || a.n_pages == 0 || !scales_in_line(a.ks, a.ks_t, a.ks_h, a.ks_p) || !scales_in_line(a.vs, a.vs_t, a.vs_h, a.vs_p)) return false;
  CodedMaps m;
  m.box_rows = a.page & (0u - a.page);                 // the largest power of two in the page size, so that a box stays in its page
  if (m.box_rows > (u32)kTileKeys) m.box_rows = kTileKeys;
  if (!codes_map(&m.k, a, a.kp, a.k_t, a.k_h, a.k_p, dim, m.box_rows) || !codes_map(&m.v, a, a.vp, a.v_t, a.v_h, a.v_p, dim, m.box_rows)) return false;
  *e = dtype == 0 ? pick_coded_chunk_dim<__nv_bfloat16, F>(a, m, dim, sms, s) : pick_coded_chunk_dim<__half, F>(a, m, dim, sms, s);
  return true;
}

}  // namespace
}  // namespace paged
}  // namespace gorio
