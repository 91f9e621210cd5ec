// What the kernels of the paged key/value cache share: the arguments of an attention call, the
// geometry of its units of work, and the plan that gives every block an equal share of them.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace gorio {
namespace paged {

typedef uint8_t u8;
typedef uint16_t u16;
typedef uint32_t u32;
typedef uint64_t u64;
typedef int64_t i64;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Everything an attention kernel needs, passed by value.  Strides are in elements.
struct Attn {
  const void *q, *kp, *vp;
  void *out;
  float *lse;                  // [n_tokens][hq] or NULL
  const int *tables, *lengths, *starts;
  const float *slopes;         // [hq] or NULL
  i64 q_t, q_h, o_t, o_h, k_p, k_h, k_t, v_p, v_h, v_t, tab_r;
  u32 n_req, n_tok, hq, hkv, group, page, n_pages, width;
  u32 causal, window;          // window 0: none
  float scale;                 // of the dot product
  float softcap;               // 0: none
  // workspace: two partial results for every block, and a counter of arrivals for each
  float *part_o, *part_ml;
  u32 *arrived;
};

// One request as the kernels see it: keys it can have at most, its new tokens and where their rows
// start.  Bad lengths or starts are cut to what the tables and the query tensor hold, so that no
// access leaves them.
struct Request {
  int len, n, q0;
};

__device__ __forceinline__ Request request_at(const Attn &a, u32 r) {
  Request x;
  const i64 cap = (i64)a.width * a.page;
  const int l = a.lengths[r], s0 = a.starts[r], s1 = a.starts[r + 1];
  x.len = l < 0 ? 0 : (i64)l > cap ? (int)cap : l;
  x.q0 = s0 < 0 ? 0 : s0 > (int)a.n_tok ? (int)a.n_tok : s0;
  const int e = s1 > (int)a.n_tok ? (int)a.n_tok : s1;
  x.n = e > x.q0 ? e - x.q0 : 0;
  return x;
}

// A unit is up to ROWS rows -- (token, query head of the group) pairs, token outer -- of one request
// and one key head.  Its visible keys are [lo, hi) over all its rows, in whole tiles of TK keys from
// tile `first`; a unit without visible keys still has one (fully masked) tile, which writes its rows.
struct Span {
  int lo, hi, first, tiles;
};

template <int ROWS, int TK>
__device__ __forceinline__ Span unit_span(const Attn &a, int len, int n, int m) {
  const u32 r0 = (u32)m * ROWS, r1 = min((u32)n * a.group, r0 + ROWS);      // n * group < 2^31
  const int ta = (int)(r0 / a.group), tb = (int)((r1 - 1) / a.group);
  Span s;
  s.hi = a.causal ? min(len, len - n + tb + 1) : len;
  s.lo = a.window ? (int)max((i64)0, (i64)len - n + ta - a.window + 1) : 0;
  if (s.hi <= s.lo) { s.lo = s.hi = 0; s.first = 0; s.tiles = 1; return s; }
  s.first = s.lo / TK;
  s.tiles = (s.hi + TK - 1) / TK - s.first;
  return s;
}

template <int ROWS>
__device__ __forceinline__ int unit_count(const Attn &a, int n) {
  return (int)(((u32)n * a.group + ROWS - 1) / ROWS);
}

// The plan.  All tiles of a call, in the order (request, key head, unit, tile), are one line; a unit's tiles are followed
// by OVER places without work, for what a unit costs besides its tiles (a block with many short units got as many
// tiles as one with a single long unit, and took twice as long).  Block i of N takes places [total*i/N,
// total*(i+1)/N).  Every block finds its own from the lengths alone, so no host step and no extra launch stands
// between the lengths and the work.  A unit that is cut by a block boundary is computed in parts, which the last of
// its blocks to finish joins in the order of the key axis: results do not depend on which block that is.
struct Cursor {
  u32 r, h;
  int m;           // unit of (r, h)
  int at;          // next place of the unit, counted from its first tile
  Request req;
  Span span;
};

struct PlanShared {
  u32 warp_sum[32];
  u32 found_r, found_before;
};

// Block i's share of `total` places begins here: the first total % n blocks have one place more than the others.
__device__ __forceinline__ u32 part_begin(u32 total, u32 i, u32 n) {
  const u32 each = total / n, more = total - each * n;
  return each * i + min(i, more);
}
// the block that owns place x
__device__ __forceinline__ u32 part_owner(u32 total, u32 x, u32 n) {
  const u32 each = total / n, more = total - each * n, first = more * (each + 1);
  return x < first ? x / (each + 1) : more + (x - first) / each;
}

// Places of request r over all its units (of one key head).  Warp-collective; lane's own request is r
// (in range where `have`); requests of many units are summed by the whole warp.
template <int ROWS, int TK, int OVER>
__device__ __forceinline__ u32 request_places(const Attn &a, u32 r, bool have) {
  const u32 lane = threadIdx.x & 31;
  Request q{0, 0, 0};
  if (have) q = request_at(a, r);
  const int units = have ? unit_count<ROWS>(a, q.n) : 0;
  u32 sum = 0;
  if (units <= 2) {
    for (int m = 0; m < units; ++m) sum += (u32)unit_span<ROWS, TK>(a, q.len, q.n, m).tiles + OVER;
  }
  u32 big = __ballot_sync(0xffffffffu, units > 2);
  while (big) {
    const int src = __ffs(big) - 1;
    big &= big - 1;
    const int len = __shfl_sync(0xffffffffu, q.len, src), n = __shfl_sync(0xffffffffu, q.n, src);
    const int cnt = __shfl_sync(0xffffffffu, units, src);
    u32 s = 0;
    for (int m = (int)lane; m < cnt; m += 32) s += (u32)unit_span<ROWS, TK>(a, len, n, m).tiles + OVER;
    s = __reduce_add_sync(0xffffffffu, s);
    if ((int)lane == src) sum = s;
  }
  return sum;
}

__device__ __forceinline__ u32 warp_scan(u32 x) {
  const u32 lane = threadIdx.x & 31;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const u32 y = __shfl_up_sync(0xffffffffu, x, d);
    if ((int)lane >= d) x += y;
  }
  return x;
}

// Inclusive sum over the block of one value a thread; `all` is the block's sum.  Two barriers.
template <int NT>
__device__ __forceinline__ u32 block_scan(u32 v, PlanShared &sh, u32 &all) {
  const u32 lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const u32 x = warp_scan(v);
  if (lane == 31) sh.warp_sum[warp] = x;
  __syncthreads();
  u32 before = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < NT / 32; ++w) {
    const u32 s = sh.warp_sum[w];
    if (w < (int)warp) before += s;
    all += s;
  }
  __syncthreads();
  return x + before;
}

// Sets the cursor to the place `offset` places after the first of request r.  Warp-collective, the same
// for all warps.
template <int ROWS, int TK, int OVER>
__device__ __forceinline__ Cursor cursor_in(const Attn &a, u32 r, u32 offset) {
  const u32 lane = threadIdx.x & 31;
  Cursor c;
  c.r = r;
  c.req = request_at(a, r);
  const int units = unit_count<ROWS>(a, c.req.n);
  u32 per_head = 0;
  for (int m = (int)lane; m < units; m += 32) per_head += (u32)unit_span<ROWS, TK>(a, c.req.len, c.req.n, m).tiles + OVER;
  per_head = __reduce_add_sync(0xffffffffu, per_head);
  c.h = offset / per_head;
  u32 o = offset - c.h * per_head;
  c.m = 0;
  c.at = 0;
  for (int base = 0; base < units; base += 32) {
    const int m = base + (int)lane;
    const u32 t = m < units ? (u32)unit_span<ROWS, TK>(a, c.req.len, c.req.n, m).tiles + OVER : 0u;
    const u32 x = warp_scan(t);
    const u32 hit = __ballot_sync(0xffffffffu, o < x);
    if (hit) {
      const int src = __ffs(hit) - 1;
      c.m = base + src;
      c.at = (int)(o - (__shfl_sync(0xffffffffu, x, src) - __shfl_sync(0xffffffffu, t, src)));
      break;
    }
    o -= __shfl_sync(0xffffffffu, x, 31);
  }
  c.span = unit_span<ROWS, TK>(a, c.req.len, c.req.n, c.m);
  return c;
}

// The next unit after the cursor's; false at the end of the line.
template <int ROWS, int TK>
__device__ __forceinline__ bool next_unit(const Attn &a, Cursor &c) {
  c.at = 0;
  if (c.m + 1 < unit_count<ROWS>(a, c.req.n)) {
    ++c.m;
  } else if (c.h + 1 < a.hkv) {
    ++c.h;
    c.m = 0;
  } else {
    do {
      if (++c.r >= a.n_req) return false;
      c.req = request_at(a, c.r);
    } while (c.req.n == 0);
    c.h = 0;
    c.m = 0;
  }
  c.span = unit_span<ROWS, TK>(a, c.req.len, c.req.n, c.m);
  return true;
}

// Moves the cursor from a place without work, or past the unit's last tile, to the next tile; `left`: places of the block's
// share from the cursor on, 0 at its end.
template <int ROWS, int TK, int OVER>
__device__ __forceinline__ void settle(const Attn &a, Cursor &c, u32 &left) {
  while (left && c.at >= c.span.tiles) {
    const u32 skip = (u32)(c.span.tiles + OVER - c.at);
    if (skip >= left) { left = 0; return; }
    left -= skip;
    if (!next_unit<ROWS, TK>(a, c)) left = 0;
  }
}

struct Plan {
  u32 total, begin, end;   // places; [begin, end) is this block's
  u32 parts;               // blocks that take part
  Cursor first;
};

__device__ __forceinline__ bool share(Plan &p, u32 total, u32 least) {
  p.total = total;
  p.parts = max(1u, min(gridDim.x, (total + least - 1) / least));
  p.begin = p.end = 0;
  if (blockIdx.x >= p.parts || total == 0) return false;
  p.begin = part_begin(total, blockIdx.x, p.parts);
  p.end = part_begin(total, blockIdx.x + 1, p.parts);
  return p.begin < p.end;
}

// By a block of NT threads; at least `least` places a block, where there are as many.  (One warp alone, without the
// barriers, took longer even for one request.)
template <int ROWS, int TK, int OVER, int NT>
__device__ __forceinline__ Plan block_plan(const Attn &a, PlanShared &sh, u32 least) {
  const u32 tid = threadIdx.x;
  u32 all = 0;
  for (u32 base = 0; base < a.n_req; base += NT) {
    u32 sum;
    block_scan<NT>(request_places<ROWS, TK, OVER>(a, base + tid, base + tid < a.n_req) * a.hkv, sh, sum);
    all += sum;
  }
  Plan p;
  if (!share(p, all, least)) return p;
  u32 before = 0;
  for (u32 base = 0; before <= p.begin; base += NT) {
    u32 sum;
    const u32 r = base + tid, mine = request_places<ROWS, TK, OVER>(a, r, r < a.n_req) * a.hkv;
    const u32 upto = before + block_scan<NT>(mine, sh, sum);
    if (upto - mine <= p.begin && p.begin < upto) { sh.found_r = r; sh.found_before = upto - mine; }
    before += sum;
  }
  __syncthreads();
  p.first = cursor_in<ROWS, TK, OVER>(a, sh.found_r, p.begin - sh.found_before);
  return p;
}

// Workspace for parts: a block leaves at most two of them, of 256 rows (or blocks on the same SM of fewer).
constexpr u32 kPartRowsPerSm = 2 * 256;
constexpr u32 kMaxDim = 128;
inline u64 part_ml_bytes(u32 sms) { return (u64)sms * kPartRowsPerSm * 2 * sizeof(float); }
inline u64 part_bytes(u32 sms) { return part_ml_bytes(sms) + (u64)sms * kPartRowsPerSm * kMaxDim * sizeof(float); }

constexpr u64 kCounterBytes = 64u << 10;   // arrival counters, one a block; zero between calls
constexpr u32 kErrorWord = (u32)(kCounterBytes / 4) - 1;   // set by a block whose waits ran out

// launchers
// False where no tensor map of the pages can be made (strides or addresses that it does not hold): nothing ran.
bool launch_chunk(const Attn &a, int dtype, int dim, u32 sms, cudaStream_t s, cudaError_t *e);
cudaError_t launch_rows(const Attn &a, int dtype, int dim, u32 sms, cudaStream_t s);

}  // namespace paged
}  // namespace gorio
