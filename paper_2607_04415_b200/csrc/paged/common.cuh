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

constexpr u64 kCounterBytes = 64u << 10;   // arrival counters, one a block; zero between calls
constexpr u32 kErrorWord = (u32)(kCounterBytes / 4) - 1;   // set by a block whose waits ran out

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
  u32 wait_ticks;              // of 1024 ns: a wait inside the chunk kernel gives up when it has lasted as long
};

// Attention over keys that the requests of a group share takes three kernels.  The first, over the shared keys, sees the groups as its
// requests (Attn's tables, lengths and n_req are theirs, `starts` are the requests' rows) and leaves each row's weighted sum of
// values, its maximum and its sum of weights in 32 bits.  Where there are few units, it leaves the parts of those that are cut, and a small second
// kernel joins them, a warp a row: in the first that would be the work of one block for each unit (64 requests over 16391 shared keys, 8
// units: 67 us, where it takes 39 without).  The last, over each request's own keys, joins what is left to its own rows before it writes them.
// Each may begin while the one before still runs, and waits for its end before it reads what that has left; the last has
// its own counters and parts.
struct PrefixAttn : Attn {
  const int *group_starts;     // [n_req + 1]: the requests of each group
  const int *own_lengths;      // [n_members]
  u32 n_members, own_places;   // requests; the most keys of its own that one can have
  float *mid_o;                // [n_tok][hq][dim]
  float2 *mid_ml;              // [n_tok][hq]: maximum in units of log2, sum
  u32 leaves_parts;
  int4 *mid_at;                // [n_tok][hq]: first and last block of its unit's parts (none: whole), row in the part, rows of a part
};
struct OwnAttn : Attn {
  const int *group_starts;
  u32 n_groups;
  const float *mid_o;
  const float2 *mid_ml;
};
__device__ __forceinline__ bool leaves_parts(const Attn &) { return false; }
__device__ __forceinline__ bool leaves_parts(const PrefixAttn &a) { return a.leaves_parts != 0; }
// A row's parts are those of blocks i0..i1, of `rows` rows, and in each in row `place`.
__device__ __forceinline__ void tell_parts(const Attn &, i64, u32, u32, int, int) {}
__device__ __forceinline__ void tell_parts(const PrefixAttn &a, i64 row, u32 i0, u32 i1, int place, int rows) {
  a.mid_at[row] = make_int4((int)i0, (int)i1, place, rows);
}
constexpr u32 kOwnCounters = (u32)(kCounterBytes / 8);     // the second kernel's counters: the other half

__device__ __forceinline__ u32 *error_word(const Attn &a) { return a.arrived + kErrorWord; }
__device__ __forceinline__ u32 *error_word(const OwnAttn &a) { return a.arrived + (kErrorWord - kOwnCounters); }

// The kernel that was launched before this one with leave to overlap has ended, and what it wrote is visible.
__device__ __forceinline__ void wait_for_kernel() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void wait_for_first(const Attn &) {}
__device__ __forceinline__ void wait_for_first(const OwnAttn &) { wait_for_kernel(); }
// The next kernel of the stream may begin where this one leaves room.
__device__ __forceinline__ void let_next_begin() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void let_second_begin(const Attn &) {}
__device__ __forceinline__ void let_second_begin(const PrefixAttn &) { let_next_begin(); }

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

// First row of the g-th group's requests, cut like the rest.
__device__ __forceinline__ int group_row(const int *group_starts, const int *starts, u32 members, u32 n_tok, u32 g) {
  const int r = group_starts[g], s = starts[r < 0 ? 0 : r > (int)members ? (int)members : r];
  return s < 0 ? 0 : s > (int)n_tok ? (int)n_tok : s;
}

__device__ __forceinline__ Request request_at(const PrefixAttn &a, u32 g) {
  Request x;
  const i64 cap = (i64)a.width * a.page;
  const int l = a.lengths[g];
  x.len = l < 0 ? 0 : (i64)l > cap ? (int)cap : l;
  x.q0 = group_row(a.group_starts, a.starts, a.n_members, a.n_tok, g);
  const int e = group_row(a.group_starts, a.starts, a.n_members, a.n_tok, g + 1);
  x.n = e > x.q0 ? e - x.q0 : 0;
  return x;
}

// The rows that belong to a group: the others have no shared keys, and the first kernel leaves nothing for them.
struct NoRows {};
struct CoveredRows {
  int from, to;
};
__device__ __forceinline__ NoRows covered_rows(const Attn &) { return NoRows{}; }
__device__ __forceinline__ CoveredRows covered_rows(const OwnAttn &a) {
  return CoveredRows{group_row(a.group_starts, a.starts, a.n_req, a.n_tok, 0), group_row(a.group_starts, a.starts, a.n_req, a.n_tok, a.n_groups)};
}

// Where the tok-th new token of a request stands on its key axis.
__device__ __forceinline__ int position_of(const Attn &, const Request &x, int tok) { return x.len - x.n + tok; }
// Of a group, whose tokens are of several requests: behind all shared keys and those that its own request holds before it.  Only
// windows and biases ask for it, so that a search for the request is made for those calls alone.
__device__ __forceinline__ int position_of(const PrefixAttn &a, const Request &x, int tok) {
  if (!a.window && !a.slopes) return x.len;
  const int row = x.q0 + tok;
  u32 lo = 0, hi = a.n_members;                          // the last request that starts at or before the row
  while (hi - lo > 1) {
    const u32 mid = (lo + hi) / 2;
    if (a.starts[mid] <= row) lo = mid; else hi = mid;
  }
  const int s0 = a.starts[lo], s1 = a.starts[lo + 1], own = a.own_lengths[lo];
  const int n = (s1 > (int)a.n_tok ? (int)a.n_tok : s1) - (s0 < 0 ? 0 : s0);
  return x.len + (own < 0 ? 0 : (u32)own > a.own_places ? (int)a.own_places : own) - n + (row - (s0 < 0 ? 0 : s0));
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

// The plan.  All tiles of a call, in the order (request, key head, unit, tile), are one line that the blocks take equal
// shares of.  Every block finds its own from the lengths alone, so no host step and no extra launch stands between the
// lengths and the work.  A unit that is cut by a block boundary is computed in parts, which the last of its blocks to
// finish joins in the order of the key axis: results do not depend on which block that is.
// Between units the line has places without work.  Where there are fewer units than blocks, each unit is filled up to
// whole shares: then no block has pieces of two units, whose starts and ends would come one after the other.  A share
// then holds at least a multiple of the square root of the longest unit's tiles, which balances the time for a share's tiles
// against the time to join a unit's parts.  Otherwise a unit's tiles are followed by OVER places, for what a unit costs
// besides its tiles (a block with many short units got as many tiles as one with a single long unit, and took twice as
// long).
struct Cursor {
  u32 r, h;
  int m;           // unit of (r, h)
  int at;          // next place of the unit, counted from its first tile
  Request req;
  Span span;
};

struct PlanShared {
  u64 warp_tiles[32];
  u32 warp_sum[32], warp_longest[32];
  u32 found_r, found_before;
};

// Shares of places: block i's begins at each * i + min(i, more).
struct Shares {
  u32 each, more;
  __device__ __forceinline__ u32 begin(u32 i) const { return each * i + min(i, more); }
  __device__ __forceinline__ u32 owner(u32 x) const {              // the block that owns place x
    const u32 first = more * (each + 1);
    return x < first ? x / (each + 1) : more + (x - first) / each;
  }
};

// Places of a unit; fill > 0: whole shares of that many.
template <int OVER>
__device__ __forceinline__ u32 unit_places(u32 tiles, u32 fill) { return fill ? (tiles + fill - 1) / fill * fill : tiles + OVER; }

// Places of request r over all its units (of one key head), its units and the most tiles of one.  Warp-collective; lane's own
// request is r (in range where `have`); requests of many units are summed by the whole warp.  Sums are cut near 2^31,
// where the plan gives up.
struct Places {
  u32 sum, units, longest;
};
template <int ROWS, int TK, int OVER, typename A>
__device__ __forceinline__ Places request_places(const A &a, u32 r, bool have, u32 fill) {
  const u32 lane = threadIdx.x & 31;
  Request q{0, 0, 0};
  if (have) q = request_at(a, r);
  Places p{0, have ? (u32)unit_count<ROWS>(a, q.n) : 0u, 0};
  if (p.units <= 4) {
    for (u32 m = 0; m < p.units; ++m) {
      const u32 t = (u32)unit_span<ROWS, TK>(a, q.len, q.n, (int)m).tiles;
      p.sum += unit_places<OVER>(t, fill);
      p.longest = max(p.longest, t);
    }
  }
  u32 big = __ballot_sync(0xffffffffu, p.units > 4);
  while (big) {
    const int src = __ffs(big) - 1;
    big &= big - 1;
    const int len = __shfl_sync(0xffffffffu, q.len, src), n = __shfl_sync(0xffffffffu, q.n, src);
    const int cnt = (int)__shfl_sync(0xffffffffu, p.units, src);
    u32 s = 0, most = 0;
    for (int m = (int)lane; m < cnt; m += 32) {
      const u32 t = (u32)unit_span<ROWS, TK>(a, len, n, m).tiles;
      s = min(s + unit_places<OVER>(t, fill), 1u << 26);
      most = max(most, t);
    }
    s = __reduce_add_sync(0xffffffffu, s);
    most = __reduce_max_sync(0xffffffffu, most);
    if ((int)lane == src) { p.sum = s; p.longest = most; }
  }
  return p;
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

// Sets the cursor to the place `offset` places after the first of request r.  Warp-collective, the same
// for all warps.
template <int ROWS, int TK, int OVER, typename A>
__device__ __forceinline__ Cursor cursor_in(const A &a, u32 r, u32 offset, u32 fill) {
  const u32 lane = threadIdx.x & 31;
  Cursor c;
  c.r = r;
  c.req = request_at(a, r);
  const int units = unit_count<ROWS>(a, c.req.n);
  u32 per_head = 0;
  for (int m = (int)lane; m < units; m += 32) per_head += unit_places<OVER>((u32)unit_span<ROWS, TK>(a, c.req.len, c.req.n, m).tiles, fill);
  per_head = __reduce_add_sync(0xffffffffu, per_head);
  c.h = offset / per_head;
  u32 o = offset - c.h * per_head;
  c.m = 0;
  c.at = 0;
  for (int base = 0; base < units; base += 32) {
    const int m = base + (int)lane;
    const u32 t = m < units ? unit_places<OVER>((u32)unit_span<ROWS, TK>(a, c.req.len, c.req.n, m).tiles, fill) : 0u;
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
template <int ROWS, int TK, typename A>
__device__ __forceinline__ bool next_unit(const A &a, Cursor &c) {
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
template <int ROWS, int TK, int OVER, typename A>
__device__ __forceinline__ void settle(const A &a, Cursor &c, u32 &left, u32 fill) {
  while (left && c.at >= c.span.tiles) {
    const u32 skip = unit_places<OVER>((u32)c.span.tiles, fill) - (u32)c.at;
    if (skip >= left) { left = 0; return; }
    left -= skip;
    if (!next_unit<ROWS, TK>(a, c)) left = 0;
  }
}

struct Plan {
  u32 begin, end;          // this block's places; equal: no work
  u32 fill;                // see unit_places
  Shares shares;
  Cursor first;
};

// By a block of NT threads.  `spread` times the square root of the longest unit: the least share of filled-up units.
// Requests are dealt out to all warps, each a run of consecutive ones, since a warp takes those of many units one by one.
template <int ROWS, int TK, int OVER, int NT, typename A>
__device__ __forceinline__ Plan block_plan(const A &a, PlanShared &sh, float spread) {
  constexpr u32 kWarpsHere = NT / 32;
  const u32 tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const u32 run = min(32u, (a.n_req + kWarpsHere - 1) / kWarpsHere), round = run * kWarpsHere;
  const u32 mine_r = lane < run ? warp * run + lane : a.n_req;       // of the first round
  Plan p;
  p.begin = p.end = 0;
  // all tiles and units, the longest unit
  u64 tiles = 0;
  u32 units = 0, longest = 0;
  Places got{0, 0, 0};
  for (u32 base = 0; base < a.n_req; base += round) {
    const u32 r = base + mine_r;
    got = request_places<ROWS, TK, OVER>(a, r, r < a.n_req, 1);
    tiles += got.sum;
    units += got.units;
    longest = max(longest, got.longest);
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) tiles += __shfl_xor_sync(0xffffffffu, tiles, d);
  units = __reduce_add_sync(0xffffffffu, units);
  longest = __reduce_max_sync(0xffffffffu, longest);
  if (lane == 0) { sh.warp_tiles[warp] = tiles; sh.warp_sum[warp] = units; sh.warp_longest[warp] = longest; }
  if (tid == 0) sh.found_r = a.n_req;
  __syncthreads();
  tiles = 0;
  u64 all_units = 0;
#pragma unroll
  for (u32 w = 0; w < kWarpsHere; ++w) { tiles += sh.warp_tiles[w]; all_units += sh.warp_sum[w]; longest = max(longest, sh.warp_longest[w]); }
  tiles *= a.hkv;
  all_units *= a.hkv;
  const u64 line = tiles + all_units * OVER;
  if (line >= (1ull << 31)) {                            // a call of hours
    if (tid == 0) *error_word(a) = 2;
    return p;
  }
  if (tiles == 0) return p;
  const u32 grid = gridDim.x, line_each = ((u32)line + grid - 1) / grid;
  p.fill = 0;
  if ((u32)all_units < grid) {
    const u32 room = grid - (u32)all_units, each = ((u32)tiles + room - 1) / room;      // all units' whole shares fit the grid then
    if (each <= line_each + 1) p.fill = max(each, (u32)(spread * sqrtf((float)longest)));
  }
  if (p.fill) {
    p.shares.each = p.fill;
    p.shares.more = 0;
  } else {
    const u32 parts = min(grid, (u32)line);
    p.shares.each = (u32)line / parts;
    p.shares.more = (u32)line - p.shares.each * parts;
    if (blockIdx.x >= parts) return p;
  }
  const u32 begin = p.shares.begin(blockIdx.x);
  u32 before = 0;
  for (u32 base = 0; base < a.n_req && before <= begin; base += round) {
    const u32 r = base + mine_r;
    if (p.fill || a.n_req > round) got = request_places<ROWS, TK, OVER>(a, r, r < a.n_req, p.fill);
    else got.sum += got.units * OVER;                    // what the one round above has found
    const u32 mine = got.sum * a.hkv;
    u32 upto = warp_scan(mine);
    __syncthreads();                                     // warp_sum has been read
    if (lane == 31) sh.warp_sum[warp] = upto;
    __syncthreads();
    upto += before;
#pragma unroll
    for (u32 w = 0; w < kWarpsHere; ++w) {
      if (w < warp) upto += sh.warp_sum[w];
      before += sh.warp_sum[w];
    }
    if (upto - mine <= begin && begin < upto) { sh.found_r = r; sh.found_before = upto - mine; }
  }
  __syncthreads();
  if (sh.found_r >= a.n_req) return p;                   // filled-up units may leave blocks without any
  p.begin = begin;
  p.end = p.fill ? begin + p.fill : p.shares.begin(blockIdx.x + 1);
  p.first = cursor_in<ROWS, TK, OVER>(a, sh.found_r, begin - sh.found_before, p.fill);
  return p;
}

// Workspace for parts: a block leaves at most two of them, of 256 rows (or blocks on the same SM of fewer).
constexpr u32 kPartRowsPerSm = 2 * 256;
constexpr u32 kMaxDim = 128;
inline u64 part_ml_bytes(u32 sms) { return (u64)sms * kPartRowsPerSm * 2 * sizeof(float); }
inline u64 part_bytes(u32 sms) { return part_ml_bytes(sms) + (u64)sms * kPartRowsPerSm * kMaxDim * sizeof(float); }

// launchers, of each kernel for each of its places
// False where no tensor map of the pages can be made (strides or addresses that it does not hold): nothing ran.
bool launch_chunk(const Attn &a, int dtype, int dim, u32 sms, cudaStream_t s, cudaError_t *e);
cudaError_t launch_rows(const Attn &a, int dtype, int dim, u32 sms, cudaStream_t s);
bool launch_chunk(const PrefixAttn &a, int dtype, int dim, u32 sms, cudaStream_t s, cudaError_t *e);
cudaError_t launch_rows(const PrefixAttn &a, int dtype, int dim, u32 sms, cudaStream_t s);
bool launch_chunk(const OwnAttn &a, int dtype, int dim, u32 sms, cudaStream_t s, cudaError_t *e);
cudaError_t launch_rows(const OwnAttn &a, int dtype, int dim, u32 sms, cudaStream_t s);

// Joins the parts that the first kernel has left of cut units.
cudaError_t launch_prefix_join(const PrefixAttn &a, int dim, u32 sms, cudaStream_t s);

// A kernel that reads what the one before leaves is launched with leave to begin before that one has ended.
struct Joining {};
template <typename A>
struct Overlaps { static constexpr bool value = false; };
template <>
struct Overlaps<OwnAttn> { static constexpr bool value = true; };
template <>
struct Overlaps<Joining> { static constexpr bool value = true; };
template <typename A, typename... Args>
cudaError_t launch_kernel(void (*kernel)(Args...), u32 blocks, u32 threads, size_t shared, cudaStream_t s, Args... args) {
  cudaLaunchAttribute overlap{};
  overlap.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  overlap.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t c{};
  c.gridDim = blocks;
  c.blockDim = threads;
  c.dynamicSmemBytes = shared;
  c.stream = s;
  c.attrs = &overlap;
  c.numAttrs = Overlaps<A>::value ? 1 : 0;
  return cudaLaunchKernelEx(&c, kernel, args...);
}

}  // namespace paged
}  // namespace gorio
