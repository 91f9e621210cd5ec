// Page tables and slot maps from request lengths, and the store of new keys and values.
#include "paged/common.cuh"
#include "paged/entries.h"

namespace gorio {
namespace paged {

namespace {

constexpr int kTabThreads = 1024;      // a block's threads, and the tokens that it describes

struct ScanShared {
  u64 n[32], need[32];
  u32 mark[32];
  int req[kTabThreads], served[kTabThreads];
  u32 start[kTabThreads];
  u64 fresh[kTabThreads];
};

// Request r: c cached tokens, n new ones, page size s.  need = ceil((c+n)/s) - ceil(c/s) pages, taken from
// the top of the stack of free pages in request order; the sums over the requests that this needs are
// prefix sums, which every block makes for itself over all requests (8 bytes each, out of L2 after the
// first block) because that is cheaper than a second launch or a wait between blocks.  A block then
// describes 1024 consecutive tokens: the requests that overlap them leave a mark at their first one,
// and a running maximum over the marks tells each token its request.  Each new page has exactly one
// new token at its start, whose thread writes the table entry, so tables cost no pass of their own.
// Bound by the latency of four dependent steps (lengths, sums, table entry, stores) for the sizes of a
// decode step; by the 16 bytes written a token for the largest.
__global__ void __launch_bounds__(kTabThreads) page_tables_kernel(const gorio_page_tables_desc a) {
  __shared__ ScanShared sh;
  const u32 tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const u32 s = a.page_size;
  const i64 n_tok = a.n_tokens;
  const i64 base = (i64)blockIdx.x * kTabThreads;
  const int fc_in = *a.free_count;
  const i64 fc = fc_in < 0 ? 0 : (u32)fc_in > a.free_capacity ? (i64)a.free_capacity : (i64)fc_in;
  u64 sum_n = 0, sum_need = 0;   // over the rounds before
  u64 top = 0;                   // pages taken by the last served request's end
  u32 mark = 0;
  sh.req[tid] = -1;
  __syncthreads();
  for (u32 round = 0, r0 = 0; r0 < a.n_requests; ++round, r0 += kTabThreads) {
    const u32 r = r0 + tid;
    i64 c = 0, n = 0;
    if (r < a.n_requests) { c = a.lengths[r]; n = a.new_lens[r]; }
    const i64 brought = n < 0 ? 0 : n > n_tok ? n_tok + 1 : n;     // the sums stay small whatever comes in
    const bool ok = c >= 0 && n >= 0 && c + n <= (i64)a.table_width * s;      // width * s < 2^31
    const u64 need = ok ? (u64)((u32)(c + n + s - 1) / s - (u32)(c + s - 1) / s) : 0;
    u64 x = (u64)brought, y = need;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const u64 xs = __shfl_up_sync(0xffffffffu, x, d), ys = __shfl_up_sync(0xffffffffu, y, d);
      if ((int)lane >= d) { x += xs; y += ys; }
    }
    if (lane == 31) { sh.n[warp] = x; sh.need[warp] = y; }
    __syncthreads();
    u64 wn = sh.n[lane], wy = sh.need[lane];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const u64 xs = __shfl_up_sync(0xffffffffu, wn, d), ys = __shfl_up_sync(0xffffffffu, wy, d);
      if ((int)lane >= d) { wn += xs; wy += ys; }
    }
    const u64 all_n = __shfl_sync(0xffffffffu, wn, 31), all_need = __shfl_sync(0xffffffffu, wy, 31);
    const u64 pn = __shfl_sync(0xffffffffu, wn, warp ? warp - 1 : 0), py = __shfl_sync(0xffffffffu, wy, warp ? warp - 1 : 0);
    x += sum_n + (warp ? pn : 0);          // tokens of requests 0..r
    y += sum_need + (warp ? py : 0);       // pages of requests 0..r
    sum_n += all_n;
    sum_need += all_need;
    const bool served = ok && y <= (u64)fc && x <= (u64)n_tok && r < a.n_requests;
    const u64 start = x - (u64)brought;
    if (served) top = y;
    if (r < a.n_requests) {
      if (round % gridDim.x == blockIdx.x) {
        if (r == 0) a.starts[0] = 0;
        a.starts[r + 1] = (int)(x > (u64)n_tok ? (u64)n_tok : x);
        a.out_lengths[r] = (int)(served ? c + n : c);
        a.out_served[r] = served ? 1 : 0;
      }
      if (brought > 0 && (i64)start < base + kTabThreads && (i64)x > base) {
        const u32 at = (i64)start > base ? (u32)((i64)start - base) : 0u;
        sh.req[at] = (int)r;
        sh.served[at] = served;
        sh.start[at] = (u32)start;
        sh.fresh[at] = y - need;
      }
    }
    __syncthreads();
  }
  if (blockIdx.x == 0) {
    // pages taken in all: the served requests' last sum
#pragma unroll
    for (int d = 16; d; d >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
    if (lane == 0) sh.need[warp] = top;
    __syncthreads();
    if (warp == 0) {
      u64 t = sh.need[lane];
#pragma unroll
      for (int d = 16; d; d >>= 1) t = max(t, __shfl_xor_sync(0xffffffffu, t, d));
      if (lane == 0) {
        *a.out_free_count = (int)(fc - (i64)t);
        if (a.n_requests == 0) a.starts[0] = 0;
      }
    }
  }
  // the last mark at or before each token
  mark = sh.req[tid] >= 0 ? tid + 1 : 0;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const u32 y = __shfl_up_sync(0xffffffffu, mark, d);
    if ((int)lane >= d) mark = max(mark, y);
  }
  if (lane == 31) sh.mark[warp] = mark;
  __syncthreads();
  {
    u32 w = lane < warp ? sh.mark[lane] : 0;
    w = __reduce_max_sync(0xffffffffu, w);
    mark = max(mark, w);
  }
  const i64 t = base + tid;
  if (t >= n_tok) return;
  i64 slot = -1;
  int pos = -1, req = -1;
  if (mark && (u64)t < sum_n) {
    const u32 at = mark - 1;
    req = sh.req[at];
    const int c = a.lengths[req];
    pos = c + (int)((u32)t - sh.start[at]);
    if (sh.served[at]) {
      const u32 page_at = (u32)pos / s, in_page = (u32)pos - page_at * s, held = (u32)(((u64)(u32)c + s - 1) / s);
      int page;
      if (page_at < held) {
        page = a.tables[(i64)req * a.table_stride + page_at];
      } else {
        page = a.free_pages[fc - 1 - (i64)(sh.fresh[at] + (page_at - held))];
        if (in_page == 0) a.tables[(i64)req * a.table_stride + page_at] = page;
      }
      slot = (i64)page * s + in_page;
    }
  }
  a.slots[t] = slot;
  a.positions[t] = pos;
  a.requests[t] = req;
}

// 16 bytes a thread and step: chunk (token, key or value, head, piece of a head) -> its slot.  A copy: each
// byte is read once and written once.
struct StoreArgs {
  gorio_cache_store_desc d;
  u32 pieces;        // 16-byte pieces of a head
  u32 per_token;     // heads * pieces
  u64 chunks;        // n_tokens * 2 * per_token
};

constexpr int kStoreThreads = 256;
constexpr int kStoreEach = 4;          // chunks in flight a thread

__global__ void __launch_bounds__(kStoreThreads) cache_store_kernel(const StoreArgs a) {
  const u64 first = (u64)blockIdx.x * (kStoreThreads * kStoreEach) + threadIdx.x;
  uint4 v[kStoreEach];
  uint4 *to[kStoreEach];
#pragma unroll
  for (int i = 0; i < kStoreEach; ++i) {
    const u64 x = first + (u64)i * kStoreThreads;
    to[i] = nullptr;
    if (x >= a.chunks) continue;
    const u32 row = (u32)(x / a.per_token), c = (u32)(x - (u64)row * a.per_token);
    const u32 t = row >> 1, h = c / a.pieces, piece = c - h * a.pieces;
    const i64 slot = a.d.slots[t];
    if (slot < 0 || slot >= (i64)a.d.n_pages * a.d.page_size) continue;
    const u32 page = (u32)slot / a.d.page_size, in_page = (u32)slot - page * a.d.page_size;
    const u16 *src, *dst;
    if (row & 1) {
      src = (const u16 *)a.d.values + (i64)t * a.d.v_token_stride + (i64)h * a.d.v_head_stride;
      dst = (const u16 *)a.d.value_pages + (i64)page * a.d.vp_page_stride + (i64)h * a.d.vp_head_stride + (i64)in_page * a.d.vp_token_stride;
    } else {
      src = (const u16 *)a.d.keys + (i64)t * a.d.k_token_stride + (i64)h * a.d.k_head_stride;
      dst = (const u16 *)a.d.key_pages + (i64)page * a.d.kp_page_stride + (i64)h * a.d.kp_head_stride + (i64)in_page * a.d.kp_token_stride;
    }
    v[i] = __ldcs((const uint4 *)(src + piece * 8));
    to[i] = (uint4 *)(dst + piece * 8);
  }
#pragma unroll
  for (int i = 0; i < kStoreEach; ++i)
    if (to[i]) *to[i] = v[i];
}

}  // namespace

cudaError_t launch_page_tables(const gorio_page_tables_desc &d, cudaStream_t s) {
  const u32 blocks = d.n_tokens > 0 ? (d.n_tokens + kTabThreads - 1) / kTabThreads : 1;
  page_tables_kernel<<<blocks, kTabThreads, 0, s>>>(d);
  return cudaGetLastError();
}

cudaError_t launch_cache_store(const gorio_cache_store_desc &d, cudaStream_t s) {
  StoreArgs a{d, d.dim / 8, d.n_heads * (d.dim / 8), 0};
  a.chunks = (u64)d.n_tokens * 2 * a.per_token;
  const u64 per_block = kStoreThreads * kStoreEach;
  cache_store_kernel<<<(u32)((a.chunks + per_block - 1) / per_block), kStoreThreads, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace paged
}  // namespace gorio
