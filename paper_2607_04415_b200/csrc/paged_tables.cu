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

__device__ __forceinline__ u64 scan_warp(u64 x) {
  const u32 lane = threadIdx.x & 31;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const u64 y = __shfl_up_sync(0xffffffffu, x, d);
    if ((int)lane >= d) x += y;
  }
  return x;
}

// Division of x < 2^31 by a page size d: x * ceil(2^(31+l) / d) >> (31+l) with 2^l >= d (Granlund and Montgomery).  All
// blocks divide for all requests; with the general division that took most of the time of a large call.
struct Divider {
  u32 mul, shift;
  __device__ __forceinline__ u32 operator()(u32 x) const { return (u32)(((u64)x * mul) >> shift); }
  __device__ __forceinline__ u32 up(u32 x) const { return x ? (*this)(x - 1) + 1 : 0u; }
};

// EACH consecutive numbers, zeros past the end
template <int EACH>
__device__ __forceinline__ void load_some(int (&v)[EACH], const int *p, u32 r, u32 end) {
  if (EACH % 4 == 0 && ((uintptr_t)p & 15) == 0 && r + EACH <= end) {
#pragma unroll
    for (int k = 0; k < EACH / 4; ++k) *(int4 *)(v + 4 * k) = *(const int4 *)(p + r + 4 * k);
  } else {
#pragma unroll
    for (int k = 0; k < EACH; ++k) v[k] = r + k < end ? p[r + k] : 0;
  }
}

// Request r: c cached tokens, n new ones, page size s.  need = ceil((c+n)/s) - ceil(c/s) pages, taken from
// the top of the stack of free pages in request order; the sums over the requests that this needs are
// prefix sums, which every block makes for itself over all requests (8 bytes each, out of L2 after the
// first block) because that is cheaper than a second launch or a wait between blocks.  A block then
// describes 1024 consecutive tokens: the requests that overlap them leave a mark at their first one,
// and a running maximum over the marks tells each token its request.  Each new page has exactly one
// new token at its start, whose thread writes the table entry, so tables cost no pass of their own.
// Bound by the latency of four dependent steps (lengths, sums, table entry, stores) for the sizes of a
// decode step.  EACH consecutive requests a thread and round: 1 where one round of a block holds all, as a
// thread's divisions then take least; 8 beyond, where rounds count.
// 32 requests of one new token take 4.3 us, 1000 mixed ones 5.0 us, 8192 requests of 266 thousand tokens (4.7 MB) 12 us
// (32 us with one request a thread).
template <int EACH>
__global__ void __launch_bounds__(kTabThreads) page_tables_kernel(const gorio_page_tables_desc a, const Divider pages_in) {
  __shared__ ScanShared sh;
  const u32 tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const u32 s = a.page_size;
  const i64 n_tok = a.n_tokens;
  const i64 base = (i64)blockIdx.x * kTabThreads;
  const int fc_in = *a.free_count;
  const i64 fc = fc_in < 0 ? 0 : (u32)fc_in > a.free_capacity ? (i64)a.free_capacity : (i64)fc_in;
  u64 sum_n = 0, sum_need = 0;   // over the rounds before
  u64 top = 0;                   // pages taken by the last served request's end
  sh.req[tid] = -1;
  for (u32 round = 0, r0 = 0; r0 < a.n_requests; ++round, r0 += kTabThreads * EACH) {
    __align__(16) int c[EACH];
    __align__(16) int n[EACH];
    u32 need[EACH];
    load_some(c, a.lengths, r0 + tid * EACH, a.n_requests);
    load_some(n, a.new_lens, r0 + tid * EACH, a.n_requests);
    auto brought = [&](int k) { return n[k] < 0 ? 0u : min((u32)n[k], a.n_tokens + 1); };      // the sums stay small whatever comes in
    auto fits = [&](int k) { return c[k] >= 0 && n[k] >= 0 && (u32)c[k] + (u32)n[k] <= a.table_width * s; };   // width * s < 2^31
    u64 x = 0, y = 0;
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      need[k] = fits(k) ? pages_in.up((u32)c[k] + (u32)n[k]) - pages_in.up((u32)c[k]) : 0u;
      x += brought(k);
      y += need[k];
    }
    const u64 xw = scan_warp(x), yw = scan_warp(y);
    if (lane == 31) { sh.n[warp] = xw; sh.need[warp] = yw; }
    __syncthreads();                                   // also after the marks were cleared
    const u64 wn = scan_warp(sh.n[lane]), wy = scan_warp(sh.need[lane]);
    const u64 pn = __shfl_sync(0xffffffffu, wn, warp ? warp - 1 : 0), py = __shfl_sync(0xffffffffu, wy, warp ? warp - 1 : 0);
    u64 upto_n = sum_n + (warp ? pn : 0) + xw - x;     // tokens and pages of the requests before this thread's
    u64 upto_need = sum_need + (warp ? py : 0) + yw - y;
    sum_n += __shfl_sync(0xffffffffu, wn, 31);
    sum_need += __shfl_sync(0xffffffffu, wy, 31);
    // Most blocks have nothing to do with most requests: a block looks closer at those that overlap its tokens and those whose
    // outputs it writes (warps' requests go round the blocks); block 0 at all, for the count of pages.
    const bool writes = (round * (kTabThreads / 32) + warp) % gridDim.x == blockIdx.x;
    const bool overlaps = (i64)upto_n < base + kTabThreads && (i64)(upto_n + x) > base;
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      const u32 r = r0 + tid * EACH + k;
      if (r >= a.n_requests || !(writes || overlaps || blockIdx.x == 0)) break;
      const u64 start = upto_n, first = upto_need;
      upto_n += brought(k);
      upto_need += need[k];
      const bool served = fits(k) && upto_need <= (u64)fc && upto_n <= (u64)n_tok;
      if (served) top = upto_need;
      if (writes) {
        if (r == 0) a.starts[0] = 0;
        a.starts[r + 1] = (int)(upto_n > (u64)n_tok ? (u64)n_tok : upto_n);
        a.out_lengths[r] = served ? c[k] + n[k] : c[k];
        a.out_served[r] = served ? 1 : 0;
      }
      if (upto_n > start && (i64)start < base + kTabThreads && (i64)upto_n > base) {
        const u32 at = (i64)start > base ? (u32)((i64)start - base) : 0u;
        sh.req[at] = (int)r;
        sh.served[at] = served;
        sh.start[at] = (u32)start;
        sh.fresh[at] = first;
      }
    }
    __syncthreads();
  }
  if (blockIdx.x == 0) {
    // pages taken in all: the served requests' last sum
#pragma unroll
    for (int d = 16; d; d >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
    __syncthreads();
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
  u32 mark = sh.req[tid] >= 0 ? tid + 1 : 0;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const u32 y = __shfl_up_sync(0xffffffffu, mark, d);
    if ((int)lane >= d) mark = max(mark, y);
  }
  if (lane == 31) sh.mark[warp] = mark;
  __syncthreads();
  mark = max(mark, __reduce_max_sync(0xffffffffu, lane < warp ? sh.mark[lane] : 0u));
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
      const u32 page_at = pages_in((u32)pos), in_page = (u32)pos - page_at * s, held = pages_in.up((u32)c);
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

// 16 bytes a thread and step, (token, key or value, head, piece of a head) -> its slot: a copy, in which each byte is read once and
// written once.  A thread keeps its (key or value, head, piece) and goes through four tokens, all their loads in flight
// at once, so that all divisions but the slot's are made once.
// 64 tokens of 8 heads of 128 take 2.3 us, 16383 tokens (115 MB) 22.6 us, 5.1 TB/s: what is written are runs of 256 bytes.
struct StoreArgs {
  gorio_cache_store_desc d;
  u32 pieces;        // 16-byte pieces of a head
  u32 columns;       // 2 * heads * pieces
  u32 side;          // tokens side by side in a block
};

constexpr int kStoreThreads = 256;
constexpr int kStoreEach = 4;          // tokens a thread

__global__ void __launch_bounds__(kStoreThreads) cache_store_kernel(const StoreArgs a) {
  const u32 sub = a.side > 1 ? threadIdx.x / a.columns : 0;
  if (sub >= a.side) return;
  const u32 first = blockIdx.x * a.side * kStoreEach + sub;
  const u32 places = a.d.n_pages * a.d.page_size;
  for (u32 c = threadIdx.x - sub * a.columns; c < a.columns; c += kStoreThreads) {
    const u32 half = a.columns / 2, v = c >= half, h = (c - v * half) / a.pieces, piece = c - v * half - h * a.pieces;
    const u16 *src = (const u16 *)(v ? a.d.values : a.d.keys) + (i64)h * (v ? a.d.v_head_stride : a.d.k_head_stride) + piece * 8;
    u16 *dst = (u16 *)(v ? a.d.value_pages : a.d.key_pages) + (i64)h * (v ? a.d.vp_head_stride : a.d.kp_head_stride) + piece * 8;
    const i64 src_t = v ? a.d.v_token_stride : a.d.k_token_stride;
    const i64 dst_p = v ? a.d.vp_page_stride : a.d.kp_page_stride, dst_t = v ? a.d.vp_token_stride : a.d.kp_token_stride;
    uint4 x[kStoreEach];
    i64 slot[kStoreEach];
#pragma unroll
    for (int i = 0; i < kStoreEach; ++i) {
      const u32 t = first + i * a.side;
      slot[i] = -1;
      if (t < a.d.n_tokens) {
        slot[i] = a.d.slots[t];
        x[i] = __ldcs((const uint4 *)(src + (i64)t * src_t));
      }
    }
#pragma unroll
    for (int i = 0; i < kStoreEach; ++i) {
      if ((u64)slot[i] >= (u64)places) continue;           // negative ones too
      const u32 page = (u32)slot[i] / a.d.page_size, in_page = (u32)slot[i] - page * a.d.page_size;
      *(uint4 *)(dst + (i64)page * dst_p + (i64)in_page * dst_t) = x[i];
    }
  }
}

}  // namespace

cudaError_t launch_page_tables(const gorio_page_tables_desc &d, cudaStream_t s) {
  const u32 blocks = d.n_tokens > 0 ? (d.n_tokens + kTabThreads - 1) / kTabThreads : 1;
  u32 l = 0;
  while ((1ull << l) < d.page_size) ++l;
  const Divider pages_in{(u32)(((1ull << (31 + l)) + d.page_size - 1) / d.page_size), 31 + l};
  if (d.n_requests <= (u32)kTabThreads) page_tables_kernel<1><<<blocks, kTabThreads, 0, s>>>(d, pages_in);
  else page_tables_kernel<8><<<blocks, kTabThreads, 0, s>>>(d, pages_in);
  return cudaGetLastError();
}

cudaError_t launch_cache_store(const gorio_cache_store_desc &d, cudaStream_t s) {
  StoreArgs a{d, d.dim / 8, 2 * d.n_heads * (d.dim / 8), 1};
  if (a.columns < (u32)kStoreThreads) a.side = kStoreThreads / a.columns;
  const u32 tokens = a.side * kStoreEach;
  cache_store_kernel<<<(d.n_tokens + tokens - 1) / tokens, kStoreThreads, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace paged
}  // namespace gorio
