// C entry points of the paged key/value cache: checks of arguments, then one launch.
#include <atomic>
#include <cmath>
#include <cstdio>
#include <mutex>

#include "../../include/gorio.h"
#include "paged/common.cuh"
#include "paged/entries.h"

namespace gorio { void set_global_error(const char *msg); }

namespace {

using namespace gorio::paged;

int bad(const char *msg) {
  gorio::set_global_error(msg);
  return GORIO_ERR_INVALID_ARG;
}

int launched(cudaError_t e, const char *what) {
  if (e == cudaSuccess) return GORIO_OK;
  char buf[160];
  std::snprintf(buf, sizeof buf, "%s: %s", what, cudaGetErrorString(e));
  gorio::set_global_error(buf);
  return GORIO_ERR_CUDA;
}

bool aligned(const void *p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

constexpr int kMaxDevices = 64;

// SMs of a device, read once
int sm_count(int dev) {
  static int known[kMaxDevices] = {};
  static std::mutex mu;
  if (dev < 0 || dev >= kMaxDevices) return 0;
  std::lock_guard<std::mutex> lk(mu);
  if (!known[dev]) {
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    known[dev] = n;
  }
  return known[dev];
}

constexpr uint64_t kWaitLimitNs = 10ull * 1000000000ull;
std::atomic<uint64_t> wait_limit{kWaitLimitNs};

// Whether the rows kernel takes a call.  It reads a request's keys once for every 16 rows ((token, query head) pairs of a key head), the
// chunk kernel once for every 256, but the chunk kernel's start and its joins cost some 14 us more.  Up to 16 rows the rows
// kernel has no work to spare.  Beyond, the two times are compared as measured (bfloat16, head sizes 64 to 128, 1 to 8
// key heads, 1 to 64 requests, 24 to 256 rows each, 150 to 131072 keys): a unit of 16 rows takes 0.6 ps for each element of a
// key, and what 384 keys take besides; one of 256 rows 1 ps an element.  The host has bounds of units and keys only.
//   8 key heads of 128, 1 request, 192 rows each:   150 keys 12 us, chunk kernel 24;     2000 keys 27 against 32
//                                    96 rows each:  8000 keys 38 against 39;            131072 keys 482 against 150
//   2 key heads of 64, 64 requests, 24 rows each:    150 keys 12 against 18;              8000 keys 94 against 88
bool takes_rows(const gorio_paged_attention_desc &d) {
  const double group = d.n_heads / d.n_kv_heads, requests = d.n_requests < d.n_tokens ? d.n_requests : d.n_tokens;
  if ((double)d.max_new * group <= 16) return true;
  auto units = [&](double rows) {
    const double alike = requests * std::ceil(d.max_new * group / rows), ragged = d.n_tokens * group / rows + requests;
    return d.n_kv_heads * (alike < ragged ? alike : ragged);
  };
  const double places = (double)d.table_width * d.page_size, seen = (double)d.window + d.max_new;
  const double keys = d.window && seen < places ? seen : places;
  return 0.6 * units(16) * (keys + 384) * d.dim <= 14e6 + units(256) * keys * d.dim;
}

}  // namespace

extern "C" int gorio_page_tables(const gorio_page_tables_desc *d, void *cuda_stream) {
  if (!d || !d->free_count || !d->starts || !d->out_free_count) return bad("page tables: null argument");
  if (d->n_requests && (!d->lengths || !d->new_lens || !d->tables || !d->out_lengths || !d->out_served))
    return bad("page tables: null argument");
  if (d->n_tokens && (!d->slots || !d->positions || !d->requests)) return bad("page tables: null argument");
  if (d->free_capacity && !d->free_pages) return bad("page tables: null argument");
  if (d->page_size < 1 || d->table_width < 1 || (uint64_t)d->page_size * d->table_width >= (1ull << 31))
    return bad("page tables: need page_size >= 1, table_width >= 1 and page_size * table_width < 2^31");
  if (d->n_requests > (1u << 20) || d->n_tokens >= (1u << 31)) return bad("page tables: at most 2^20 requests and 2^31 - 1 tokens");
  if (d->table_stride < (int64_t)d->table_width && d->n_requests > 1) return bad("page tables: rows of the table overlap");
  return launched(launch_page_tables(*d, (cudaStream_t)cuda_stream), "page tables");
}

extern "C" int gorio_cache_store(const gorio_cache_store_desc *d, void *cuda_stream) {
  if (!d) return bad("cache store: null argument");
  if (d->n_tokens == 0 || d->n_heads == 0 || d->n_pages == 0) return GORIO_OK;
  if (!d->keys || !d->values || !d->key_pages || !d->value_pages || !d->slots) return bad("cache store: null argument");
  if (d->dim == 0 || d->dim % 8 != 0 || d->page_size < 1 || (uint64_t)d->n_pages * d->page_size >= (1ull << 31))
    return bad("cache store: need dim a multiple of 8, page_size >= 1 and n_pages * page_size < 2^31");
  const int64_t strides = d->k_token_stride | d->k_head_stride | d->v_token_stride | d->v_head_stride | d->kp_page_stride | d->kp_head_stride |
                          d->kp_token_stride | d->vp_page_stride | d->vp_head_stride | d->vp_token_stride;
  if (strides & 7) return bad("cache store: every stride must be a multiple of 8 elements");
  if (!aligned(d->keys, 16) || !aligned(d->values, 16) || !aligned(d->key_pages, 16) || !aligned(d->value_pages, 16))
    return bad("cache store: keys, values and pages must be 16-byte aligned");
  if (d->n_tokens >= (1u << 31)) return bad("cache store: at most 2^31 - 1 tokens");        // the kernel counts past them in 32 bits
  if (d->n_heads > 65536 || d->dim > 65536 || (uint64_t)d->n_tokens * d->n_heads * d->dim >= (1ull << 40))
    return bad("cache store: too large");
  return launched(launch_cache_store(*d, (cudaStream_t)cuda_stream), "cache store");
}

extern "C" uint64_t gorio_attention_workspace_bytes(int cuda_device) {
  const int sms = sm_count(cuda_device);
  return sms ? kCounterBytes + part_bytes((u32)sms) : 0;
}

extern "C" int gorio_attention_wait_limit(uint64_t nanoseconds) {
  wait_limit.store(nanoseconds ? nanoseconds : kWaitLimitNs, std::memory_order_relaxed);
  return GORIO_OK;
}

extern "C" int gorio_attention_check(void *workspace, void *cuda_stream) {
  if (!workspace) return bad("attention check: null argument");
  u32 word = 0;
  const cudaStream_t s = (cudaStream_t)cuda_stream;
  cudaError_t e = cudaMemcpyAsync(&word, (u32 *)workspace + kErrorWord, sizeof word, cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e != cudaSuccess || word == 0) return launched(e, "attention check");
  e = cudaMemsetAsync(workspace, 0, kCounterBytes, s);
  if (e != cudaSuccess) return launched(e, "attention check");
  if (word == 2) {
    gorio::set_global_error("paged attention: a call had 2^31 or more tiles of keys and was not computed");
    return GORIO_ERR_CAPACITY;
  }
  gorio::set_global_error("paged attention: a wait inside a kernel lasted longer than its limit; the results of calls with this workspace are not valid");
  return GORIO_ERR_TIMEOUT;
}

extern "C" int gorio_paged_attention(const gorio_paged_attention_desc *d, void *cuda_stream) {
  if (!d) return bad("paged attention: null argument");
  if (d->n_requests == 0 || d->n_tokens == 0) return GORIO_OK;
  if (!d->q || !d->out || !d->tables || !d->lengths || !d->starts || !d->workspace) return bad("paged attention: null argument");
  if (d->n_pages && (!d->key_pages || !d->value_pages)) return bad("paged attention: null argument");
  if (d->dtype > GORIO_KV_FP16) return bad("paged attention: unknown dtype");
  if (d->dim != 64 && d->dim != 96 && d->dim != 128) return bad("paged attention: dim must be 64, 96 or 128");
  if (d->n_kv_heads < 1 || d->n_heads < 1 || d->n_heads % d->n_kv_heads != 0 || d->n_heads > 65536)
    return bad("paged attention: n_heads must be a multiple of n_kv_heads");
  if (d->page_size < 8 || d->page_size % 8 != 0 || d->table_width < 1 || (uint64_t)d->page_size * d->table_width >= (1ull << 31) ||
      (uint64_t)d->n_pages * d->page_size >= (1ull << 31))
    return bad("paged attention: need page_size a multiple of 8 and fewer than 2^31 places in a table row and in the cache");
  if (d->n_requests > (1u << 20) || d->n_tokens >= (1u << 31)) return bad("paged attention: at most 2^20 requests and 2^31 - 1 tokens");
  if (!(d->scale > 0.0f) || !std::isfinite(d->scale) || !(d->softcap >= 0.0f) || !std::isfinite(d->softcap))
    return bad("paged attention: need a finite scale > 0 and a finite softcap >= 0");
  if ((uint64_t)d->n_tokens * d->n_heads >= (1ull << 31)) return bad("paged attention: n_tokens * n_heads must be below 2^31");
  const int64_t strides = d->q_token_stride | d->q_head_stride | d->o_token_stride | d->o_head_stride | d->kp_page_stride | d->kp_head_stride |
                          d->kp_token_stride | d->vp_page_stride | d->vp_head_stride | d->vp_token_stride;
  if (strides & 7) return bad("paged attention: every stride must be a multiple of 8 elements");
  if (!aligned(d->q, 16) || !aligned(d->out, 16) || !aligned(d->key_pages, 16) || !aligned(d->value_pages, 16))
    return bad("paged attention: q, out and pages must be 16-byte aligned");
  if (!aligned(d->workspace, 256)) return bad("paged attention: the workspace must be 256-byte aligned");
  int dev = 0;
  const cudaError_t found = cudaGetDevice(&dev);
  if (found != cudaSuccess) return launched(found, "paged attention");
  const int sms = sm_count(dev);
  if (sms < 1) return launched(cudaErrorInvalidDevice, "paged attention");

  Attn a{};
  a.q = d->q; a.kp = d->key_pages; a.vp = d->value_pages; a.out = d->out; a.lse = d->lse;
  a.tables = d->tables; a.lengths = d->lengths; a.starts = d->starts; a.slopes = d->slopes;
  a.q_t = d->q_token_stride; a.q_h = d->q_head_stride; a.o_t = d->o_token_stride; a.o_h = d->o_head_stride;
  a.k_p = d->kp_page_stride; a.k_h = d->kp_head_stride; a.k_t = d->kp_token_stride;
  a.v_p = d->vp_page_stride; a.v_h = d->vp_head_stride; a.v_t = d->vp_token_stride;
  if (d->n_pages == 0) {                                     // nothing is read, but the copies of no bytes name an address
    a.kp = a.vp = d->workspace;
    a.k_p = a.k_h = a.k_t = a.v_p = a.v_h = a.v_t = 0;
  }
  a.tab_r = d->table_stride;
  a.n_req = d->n_requests; a.n_tok = d->n_tokens; a.hq = d->n_heads; a.hkv = d->n_kv_heads; a.group = d->n_heads / d->n_kv_heads;
  a.page = d->page_size; a.n_pages = d->n_pages; a.width = d->table_width;
  a.causal = d->causal != 0; a.window = d->window;
  a.scale = d->scale; a.softcap = d->softcap;
  const uint64_t ticks = wait_limit.load(std::memory_order_relaxed) >> 10;
  a.wait_ticks = ticks < 0xffffffffu ? (u32)ticks : 0xffffffffu;
  a.arrived = (u32 *)d->workspace;
  a.part_ml = (float *)((char *)d->workspace + kCounterBytes);
  a.part_o = (float *)((char *)a.part_ml + part_ml_bytes((u32)sms));
  if (!takes_rows(*d)) {
    cudaError_t e = cudaSuccess;
    if (launch_chunk(a, (int)d->dtype, (int)d->dim, (u32)sms, (cudaStream_t)cuda_stream, &e)) return launched(e, "paged attention");
  }
  return launched(launch_rows(a, (int)d->dtype, (int)d->dim, (u32)sms, (cudaStream_t)cuda_stream), "paged attention");
}
