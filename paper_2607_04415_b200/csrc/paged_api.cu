// C entry points of the paged key/value cache: checks of arguments, then one launch.
#include <atomic>
#include <cmath>
#include <cstdio>
#include <mutex>

#include "../../include/gorio.h"
#include "paged/coded.cuh"
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
// For 8-bit codes both kernels pay for taking them apart: a unit of 16 rows 0.5 ps for half the bytes, one of the chunk kernel 1.12 ps, and with
// at most 128 rows, one row tile, 1.44 (16 requests, 8 key heads of 128, 65536 keys: 16 rows 542 us, 24 rows some 1090 against 1550, 48 rows 1626
// against 1551, 192 rows 6500 against 1183).
struct Costs {
  double row_unit, chunk_unit, chunk_tile;       // ps an element of a key
};
constexpr Costs kWideCosts{0.6, 1.0, 1.0}, kCodedCosts{0.5, 1.12, 1.44};

bool takes_rows(const gorio_paged_attention_desc &d, const Costs &c = kWideCosts) {
  const double group = d.n_heads / d.n_kv_heads, requests = d.n_requests < d.n_tokens ? d.n_requests : d.n_tokens;
  if ((double)d.max_new * group <= 16) return true;
  auto units = [&](double rows) {
    const double alike = requests * std::ceil(d.max_new * group / rows), ragged = d.n_tokens * group / rows + requests;
    return d.n_kv_heads * (alike < ragged ? alike : ragged);
  };
  const double places = (double)d.table_width * d.page_size, seen = (double)d.window + d.max_new;
  const double keys = d.window && seen < places ? seen : places;
  const double chunk = d.max_new * group <= 128 ? c.chunk_tile : c.chunk_unit;
  return c.row_unit * units(16) * (keys + 384) * d.dim <= 14e6 + chunk * units(256) * keys * d.dim;
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

namespace {

// Checks of the numbers and addresses of an attention call; its workspace's among them.
int check_attention(const gorio_paged_attention_desc *d) {
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
  return GORIO_OK;
}

// SMs of the current device
int current_sms(int *sms, const char *what) {
  int dev = 0;
  const cudaError_t found = cudaGetDevice(&dev);
  if (found != cudaSuccess) return launched(found, what);
  *sms = sm_count(dev);
  return *sms < 1 ? launched(cudaErrorInvalidDevice, what) : GORIO_OK;
}

void fill_attention(Attn &a, const gorio_paged_attention_desc *d, int sms) {
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
}

// One of the two kernels, by the bounds of rows and keys in `d`.
template <typename A>
cudaError_t launch_attention(const A &a, const gorio_paged_attention_desc &d, int sms, cudaStream_t s) {
  if (!takes_rows(d)) {
    cudaError_t e = cudaSuccess;
    if (launch_chunk(a, (int)d.dtype, (int)d.dim, (u32)sms, s, &e)) return e;
  }
  return launch_rows(a, (int)d.dtype, (int)d.dim, (u32)sms, s);
}

}  // namespace

extern "C" int gorio_paged_attention(const gorio_paged_attention_desc *d, void *cuda_stream) {
  if (!d) return bad("paged attention: null argument");
  if (d->n_requests == 0 || d->n_tokens == 0) return GORIO_OK;
  int sms = 0, st = check_attention(d);
  if (st == GORIO_OK) st = current_sms(&sms, "paged attention");
  if (st != GORIO_OK) return st;
  Attn a{};
  fill_attention(a, d, sms);
  return launched(launch_attention(a, *d, sms, (cudaStream_t)cuda_stream), "paged attention");
}

namespace {

// What a call on shared keys needs besides the workspace: the last kernel's parts, then the first one's results.
uint64_t mid_ml_bytes(uint64_t rows) { return (rows * sizeof(float2) + 255) / 256 * 256; }
uint64_t scratch_bytes(int sms, uint64_t rows, uint64_t dim) { return part_bytes((u32)sms) + 3 * mid_ml_bytes(rows) + rows * dim * sizeof(float); }

}  // namespace

extern "C" uint64_t gorio_prefix_scratch_bytes(int cuda_device, uint32_t n_tokens, uint32_t n_heads, uint32_t dim) {
  const int sms = sm_count(cuda_device);
  return sms ? scratch_bytes(sms, (uint64_t)n_tokens * n_heads, dim) : 0;
}

extern "C" int gorio_prefix_attention(const gorio_prefix_attention_desc *d, void *cuda_stream) {
  if (!d) return bad("prefix attention: null argument");
  const gorio_paged_attention_desc &own = d->own;
  if (own.n_requests == 0 || own.n_tokens == 0) return GORIO_OK;
  int sms = 0, st = check_attention(&own);
  if (st != GORIO_OK) return st;
  if (!d->prefix_tables || !d->prefix_lengths || !d->group_starts || !d->scratch) return bad("prefix attention: null argument");
  if (d->n_groups < 1 || d->n_groups > (1u << 20) || d->prefix_width < 1 || (uint64_t)own.page_size * d->prefix_width >= (1ull << 31))
    return bad("prefix attention: need 1 to 2^20 groups and fewer than 2^31 places in a row of their tables");
  if (((uint64_t)d->prefix_width + own.table_width) * own.page_size + own.n_tokens >= (1ull << 31))
    return bad("prefix attention: positions must stay below 2^31");
  if (!aligned(d->scratch, 256)) return bad("prefix attention: the scratch must be 256-byte aligned");
  st = current_sms(&sms, "prefix attention");
  if (st != GORIO_OK) return st;

  const uint64_t rows = (uint64_t)own.n_tokens * own.n_heads;
  float2 *const mid_ml = (float2 *)((char *)d->scratch + part_bytes((u32)sms));
  int4 *const mid_at = (int4 *)((char *)mid_ml + mid_ml_bytes(rows));             // twice as large
  float *const mid_o = (float *)((char *)mid_at + 2 * mid_ml_bytes(rows));
  PrefixAttn p{};
  fill_attention(p, &own, sms);
  p.tables = d->prefix_tables; p.lengths = d->prefix_lengths; p.tab_r = d->prefix_table_stride;
  p.n_req = d->n_groups; p.width = d->prefix_width;
  p.causal = 0;                                              // shared keys stand before all new tokens
  p.group_starts = d->group_starts; p.own_lengths = own.lengths;
  p.n_members = own.n_requests; p.own_places = own.table_width * own.page_size;
  p.mid_o = mid_o; p.mid_ml = mid_ml; p.mid_at = mid_at;
  gorio_paged_attention_desc shared = own;                   // bounds of the first kernel's rows and keys
  shared.n_requests = d->n_groups; shared.table_width = d->prefix_width; shared.max_new = own.n_tokens;
  // Units of the first kernel, by their bounds: with few, joining their parts is a kernel of its own.  9 groups of 1155 tokens in all, 2 key heads of 7:
  // some 80 units, 84 us with the joins in the first kernel and 94 with their own.
  const bool rows_kernel = takes_rows(shared);
  const double per_unit = rows_kernel ? 16 : 256, units = own.n_kv_heads * ((double)own.n_tokens * (own.n_heads / own.n_kv_heads) / per_unit + d->n_groups);
  p.leaves_parts = units < sms / 2;
  cudaError_t e = launch_attention(p, shared, sms, (cudaStream_t)cuda_stream);
  if (e == cudaSuccess && p.leaves_parts) e = launch_prefix_join(p, (int)own.dim, (u32)sms, (cudaStream_t)cuda_stream);
  if (e != cudaSuccess) return launched(e, "prefix attention");

  OwnAttn o{};
  fill_attention(o, &own, sms);
  o.arrived += kOwnCounters;
  o.part_ml = (float *)d->scratch;
  o.part_o = (float *)((char *)d->scratch + part_ml_bytes((u32)sms));
  o.group_starts = d->group_starts; o.n_groups = d->n_groups;
  o.mid_o = mid_o; o.mid_ml = mid_ml;
  return launched(launch_attention(o, own, sms, (cudaStream_t)cuda_stream), "prefix attention");
}

namespace {

// Both calls on rows of a quantised cache.
int quantized_rows(const gorio_quantized_rows_desc *d, bool store, void *cuda_stream) {
  const char *const what = store ? "quantized store" : "quantized load";
  if (!d) return bad("quantized rows: null argument");
  if (d->n_tokens == 0 || d->n_heads == 0 || (store && d->n_pages == 0)) return GORIO_OK;
  if (!d->keys || !d->values || !d->slots) return bad("quantized rows: null argument");
  if (d->n_pages && (!d->key_pages || !d->value_pages || !d->key_scales || !d->value_scales)) return bad("quantized rows: null argument");
  if (d->dtype > GORIO_KV_FP16 || d->format > GORIO_CODES_INT8) return bad("quantized rows: unknown dtype or format");
  if (d->dim == 0 || d->dim % 16 != 0 || d->dim > 256 || d->page_size < 1 || (uint64_t)d->n_pages * d->page_size >= (1ull << 31))
    return bad("quantized rows: need dim a multiple of 16 and at most 256, page_size >= 1 and n_pages * page_size < 2^31");
  const int64_t wide = d->k_token_stride | d->k_head_stride | d->v_token_stride | d->v_head_stride;
  const int64_t codes = d->kp_page_stride | d->kp_head_stride | d->kp_token_stride | d->vp_page_stride | d->vp_head_stride | d->vp_token_stride;
  if ((wide & 7) || (codes & 15)) return bad("quantized rows: strides must be multiples of 8 elements, of the pages of 16");
  if (!aligned(d->keys, 16) || !aligned(d->values, 16) || !aligned(d->key_pages, 16) || !aligned(d->value_pages, 16))
    return bad("quantized rows: keys, values and pages must be 16-byte aligned");
  if (!aligned(d->key_scales, 4) || !aligned(d->value_scales, 4)) return bad("quantized rows: scales must be 4-byte aligned");
  if (d->n_tokens >= (1u << 31) || d->n_heads > 65536 || (uint64_t)d->n_tokens * d->n_heads >= (1ull << 31))
    return bad("quantized rows: n_tokens * n_heads must be below 2^31");
  return launched(launch_quantized_rows(*d, store, (cudaStream_t)cuda_stream), what);
}

}  // namespace

extern "C" int gorio_cache_store_quantized(const gorio_quantized_rows_desc *d, void *cuda_stream) { return quantized_rows(d, true, cuda_stream); }
extern "C" int gorio_cache_load_quantized(const gorio_quantized_rows_desc *d, void *cuda_stream) { return quantized_rows(d, false, cuda_stream); }

extern "C" int gorio_paged_attention_quantized(const gorio_quantized_attention_desc *d, void *cuda_stream) {
  if (!d) return bad("quantized attention: null argument");
  const gorio_paged_attention_desc &p = d->attention;
  if (p.n_requests == 0 || p.n_tokens == 0) return GORIO_OK;
  int sms = 0, st = check_attention(&p);
  if (st != GORIO_OK) return st;
  if (d->format > GORIO_CODES_INT8) return bad("quantized attention: unknown format");
  if (p.n_pages && (!d->key_scales || !d->value_scales)) return bad("quantized attention: null argument");
  if (!aligned(d->key_scales, 4) || !aligned(d->value_scales, 4)) return bad("quantized attention: scales must be 4-byte aligned");
  if ((p.kp_page_stride | p.kp_head_stride | p.kp_token_stride | p.vp_page_stride | p.vp_head_stride | p.vp_token_stride) & 15)
    return bad("quantized attention: strides of the pages must be multiples of 16");
  st = current_sms(&sms, "quantized attention");
  if (st != GORIO_OK) return st;
  CodedAttn a{};
  fill_attention(a, &p, sms);
  a.ks = d->key_scales; a.vs = d->value_scales;
  a.ks_p = d->ks_page_stride; a.ks_h = d->ks_head_stride; a.ks_t = d->ks_token_stride;
  a.vs_p = d->vs_page_stride; a.vs_h = d->vs_head_stride; a.vs_t = d->vs_token_stride;
  if (p.n_pages == 0) {                                      // as for the pages
    a.ks = a.vs = (const float *)p.workspace;
    a.ks_p = a.ks_h = a.ks_t = a.vs_p = a.vs_h = a.vs_t = 0;
  }
  const cudaStream_t s = (cudaStream_t)cuda_stream;
  cudaError_t e = cudaSuccess;
  if (!takes_rows(p, kCodedCosts)) {
    const bool ran = d->format == GORIO_CODES_E4M3 ? launch_coded_chunk_e4m3(a, (int)p.dtype, (int)p.dim, (u32)sms, s, &e)
                                                   : launch_coded_chunk_int8(a, (int)p.dtype, (int)p.dim, (u32)sms, s, &e);
    if (ran) return launched(e, "quantized attention");
  }
  const bool few = (uint64_t)p.max_new * (p.n_heads / p.n_kv_heads) <= 8;
  e = d->format == GORIO_CODES_E4M3 ? launch_coded_rows_e4m3(a, (int)p.dtype, (int)p.dim, few, (u32)sms, s)
                                    : launch_coded_rows_int8(a, (int)p.dtype, (int)p.dim, few, (u32)sms, s);
  return launched(e, "quantized attention");
}
