// Host side of include/rtams_cache.h: layout of the pool, checks, and the enqueue-only entry points.
#include "../../include/rtams_cache.h"

#include <cmath>
#include <cstring>
#include <mutex>
#include <new>

#include "cache.h"
#include "host.h"

using namespace rtams;

struct rtams_cache {
  rtams_cache_config cfg{};
  CacheDev dev{};
  CacheMirror *mirror = nullptr;
  std::mutex mutex;  // calls of one cache are enqueued one after another
  hipStream_t stream = nullptr;  // of the last call
  bool have_stream = false;
  hipEvent_t done = nullptr;
  bool forked = false;  // sequences may share pages
};

namespace {

constexpr size_t kAlign = 256;
constexpr int64_t kMaxItems = kCacheMaxSeqs;

struct CacheLayout {
  size_t ctrl, free_bits, refs, lengths, table, items, picked, pair_src, pair_dst, map, data, total;
  int64_t page_bytes, pages;
};

bool cache_config_ok(const rtams_cache_config *c, bool need_memory) {
  if (!c) return fail(RTAMS_EINVAL, "config is NULL"), false;
  if (c->layers < 1 || c->layers > 1024) return fail(RTAMS_EINVAL, "layers must be in 1..1024, got %d", c->layers), false;
  if (c->kv_heads < 1 || c->kv_heads > 1024) return fail(RTAMS_EINVAL, "kv_heads must be in 1..1024, got %d", c->kv_heads), false;
  if (c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128 && c->head_dim != 256)
    return fail(RTAMS_EINVAL, "head_dim must be 64, 96, 128 or 256, got %d", c->head_dim), false;
  if (c->page_tokens < kBlockTokens || c->page_tokens % kBlockTokens || c->page_tokens > 1024)
    return fail(RTAMS_EINVAL, "page_tokens must be a multiple of 32 in 32..1024, got %d", c->page_tokens), false;
  if (c->max_seqs < 1 || c->max_seqs > kCacheMaxSeqs) return fail(RTAMS_EINVAL, "max_seqs must be in 1..%d, got %d", kCacheMaxSeqs, c->max_seqs), false;
  if (c->max_pages < 1 || (int64_t)c->max_pages * c->page_tokens >= ((int64_t)1 << 30))
    return fail(RTAMS_EINVAL, "max_pages must be positive and max_pages * page_tokens below 2^30, got %d", c->max_pages), false;
  if (need_memory) {
    if (!c->d_pool || !c->d_scratch) return fail(RTAMS_EINVAL, "pool and scratch must be given"), false;
    if (((uintptr_t)c->d_pool | (uintptr_t)c->d_scratch) % kAlign)
      return fail(RTAMS_EINVAL, "pool and scratch must be %zu-byte aligned", kAlign), false;
  }
  return true;
}

void cache_lay_out(const rtams_cache_config *c, int64_t pages, CacheLayout *L) {
  size_t o = 0;
  auto take = [&](size_t bytes) { size_t at = o; o = up(o + bytes, kAlign); return at; };
  L->pages = pages;
  L->page_bytes = (int64_t)c->page_tokens / kBlockTokens * c->kv_heads * (40 * c->head_dim);
  L->ctrl = take(sizeof(CacheCtrl));
  L->free_bits = take(((size_t)pages + 31) / 32 * 4);
  L->refs = take((size_t)pages * 4);
  L->lengths = take((size_t)c->max_seqs * 4);
  L->table = take((size_t)c->max_seqs * c->max_pages * 4);
  L->items = take((size_t)c->max_seqs * sizeof(CacheItem));
  L->picked = take((size_t)pages * 4);
  L->pair_src = take((size_t)pages * 4);
  L->pair_dst = take((size_t)pages * 4);
  L->map = take((size_t)pages * 4);
  L->data = o;
  L->total = o + (size_t)pages * c->layers * L->page_bytes;
}

// Clears the tables, marks every page free and gives what pages hold finite steps.
__global__ void k_cache_clear(CacheDev d, uint4 *data, uint64_t chunks) {
  const uint64_t at = blockIdx.x * (uint64_t)blockDim.x + threadIdx.x, all = (uint64_t)gridDim.x * blockDim.x;
  for (uint64_t i = at; i < chunks; i += all) data[i] = make_uint4(0, 0, 0, 0);
  for (uint64_t i = at; i < d.pages; i += all) d.refs[i] = 0;
  for (uint64_t i = at; i < (uint64_t)d.max_seqs; i += all) d.lengths[i] = 0;
  for (uint64_t i = at; i < (uint64_t)d.max_seqs * d.max_pages; i += all) d.table[i] = -1;
  for (uint64_t i = at; i < ((uint64_t)d.pages + 31) / 32; i += all)
    d.free_bits[i] = d.pages - i * 32 >= 32 ? ~0u : (1u << (d.pages - i * 32)) - 1u;
  if (at == 0) *d.ctrl = CacheCtrl{d.pages, 0, 0, 0, 0, {}};
}

__global__ void k_cache_clear_stop(CacheDev d) {
  d.ctrl->stopped = 0;
  d.mirror->error = 0;
}

__global__ void k_cache_clear_words(uint32_t *p, uint64_t n) {
  for (uint64_t i = blockIdx.x * (uint64_t)blockDim.x + threadIdx.x; i < n; i += (uint64_t)gridDim.x * blockDim.x) p[i] = 0;
}

// Orders the call behind the cache's work on another stream.  (Not a recorded call, which the graph orders.)
int cache_enter(rtams_cache *c, hipStream_t s, bool *recorded = nullptr) {
  hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(s, &capture) != hipSuccess) (void)hipGetLastError();
  if (recorded) *recorded = capture == hipStreamCaptureStatusActive;
  if (capture == hipStreamCaptureStatusActive) return RTAMS_OK;
  if (c->have_stream && c->stream != s) {
    HIP_TRY(hipEventRecord(c->done, c->stream));
    HIP_TRY(hipStreamWaitEvent(s, c->done, 0));
  }
  c->stream = s;
  c->have_stream = true;
  return RTAMS_OK;
}

int launched(const char *what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? RTAMS_OK : fail(RTAMS_EHIP, "%s launch failed: %s", what, hipGetErrorString(e));
}

int check_items(const rtams_cache *c, int64_t n, const int32_t *d_seqs) {
  if (!c) return fail(RTAMS_EINVAL, "cache is NULL");
  if (n < 0 || n > kMaxItems) return fail(RTAMS_EINVAL, "n must be in 0..%lld, got %lld", (long long)kMaxItems, (long long)n);
  if (n > c->cfg.max_seqs) return fail(RTAMS_EINVAL, "n %lld is more than the cache's %d sequences", (long long)n, c->cfg.max_seqs);
  (void)d_seqs;
  return RTAMS_OK;
}

int check_rows(const rtams_cache *c, int32_t layer, int64_t n, const int32_t *d_starts, int64_t rows, int32_t max_new) {
  if (layer < 0 || layer >= c->cfg.layers) return fail(RTAMS_EINVAL, "layer %d outside 0..%d", layer, c->cfg.layers - 1);
  if (rows < 0 || rows > 0x7fffffff) return fail(RTAMS_EINVAL, "rows must be in 0..2^31 - 1, got %lld", (long long)rows);
  if (!d_starts && rows != n) return fail(RTAMS_EINVAL, "without d_starts every item has one row: %lld rows for %lld items", (long long)rows, (long long)n);
  if (max_new < 1) return fail(RTAMS_EINVAL, "max_new must be positive, got %d", max_new);
  if (n * (int64_t)c->cfg.kv_heads * ((d_starts ? (max_new < rows ? (int64_t)max_new : rows) : 1) / kBlockTokens + 2) > 0x7fffffff)
    return fail(RTAMS_EINVAL, "%lld items of up to %d rows are too many for one call", (long long)n, max_new);
  return RTAMS_OK;
}

CacheRows items_of(int64_t n, const int32_t *d_seqs, const int32_t *d_starts, int64_t rows, int32_t max_new) {
  CacheRows r{};
  r.n = (int32_t)n;
  r.seqs = d_seqs;
  r.starts = d_starts;
  r.rows = rows;
  r.max_new = d_starts ? (max_new < rows ? max_new : (int32_t)rows) : 1;
  return r;
}

}  // namespace

extern "C" {

size_t rtams_cache_pool_bytes_for(const rtams_cache_config *cfg, int64_t pages) {
  if (!cache_config_ok(cfg, false)) return 0;
  if (pages < 1 || pages > 0x7fffffff) return fail(RTAMS_EINVAL, "pages must be in 1..2^31 - 1, got %lld", (long long)pages), 0;
  CacheLayout L;
  cache_lay_out(cfg, pages, &L);
  return L.total;
}

size_t rtams_cache_scratch_bytes_for(const rtams_cache_config *cfg) {
  if (!cache_config_ok(cfg, false)) return 0;
  return up(cache_arrived_words(cfg->max_seqs, cfg->kv_heads) * 4, kAlign) + up(cache_part_ml_floats(cfg->head_dim) * 4, kAlign) +
         up(cache_part_floats(cfg->head_dim) * 4, kAlign);
}

int rtams_cache_create(const rtams_cache_config *cfg, rtams_cache **out) {
  if (!out) return fail(RTAMS_EINVAL, "out is NULL");
  *out = nullptr;
  if (!cache_config_ok(cfg, true)) return RTAMS_EINVAL;
  // as many pages as fit: the tables grow with the pages, so from above
  CacheLayout L;
  cache_lay_out(cfg, 1, &L);
  int64_t pages = (int64_t)(cfg->pool_bytes / ((size_t)L.page_bytes * cfg->layers));
  if (pages > 0x7fffffff) pages = 0x7fffffff;
  for (; pages > 0; --pages) {
    cache_lay_out(cfg, pages, &L);
    if (L.total <= cfg->pool_bytes) break;
    const int64_t over = (int64_t)((L.total - cfg->pool_bytes) / ((size_t)L.page_bytes * cfg->layers + 32));
    if (over > 1) pages -= over - 1;
  }
  if (pages < 1) return fail(RTAMS_EINVAL, "pool_bytes %zu holds no page (one takes %zu)", cfg->pool_bytes, rtams_cache_pool_bytes_for(cfg, 1));
  const size_t scratch = rtams_cache_scratch_bytes_for(cfg);
  if (cfg->scratch_bytes < scratch) return fail(RTAMS_EINVAL, "scratch_bytes %zu, %zu are needed", cfg->scratch_bytes, scratch);
  rtams_cache *c = new (std::nothrow) rtams_cache;
  if (!c) return fail(RTAMS_EINVAL, "out of host memory");
  c->cfg = *cfg;
  CacheDev &d = c->dev;
  char *p = static_cast<char *>(cfg->d_pool);
  d.layers = cfg->layers;
  d.kv_heads = cfg->kv_heads;
  d.head_dim = cfg->head_dim;
  d.page_tokens = cfg->page_tokens;
  d.max_seqs = cfg->max_seqs;
  d.max_pages = cfg->max_pages;
  d.pages = (uint32_t)pages;
  d.page_blocks = (uint32_t)cfg->page_tokens / kBlockTokens;
  d.page_blocks_magic = d.page_blocks == 1 ? 0 : (uint32_t)((((uint64_t)1 << 32) + d.page_blocks - 1) / d.page_blocks);
  d.block_bytes = 40u * (uint32_t)cfg->head_dim;
  d.page_bytes = L.page_bytes;
  d.ctrl = reinterpret_cast<CacheCtrl *>(p + L.ctrl);
  d.free_bits = reinterpret_cast<uint32_t *>(p + L.free_bits);
  d.refs = reinterpret_cast<int32_t *>(p + L.refs);
  d.lengths = reinterpret_cast<int32_t *>(p + L.lengths);
  d.table = reinterpret_cast<int32_t *>(p + L.table);
  d.items = reinterpret_cast<CacheItem *>(p + L.items);
  d.picked = reinterpret_cast<int32_t *>(p + L.picked);
  d.pair_src = reinterpret_cast<int32_t *>(p + L.pair_src);
  d.pair_dst = reinterpret_cast<int32_t *>(p + L.pair_dst);
  d.map = reinterpret_cast<int32_t *>(p + L.map);
  d.data = reinterpret_cast<unsigned char *>(p + L.data);
  char *q = static_cast<char *>(cfg->d_scratch);
  const size_t arrived = cache_arrived_words(cfg->max_seqs, cfg->kv_heads);
  d.arrived = reinterpret_cast<uint32_t *>(q);
  q += up(arrived * 4, kAlign);
  d.part_ml = reinterpret_cast<float *>(q);
  q += up(cache_part_ml_floats(cfg->head_dim) * 4, kAlign);
  d.part = reinterpret_cast<float *>(q);
  auto bail = [&](int code) { rtams_cache_destroy(c); return code; };
  if (allow_large_lds_cache_attend() != hipSuccess || allow_large_lds_cache_prompt() != hipSuccess) return bail(fail(RTAMS_EHIP, "hipFuncSetAttribute failed"));
  void *hm = nullptr, *dm = nullptr;
  if (hipHostMalloc(&hm, sizeof(CacheMirror), hipHostMallocMapped) != hipSuccess) return bail(fail(RTAMS_EHIP, "hipHostMalloc failed"));
  c->mirror = static_cast<CacheMirror *>(hm);
  memset(hm, 0, sizeof(CacheMirror));
  if (hipHostGetDevicePointer(&dm, hm, 0) != hipSuccess) return bail(fail(RTAMS_EHIP, "hipHostGetDevicePointer failed"));
  d.mirror = static_cast<CacheMirror *>(dm);
  if (hipEventCreateWithFlags(&c->done, hipEventDisableTiming) != hipSuccess) return bail(fail(RTAMS_EHIP, "hipEventCreate failed"));
  k_cache_clear<<<2048, 256>>>(d, reinterpret_cast<uint4 *>(d.data), (uint64_t)pages * cfg->layers * (uint64_t)L.page_bytes / 16);
  k_cache_clear_words<<<256, 256>>>(d.arrived, arrived);
  if (hipGetLastError() != hipSuccess || hipDeviceSynchronize() != hipSuccess) return bail(fail(RTAMS_EHIP, "clearing the pool failed"));
  *out = c;
  return RTAMS_OK;
}

int rtams_cache_destroy(rtams_cache *c) {
  if (!c) return RTAMS_OK;
  if (c->have_stream) (void)hipStreamSynchronize(c->stream);
  if (c->done) (void)hipEventDestroy(c->done);
  if (c->mirror) (void)hipHostFree(c->mirror);
  delete c;
  return RTAMS_OK;
}

int rtams_cache_layout(const rtams_cache *c, rtams_cache_view *out) {
  if (!c || !out) return fail(RTAMS_EINVAL, "cache or out is NULL");
  out->d_table = c->dev.table;
  out->d_lengths = c->dev.lengths;
  out->d_refs = c->dev.refs;
  out->d_pages = c->dev.data;
  out->pages = c->dev.pages;
  out->page_bytes = c->dev.page_bytes;
  return RTAMS_OK;
}

int rtams_cache_extend(rtams_cache *c, int64_t n, const int32_t *d_seqs, const int32_t *d_starts, void *hip_stream) {
  int rc = check_items(c, n, d_seqs);
  if (rc || n == 0) return rc;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  std::lock_guard<std::mutex> g(c->mutex);
  bool recorded = false;
  if ((rc = cache_enter(c, s, &recorded))) return rc;
  CacheRows r = items_of(n, d_seqs, d_starts, 0x7fffffff, 0x7fffffff);
  // (without a fork before this call no page can be shared; a recorded call may be launched behind a later fork)
  launch_cache_extend(c->dev, r, c->forked || recorded, s);
  return launched("extend");
}

int rtams_cache_write(rtams_cache *c, int32_t layer, int64_t n, const int32_t *d_seqs, const int32_t *d_starts, int64_t rows, int32_t max_new,
                      const void *d_k, const void *d_v, int64_t row_stride, int64_t head_stride, int32_t type, void *hip_stream) {
  int rc = check_items(c, n, d_seqs);
  if (!rc) rc = check_rows(c, layer, n, d_starts, rows, max_new);
  if (rc) return rc;
  if (type != RTAMS_TYPE_BF16 && type != RTAMS_TYPE_F16) return fail(RTAMS_EINVAL, "keys and values are bfloat16 or halves, got type %d", type);
  // (of one row, or of one head, the stride says nothing)
  if (rows == 1) row_stride = 0;
  if (c->cfg.kv_heads == 1) head_stride = 0;
  if (row_stride < 0 || row_stride >= 1 << 24 || head_stride < 0 || head_stride >= (int64_t)1 << 40)
    return fail(RTAMS_EINVAL, "strides must be in 0..2^24 - 1 elements for rows and 0..2^40 - 1 for heads, got %lld and %lld", (long long)row_stride, (long long)head_stride);
  if (n == 0 || rows == 0) return RTAMS_OK;
  if (!d_k || !d_v) return fail(RTAMS_EINVAL, "keys or values are NULL");
  if (((uintptr_t)d_k | (uintptr_t)d_v) % 2) return fail(RTAMS_EINVAL, "keys and values must be 2-byte aligned");
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  std::lock_guard<std::mutex> g(c->mutex);
  if ((rc = cache_enter(c, s))) return rc;
  const bool vec = ((uintptr_t)d_k | (uintptr_t)d_v) % 16 == 0 && row_stride % 8 == 0 && head_stride % 8 == 0;
  launch_cache_write(c->dev, items_of(n, d_seqs, d_starts, rows, max_new), layer, d_k, d_v, row_stride, head_stride, type == RTAMS_TYPE_F16, vec, s);
  return launched("write");
}

int rtams_cache_read(rtams_cache *c, int32_t layer, int64_t n, const int32_t *d_seqs, const int32_t *d_starts, int64_t rows, int32_t max_new,
                     void *d_k, void *d_v, int32_t type, void *hip_stream) {
  int rc = check_items(c, n, d_seqs);
  if (!rc) rc = check_rows(c, layer, n, d_starts, rows, max_new);
  if (rc) return rc;
  if (type < RTAMS_TYPE_BF16 || type > RTAMS_TYPE_F32) return fail(RTAMS_EINVAL, "unknown type %d", type);
  if (n == 0 || rows == 0) return RTAMS_OK;
  if (!d_k || !d_v) return fail(RTAMS_EINVAL, "keys or values are NULL");
  if (((uintptr_t)d_k | (uintptr_t)d_v) % 16) return fail(RTAMS_EINVAL, "keys and values must be 16-byte aligned");
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  std::lock_guard<std::mutex> g(c->mutex);
  if ((rc = cache_enter(c, s))) return rc;
  launch_cache_read(c->dev, items_of(n, d_seqs, d_starts, rows, max_new), layer, d_k, d_v, type, s);
  return launched("read");
}

int rtams_cache_attend(rtams_cache *c, const rtams_cache_query *q, int64_t n, const int32_t *d_seqs, const int32_t *d_starts, int64_t rows,
                       void *hip_stream) {
  int rc = check_items(c, n, d_seqs);
  if (rc) return rc;
  if (!q) return fail(RTAMS_EINVAL, "query is NULL");
  if ((rc = check_rows(c, q->layer, n, d_starts, rows, q->max_new))) return rc;
  if (q->q_heads < 1 || q->q_heads % c->cfg.kv_heads || q->q_heads > 65536)
    return fail(RTAMS_EINVAL, "q_heads must be a multiple of the cache's %d heads, got %d", c->cfg.kv_heads, q->q_heads);
  if (q->type != RTAMS_TYPE_BF16 && q->type != RTAMS_TYPE_F16) return fail(RTAMS_EINVAL, "queries are bfloat16 or halves, got type %d", q->type);
  if (q->window < 0 || (q->window > 0 && !q->causal)) return fail(RTAMS_EINVAL, "window %d: not negative, and causal only", q->window);
  if (!std::isfinite(q->scale)) return fail(RTAMS_EINVAL, "scale must be finite");
  if (n == 0 || rows == 0) return RTAMS_OK;
  if (!q->d_q || !q->d_out) return fail(RTAMS_EINVAL, "queries or output are NULL");
  if (((uintptr_t)q->d_q | (uintptr_t)q->d_out) % 2 || (uintptr_t)q->d_lse % 4) return fail(RTAMS_EINVAL, "queries, output or logarithms are not aligned to their type");
  // what the kernels count in 32 bits: rows of an item, workgroups, steps of 128 tokens
  const int64_t most = d_starts ? (q->max_new < rows ? (int64_t)q->max_new : rows) : 1, share = q->q_heads / c->cfg.kv_heads;
  const int64_t heads = n * c->cfg.kv_heads, steps = (int64_t)c->cfg.max_pages * c->cfg.page_tokens / 128 + 1;
  if (share * most >= (int64_t)1 << 30 || heads >= 1 << 22 || heads * (share * most / 128 + 1) >= 1 << 28 || heads * steps >= (int64_t)1 << 32)
    return fail(RTAMS_EINVAL, "%lld items of up to %lld rows, %d heads, are too many for one call", (long long)n, (long long)most, q->q_heads);
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  std::lock_guard<std::mutex> g(c->mutex);
  if ((rc = cache_enter(c, s))) return rc;
  CacheQuery k{};
  k.r = items_of(n, d_seqs, d_starts, rows, q->max_new);
  k.layer = q->layer;
  k.q_heads = q->q_heads;
  k.share = q->q_heads / c->cfg.kv_heads;
  k.half_type = q->type == RTAMS_TYPE_F16;
  k.causal = q->causal != 0;
  k.window = q->window;
  int twos = 0;
  const double times = (double)q->scale * 1.4426950408889634;
  std::frexp(times, &twos);
  k.scale_two = times == 0.0 ? 0.0f : (float)std::copysign(std::ldexp(1.0, twos - 1 < 127 ? twos - 1 : 127), times);
  k.scale_rest = k.scale_two == 0.0f ? 1.0f : (float)(times / k.scale_two);
  k.q = static_cast<const uint16_t *>(q->d_q);
  k.q_row = q->q_row_stride;
  k.q_head = q->q_head_stride;
  k.out = static_cast<uint16_t *>(q->d_out);
  k.out_row = q->out_row_stride;
  k.out_head = q->out_head_stride;
  k.lse = q->d_lse;
  k.vec = ((uintptr_t)q->d_q | (uintptr_t)q->d_out) % 16 == 0 && (k.q_row | k.q_head | k.out_row | k.out_head) % 8 == 0;
  launch_cache_attend(c->dev, k, s);
  return launched("attend");
}

int rtams_cache_fork(rtams_cache *c, int64_t n, const int32_t *d_src, const int32_t *d_dst, int32_t copy, void *hip_stream) {
  int rc = check_items(c, n, d_src);
  if (rc || n == 0) return rc;
  if (!d_src || !d_dst) return fail(RTAMS_EINVAL, "sources or destinations are NULL");
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  std::lock_guard<std::mutex> g(c->mutex);
  if ((rc = cache_enter(c, s))) return rc;
  c->forked |= copy == 0;
  launch_cache_fork(c->dev, (int32_t)n, d_src, d_dst, copy != 0, s);
  return launched("fork");
}

int rtams_cache_trim(rtams_cache *c, int64_t n, const int32_t *d_seqs, const int32_t *d_lengths, void *hip_stream) {
  int rc = check_items(c, n, d_seqs);
  if (rc || n == 0) return rc;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  std::lock_guard<std::mutex> g(c->mutex);
  if ((rc = cache_enter(c, s))) return rc;
  launch_cache_trim(c->dev, (int32_t)n, d_seqs, d_lengths, s);
  return launched("trim");
}

int rtams_cache_compact(rtams_cache *c, void *hip_stream) {
  if (!c) return fail(RTAMS_EINVAL, "cache is NULL");
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  std::lock_guard<std::mutex> g(c->mutex);
  int rc = cache_enter(c, s);
  if (rc) return rc;
  launch_cache_compact(c->dev, s);
  return launched("compact");
}

int rtams_cache_free_pages(rtams_cache *c, int64_t *out) {
  if (!c || !out) return fail(RTAMS_EINVAL, "cache or out is NULL");
  std::lock_guard<std::mutex> g(c->mutex);
  if (c->have_stream) HIP_TRY(hipStreamSynchronize(c->stream));
  uint32_t v = 0;
  HIP_TRY(hipMemcpy(&v, &c->dev.ctrl->free, 4, hipMemcpyDeviceToHost));
  *out = v;
  return RTAMS_OK;
}

int rtams_cache_poll_error(rtams_cache *c) {
  if (!c) return fail(RTAMS_EINVAL, "cache is NULL");
  const int e = __atomic_load_n(&c->mirror->error, __ATOMIC_RELAXED);
  if (e == RTAMS_EPOOL) return fail(e, "an extend or a copying fork found too few free pages and was dropped");
  if (e != RTAMS_OK) return fail(e, "a call's items were not what it asks for");
  return RTAMS_OK;
}

int rtams_cache_clear_error(rtams_cache *c) {
  if (!c) return fail(RTAMS_EINVAL, "cache is NULL");
  std::lock_guard<std::mutex> g(c->mutex);
  if (c->have_stream) HIP_TRY(hipStreamSynchronize(c->stream));
  k_cache_clear_stop<<<1, 1, 0, c->stream>>>(c->dev);
  int rc = launched("clear_error");
  if (rc) return rc;
  HIP_TRY(hipStreamSynchronize(c->stream));
  return RTAMS_OK;
}

}  // extern "C"
