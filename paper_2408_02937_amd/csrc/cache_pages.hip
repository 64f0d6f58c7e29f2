// Pages of the cache: room for new rows with copy on write, forks, copies, trims and compaction (include/rtams_cache.h).
//
// One workgroup of 1024 lanes plans a call: it checks every item before it changes anything, numbers the new pages by a
// prefix sum over the items and takes the lowest free ones from a bitmap, 32,768 pages a step.  What a call does is thereby
// a function of the table: counts are added with atomics, whose order shows nowhere.  Tables are small (four bytes a page); what
// moves bytes, a copy of whole pages, runs on the whole chip in pieces of 16 KiB.
//
// Planning is a chain of loads and barriers on one compute unit: 4.8 us for a token each of 48 sequences, 2 to 4 for a trim, 5.8 for a fork of 32, 6.1
// for the plan of a compaction.  Copies are bound by memory: 3.3 GB read and written in 655 us, 5.1 TB/s; 354 MB in 76 us, 4.6.
#include "../../include/rtams_cache.h"

#include "cache.h"
#include "rtams_dev.h"

namespace rtams {

namespace {

constexpr int kPlanLanes = 1024;
constexpr int kCopyBytes = 16384;   // a workgroup's piece
constexpr int kPicked = 2048;       // new pages that it keeps in LDS
constexpr int kFewEntries = kPlanLanes;  // table entries that it walks by itself

__device__ inline uint32_t lane_id() { return threadIdx.x & 63; }

struct Plan {
  uint32_t seen[kCacheMaxSeqs / 32];
  uint32_t waves[kPlanLanes / 64];
  int32_t picked[kPicked];
  // of 1024 items: sequence, first new entry and the first page for it, and how many new entries the items in front have
  int32_t seq[kPlanLanes], page0[kPlanLanes];
  uint32_t off[kPlanLanes], before[kPlanLanes];
  uint32_t pairs, freed;
};

// Exclusive prefix sum over the workgroup; *total to every lane, in 64 bits: a lane may ask for all pages of a long sequence, 2^25 of
// them, which 64 lanes do within 32 bits and 1024 do not.  (Where *total is beyond 32 bits the prefix sums are not to be used.)
__device__ inline uint32_t scan_lanes(uint32_t v, uint64_t *total, Plan &sh) {
  const uint32_t inc = wave_running_sum(v);
  __syncthreads();
  if (lane_id() == 63) sh.waves[threadIdx.x >> 6] = inc;
  __syncthreads();
  uint32_t before = 0;
  uint64_t all = 0;
#pragma unroll
  for (int w = 0; w < kPlanLanes / 64; ++w) {
    const uint32_t x = sh.waves[w];
    before += w < (int)(threadIdx.x >> 6) ? x : 0;
    all += x;
  }
  *total = all;
  return before + inc - v;
}

// Takes the `total` lowest free pages, which there are, in order: the first ones into LDS, the others into memory.
__device__ void pick_pages(const CacheDev &d, uint32_t total, Plan &sh) {
  const uint32_t words = (d.pages + 31) / 32;
  uint32_t found = 0;
  for (uint32_t base = 0; base < words && found < total; base += kPlanLanes) {
    const uint32_t at = base + threadIdx.x;
    uint32_t w = at < words ? d.free_bits[at] : 0;
    uint64_t here;
    uint32_t rank = found + scan_lanes(__popc(w), &here, sh);
    const uint32_t before = w;
    for (uint32_t x = w; x && rank < total; x &= x - 1, ++rank) {
      const int bit = __ffs(x) - 1;
      if (rank < kPicked) sh.picked[rank] = (int32_t)(at * 32 + bit);
      else d.picked[rank] = (int32_t)(at * 32 + bit);
      w &= ~(1u << bit);
    }
    if (w != before) d.free_bits[at] = w;
    found += (uint32_t)here;
  }
  __syncthreads();
}

__device__ inline int32_t picked_page(const CacheDev &d, const Plan &sh, uint32_t rank) { return rank < kPicked ? sh.picked[rank] : d.picked[rank]; }

__device__ inline void put_back(const CacheDev &d, int32_t page) { atomicOr(&d.free_bits[page >> 5], 1u << (page & 31)); }

__device__ inline bool named_before(uint32_t *seen, int32_t seq) { return (atomicOr(&seen[seq >> 5], 1u << (seq & 31)) >> (seq & 31)) & 1; }

__device__ inline int32_t pages_for(const CacheDev &d, int64_t tokens) { return (int32_t)((tokens + d.page_tokens - 1) / d.page_tokens); }

__device__ inline void clear_seen(const CacheDev &d, Plan &sh) {
  for (int i = threadIdx.x; i < (d.max_seqs + 31) / 32; i += kPlanLanes) sh.seen[i] = 0;
  if (threadIdx.x == 0) sh.pairs = sh.freed = 0;
  __syncthreads();
}

// The call is dropped.
__device__ inline void drop(const CacheDev &d, int code) {
  if (threadIdx.x == 0) {
    d.ctrl->pairs = 0;
    d.ctrl->ok = 0;
    cache_raise(d, code);
  }
}

// Entry e of the up to 1024 items in LDS: which of them it is.
__device__ inline int item_of(const Plan &sh, uint32_t e) {
  int lo = 0, hi = kPlanLanes - 1;
  while (lo < hi) {  // the last one that begins at e or before
    const int mid = (lo + hi + 1) / 2;
    if (sh.before[mid] <= e) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__global__ __launch_bounds__(kPlanLanes) void k_cache_extend(CacheDev d, CacheRows r) {
  __shared__ Plan sh;
  clear_seen(d, sh);
  uint32_t total = 0;
  int bad = 0, short_of = 0;
  CacheItem it{};
  for (int base = 0; base < r.n; base += kPlanLanes) {
    const int i = base + threadIdx.x;
    uint32_t need = 0;
    it = CacheItem{};
    if (i < r.n) {
      int64_t first;
      int count;
      const int s = cache_item_seq(r, i);
      const bool rows = cache_item_rows(r, i, &first, &count);
      if (!rows || (uint32_t)s >= (uint32_t)d.max_seqs || named_before(sh.seen, s)) {
        bad = 1;
      } else {
        const int length = d.lengths[s];
        if ((int64_t)length + count > (int64_t)d.max_pages * d.page_tokens) {
          bad = 1;
        } else {
          it.seq = s;
          it.src = length + count;
          it.have = pages_for(d, length);
          it.want = pages_for(d, (int64_t)length + count);
          it.copy = count > 0 && length % d.page_tokens && d.refs[d.table[(int64_t)s * d.max_pages + it.have - 1]] > 1;
          need = (uint32_t)(it.want - it.have + it.copy);
        }
      }
    }
    uint64_t here;
    it.off = total + scan_lanes(need, &here, sh);
    if (r.n > kPlanLanes && i < r.n) d.items[i] = it;
    short_of = here > d.pages - total;
    bad = __syncthreads_or(bad);
    if (bad || short_of) break;
    total += (uint32_t)here;
  }
  if (bad || short_of || total > d.ctrl->free) {
    __syncthreads();
    if (threadIdx.x == 0) d.ctrl->stopped = 1;
    return drop(d, bad ? RTAMS_EINVAL : RTAMS_EPOOL);
  }
  if (total) pick_pages(d, total, sh);
  // few new entries, or a row for each item and so a page at most, are this workgroup's work, others the next launch's
  const bool here_too = total <= kPlanLanes || !r.starts;
  for (int base = 0; base < r.n; base += kPlanLanes) {
    const int i = base + threadIdx.x;
    if (r.n > kPlanLanes) it = i < r.n ? d.items[i] : CacheItem{};
    else if (!here_too && i < r.n) d.items[i] = it;
    if (i < r.n) {
      if (it.copy) {
        int32_t *last = d.table + (int64_t)it.seq * d.max_pages + it.have - 1;
        const int32_t from = *last, to = picked_page(d, sh, it.off);
        *last = to;
        d.refs[to] = 1;
        if (atomicSub(&d.refs[from], 1) == 1) {  // all that shared it got copies
          put_back(d, from);
          atomicAdd(&sh.freed, 1u);
        }
        const uint32_t at = atomicAdd(&sh.pairs, 1u);
        d.pair_src[at] = from;
        d.pair_dst[at] = to;
      }
      d.lengths[it.seq] = it.src;
    }
    if (!here_too) continue;
    uint64_t fresh;
    sh.before[threadIdx.x] = scan_lanes(i < r.n ? (uint32_t)(it.want - it.have) : 0, &fresh, sh);
    if (fresh == 0) continue;
    sh.seq[threadIdx.x] = it.seq;
    sh.page0[threadIdx.x] = it.have;
    sh.off[threadIdx.x] = it.off + it.copy;
    __syncthreads();
    if (threadIdx.x < fresh) {
      const int x = item_of(sh, threadIdx.x);
      const uint32_t nth = threadIdx.x - sh.before[x];
      const int32_t page = picked_page(d, sh, sh.off[x] + nth);
      d.table[(int64_t)sh.seq[x] * d.max_pages + sh.page0[x] + nth] = page;
      d.refs[page] = 1;
    }
    __syncthreads();
  }
  if (!here_too)
    for (uint32_t x = threadIdx.x; x < total && x < kPicked; x += kPlanLanes) d.picked[x] = sh.picked[x];
  __syncthreads();
  if (threadIdx.x == 0) {
    d.ctrl->free += sh.freed - total;
    d.ctrl->pairs = sh.pairs;
    d.ctrl->ok = here_too ? 0 : 1;  // whether entries are left to the next launch
    d.ctrl->stopped = 0;
  }
}

// Table entries of the call's items, 64 at a time.
template <class F>
__device__ void each_entry(const CacheDev &d, int n, F f) {
  const uint32_t per = (uint32_t)(d.max_pages + 63) / 64;
  uint32_t i = (blockIdx.x * 4 + (threadIdx.x >> 6)) / per, chunk = (blockIdx.x * 4 + (threadIdx.x >> 6)) % per;
  const uint32_t step_i = gridDim.x * 4 / per, step_chunk = gridDim.x * 4 % per;
  while (i < (uint32_t)n) {
    f(d.items[i], (int)(chunk * 64 + lane_id()));
    i += step_i;
    chunk += step_chunk;
    if (chunk >= per) {
      chunk -= per;
      ++i;
    }
  }
}

__global__ __launch_bounds__(256) void k_cache_extend_entries(CacheDev d, int32_t n) {
  if (!d.ctrl->ok) return;
  each_entry(d, n, [&](const CacheItem &it, int p) {
    if (p < it.have || p >= it.want) return;
    const int32_t page = d.picked[it.off + it.copy + (p - it.have)];
    d.table[(int64_t)it.seq * d.max_pages + p] = page;
    d.refs[page] = 1;
  });
}

// Entry p of a sequence that gives it up; true where the page is free now.
__device__ inline bool give_up(const CacheDev &d, int32_t seq, int p) {
  int32_t *e = d.table + (int64_t)seq * d.max_pages + p;
  const int32_t page = *e;
  *e = -1;
  const bool gone = atomicSub(&d.refs[page], 1) == 1;
  if (gone) put_back(d, page);
  return gone;
}

// few: at most 1024 items, and their entries are this workgroup's work.
__global__ __launch_bounds__(kPlanLanes) void k_cache_trim(CacheDev d, int32_t n, const int32_t *seqs, const int32_t *lengths, int few) {
  __shared__ Plan sh;
  clear_seen(d, sh);
  int bad = 0;
  CacheItem it{};
  for (int i = threadIdx.x; i < n; i += kPlanLanes) {
    const int s = seqs ? seqs[i] : i, to = lengths ? lengths[i] : 0;
    if ((uint32_t)s >= (uint32_t)d.max_seqs || named_before(sh.seen, s)) {
      bad = 1;
    } else {
      const int length = d.lengths[s];
      bad |= to < 0 || to > length;
      it.seq = s;
      it.src = to;
      it.have = pages_for(d, length);
      it.want = pages_for(d, to);
      if (!few) d.items[i] = it;
    }
  }
  if (__syncthreads_or(bad)) return drop(d, RTAMS_EINVAL);
  if (threadIdx.x == 0) d.ctrl->ok = 1;
  if (!few) return;
  if ((int)threadIdx.x < n) d.lengths[it.seq] = it.src;
  uint64_t entries;
  sh.before[threadIdx.x] = scan_lanes((uint32_t)(it.have - it.want), &entries, sh);
  sh.seq[threadIdx.x] = it.seq;
  sh.page0[threadIdx.x] = it.want;
  __syncthreads();
  uint32_t gone = 0;
  for (uint32_t e = threadIdx.x; e < entries; e += kPlanLanes) {
    const int x = item_of(sh, e);
    gone += give_up(d, sh.seq[x], sh.page0[x] + (int)(e - sh.before[x]));
  }
  if (gone) atomicAdd(&d.ctrl->free, gone);
}

__global__ __launch_bounds__(256) void k_cache_trim_entries(CacheDev d, int32_t n) {
  if (!d.ctrl->ok) return;
  each_entry(d, n, [&](const CacheItem &it, int p) {
    if (p == 0) d.lengths[it.seq] = it.src;
    const uint64_t all = __ballot(p >= it.want && p < it.have && give_up(d, it.seq, p));
    if (all && lane_id() == 0) atomicAdd(&d.ctrl->free, (uint32_t)__popcll(all));
  });
}

// Of rows that are kept: the items, and whether the call holds.  src: position of the first row, off: rows kept, copy: rows.
__global__ __launch_bounds__(kPlanLanes) void k_cache_keep_plan(CacheDev d, CacheRows r, const int32_t *path, const int32_t *kept) {
  __shared__ Plan sh;
  clear_seen(d, sh);
  int bad = 0;
  for (int i = threadIdx.x; i < r.n; i += kPlanLanes) {
    int64_t first;
    int count;
    const int s = cache_item_seq(r, i), k = kept[i];
    const bool rows = cache_item_rows(r, i, &first, &count);
    if (!rows || (uint32_t)s >= (uint32_t)d.max_seqs || named_before(sh.seen, s)) {
      bad = 1;
      continue;
    }
    const int length = d.lengths[s], base = length - count;
    if (count > length || k < 0 || k > count) {
      bad = 1;
      continue;
    }
    int before = -1, moved = k;  // (the first row that moves: those behind it do)
    for (int j = 0; j < k; j += 8) {
      int p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = path[first + min(j + e, k - 1)];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (j + e >= k) break;
        bad |= p[e] <= before || p[e] >= count;
        before = p[e];
        if (p[e] != j + e) moved = min(moved, j + e);
      }
    }
    // (another sequence's rows are not written over)
    for (int page = (base + moved) / d.page_tokens; moved < k && page <= (base + k - 1) / d.page_tokens; ++page) bad |= d.refs[d.table[(int64_t)s * d.max_pages + page]] != 1;
    d.items[i] = CacheItem{s, base, pages_for(d, length), pages_for(d, (int64_t)base + k), (uint32_t)k, count, {}};
  }
  if (__syncthreads_or(bad)) return drop(d, RTAMS_EINVAL);
  if (threadIdx.x == 0) d.ctrl->ok = d.ctrl->stopped == 0;
}

__global__ __launch_bounds__(256) void k_cache_keep_cut(CacheDev d, int32_t n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (!d.ctrl->ok || i >= n) return;
  const CacheItem it = d.items[i];
  d.lengths[it.seq] = it.src + (int)it.off;
  uint32_t gone = 0;
  for (int p = it.want; p < it.have; ++p) gone += give_up(d, it.seq, p);
  if (gone) atomicAdd(&d.ctrl->free, gone);
}

// Entry p of a fork's destination; copy: a page of its own, pair `pair` of the call.
__device__ inline void take_over(const CacheDev &d, int32_t src, int32_t dst, int p, bool copy, uint32_t pair, int32_t own) {
  const int32_t page = d.table[(int64_t)src * d.max_pages + p];
  d.table[(int64_t)dst * d.max_pages + p] = copy ? own : page;
  if (copy) {
    d.refs[own] = 1;
    d.pair_src[pair] = page;
    d.pair_dst[pair] = own;
  } else {
    atomicAdd(&d.refs[page], 1);
  }
}

__global__ __launch_bounds__(kPlanLanes) void k_cache_fork(CacheDev d, int32_t n, const int32_t *src, const int32_t *dst, int copy, int few) {
  __shared__ Plan sh;
  clear_seen(d, sh);
  int bad = 0, short_of = 0;
  for (int i = threadIdx.x; i < n; i += kPlanLanes) {
    const int s = dst[i];
    bad |= (uint32_t)s >= (uint32_t)d.max_seqs || named_before(sh.seen, s) || d.lengths[s] != 0;
  }
  bad = __syncthreads_or(bad);
  uint32_t total = 0;
  CacheItem it{};
  for (int base = 0; base < n && !bad && !short_of; base += kPlanLanes) {
    const int i = base + threadIdx.x;
    uint32_t need = 0;
    uint64_t here;
    it = CacheItem{};
    if (i < n) {
      const int s = src[i];
      if ((uint32_t)s >= (uint32_t)d.max_seqs || (sh.seen[s >> 5] >> (s & 31)) & 1) {
        bad = 1;
      } else {
        it.seq = dst[i];
        it.src = s;
        it.want = d.lengths[s];
        it.have = pages_for(d, it.want);
        it.copy = copy;
        need = copy ? (uint32_t)it.have : 0;
      }
    }
    it.off = total + scan_lanes(need, &here, sh);
    if (i < n && !few) d.items[i] = it;
    short_of = here > d.pages - total;  // (a source may be named by every item: the sum is not bounded by the pages there are)
    total += (uint32_t)here;
    bad = __syncthreads_or(bad);
  }
  if (bad || short_of || total > d.ctrl->free) {
    __syncthreads();
    return drop(d, bad ? RTAMS_EINVAL : RTAMS_EPOOL);
  }
  if (total) pick_pages(d, total, sh);
  __syncthreads();
  if (threadIdx.x == 0) {
    d.ctrl->free -= total;
    d.ctrl->pairs = total;
    d.ctrl->ok = 1;
  }
  if (!few) {
    for (uint32_t x = threadIdx.x; x < total && x < kPicked; x += kPlanLanes) d.picked[x] = sh.picked[x];
    return;
  }
  if ((int)threadIdx.x < n) d.lengths[it.seq] = it.want;
  uint64_t entries;
  sh.before[threadIdx.x] = scan_lanes((uint32_t)it.have, &entries, sh);
  sh.seq[threadIdx.x] = it.seq;
  sh.page0[threadIdx.x] = it.src;
  sh.off[threadIdx.x] = it.off;
  __syncthreads();
  for (uint32_t e = threadIdx.x; e < entries; e += kPlanLanes) {
    const int x = item_of(sh, e);
    const uint32_t p = e - sh.before[x], pair = sh.off[x] + p;
    take_over(d, sh.page0[x], sh.seq[x], (int)p, copy, pair, copy ? picked_page(d, sh, pair) : 0);
  }
}

__global__ __launch_bounds__(256) void k_cache_fork_entries(CacheDev d, int32_t n) {
  if (!d.ctrl->ok) return;
  each_entry(d, n, [&](const CacheItem &it, int p) {
    if (p == 0) d.lengths[it.seq] = it.want;
    if (p < it.have) take_over(d, it.src, it.seq, p, it.copy, it.off + p, it.copy ? d.picked[it.off + p] : 0);
  });
}

// Which pages go where.  Free pages below the number in use and used ones from there on are equally many.
__global__ __launch_bounds__(kPlanLanes) void k_cache_compact(CacheDev d) {
  __shared__ Plan sh;
  const uint32_t used = d.pages - d.ctrl->free, words = (d.pages + 31) / 32;
  uint32_t holes = 0, movers = 0;
  for (uint32_t base = 0; base < words; base += kPlanLanes) {
    const uint32_t at = base + threadIdx.x;
    uint32_t low = 0, high = 0;  // free below `used`, used above
    if (at < words) {
      const uint32_t w = d.free_bits[at], first = at * 32;
      const uint32_t real = d.pages - first >= 32 ? ~0u : (1u << (d.pages - first)) - 1u;
      const uint32_t below = used <= first ? 0 : used - first >= 32 ? ~0u : (1u << (used - first)) - 1u;
      low = w & below;
      high = ~w & real & ~below;
      if (low | high) d.free_bits[at] = real & ~below;
    }
    uint64_t all_low, all_high;
    uint32_t a = holes + scan_lanes(__popc(low), &all_low, sh), b = movers + scan_lanes(__popc(high), &all_high, sh);
    for (uint32_t x = low; x; x &= x - 1) d.pair_dst[a++] = (int32_t)(at * 32 + __ffs(x) - 1);
    for (uint32_t x = high; x; x &= x - 1) d.pair_src[b++] = (int32_t)(at * 32 + __ffs(x) - 1);
    holes += (uint32_t)all_low;
    movers += (uint32_t)all_high;
  }
  __syncthreads();
  for (uint32_t j = threadIdx.x; j < movers; j += kPlanLanes) {
    const int32_t from = d.pair_src[j], to = d.pair_dst[j];
    d.map[from] = to;
    d.refs[to] = d.refs[from];
    d.refs[from] = 0;
  }
  if (threadIdx.x == 0) {
    d.ctrl->pairs = movers;
    d.ctrl->used = used;
  }
}

// Copies the call's pairs of pages, all layers; the first `renames` workgroups rewrite the table after a compaction instead.
__global__ __launch_bounds__(256) void k_cache_move(CacheDev d, int renames) {
  const uint32_t pairs = d.ctrl->pairs;
  if (pairs == 0) return;
  if ((int)blockIdx.x < renames) {
    const uint32_t used = d.ctrl->used;
    for (int s = blockIdx.x; s < d.max_seqs; s += renames)
      for (int p = threadIdx.x, n = pages_for(d, d.lengths[s]); p < n; p += 256) {
        int32_t *e = d.table + (int64_t)s * d.max_pages + p;
        if ((uint32_t)*e >= used) *e = d.map[*e];
      }
    return;
  }
  const uint32_t pieces = (uint32_t)((d.page_bytes + kCopyBytes - 1) / kCopyBytes), per_pair = pieces * (uint32_t)d.layers;
  const uint64_t units = (uint64_t)pairs * per_pair;
  for (uint64_t u = blockIdx.x - renames; u < units; u += gridDim.x - renames) {
    const uint32_t pair = (uint32_t)(u / per_pair), rest = (uint32_t)(u % per_pair), layer = rest / pieces, piece = rest % pieces;
    const int64_t at = (int64_t)piece * kCopyBytes, page0 = (int64_t)layer * d.pages;
    const uint4 *from = reinterpret_cast<const uint4 *>(d.data + (page0 + d.pair_src[pair]) * d.page_bytes + at);
    uint4 *to = reinterpret_cast<uint4 *>(d.data + (page0 + d.pair_dst[pair]) * d.page_bytes + at);
    const int n = (int)((d.page_bytes - at < kCopyBytes ? d.page_bytes - at : kCopyBytes) / 16);
    uint4 x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = (int)threadIdx.x + 256 * j < n ? from[threadIdx.x + 256 * j] : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if ((int)threadIdx.x + 256 * j < n) to[threadIdx.x + 256 * j] = x[j];
  }
}

// Workgroups for a copy of at most `pairs` pages: a piece each, up to eight to a compute unit.
int copy_groups(const CacheDev &d, int64_t pairs) {
  const int64_t units = pairs * d.layers * ((d.page_bytes + kCopyBytes - 1) / kCopyBytes);
  return (int)(units < 2048 ? units : 2048);
}

int entry_groups(const CacheDev &d, int64_t n) {
  const int64_t groups = (n * ((d.max_pages + 63) / 64) + 3) / 4;
  return (int)(groups < 2048 ? groups : 2048);
}

}  // namespace

// An entry to a lane of the planning workgroup costs what a launch does (64 sequences of 16 pages trimmed and extended: 26 us, 24 with launches
// of their own; 4 of 16: 16 and 19), two more (8 of 256: 39 and 27), sixteen far more (64 of 256: 155 and 32).
static bool few_entries(const CacheDev &d, int64_t n) { return n <= kPlanLanes && n * d.max_pages <= kFewEntries; }

void launch_cache_extend(const CacheDev &d, const CacheRows &r, bool copies, hipStream_t s) {
  k_cache_extend<<<1, kPlanLanes, 0, s>>>(d, r);
  if (r.starts && (int64_t)r.n * d.max_pages > kPlanLanes) k_cache_extend_entries<<<entry_groups(d, r.n), 256, 0, s>>>(d, r.n);
  if (copies) k_cache_move<<<copy_groups(d, r.n), 256, 0, s>>>(d, 0);
}

void launch_cache_trim(const CacheDev &d, int32_t n, const int32_t *seqs, const int32_t *lengths, hipStream_t s) {
  const bool few = few_entries(d, n);
  k_cache_trim<<<1, kPlanLanes, 0, s>>>(d, n, seqs, lengths, few);
  if (!few) k_cache_trim_entries<<<entry_groups(d, n), 256, 0, s>>>(d, n);
}

void launch_cache_keep_plan(const CacheDev &d, const CacheRows &r, const int32_t *path, const int32_t *kept, hipStream_t s) {
  k_cache_keep_plan<<<1, kPlanLanes, 0, s>>>(d, r, path, kept);
}

void launch_cache_keep_cut(const CacheDev &d, int32_t n, hipStream_t s) { k_cache_keep_cut<<<(n + 255) / 256, 256, 0, s>>>(d, n); }

void launch_cache_fork(const CacheDev &d, int32_t n, const int32_t *src, const int32_t *dst, bool copy, hipStream_t s) {
  const bool few = few_entries(d, n);
  k_cache_fork<<<1, kPlanLanes, 0, s>>>(d, n, src, dst, copy, few);
  if (!few) k_cache_fork_entries<<<entry_groups(d, n), 256, 0, s>>>(d, n);
  if (copy) k_cache_move<<<copy_groups(d, (int64_t)n * d.max_pages), 256, 0, s>>>(d, 0);
}

void launch_cache_compact(const CacheDev &d, hipStream_t s) {
  k_cache_compact<<<1, kPlanLanes, 0, s>>>(d);
  const int renames = d.max_seqs < 1024 ? d.max_seqs : 1024;
  k_cache_move<<<renames + copy_groups(d, d.pages), 256, 0, s>>>(d, renames);
}

}  // namespace rtams
