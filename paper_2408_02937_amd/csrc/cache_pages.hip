// Pages of the cache: room for new rows with copy on write, forks, copies, trims and compaction (include/rtams_cache.h).
//
// One workgroup of 1024 lanes plans a call: it checks every item before it changes anything, numbers the new pages by a
// prefix sum over the items and takes the lowest free ones from a bitmap, 32,768 pages a step.  What a call does is thereby
// a function of the table: counts are added with atomics, whose order shows nowhere.  Tables are small (four bytes a page); what
// moves bytes, a copy of whole pages, runs on the whole chip in pieces of 16 KiB.
#include "../../include/rtams_cache.h"

#include "cache.h"

namespace rtams {

namespace {

constexpr int kPlanLanes = 1024;
constexpr int kCopyBytes = 16384;   // a workgroup's piece
constexpr int kInlineSlots = 16384; // table entries that the planning workgroup walks by itself

__device__ inline uint32_t lane_id() { return threadIdx.x & 63; }

// Exclusive prefix sum over the workgroup; *total to every lane.
__device__ inline uint32_t scan_lanes(uint32_t v, uint32_t *total) {
  __shared__ uint32_t waves[kPlanLanes / 64];
  uint32_t inc = v;
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t x = __shfl_up(inc, o);
    if (lane_id() >= (uint32_t)o) inc += x;
  }
  __syncthreads();
  if (lane_id() == 63) waves[threadIdx.x >> 6] = inc;
  __syncthreads();
  uint32_t before = 0, all = 0;
  for (int w = 0; w < kPlanLanes / 64; ++w) {
    const uint32_t x = waves[w];
    before += w < (int)(threadIdx.x >> 6) ? x : 0;
    all += x;
  }
  *total = all;
  return before + inc - v;
}

// Takes the `total` lowest free pages, which there are, in order into picked.
__device__ void pick_pages(const CacheDev &d, uint32_t total) {
  const uint32_t words = (d.pages + 31) / 32;
  uint32_t found = 0;
  for (uint32_t base = 0; base < words && found < total; base += kPlanLanes) {
    const uint32_t at = base + threadIdx.x;
    uint32_t w = at < words ? d.free_bits[at] : 0, here;
    uint32_t rank = found + scan_lanes(__popc(w), &here);
    const uint32_t before = w;
    for (uint32_t x = w; x && rank < total; x &= x - 1, ++rank) {
      const int bit = __ffs(x) - 1;
      d.picked[rank] = (int32_t)(at * 32 + bit);
      w &= ~(1u << bit);
    }
    if (w != before) d.free_bits[at] = w;
    found += here;
  }
  __syncthreads();
}

__device__ inline void put_back(const CacheDev &d, int32_t page) { atomicOr(&d.free_bits[page >> 5], 1u << (page & 31)); }

__device__ inline bool named_before(uint32_t *seen, int32_t seq) { return (atomicOr(&seen[seq >> 5], 1u << (seq & 31)) >> (seq & 31)) & 1; }

__device__ inline int32_t pages_for(const CacheDev &d, int64_t tokens) { return (int32_t)((tokens + d.page_tokens - 1) / d.page_tokens); }

// The call is dropped.
__device__ inline void drop(const CacheDev &d, int code) {
  if (threadIdx.x == 0) {
    d.ctrl->pairs = 0;
    d.ctrl->ok = 0;
    cache_raise(d, code);
  }
}

__global__ __launch_bounds__(kPlanLanes) void k_cache_extend(CacheDev d, CacheRows r) {
  __shared__ uint32_t seen[kCacheMaxSeqs / 32];
  __shared__ int32_t big[kPlanLanes];
  __shared__ uint32_t nbig, npairs, nfreed;
  for (int i = threadIdx.x; i < (d.max_seqs + 31) / 32; i += kPlanLanes) seen[i] = 0;
  if (threadIdx.x == 0) npairs = nfreed = 0;
  __syncthreads();
  uint32_t total = 0;
  int bad = 0, short_of = 0;
  for (int base = 0; base < r.n; base += kPlanLanes) {
    const int i = base + threadIdx.x;
    uint32_t need = 0;
    CacheItem it{};
    if (i < r.n) {
      int64_t first;
      int count;
      const int s = cache_item_seq(r, i);
      if (!cache_item_rows(r, i, &first, &count) || (uint32_t)s >= (uint32_t)d.max_seqs || named_before(seen, s) ||
          (int64_t)d.lengths[s] + count > (int64_t)d.max_pages * d.page_tokens) {
        bad = 1;
      } else {
        const int length = d.lengths[s];
        it.seq = s;
        it.src = length + count;
        it.have = pages_for(d, length);
        it.want = pages_for(d, (int64_t)length + count);
        it.copy = count > 0 && length % d.page_tokens && d.refs[d.table[(int64_t)s * d.max_pages + it.have - 1]] > 1;
        need = (uint32_t)(it.want - it.have + it.copy);
      }
    }
    uint32_t here;
    it.off = total + scan_lanes(need, &here);
    if (i < r.n) d.items[i] = it;
    short_of |= here > d.pages - total;  // (sums of a call stay below 2^32)
    if (__syncthreads_or(bad | short_of)) break;
    total += here;
  }
  bad = __syncthreads_or(bad);
  short_of = __syncthreads_or(short_of);
  if (bad || short_of || total > d.ctrl->free) {
    __syncthreads();
    if (threadIdx.x == 0) d.ctrl->stopped = 1;
    return drop(d, bad ? RTAMS_EINVAL : RTAMS_EPOOL);
  }
  if (total) pick_pages(d, total);
  for (int base = 0; base < r.n; base += kPlanLanes) {
    if (threadIdx.x == 0) nbig = 0;
    __syncthreads();
    const int i = base + threadIdx.x;
    if (i < r.n) {
      const CacheItem it = d.items[i];
      int32_t *row = d.table + (int64_t)it.seq * d.max_pages;
      if (it.copy) {
        const int32_t from = row[it.have - 1], to = d.picked[it.off];
        row[it.have - 1] = to;
        d.refs[to] = 1;
        if (atomicSub(&d.refs[from], 1) == 1) {  // all that shared it got copies
          put_back(d, from);
          atomicAdd(&nfreed, 1u);
        }
        const uint32_t at = atomicAdd(&npairs, 1u);
        d.pair_src[at] = from;
        d.pair_dst[at] = to;
      }
      if (it.want - it.have <= 4) {
        for (int p = it.have; p < it.want; ++p) {
          const int32_t page = d.picked[it.off + it.copy + (p - it.have)];
          row[p] = page;
          d.refs[page] = 1;
        }
      } else {
        big[atomicAdd(&nbig, 1u)] = i;
      }
      d.lengths[it.seq] = it.src;
    }
    __syncthreads();
    for (uint32_t b = 0; b < nbig; ++b) {
      const CacheItem it = d.items[big[b]];
      int32_t *row = d.table + (int64_t)it.seq * d.max_pages;
      for (int p = it.have + (int)threadIdx.x; p < it.want; p += kPlanLanes) {
        const int32_t page = d.picked[it.off + it.copy + (p - it.have)];
        row[p] = page;
        d.refs[page] = 1;
      }
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    d.ctrl->free += nfreed - total;
    d.ctrl->pairs = npairs;
    d.ctrl->ok = 1;
    d.ctrl->stopped = 0;
  }
}

// Table entries of the call's items, 64 at a time, by `waves` wavefronts of which this is number `wave`.
template <class F>
__device__ void each_entry(const CacheDev &d, int n, int wave, int waves, F f) {
  const int per = (d.max_pages + 63) / 64;
  for (int64_t u = wave; u < (int64_t)n * per; u += waves) {
    const int i = (int)(u / per);
    f(i, d.items[i], (int)(u % per) * 64 + (int)lane_id());
  }
}

__device__ void trim_entries(const CacheDev &d, int n, int wave, int waves) {
  each_entry(d, n, wave, waves, [&](int, const CacheItem &it, int p) {
    bool gone = false;
    if (p >= it.want && p < it.have) {
      int32_t *e = d.table + (int64_t)it.seq * d.max_pages + p;
      const int32_t page = *e;
      *e = -1;
      gone = atomicSub(&d.refs[page], 1) == 1;
      if (gone) put_back(d, page);
    }
    const uint64_t all = __ballot(gone);
    if (all && lane_id() == 0) atomicAdd(&d.ctrl->free, (uint32_t)__popcll(all));
  });
}

__global__ __launch_bounds__(kPlanLanes) void k_cache_trim(CacheDev d, int32_t n, const int32_t *seqs, const int32_t *lengths, int inline_too) {
  __shared__ uint32_t seen[kCacheMaxSeqs / 32];
  for (int i = threadIdx.x; i < (d.max_seqs + 31) / 32; i += kPlanLanes) seen[i] = 0;
  __syncthreads();
  int bad = 0;
  for (int i = threadIdx.x; i < n; i += kPlanLanes) {
    const int s = seqs ? seqs[i] : i, to = lengths ? lengths[i] : 0;
    if ((uint32_t)s >= (uint32_t)d.max_seqs || named_before(seen, s) || to < 0 || to > d.lengths[s]) {
      bad = 1;
    } else {
      CacheItem it{};
      it.seq = s;
      it.src = to;
      it.have = pages_for(d, d.lengths[s]);
      it.want = pages_for(d, to);
      d.items[i] = it;
    }
  }
  if (__syncthreads_or(bad)) return drop(d, RTAMS_EINVAL);
  for (int i = threadIdx.x; i < n; i += kPlanLanes) d.lengths[d.items[i].seq] = d.items[i].src;
  if (threadIdx.x == 0) d.ctrl->ok = 1;
  if (inline_too) trim_entries(d, n, threadIdx.x >> 6, kPlanLanes / 64);
}

__global__ __launch_bounds__(256) void k_cache_trim_entries(CacheDev d, int32_t n) {
  if (d.ctrl->ok) trim_entries(d, n, blockIdx.x * 4 + (threadIdx.x >> 6), gridDim.x * 4);
}

__device__ void fork_entries(const CacheDev &d, int n, int wave, int waves) {
  each_entry(d, n, wave, waves, [&](int, const CacheItem &it, int p) {
    if (p == 0) d.lengths[it.seq] = d.lengths[it.src];
    if (p >= it.have) return;
    const int32_t page = d.table[(int64_t)it.src * d.max_pages + p];
    int32_t *to = d.table + (int64_t)it.seq * d.max_pages + p;
    if (it.copy) {
      const int32_t own = d.picked[it.off + p];
      *to = own;
      d.refs[own] = 1;
      d.pair_src[it.off + p] = page;
      d.pair_dst[it.off + p] = own;
    } else {
      *to = page;
      atomicAdd(&d.refs[page], 1);
    }
  });
}

__global__ __launch_bounds__(kPlanLanes) void k_cache_fork(CacheDev d, int32_t n, const int32_t *src, const int32_t *dst, int copy, int inline_too) {
  __shared__ uint32_t seen[kCacheMaxSeqs / 32];
  for (int i = threadIdx.x; i < (d.max_seqs + 31) / 32; i += kPlanLanes) seen[i] = 0;
  __syncthreads();
  int bad = 0, short_of = 0;
  for (int i = threadIdx.x; i < n; i += kPlanLanes) {
    const int s = dst[i];
    bad |= (uint32_t)s >= (uint32_t)d.max_seqs || named_before(seen, s) || d.lengths[s] != 0;
  }
  bad = __syncthreads_or(bad);
  uint32_t total = 0;
  for (int base = 0; base < n && !bad && !short_of; base += kPlanLanes) {
    const int i = base + threadIdx.x;
    uint32_t need = 0, here;
    CacheItem it{};
    if (i < n) {
      const int s = src[i];
      if ((uint32_t)s >= (uint32_t)d.max_seqs || (seen[s >> 5] >> (s & 31)) & 1) {
        bad = 1;
      } else {
        it.seq = dst[i];
        it.src = s;
        it.have = it.want = pages_for(d, d.lengths[s]);
        it.copy = copy;
        need = copy ? (uint32_t)it.have : 0;
      }
    }
    it.off = total + scan_lanes(need, &here);
    if (i < n) d.items[i] = it;
    short_of = here > d.pages - total;
    total += here;
    bad = __syncthreads_or(bad);
  }
  if (bad || short_of || total > d.ctrl->free) {
    __syncthreads();
    return drop(d, bad ? RTAMS_EINVAL : RTAMS_EPOOL);
  }
  if (total) pick_pages(d, total);
  __syncthreads();
  if (threadIdx.x == 0) {
    d.ctrl->free -= total;
    d.ctrl->pairs = total;
    d.ctrl->ok = 1;
  }
  if (inline_too) fork_entries(d, n, threadIdx.x >> 6, kPlanLanes / 64);
}

__global__ __launch_bounds__(256) void k_cache_fork_entries(CacheDev d, int32_t n) {
  if (d.ctrl->ok) fork_entries(d, n, blockIdx.x * 4 + (threadIdx.x >> 6), gridDim.x * 4);
}

// Which pages go where.  Free pages below the number in use and used ones from there on are equally many.
__global__ __launch_bounds__(kPlanLanes) void k_cache_compact(CacheDev d) {
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
    uint32_t all_low, all_high;
    uint32_t a = holes + scan_lanes(__popc(low), &all_low), b = movers + scan_lanes(__popc(high), &all_high);
    for (uint32_t x = low; x; x &= x - 1) d.pair_dst[a++] = (int32_t)(at * 32 + __ffs(x) - 1);
    for (uint32_t x = high; x; x &= x - 1) d.pair_src[b++] = (int32_t)(at * 32 + __ffs(x) - 1);
    holes += all_low;
    movers += all_high;
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
    const int per = (d.max_pages + 63) / 64;
    const uint32_t used = d.ctrl->used;
    for (int64_t u = blockIdx.x * 4 + (threadIdx.x >> 6); u < (int64_t)d.max_seqs * per; u += renames * 4) {
      const int s = (int)(u / per), p = (int)(u % per) * 64 + (int)lane_id();
      if (p >= pages_for(d, d.lengths[s])) continue;
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

// A call of few table entries takes one launch: the planning workgroup walks them too.
bool walks_inline(const CacheDev &d, int64_t n) { return n * (int64_t)d.max_pages <= kInlineSlots; }

}  // namespace

void launch_cache_extend(const CacheDev &d, const CacheRows &r, hipStream_t s) {
  k_cache_extend<<<1, kPlanLanes, 0, s>>>(d, r);
  k_cache_move<<<copy_groups(d, r.n), 256, 0, s>>>(d, 0);
}

void launch_cache_trim(const CacheDev &d, int32_t n, const int32_t *seqs, const int32_t *lengths, hipStream_t s) {
  const bool one = walks_inline(d, n);
  k_cache_trim<<<1, kPlanLanes, 0, s>>>(d, n, seqs, lengths, one);
  if (!one) k_cache_trim_entries<<<entry_groups(d, n), 256, 0, s>>>(d, n);
}

void launch_cache_fork(const CacheDev &d, int32_t n, const int32_t *src, const int32_t *dst, bool copy, hipStream_t s) {
  const bool one = walks_inline(d, n);
  k_cache_fork<<<1, kPlanLanes, 0, s>>>(d, n, src, dst, copy, one);
  if (!one) k_cache_fork_entries<<<entry_groups(d, n), 256, 0, s>>>(d, n);
  if (copy) k_cache_move<<<copy_groups(d, (int64_t)n * d.max_pages), 256, 0, s>>>(d, 0);
}

void launch_cache_compact(const CacheDev &d, hipStream_t s) {
  k_cache_compact<<<1, kPlanLanes, 0, s>>>(d);
  const int renames = entry_groups(d, d.max_seqs);
  k_cache_move<<<renames + copy_groups(d, d.pages), 256, 0, s>>>(d, renames);
}

}  // namespace rtams
