// Trees of drafted tokens over the cache (include/rtams_cache.h): what each row of a tree sees and where it stands, the path that the
// choices follow, and the rows of that path moved to the front of their item's.  (Their attention: cache_attend.hip, cache_prompt.hip.)
//
// All are chains of look-ups over little data.  A row's ancestors are found by doubling: it takes over what the row it points to has, which then
// points twice as far.  The path is walked by one wavefront, whose lanes each know whether their row is the token that was chosen behind
// its parent; a step is a comparison and a ballot.  Rows are moved within a sequence, always to the front, so a workgroup, which has one layer and
// head of an item, takes the blocks of 32 tokens in order: it reads all that goes into one, then writes it.
#include "../../include/rtams_cache.h"

#include "cache_mm.h"

namespace rtams {

namespace {

constexpr int kLanes = 256;
constexpr int kMostRows = 1024;  // of a tree

// ------------------------------------------------------------------ parents to ancestors
// Up to 64 rows, a row to a lane of one wavefront: no LDS, no barriers.  48 trees of 31 rows: 3.4 us, by a workgroup
// with LDS, as larger ones are, 6.0.
__global__ __launch_bounds__(64) void k_cache_tree_few(CacheDev d, CacheRows r, const int32_t *parents, uint32_t *tree, int words, int32_t *positions) {
  const int item = blockIdx.x, seq = cache_item_seq(r, item), j = threadIdx.x;
  int64_t row0;
  int count;
  bool bad = !cache_item_rows(r, item, &row0, &count) || (uint32_t)seq >= (uint32_t)d.max_seqs;
  const int length = d.lengths[bad ? 0 : seq];
  bad = bad || count > length;
  int up = !bad && j < count ? parents[row0 + j] : -1;
  bad |= up < -1 || up >= j;
  if (__any(bad)) {
    if (j == 0) cache_raise(d, RTAMS_EINVAL);
    return;
  }
  uint32_t low = j < 32 ? 1u << j : 0, high = j < 32 ? 0 : 1u << (j - 32);
  while (__any(up >= 0)) {
    const int from = max(up, 0);
    const uint32_t more_low = (uint32_t)__shfl((int)low, from), more_high = (uint32_t)__shfl((int)high, from);
    const int next = __shfl(up, from);
    if (up >= 0) {
      low |= more_low;
      high |= more_high;
      up = next;
    }
  }
  if (j >= count) return;
  for (int w = 0; w < words; ++w) tree[(row0 + j) * words + w] = w == 0 ? low : w == 1 ? high : 0;
  if (positions) positions[row0 + j] = length - count + __popc(low) + __popc(high) - 1;
}

__global__ __launch_bounds__(kLanes) void k_cache_tree(CacheDev d, CacheRows r, const int32_t *parents, uint32_t *tree, int words, int32_t *positions) {
  extern __shared__ uint32_t kin[];  // [count][words]
  __shared__ int32_t points[2][kMostRows];
  const int item = blockIdx.x, seq = cache_item_seq(r, item);
  int64_t row0;
  int count;
  bool bad = !cache_item_rows(r, item, &row0, &count) || (uint32_t)seq >= (uint32_t)d.max_seqs;
  const int length = d.lengths[bad ? 0 : seq];
  bad = bad || count > length;
  if (!bad)
    for (int j = threadIdx.x; j < count; j += kLanes) {
      const int p = parents[row0 + j];
      bad |= p < -1 || p >= j;
      points[0][j] = p;
    }
  if (__syncthreads_or(bad)) {
    if (threadIdx.x == 0) cache_raise(d, RTAMS_EINVAL);
    return;
  }
  const int all = count * words;
  for (int u = threadIdx.x; u < all; u += kLanes) {
    const int j = u / words, w = u % words;
    kin[u] = j / 32 == w ? 1u << (j % 32) : 0;
  }
  int32_t *up = points[0], *next = points[1];
  for (int some = 1; some;) {
    __syncthreads();
    // (a row that another lane has already brought further on has more of the same ancestors)
    for (int u = threadIdx.x; u < all; u += kLanes) {
      const int p = up[u / words];
      if (p < 0) continue;
      const uint32_t more = __hip_atomic_load(&kin[p * words + u % words], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
      __hip_atomic_store(&kin[u], kin[u] | more, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    }
    some = 0;
    for (int j = threadIdx.x; j < count; j += kLanes) {
      const int p = up[j];
      next[j] = p < 0 ? -1 : up[p];
      some |= next[j] >= 0;
    }
    some = __syncthreads_or(some);
    int32_t *const swap = up;
    up = next;
    next = swap;
  }
  for (int u = threadIdx.x; u < all; u += kLanes) tree[row0 * words + u] = kin[u];
  if (positions)
    for (int j = threadIdx.x; j < count; j += kLanes) {
      int depth = -1;
      for (int w = 0; w < words; ++w) depth += __popc(kin[j * words + w]);
      positions[row0 + j] = length - count + depth;
    }
}

// ------------------------------------------------------------------ the path of the choices
// EACH rows to a lane.
template <int EACH>
__global__ __launch_bounds__(64) void k_cache_walk(CacheDev d, CacheRows r, const int32_t *parents, const int32_t *tokens, const int32_t *chosen, int32_t *path,
                                                   int32_t *kept, int32_t *next) {
  __shared__ int32_t choice[64 * EACH];
  const int item = blockIdx.x, lane = threadIdx.x;
  int64_t row0;
  int count;
  if (!cache_item_rows(r, item, &row0, &count)) {
    if (lane == 0) {
      cache_raise(d, RTAMS_EINVAL);
      kept[item] = next[item] = -1;
    }
    return;
  }
  int from[EACH], token[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int j = i * 64 + lane;
    from[i] = token[i] = -1;
    if (j < count) {
      from[i] = parents[row0 + j];
      token[i] = tokens[row0 + j];
      choice[j] = chosen[row0 + j];
    }
  }
  __syncthreads();
  bool bad = false;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {  // from: the parent of row lane + 64 i, if it is what was chosen there
    const bool right = from[i] >= -1 && from[i] < i * 64 + lane;
    bad |= !right;
    if (!right || from[i] < 0 || token[i] < 0 || choice[right ? max(from[i], 0) : 0] != token[i]) from[i] = -1;
  }
  bad = __any(bad);
  int len = 0, last = -1;
  if (!bad && count > 0) {
    last = 0;
    for (len = 1;; ++len) {
      if (lane == 0) path[row0 + len - 1] = last;
      int found = -1;
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        const uint64_t who = found < 0 && i * 64 < count ? __ballot(from[i] == last) : 0;
        if (who) found = i * 64 + __ffsll((unsigned long long)who) - 1;
      }
      if (found < 0) break;
      last = found;
    }
  }
  for (int j = len + lane; j < count; j += 64) path[row0 + j] = -1;
  if (lane == 0) {
    if (bad) cache_raise(d, RTAMS_EINVAL);
    kept[item] = bad ? -1 : len;
    next[item] = last >= 0 ? choice[last] : -1;
  }
}

// ------------------------------------------------------------------ rows of a path to the front
// items[i], planned ahead: src: position of the first row, off: rows kept, copy: rows.
template <int D>
__global__ __launch_bounds__(kLanes) void k_cache_keep(CacheDev d, CacheRows r, const int32_t *path, uint32_t first_unit) {
  constexpr int W = D / 8, G = D / 32, VC = value_chunk(D), kPages = kMostRows / kBlockTokens + 2;
  constexpr int kKeys = (kBlockTokens * (W + G) + kLanes - 1) / kLanes, kValues = (4 * D + kLanes - 1) / kLanes, kMeta = (kBlockTokens * 2 * G + kLanes - 1) / kLanes;
  __shared__ int32_t from[kMostRows], pages[kPages];
  __shared__ int first_moved;
  const uint32_t u0 = first_unit + blockIdx.x, head = u0 % d.kv_heads, rest = u0 / d.kv_heads;
  const int layer = rest % d.layers, item = rest / d.layers;
  const uint32_t ok = d.ctrl->ok;
  const CacheItem it = d.items[item];
  const int64_t row0 = r.starts ? r.starts[item] : item;
  if (!ok) return;
  const int base = uniform(it.src), kept = uniform(it.off), count = uniform(it.copy), seq = uniform(it.seq);
  if (threadIdx.x == 0) first_moved = kMostRows;
  __syncthreads();
  const int page0 = base / d.page_tokens;
  for (int j = threadIdx.x; j < kept; j += kLanes) {
    const int p = path[row0 + j];
    from[j] = p;
    if (p != j) atomicMin(&first_moved, j);
  }
  if (count > 0 && (int)threadIdx.x <= (base + count - 1) / d.page_tokens - page0) pages[threadIdx.x] = d.table[(int64_t)seq * d.max_pages + page0 + threadIdx.x];
  __syncthreads();
  const int j0 = uniform(first_moved);
  if (j0 >= kept) return;
  const auto block_of = [&](int pos) {
    const uint32_t block = (uint32_t)pos / kBlockTokens, pg = cache_page_of(d, block);
    return cache_block(d, layer, pages[pg - page0], (int)head, block - pg * d.page_blocks);
  };
  for (int block = (base + j0) / kBlockTokens; block * kBlockTokens < base + kept; ++block) {
    unsigned char *const to = block_of(block * kBlockTokens);
    const int shift = block * kBlockTokens - base;  // token t of the block is row t + shift
    // a token of the block that is moved into: its source
    const auto source = [&](int t) {
      const int j = t + shift;
      return j >= j0 && j < kept ? base + from[j] : -1;
    };
    uint32_t key[kKeys], value[kValues];
    uint16_t meta[kMeta];
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
      const int u = i * kLanes + threadIdx.x, t = u / (W + G), w = u % (W + G), pos = u < kBlockTokens * (W + G) ? source(t) : -1;
      key[i] = 0;
      if (pos < 0) continue;
      const unsigned char *p = block_of(pos);
      const int s = pos % kBlockTokens;
      key[i] = *reinterpret_cast<const uint32_t *>(w < W ? p + s * (D / 2) + w * 4 : p + 16 * D + (s * G + w - W) * 4);
    }
#pragma unroll
    for (int i = 0; i < kValues; ++i) {
      const int u = i * kLanes + threadIdx.x, b = u / VC % 64 / 16;
      value[i] = 0;
      if (u >= 4 * D) continue;
      uint32_t x = reinterpret_cast<const uint32_t *>(to + 20 * D)[u];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int pos = source((b / 2) * 16 + (b % 2) * 4 + (e / 4) * 8 + e % 4);
        if (pos < 0) continue;
        const int s = pos % kBlockTokens;
        const uint32_t y = reinterpret_cast<const uint32_t *>(block_of(pos) + 20 * D)[u + (value_group(s) - b) * 16 * VC];
        x = (x & ~(15u << element_shift(e))) | ((y >> element_shift(value_element(s))) & 15u) << element_shift(e);
      }
      value[i] = x;
    }
#pragma unroll
    for (int i = 0; i < kMeta; ++i) {
      const int u = i * kLanes + threadIdx.x, t = u % kBlockTokens, g = u / kBlockTokens, pos = g < 2 * G ? source(t) : -1;
      meta[i] = 0;
      if (pos < 0) continue;
      const int s = pos % kBlockTokens;
      meta[i] = reinterpret_cast<const uint16_t *>(block_of(pos) + 36 * D)[g * kBlockTokens + value_group(s) * 8 + value_element(s)];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
      const int u = i * kLanes + threadIdx.x, t = u / (W + G), w = u % (W + G);
      if (u < kBlockTokens * (W + G) && source(t) >= 0) *reinterpret_cast<uint32_t *>(w < W ? to + t * (D / 2) + w * 4 : to + 16 * D + (t * G + w - W) * 4) = key[i];
    }
#pragma unroll
    for (int i = 0; i < kValues; ++i)
      if (i * kLanes + (int)threadIdx.x < 4 * D) reinterpret_cast<uint32_t *>(to + 20 * D)[i * kLanes + threadIdx.x] = value[i];
#pragma unroll
    for (int i = 0; i < kMeta; ++i) {
      const int u = i * kLanes + threadIdx.x, t = u % kBlockTokens, g = u / kBlockTokens;
      if (g < 2 * G && source(t) >= 0) reinterpret_cast<uint16_t *>(to + 36 * D)[g * kBlockTokens + value_group(t) * 8 + value_element(t)] = meta[i];
    }
    __syncthreads();
  }
}

}  // namespace

void launch_cache_tree(const CacheDev &d, const CacheRows &r, const int32_t *parents, uint32_t *tree, int words, int32_t *positions, hipStream_t s) {
  if (r.max_new <= 64) k_cache_tree_few<<<r.n, 64, 0, s>>>(d, r, parents, tree, words, positions);
  else k_cache_tree<<<r.n, kLanes, (size_t)r.max_new * words * 4, s>>>(d, r, parents, tree, words, positions);
}

void launch_cache_walk(const CacheDev &d, const CacheRows &r, const int32_t *parents, const int32_t *tokens, const int32_t *chosen, int32_t *path, int32_t *kept,
                       int32_t *next, hipStream_t s) {
  const auto go = [&](auto kernel) { kernel<<<r.n, 64, 0, s>>>(d, r, parents, tokens, chosen, path, kept, next); };
  if (r.max_new <= 64) go(k_cache_walk<1>);
  else if (r.max_new <= 256) go(k_cache_walk<4>);
  else go(k_cache_walk<kMostRows / 64>);
}

void launch_cache_keep(const CacheDev &d, const CacheRows &r, const int32_t *path, const int32_t *kept, hipStream_t s) {
  launch_cache_keep_plan(d, r, path, kept, s);
  const int64_t units = (int64_t)r.n * d.layers * d.kv_heads, most = 1 << 22;
  for (int64_t at = 0; at < units; at += most) {
    const uint32_t grid = (uint32_t)(units - at < most ? units - at : most);
    switch (d.head_dim) {
      case 64: k_cache_keep<64><<<grid, kLanes, 0, s>>>(d, r, path, (uint32_t)at); break;
      case 96: k_cache_keep<96><<<grid, kLanes, 0, s>>>(d, r, path, (uint32_t)at); break;
      case 128: k_cache_keep<128><<<grid, kLanes, 0, s>>>(d, r, path, (uint32_t)at); break;
      default: k_cache_keep<256><<<grid, kLanes, 0, s>>>(d, r, path, (uint32_t)at); break;
    }
  }
  launch_cache_keep_cut(d, r.n, s);
}

hipError_t allow_large_lds_cache_tree() {
  return hipFuncSetAttribute(reinterpret_cast<const void *>(k_cache_tree), hipFuncAttributeMaxDynamicSharedMemorySize, kMostRows * (kMostRows / 32) * 4);
}

}  // namespace rtams
