// Device-side view of the paged cache of keys and values in 4 bits (include/rtams_cache.h) and the launches of its
// kernels.  Internal to the library.
//
// A page holds page_tokens tokens of every layer; of one layer and head it is page_tokens / 32 blocks of 32 tokens, each 40 *
// head_dim bytes and laid out as the attention's matrix instructions take it, so that a wavefront reads whole lines and
// needs no transposition:
//   key codes     [32 tokens][head_dim / 8 words]        a word: 8 channels of a token
//   key meta      [32 tokens][head_dim / 32]             step (low half), zero (high half)
//   value codes   [words / kVChunk][64 lanes][kVChunk]   a word: 8 tokens of a channel (see value_word)
//   value meta    [head_dim / 32][step, zero][32 tokens in the order of the value words] halves
// In a word, element i of the 8 lies at bit 4 * (i / 2) + 16 * (i % 2): two and's give two neighbours in the halves of a register.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rtams {

constexpr int kBlockTokens = 32;
constexpr int kGroup = 32;          // channels that share a step and a zero
constexpr float kCacheMost = 60000.0f;
constexpr int kCacheMaxSeqs = 65536;

struct CacheCtrl {
  uint32_t free;     // pages that nobody names
  uint32_t pairs;    // pages to copy, of the call being run
  uint32_t ok;       // the plan of the call being run holds
  uint32_t stopped;  // the last extend was dropped: writes are dropped too
  uint32_t used;     // of a compaction: pages in use
  uint32_t pad[59];
};

struct CacheItem {  // of the call being run
  int32_t seq, src;    // (src: fork)
  int32_t have, want;  // pages before and after
  uint32_t off;        // first of its new pages among the call's
  int32_t copy;        // its last page is replaced by a copy
  int32_t pad[2];
};

struct CacheMirror {  // pinned host memory
  int32_t error;
};

struct CacheDev {
  int32_t layers, kv_heads, head_dim, page_tokens, max_seqs, max_pages;
  uint32_t pages;
  uint32_t page_blocks;        // page_tokens / 32
  uint32_t page_blocks_magic;  // block / page_blocks == block * magic >> 32 for block < 2^27 (page_blocks > 1)
  uint32_t block_bytes;        // 40 * head_dim
  int64_t page_bytes;          // of one layer
  CacheCtrl *ctrl;
  uint32_t *free_bits;  // a bit for each page
  int32_t *refs, *lengths, *table;
  CacheItem *items;
  int32_t *picked;                // new pages of the call, in order
  int32_t *pair_src, *pair_dst;   // pages to copy
  int32_t *map;                   // of a compaction: where a page went
  unsigned char *data;
  CacheMirror *mirror;
  float *part;        // attention: parts of rows
  float *part_ml;     // their maxima and sums
  uint32_t *arrived;  // parts of an item that are there
  uint32_t *joins;    // of a head's row tile: how many parts (upper half) and the first of them, for a launch that joins them
};

struct CacheRows {  // the items of a call, and rows that lie `row_stride` elements apart
  int32_t n;
  int32_t max_new;
  int64_t rows;
  const int32_t *seqs, *starts;
};

// First row and number of rows of item i; false where they are not inside the call's rows.
__device__ inline bool cache_item_rows(const CacheRows &r, int i, int64_t *first, int *count) {
  if (!r.starts) {
    *first = i;
    *count = 1;
    return i < r.rows;
  }
  const int a = r.starts[i], b = r.starts[i + 1];
  *first = a;
  *count = b - a;
  return a >= 0 && b >= a && b <= r.rows && b - a <= r.max_new;
}

__device__ inline int cache_item_seq(const CacheRows &r, int i) { return r.seqs ? r.seqs[i] : i; }

__device__ inline void cache_raise(const CacheDev &d, int code) {
  int zero = 0;
  __hip_atomic_compare_exchange_strong(&d.mirror->error, &zero, code, __ATOMIC_RELAXED, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
}

__host__ __device__ inline uint32_t cache_page_of(const CacheDev &d, uint32_t block) {
  return d.page_blocks == 1 ? block : (uint32_t)(((uint64_t)block * d.page_blocks_magic) >> 32);
}

__device__ inline unsigned char *cache_block(const CacheDev &d, int layer, int page, int head, uint32_t block_in_page) {
  return d.data + ((int64_t)layer * d.pages + page) * d.page_bytes +
         (int64_t)((uint32_t)head * d.page_blocks + block_in_page) * d.block_bytes;
}

// The word of value codes that channel ch and lane group b (0..3) of a block have: tokens 16 * (b / 2) + 4 * (b % 2) +
// {0, 1, 2, 3, 8, 9, 10, 11}, which is what one lane of the matrix instructions holds of a column of probabilities.
__host__ __device__ constexpr int value_chunk(int head_dim) { return head_dim / 16 % 4 == 0 ? 4 : 2; }
__host__ __device__ inline int value_word(int head_dim, int ch, int b) {
  const int vc = value_chunk(head_dim), tile = ch / 16;
  return ((tile / vc) * 64 + b * 16 + ch % 16) * vc + tile % vc;
}
// Where token t of a block is in the value words: lane group and element.
__host__ __device__ inline int value_group(int t) { return (t / 16) * 2 + (t / 4) % 2; }
__host__ __device__ inline int value_element(int t) { return (t / 8) % 2 * 4 + t % 4; }
__host__ __device__ inline int element_shift(int e) { return 4 * (e / 2) + 16 * (e % 2); }

struct CacheQuery {
  CacheRows r;
  int32_t layer, q_heads, share;  // share: query heads of a kv head
  int32_t half_type;              // 1: halves, 0: bfloat16
  int32_t causal, window;
  int32_t vec;                    // q and out may be read and written 16 and 8 bytes at a time
  float scale_two, scale_rest;    // scale * log2(e): a power of two, with its sign, times a number from 1 to 2
  const uint16_t *q;
  int64_t q_row, q_head;
  uint16_t *out;
  int64_t out_row, out_head;
  float *lse;
};

struct CacheSight {  // what rows see besides the last positions of a window and, of each other, the ones before
  int32_t sinks;         // with a window: the first so many positions
  int32_t words;         // of a row of tree
  const uint32_t *tree;  // bit i of row j's words: it sees row i of its item; NULL: the rows up to itself
};

void launch_cache_extend(const CacheDev &d, const CacheRows &r, bool copies, hipStream_t s);  // copies: pages may be shared
void launch_cache_fork(const CacheDev &d, int32_t n, const int32_t *src, const int32_t *dst, bool copy, hipStream_t s);
void launch_cache_trim(const CacheDev &d, int32_t n, const int32_t *seqs, const int32_t *lengths, hipStream_t s);
void launch_cache_compact(const CacheDev &d, hipStream_t s);
void launch_cache_write(const CacheDev &d, const CacheRows &r, int layer, const void *k, const void *v, int64_t row_stride,
                        int64_t head_stride, bool half_type, bool vec, hipStream_t s);
void launch_cache_read(const CacheDev &d, const CacheRows &r, int layer, void *k, void *v, int type, hipStream_t s);
void launch_cache_attend(const CacheDev &d, const CacheQuery &q, const CacheSight *sight, hipStream_t s);  // (sight: NULL where it says nothing)
void launch_cache_prompt(const CacheDev &d, const CacheQuery &q, const CacheSight *sight, hipStream_t s);  // (many rows; launch_cache_attend chooses)
void launch_cache_tree(const CacheDev &d, const CacheRows &r, const int32_t *parents, uint32_t *tree, int words, int32_t *positions, hipStream_t s);
void launch_cache_walk(const CacheDev &d, const CacheRows &r, const int32_t *parents, const int32_t *tokens, const int32_t *chosen, int32_t *path, int32_t *kept,
                       int32_t *next, hipStream_t s);
void launch_cache_keep(const CacheDev &d, const CacheRows &r, const int32_t *path, const int32_t *kept, hipStream_t s);
void launch_cache_keep_plan(const CacheDev &d, const CacheRows &r, const int32_t *path, const int32_t *kept, hipStream_t s);  // checks, and d.items
void launch_cache_keep_cut(const CacheDev &d, int32_t n, hipStream_t s);                                                     // lengths, and pages given up
hipError_t allow_large_lds_cache_tree();
hipError_t allow_large_lds_cache_attend();
hipError_t allow_large_lds_cache_prompt();
size_t cache_prompt_part_rows();
size_t cache_prompt_groups();
size_t cache_part_floats(int head_dim);    // room for parts of rows: values,
size_t cache_part_ml_floats(int head_dim); // maxima and sums,
size_t cache_arrived_words(int max_seqs, int kv_heads);

}  // namespace rtams
