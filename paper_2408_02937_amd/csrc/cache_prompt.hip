// Attention of many rows over the cache in 4 bits: prompts, and pieces of prompts behind what the cache already holds.
//
// The formulas are those of cache_attend.hip; here arithmetic bounds: 4 * head_dim flops for a row and token.  A workgroup has
// 32 rows for each wavefront (a row: a token's query head of those that share a kv head) and goes over the tokens that they see
// 64 at a time (32 where head_dim is 256): all its lanes turn their codes into halves in LDS, once for all rows, while the loads of the next
// tokens are under way; two buffers, one barrier.  Scores are S^T = K Q^T with Q in registers; a lane has one row's scores and its
// probabilities are the operand that O^T = V^T P^T takes.  The running maximum enters as the start of the scores' sums and moves
// only where a score has left it 8 behind.  LDS holds operands in the order in which the lanes take them, 16 bytes each; the slots are
// swapped so that writing meets no bank twice.  Where rows are too few to fill the chip the tokens are split, and the last
// part of a row to arrive joins them.
#include "../../include/rtams_cache.h"

#include "cache_mm.h"

namespace rtams {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int tile_blocks(int head_dim) { return head_dim == 256 ? 1 : 2; }  // of 32 tokens; registers decide
constexpr int kParts = 256;      // workgroups that may leave parts

template <int D>
struct Staging {  // of a tile in LDS: operands of 16 bytes
  uint4 k[tile_blocks(D) * 4 * D];  // [block][word][token]
  uint4 v[tile_blocks(D) * 4 * D];  // [block][32 channels][lane group][channel]
};

__device__ inline int key_slot(int word, int token) { return token ^ (((word >> 1) & 7) << 1); }
__device__ inline int value_slot(int tile, int ch) { return ch ^ ((tile & 1) << 3); }

template <int D>
struct Piece {  // two words of keys or values with their steps and zeros
  uint2 code;
  HalfWords step, zero;  // keys: w[0] holds both
};

// Pieces of a tile whose blocks are at blk0 and blk1: the first kPieces<D> are keys, as many more values.
template <int D>
constexpr int kPieces = tile_blocks(D) * 2 * D;
template <int D>
__device__ inline void load_piece(Piece<D> &p, int u, const unsigned char *blk0, const unsigned char *blk1) {
  constexpr int WP = D / 16, VC = value_chunk(D);
  if (u < kPieces<D>) {
    const int token = u / WP, wp = u % WP;
    const unsigned char *blk = token < 32 ? blk0 : blk1;
    p.code = *reinterpret_cast<const uint2 *>(blk + (token & 31) * (D / 2) + wp * 8);
    p.step.w[0] = *reinterpret_cast<const uint32_t *>(blk + 16 * D + ((token & 31) * (D / 32) + (wp >> 1)) * 4);
  } else {
    const int x = u - kPieces<D>, idx = x % (2 * D);
    const unsigned char *blk = x < 2 * D ? blk0 : blk1;
    p.code = *reinterpret_cast<const uint2 *>(blk + 20 * D + idx * 8);
    const int group = VC == 4 ? (idx >> 7) * 2 + (idx & 1) : idx >> 6, b = VC == 4 ? (idx >> 5) & 3 : (idx >> 4) & 3;
    const uint4 s = *reinterpret_cast<const uint4 *>(blk + 36 * D + group * 128 + b * 16), z = *reinterpret_cast<const uint4 *>(blk + 36 * D + group * 128 + 64 + b * 16);
    __builtin_memcpy(&p.step, &s, 16);
    __builtin_memcpy(&p.zero, &z, 16);
  }
}

template <int D>
__device__ inline void put_piece(const Piece<D> &p, int u, Staging<D> &sh) {
  constexpr int WP = D / 16, VC = value_chunk(D);
  if (u < kPieces<D>) {
    const int token = u / WP, wp = u % WP;
    const half2v step = {half_at(p.step.w[0], 0), half_at(p.step.w[0], 0)}, zero = {half_at(p.step.w[0], 1), half_at(p.step.w[0], 1)};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      HalfWords x = codes_of(i ? p.code.y : p.code.x);
#pragma unroll
      for (int j = 0; j < 4; ++j) x.p[j] = __builtin_elementwise_fma(x.p[j], step, zero);
      const int word = wp * 2 + i;
      sh.k[((token >> 5) * (D / 8) + word) * 32 + key_slot(word, token & 31)] = make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]);
    }
  } else {
    const int y = u - kPieces<D>, idx = y % (2 * D), block = y / (2 * D);
    const int tile = VC == 4 ? (idx >> 7) * 2 + (idx & 1) : idx >> 6, lane = VC == 4 ? (idx >> 1) & 63 : idx & 63;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      HalfWords x = codes_of(i ? p.code.y : p.code.x);
#pragma unroll
      for (int j = 0; j < 4; ++j) x.p[j] = __builtin_elementwise_fma(x.p[j], p.step.p[j], p.zero.p[j]);
      sh.v[((block * (D / 32) + tile) * 4 + (lane >> 4)) * 32 + value_slot(tile, i * 16 + (lane & 15))] = make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]);
    }
  }
}

template <int D, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void k_cache_prompt(CacheDev d, CacheQuery q, int tiles, int splits) {
  constexpr int kLanes = WAVES * 64, kRows = WAVES * 32, NS = D / 16, NC = D / 32, NP = (2 * kPieces<D> + kLanes - 1) / kLanes;
  constexpr int TB = tile_blocks(D), kTile = TB * kBlockTokens;
  extern __shared__ uint4 lds[];
  Staging<D> *sh = reinterpret_cast<Staging<D> *>(lds);
  __shared__ int last;
  // heads fastest (a head's cache stays on one die), then the items, the splits, and the row tiles from the longest on
  uint32_t at = blockIdx.x;
  const int head = at % d.kv_heads;
  at /= d.kv_heads;
  const int item = at % q.r.n;
  at /= q.r.n;
  const int split = at % splits, tile = tiles - 1 - (int)(at / splits);
  int64_t row0;
  int count;
  const int seq = cache_item_seq(q.r, item);
  if (!cache_item_rows(q.r, item, &row0, &count) || (uint32_t)seq >= (uint32_t)d.max_seqs) {
    if (threadIdx.x == 0) cache_raise(d, RTAMS_EINVAL);
    return;
  }
  const int length = d.lengths[seq], rows = q.share * count - tile * kRows;  // of the item, from this tile on
  if (q.causal && count > length && threadIdx.x == 0) cache_raise(d, RTAMS_EINVAL);
  if (rows <= 0) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 31, h = lane >> 5;

  // this lane's row
  const int row = wave * 32 + col, mine = tile * kRows + row;
  const bool real = row < rows;
  const int j = real ? mine / q.share : 0, qh = head * q.share + (real ? mine % q.share : 0);
  const int pos = length - count + j;
  const int see_to = !real ? 0 : q.causal ? pos + 1 : length;
  const int see_from = q.causal && q.window ? pos - q.window + 1 : 0;
  half8 qf[NS];
  {
    const uint16_t *p = q.q + (row0 + j) * q.q_row + (int64_t)qh * q.q_head + h * 8;
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[s] = real ? load_query(p + s * 16, q.half_type, q.vec, q.scale_log2) : half8{};
  }
  // what the wavefront's rows see, what all of them see, and what the workgroup goes over
  const int w_first = tile * kRows + wave * 32, w_last = min(w_first + 31, q.share * count - 1);
  const bool busy = wave * 32 < rows;
  const int j_first = w_first / q.share, j_last = w_last / q.share;
  const int any_to = !busy ? 0 : q.causal ? length - count + j_last + 1 : length, all_to = q.causal ? length - count + j_first + 1 : length;
  const int any_from = q.causal && q.window ? length - count + j_first - q.window + 1 : 0, all_from = q.causal && q.window ? length - count + j_last - q.window + 1 : 0;
  const int g_last = min(tile * kRows + kRows - 1, q.share * count - 1) / q.share;
  const int to = q.causal ? length - count + g_last + 1 : length;
  const int from = q.causal && q.window ? max(0, length - count + tile * kRows / q.share - q.window + 1) & ~(kBlockTokens - 1) : 0;
  const int steps = to > from ? (to - from + kTile - 1) / kTile : 0;
  const int parts = max(1, min(splits, steps));
  if (split >= parts) return;
  const int t0 = (int)((int64_t)steps * split / parts), t1 = (int)((int64_t)steps * (split + 1) / parts);

  f32x16 o[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[c][e] = 0.0f;
  float m = -INFINITY, l = 0.0f;
  f32x16 start;  // of the scores' sums: less the maximum
#pragma unroll
  for (int e = 0; e < 16; ++e) start[e] = 0.0f;

  const int32_t *table = d.table + (int64_t)seq * d.max_pages;
  const int last_block = (length - 1) / kBlockTokens;
  const auto block_at = [&](int block) {  // (a tile's second block may lie behind the last)
    const uint32_t b = (uint32_t)min(block, last_block), pg = cache_page_of(d, b);
    return cache_block(d, q.layer, table[pg], head, b - pg * d.page_blocks);
  };
  Piece<D> next[NP];
  const auto load_tile = [&](int t) {
    const int block = (from + t * kTile) / kBlockTokens;
    const unsigned char *b0 = block_at(block), *b1 = TB == 2 ? block_at(block + 1) : b0;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int u = i * kLanes + threadIdx.x;
      if (2 * kPieces<D> % kLanes == 0 || u < 2 * kPieces<D>) load_piece<D>(next[i], u, b0, b1);
    }
  };
  const auto put_tile = [&](Staging<D> &to_lds) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int u = i * kLanes + threadIdx.x;
      if (2 * kPieces<D> % kLanes == 0 || u < 2 * kPieces<D>) put_piece<D>(next[i], u, to_lds);
    }
  };
  if (t0 < t1) {
    load_tile(t0);
    put_tile(sh[0]);
  }
  __syncthreads();
  for (int t = t0; t < t1; ++t) {
    const Staging<D> &s = sh[(t - t0) & 1];
    if (t + 1 < t1) load_tile(t + 1);
    const int tok0 = from + t * kTile;
    if (tok0 < any_to && tok0 + kTile > any_from) {
      f32x16 sc[TB];
#pragma unroll
      for (int x = 0; x < TB; ++x) sc[x] = start;
#pragma unroll
      for (int k = 0; k < NS; ++k)
#pragma unroll
        for (int x = 0; x < TB; ++x) {
          const int word = 2 * k + h;
          const uint4 a = s.k[(x * (D / 8) + word) * 32 + key_slot(word, col)];
          half8 kh;
          __builtin_memcpy(&kh, &a, 16);
          sc[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kh, qf[k], sc[x], 0, 0, 0);
        }
      if (tok0 + kTile > all_to || tok0 < all_from) {
#pragma unroll
        for (int x = 0; x < TB; ++x)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int token = tok0 + 32 * x + 8 * (e >> 2) + 4 * h + (e & 3);
            if (token >= see_to || token < see_from) sc[x][e] = -INFINITY;
          }
      }
      float top = -INFINITY;
#pragma unroll
      for (int x = 0; x < TB; ++x)
#pragma unroll
        for (int e = 0; e < 16; e += 2) top = fmaxf(top, fmaxf(sc[x][e], sc[x][e + 1]));
      top = fmaxf(top, __shfl_xor(top, 32));
      const bool move = top > 8.0f || (m == -INFINITY && top > -INFINITY);  // (scores are relative to the maximum)
      if (__any(move)) {
        const float by = move ? top : 0.0f, shrink = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(-by);
        if (move) m = (m == -INFINITY ? 0.0f : m) + by;
        l *= shrink;
#pragma unroll
        for (int c = 0; c < NC; ++c) o[c] *= shrink;
#pragma unroll
        for (int x = 0; x < TB; ++x) sc[x] -= by;
        start -= by;
      }
      half8 pf[TB][2];
#pragma unroll
      for (int x = 0; x < TB; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          float p[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            p[e] = __builtin_amdgcn_exp2f(sc[x][8 * y + e]);
            l += p[e];
          }
          pf[x][y] = to_half8(p);
        }
#pragma unroll
      for (int x = 0; x < TB; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            const uint4 a = s.v[((x * NC + c) * 4 + 2 * y + h) * 32 + value_slot(c, col)];
            half8 vh;
            __builtin_memcpy(&vh, &a, 16);
            o[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vh, pf[x][y], o[c], 0, 0, 0);
          }
    }
    if (t + 1 < t1) put_tile(sh[(t + 1 - t0) & 1]);
    __syncthreads();
  }
  l += __shfl_xor(l, 32);

  if (parts == 1) {
    if (real)
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < 16; e += 4)
          store_row(q, row0 + j, qh, c * 32 + 2 * e + 4 * h, f32x4{o[c][e], o[c][e + 1], o[c][e + 2], o[c][e + 3]}, m, l);
    return;
  }
  const int64_t group = ((int64_t)tile * q.r.n + item) * d.kv_heads + head;
  float *part = d.part + (group * splits + split) * kRows * D, *ml = d.part_ml + (group * splits + split) * kRows * 2;
  if (real) {
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < 16; e += 2) put_pair(part + row * D + c * 32 + 8 * (e >> 2) + 4 * h + (e & 3), o[c][e], o[c][e + 1]);
    if (h == 0) put_pair(ml + row * 2, m, l);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wavefront's part is out ...
  __syncthreads();                                  // ... and that of the others
  if (threadIdx.x == 0) {
    last = __hip_atomic_fetch_add(d.arrived + group, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)parts - 1;
    if (last) __hip_atomic_store(d.arrived + group, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (!last) return;
  part = d.part + group * splits * kRows * D;
  ml = d.part_ml + group * splits * kRows * 2;
  for (int u = threadIdx.x; u < min(rows, kRows) * (D / 4); u += kLanes) {
    const int r = u / (D / 4), c = u % (D / 4) * 4, i = tile * kRows + r;
    join_parts(q, row0 + i / q.share, head * q.share + i % q.share, c, parts, part + r * D + c, ml + r * 2, D, kRows);
  }
}

template <int D, int WAVES>
void launch(const CacheDev &d, const CacheQuery &q, hipStream_t s) {
  const int64_t rows = (int64_t)q.share * q.r.max_new;
  const int tiles = (int)((rows + WAVES * 32 - 1) / (WAVES * 32));
  const int64_t groups = (int64_t)tiles * q.r.n * d.kv_heads;
  const int splits = groups >= kParts ? 1 : (int)(kParts / groups);
  k_cache_prompt<D, WAVES><<<(uint32_t)(groups * splits), WAVES * 64, 2 * sizeof(Staging<D>), s>>>(d, q, tiles, splits);
}

}  // namespace

size_t cache_prompt_part_rows() { return (size_t)kParts * 256; }
size_t cache_prompt_groups() { return kParts; }

void launch_cache_prompt(const CacheDev &d, const CacheQuery &q, hipStream_t s) {
  switch (d.head_dim) {
    case 64: return launch<64, 8>(d, q, s);
    case 96: return launch<96, 8>(d, q, s);
    case 128: return launch<128, 8>(d, q, s);
    default: return launch<256, 4>(d, q, s);
  }
}

hipError_t allow_large_lds_cache_prompt() {
  const auto allow = [](const void *f, int bytes) { return hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, bytes); };
  return allow(reinterpret_cast<const void *>(k_cache_prompt<256, 4>), 2 * (int)sizeof(Staging<256>));
}

}  // namespace rtams
