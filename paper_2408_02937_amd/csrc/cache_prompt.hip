// Attention of many rows over the cache in 4 bits: prompts, and pieces of prompts behind what the cache already holds.
//
// The formulas are those of cache_attend.hip; here arithmetic bounds: 4 * head_dim flops for a row and token.  A workgroup has
// 32 rows for each wavefront (a row: a token's query head of those that share a kv head) and goes over the tokens that they see
// 64 at a time (32 where head_dim is 256): all its lanes turn their codes into halves in LDS, once for all rows, a tile ahead of the products, while the
// next tiles' codes are on their way to registers or to LDS (by_copies); two buffers, one barrier a tile.  Scores are S^T = K Q^T with Q in registers; a lane has one row's scores and its
// probabilities are the operand that O^T = V^T P^T takes.  The running maximum enters as the start of the scores' sums and moves
// only where a score has left it far behind (kLag).  LDS holds operands in the order in which the lanes take them, 16 bytes each; the slots are
// swapped so that writing meets no bank twice.  Where rows are too few to fill the chip the tokens are split, and the last
// part of a row to arrive joins them.
//
// The scale's power of two is in the query, exact as an operand; what is left of it multiplies scores in 32 bits (in the query and rounded there:
// 576 us instead of 580, and half outputs 1.6 to 1.8 times as far from 64 bits as their own rounding alone, not 1.5 to 1.6).
//
// Measured: a prompt of 8,192 tokens, 32 heads of 128 over 8: 567 to 640 us from card to card for 550 GFLOP, 860 to 970 TFLOP/s where a plain product
// of 8,192 squared reaches 1,140 in bfloat16 and 1,084 in halves.  Vector instructions (exponentials, masks, codes) take 48 % of the cycles, matrix
// instructions 41 %, and two wavefronts of a SIMD overlap them in part.  Heads of 64, 96, 128, 256 on one card: 386, 484, 568, 2,312 us; 712, 852, 968,
// 476 TFLOP/s: the fewer the channels, the more exponentials for a flop; at 256 one wavefront fits a SIMD.  At 128 channels, on a card of 580 us:
// 4 wavefronts a workgroup 710, wavefronts half a tile apart 610.
// What bounds it: a tile of 64 tokens takes a compute unit 2.5 us, of which products and exponentials alone take 1.9, 0.93 of them the matrix instructions' own
// time; at their full rate they would read LDS at its own.  With the SIMD's two wavefronts changing places between matrix and vector instructions behind a
// barrier each 252 us where 206 are taken here, with the next tile's scores between this one's exponentials 226 (252 rows behind 4 sequences of up to 60,063).
//
// With a sight (CacheSight: sinks, trees) a tile's tokens are counted without those between the sinks and the window; what a row sees of 32 tokens are
// the bits of a word.  Parts of rows are joined by a launch of their own.  8,192 rows under a window of 1,000 with 64 sinks: 201 us for 133 GFLOP; vector
// instructions have 0.38 of the cycles, matrix instructions 0.28, LDS 0.26 of a unit's.
#include "../../include/rtams_cache.h"

#include <climits>
#include <type_traits>

#include "cache_mm.h"
#include "rtams_dev.h"

namespace rtams {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int tile_blocks(int head_dim) { return head_dim == 256 ? 1 : 2; }  // of 32 tokens; registers decide
constexpr int kRows = 256;       // of a workgroup's parts at most

// Workgroups that a compute unit runs at once: registers decide.
constexpr int at_once(int head_dim, int waves) { return waves == 8 || head_dim == 256 ? 1 : 2; }

constexpr int kRing = 4;  // tiles on their way or being unpacked

// Whether codes come to LDS as they are, by copies that run three tiles ahead; others are loaded into registers two tiles ahead.  Without a sight, in registers
// and by copies, one card: a prompt of 8,192 tokens, 32 heads of 64, 96, 128, 256 channels over 8: 398 and 386, 483 and 483, 567 and 570, 2,312 and 2,352 us;
// 600 rows behind each of 8 sequences of up to 5,000, 8 heads: 97 and 94, 113 and 112, 123 and 127, 347 and 351.  (With a sight the blocks of a tile may lie
// apart; there they are copied one by one.)
constexpr bool by_copies(int head_dim, bool sight) { return sight || head_dim == 64; }

template <int D, int TB, bool RING>
struct Staging {  // tiles in LDS: operands of 16 bytes
  uint4 k[2][TB * 4 * D];  // [block][word][token]
  uint4 v[2][TB * 4 * D];  // [block][32 channels][lane group][channel]
};
template <int D, int TB>
struct Staging<D, TB, true> : Staging<D, TB, false> {
  uint4 raw[kRing][TB * 40 * D / 16];  // as the cache holds them
};

__device__ inline int key_slot(int word, int token) { return token ^ (((word >> 1) & 7) << 1); }
__device__ inline int value_slot(int tile, int ch) { return ch ^ ((tile & 1) << 3); }

template <int D>
struct Words {  // two words of keys or values with their steps and zeros
  uint2 code;
  HalfWords step, zero;  // keys: w[0] holds both
};

// Pairs of words of a tile whose blocks are at blk0 and blk1: the first kPairs<D, TB> are keys, as many more values.
template <int D, int TB>
constexpr int kPairs = TB * 2 * D;
template <int D, int TB>
__device__ inline void load_words(Words<D> &p, int u, const unsigned char *blk0, const unsigned char *blk1) {
  constexpr int WP = D / 16, VC = value_chunk(D);
  if (u < kPairs<D, TB>) {
    const int token = u / WP, wp = u % WP;
    const unsigned char *blk = token < 32 ? blk0 : blk1;
    p.code = *reinterpret_cast<const uint2 *>(blk + (token & 31) * (D / 2) + wp * 8);
    p.step.w[0] = *reinterpret_cast<const uint32_t *>(blk + 16 * D + ((token & 31) * (D / 32) + (wp >> 1)) * 4);
  } else {
    const int x = u - kPairs<D, TB>, idx = x % (2 * D);
    const unsigned char *blk = x < 2 * D ? blk0 : blk1;
    p.code = *reinterpret_cast<const uint2 *>(blk + 20 * D + idx * 8);
    const int group = VC == 4 ? (idx >> 7) * 2 + (idx & 1) : idx >> 6, b = VC == 4 ? (idx >> 5) & 3 : (idx >> 4) & 3;
    const uint4 s = *reinterpret_cast<const uint4 *>(blk + 36 * D + group * 128 + b * 16), z = *reinterpret_cast<const uint4 *>(blk + 36 * D + group * 128 + 64 + b * 16);
    __builtin_memcpy(&p.step, &s, 16);
    __builtin_memcpy(&p.zero, &z, 16);
  }
}

template <int D, int TB>
__device__ inline void put_words(const Words<D> &p, int u, uint4 *k, uint4 *v) {
  constexpr int WP = D / 16, VC = value_chunk(D);
  if (u < kPairs<D, TB>) {
    const int token = u / WP, wp = u % WP;
    const half2v step = {half_at(p.step.w[0], 0), half_at(p.step.w[0], 0)}, zero = {half_at(p.step.w[0], 1), half_at(p.step.w[0], 1)};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      HalfWords x = codes_of(i ? p.code.y : p.code.x);
#pragma unroll
      for (int j = 0; j < 4; ++j) x.p[j] = __builtin_elementwise_fma(x.p[j], step, zero);
      const int word = wp * 2 + i;
      k[((token >> 5) * (D / 8) + word) * 32 + key_slot(word, token & 31)] = make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]);
    }
  } else {
    const int y = u - kPairs<D, TB>, idx = y % (2 * D), block = y / (2 * D);
    const int tile = VC == 4 ? (idx >> 7) * 2 + (idx & 1) : idx >> 6, lane = VC == 4 ? (idx >> 1) & 63 : idx & 63;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      HalfWords x = codes_of(i ? p.code.y : p.code.x);
#pragma unroll
      for (int j = 0; j < 4; ++j) x.p[j] = __builtin_elementwise_fma(x.p[j], p.step.p[j], p.zero.p[j]);
      v[((block * (D / 32) + tile) * 4 + (lane >> 4)) * 32 + value_slot(tile, i * 16 + (lane & 15))] = make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]);
    }
  }
}

typedef const __attribute__((address_space(4))) int32_t *ScalarInts;

struct Span {  // what the rows of a tile of an item go over
  int64_t row0;
  int seq, count, length, from, steps;  // from: first position, at a block's begin (with sinks: behind them, less what they take)
};

// Row tile `tile` (of `rows` rows) of an item; count 0: none.
template <bool SIGHT>
__device__ inline Span find_span(const CacheDev &d, const CacheQuery &q, const CacheSight &g, int item, int tile, int rows, int step_tokens, bool tell) {
  Span s{};
  s.seq = cache_item_seq(q.r, item);
  if (!cache_item_rows(q.r, item, &s.row0, &s.count) || (uint32_t)s.seq >= (uint32_t)d.max_seqs) {
    if (tell) cache_raise(d, RTAMS_EINVAL);
    s.count = 0;
    return s;
  }
  s.length = d.lengths[s.seq];
  if (q.causal && s.count > s.length) {
    if (tell) cache_raise(d, RTAMS_EINVAL);
    s.count = 0;
    return s;
  }
  if (tile * rows >= q.share * s.count) {
    s.count = 0;
    return s;
  }
  const int last = min(tile * rows + rows - 1, q.share * s.count - 1) / q.share;
  const bool tree = SIGHT && g.tree;
  int to = q.causal && !tree ? s.length - s.count + last + 1 : s.length;
  // (a tree's row may see no row of its item, itself included)
  s.from = q.causal && q.window ? max(0, s.length - s.count + (tree ? -1 : tile * rows / q.share) - q.window + 1) & ~(kBlockTokens - 1) : 0;
  if (SIGHT) {
    s.from = max(0, s.from - sink_blocks(g));
    to = max(to, s.from);  // (a first row's window may begin behind the last one's end)
  }
  s.steps = to > s.from ? (to - s.from + step_tokens - 1) / step_tokens : 1;  // (one, also where the rows see nothing)
  return s;
}

struct Piece {
  int entry, head;       // entry: row tiles from the longest on, the items of each
  int parts, nth, part;  // pieces of the head's row tile; which one this is; where its parts begin, if there are several
};

// From so many times the workgroups that run at once (one item: from as many) nothing is planned.  With a plan and without, 8 heads: 8 items of up to
// 5,000 tokens and 600 rows, 12 of up to 3,000 and 512 rows, 2 of up to 4,000 and 2,000 rows, ragged and then all as long:
//    64 channels  232, 161, 122 us and 298, 184, 150   341, 224, 161 us and 333, 213, 152
//    96           252, 187, 141        340, 211, 174   397, 269, 191        390, 256, 186
//   128           304, 222, 170        401, 253, 214   482, 331, 237        477, 321, 234
//   256           1535, 960, 634       1540, 960, 876  1673, 1221, 901      1674, 1221, 881
// One prompt of 3,000, 128 channels: 101 and 101, of 7,000: 447 and 430.
constexpr int kSplit = 4;
constexpr int kMostEntries = 1024;  // row tiles of items that are planned
constexpr int kClasses = 8;         // of their pieces, by length

template <int D, int TB, bool RING>
union Shared {
  Staging<D, TB, RING> tile;
  float steps[kMostEntries];  // in front of them
};

// Which piece is workgroup blockIdx.x's, where tokens are split (find_piece in cache_attend.hip has the same for few rows).  One wavefront's work.
template <bool SIGHT>
__device__ inline bool find_piece(const CacheDev &d, const CacheQuery &q, const CacheSight &g, int tiles, int rows, int step_tokens, uint32_t workers, float *steps, Piece *piece) {
  const int lane = threadIdx.x & 63, n = q.r.n * tiles;
  uint32_t all = 0;
  float longest = 1.0f;
  for (int base = 0; base < (n + 255) / 256 * 256; base += 64) {
    const int e = base + lane;
    const Span sp = e < n ? find_span<SIGHT>(d, q, g, e % q.r.n, tiles - 1 - e / q.r.n, rows, step_tokens, blockIdx.x == 0) : Span{};
    const int mine = sp.count ? sp.steps : 0;
    steps[e] = (float)mine;
    longest = fmaxf(longest, (float)mine);
    all += last_lane(wave_running_sum((uint32_t)mine));
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) longest = fmaxf(longest, __shfl_xor(longest, o));
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  // (never less than an even share: scratch has room for twice as many parts as there are workers, as in cache_attend.hip)
  const uint32_t share = max(1u, (all * (uint32_t)d.kv_heads + workers - 1) / workers), size = share > 1 ? piece_steps(steps, n, d.kv_heads, share, workers, SIGHT ? 1 : 0) : 1;
  // pieces from the longest on, by eighths: what comes last then fills what is left
  const float one_over = 1.0f / (float)size, per_class = kClasses / fminf((float)size, longest);
  uint32_t before = 0, parts_before = 0;
  for (int c = kClasses; c > 0; --c)
    for (int base = 0; base < n; base += 64) {
      const int e = base + lane;
      const uint32_t mine = e < n ? (uint32_t)steps[e] : 0, parts = div_up(mine, size, one_over);
      const bool now = parts > 0 && min(kClasses, (int)((float)mine * per_class / (float)parts) + 1) == c;
      if (!__any(now)) continue;
      const uint32_t pieces = now ? parts * (uint32_t)d.kv_heads : 0, shared = parts > 1 ? pieces : 0;
      const uint32_t upto = wave_running_sum(pieces), upto_shared = wave_running_sum(shared), x = blockIdx.x - (before + upto - pieces);
      if (x < pieces) *piece = Piece{e, (int)(x / parts), (int)parts, (int)(x % parts), (int)(parts_before + upto_shared - shared + x - x % parts)};
      if (__any(x < pieces)) return true;
      before += last_lane(upto);
      parts_before += last_lane(upto_shared);
    }
  return false;
}

// Orders a run of N matrix instructions, each of which takes an operand from LDS: kAhead reads go out in front of the first.  (Left alone the
// compiler asks for a pair and waits for it, a trip to LDS for every two instructions.)
template <int N>
__device__ __forceinline__ void reads_ahead() {
  constexpr int kAhead = N < 6 ? N : 6, kRead = 0x100, kMfma = 0x8;
  __builtin_amdgcn_sched_group_barrier(kRead, kAhead, 0);
#pragma unroll
  for (int i = 0; i < N - kAhead; ++i) {
    __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
    __builtin_amdgcn_sched_group_barrier(kRead, 1, 0);
  }
  __builtin_amdgcn_sched_group_barrier(kMfma, kAhead, 0);
}

// The other wavefronts' writes to LDS, and copies that they waited for, are there.  (Not __syncthreads: that would wait for all copies.)
__device__ __forceinline__ void meet() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <int D, int WAVES, int TB, bool SIGHT>
__device__ __forceinline__ void attend_many(const CacheDev &d, const CacheQuery &q, const CacheSight &g, int tiles, int tile_rows, int split, uint32_t first) {
  constexpr int kLanes = WAVES * 64, NS = D / 16, NC = D / 32, NP = (2 * kPairs<D, TB> + kLanes - 1) / kLanes;
  constexpr int kTile = TB * kBlockTokens;
  extern __shared__ uint4 lds[];
  constexpr bool RING = by_copies(D, SIGHT);
  Shared<D, TB, RING> &shared = *reinterpret_cast<Shared<D, TB, RING> *>(lds);
  Staging<D, TB, RING> &sh = shared.tile;
  __shared__ Piece piece;
  __shared__ int flag;
  Piece pc;
  if (split) {
    if (threadIdx.x < 64) {
      const bool found = find_piece<SIGHT>(d, q, g, tiles, tile_rows, kTile, kUnits * at_once(D, WAVES), shared.steps, &piece);
      if (threadIdx.x == 0) flag = found;
    }
    __syncthreads();
    if (!flag) return;
    pc = Piece{uniform(piece.entry), uniform(piece.head), uniform(piece.parts), uniform(piece.nth), uniform(piece.part)};
    __syncthreads();
  } else {  // heads fastest (a head's cache stays on one die), then the items, and the row tiles from the longest on
    const uint32_t x = first + blockIdx.x;
    pc = Piece{(int)(x / d.kv_heads), (int)(x % d.kv_heads), 1, 0, 0};
  }
  const int item = pc.entry % q.r.n, tile = tiles - 1 - pc.entry / q.r.n, head = pc.head;
  const Span sp = find_span<SIGHT>(d, q, g, item, tile, tile_rows, kTile, !split && tile == 0 && head == 0 && threadIdx.x == 0);
  const int count = uniform(sp.count);
  if (!count) return;
  const int64_t row0 = sp.row0;
  const int seq = uniform(sp.seq), length = uniform(sp.length), from = uniform(sp.from), steps = uniform(sp.steps), rows = q.share * count - tile * tile_rows;  // rows: from this tile on
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), col = lane & 31, h = lane >> 5;

  // this lane's row
  const int row = wave * 32 + col, mine = tile * tile_rows + row;
  const bool real = row < min(rows, tile_rows);
  const int j = real ? mine / q.share : 0, qh = head * q.share + (real ? mine % q.share : 0);
  const bool tree = SIGHT && g.tree;
  const int base_pos = length - count;
  const uint32_t *const kin = tree ? g.tree + (row0 + j) * g.words : nullptr;
  int pos = length - count + j;
  if (tree && q.window) {
    pos = base_pos - 1;
    for (int w = 0; w * 32 < count; ++w) pos += __popc(kin[w] & low_bits(count - w * 32));
  }
  const int see_from = q.causal && q.window ? pos - q.window + 1 : 0;
  const uint32_t sees = !real ? 0 : (uint32_t)max(0, (q.causal ? pos + 1 : length) - see_from);  // positions from see_from on
  // with a sight: of the 32 positions from tok on, as bits
  const auto sees_at = [&](int tok) {
    if (!real) return 0u;
    uint32_t x = low_bits((tree ? base_pos : q.causal ? pos + 1 : length) - tok) & (~low_bits(see_from - tok) | low_bits(g.sinks - tok));
    const int at = tok - base_pos;
    if (tree && at > -32 && at < count) {
      const int w = at >> 5, by = at & 31;
      const uint32_t lo = w >= 0 ? kin[w] : 0, hi = (w + 1) * 32 < count ? kin[w + 1] : 0;
      x |= (uint32_t)(((uint64_t)hi << 32 | lo) >> by) & low_bits(count - at);
    }
    return x;
  };
  half8 qf[NS];
  {
    const uint16_t *p = q.q + (row0 + j) * q.q_row + (int64_t)qh * q.q_head + h * 8;
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[s] = real ? load_query(p + s * 16, q.half_type, q.vec, q.scale_two) : half8{};
  }
  // what some of the wavefront's rows see, and what all of them do
  const int w_first = tile * tile_rows + wave * 32, w_last = min(w_first + 31, q.share * count - 1);  // (tile_rows: whole wavefronts)
  const bool busy = wave * 32 < min(rows, tile_rows);
  const int j_first = w_first / q.share, j_last = w_last / q.share;
  const int any_to = !busy ? INT_MIN : q.causal && !tree ? length - count + j_last + 1 : length, all_to = tree ? base_pos : q.causal ? length - count + j_first + 1 : length;
  const int any_from = q.causal && q.window ? length - count + (tree ? -1 : j_first) - q.window + 1 : 0;
  const int all_from = q.causal && q.window ? length - count + (tree ? count - 1 : j_last) - q.window + 1 : 0;
  const int each = steps / pc.parts, longer = steps - each * pc.parts;  // steps in equal pieces, the first ones one longer
  const int t0 = each * pc.nth + min(pc.nth, longer), t1 = t0 + each + (pc.nth < longer);

  f32x16 o[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[c][e] = 0.0f;
  const float rest = q.scale_rest;  // scores and their maximum are what it multiplies
  float m = real ? -INFINITY : 0.0f, l = 0.0f;
  f32x16 start;  // of the scores' sums: less the maximum
#pragma unroll
  for (int e = 0; e < 16; ++e) start[e] = 0.0f;

  const ScalarInts table = (ScalarInts)(uintptr_t)(d.table + (int64_t)seq * d.max_pages);
  const int last_block = max(0, length - 1) / kBlockTokens;
  const auto block_at = [&](int block) {  // (a tile's second block may lie behind the last)
    const uint32_t b = (uint32_t)min(block, last_block), pg = cache_page_of(d, b);
    return cache_block(d, q.layer, table[pg], head, b - pg * d.page_blocks);
  };
  // (with a sight a tile's tokens are counted from the first one on, without those between the sinks and the window)
  const int sinks = SIGHT ? sink_blocks(g) : 0;
  const auto place = [&](int at) { return !SIGHT || at >= sinks ? at + from : at; };
  f32x16 sc[TB];
  half8 pf[TB][2];
  const auto scores = [&](const uint4 *kt) {
#pragma unroll
    for (int x = 0; x < TB; ++x) sc[x] = start;
#pragma unroll
    for (int k = 0; k < NS; ++k)
#pragma unroll
      for (int x = 0; x < TB; ++x) {
        const int word = 2 * k + h;
        const uint4 a = kt[(x * (D / 8) + word) * 32 + key_slot(word, col)];
        half8 kh;
        __builtin_memcpy(&kh, &a, 16);
        sc[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kh, qf[k], sc[x], 0, 0, 0);
      }
    reads_ahead<NS * TB>();
  };
  // Probabilities, and whether one is beyond what the maximum may be left behind.
  const auto powers = [&]() {
    half2v most = {(_Float16)0.0f, (_Float16)0.0f};
#pragma unroll
    for (int x = 0; x < TB; ++x)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        HalfWords w;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          w.p[e] = half2v{(_Float16)__builtin_amdgcn_exp2f(sc[x][8 * y + 2 * e] * rest), (_Float16)__builtin_amdgcn_exp2f(sc[x][8 * y + 2 * e + 1] * rest)};
          most = __builtin_elementwise_max(most, w.p[e]);
        }
        pf[x][y] = w.h;
      }
    constexpr _Float16 kMost = (_Float16)(1 << (int)(kTop + kLag));
    return most[0] > kMost || most[1] > kMost;
  };
  const auto probabilities = [&](int tok0, int tok1) {
    if constexpr (SIGHT) {
#pragma unroll
      for (int x = 0; x < TB; ++x) {
        const int tok = x ? tok1 : tok0;
        if (tok + kBlockTokens <= all_to && (tok >= all_from || tok + kBlockTokens <= g.sinks)) continue;
        const uint32_t mine = sees_at(tok) >> (4 * h);
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (!(mine >> (8 * (e >> 2) + (e & 3)) & 1)) sc[x][e] = -INFINITY;
      }
    } else if (tok0 + kTile > all_to || tok0 < all_from) {
      const uint32_t at = (uint32_t)(tok0 + 4 * h - see_from);
#pragma unroll
      for (int x = 0; x < TB; ++x)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (at + 32 * x + 8 * (e >> 2) + (e & 3) >= sees) sc[x][e] = -INFINITY;
    }
    if (__any(powers() || m == -INFINITY)) {
      float top = -INFINITY;
#pragma unroll
      for (int x = 0; x < TB; ++x)
#pragma unroll
        for (int e = 0; e < 16; e += 2) top = fmaxf(top, fmaxf(sc[x][e], sc[x][e + 1]));
      top = fmaxf(top, __shfl_xor(top, 32));
      const bool move = top * rest > kTop + kLag || (m == -INFINITY && top > -INFINITY);  // (scores are relative to the maximum)
      const float by = move ? top - kTop * __builtin_amdgcn_rcpf(rest) : 0.0f, shrink = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(-by * rest);
      if (move) m = (m == -INFINITY ? 0.0f : m) + by;
      l *= shrink;
#pragma unroll
      for (int c = 0; c < NC; ++c) o[c] *= shrink;
#pragma unroll
      for (int x = 0; x < TB; ++x) sc[x] -= by;
      start -= by;
      powers();
    }
    // (32 tokens first: a long tail's probabilities one by one would be lost in the row's sum.  The row's sum itself, 64 tokens, 32: heads of 64, 96, 128, 256
    // channels, prompts of 4,534, 2 heads of 8: 111, 124, 144, 417 us; 113, 127, 142, 407; 112, 125, 142, 408)
#pragma unroll
    for (int x = 0; x < TB; ++x) l += add_up(add_up(0.0f, pf[x][0]), pf[x][1]);
  };
  const auto weigh = [&](const uint4 *vt) {
#pragma unroll
    for (int x = 0; x < TB; ++x)
#pragma unroll
      for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const uint4 a = vt[((x * NC + c) * 4 + 2 * y + h) * 32 + value_slot(c, col)];
          half8 vh;
          __builtin_memcpy(&vh, &a, 16);
          o[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vh, pf[x][y], o[c], 0, 0, 0);
        }
    reads_ahead<NC * TB * 2>();
  };
  if (length > 0) {  // (an empty sequence has one step and no page)
    if constexpr (RING) {
      // A tile is copied in chunks of 1 KiB, one to a wavefront after the other.
      constexpr int kChunks = (40 * D + 1023) / 1024, kAll = TB * kChunks, kMost = (kAll + WAVES - 1) / WAVES, kLess = kAll / WAVES;
      const uint32_t ring = (uint32_t)uniform((int)lds_address(sh.raw[0]));
      const auto copy = [&](int t) {
        const uint32_t slot = ring + (uint32_t)(t - t0) % kRing * (TB * 40 * D);
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
          const int c = i * WAVES + wave, x = c / kChunks, at = c % kChunks * 1024;
          if (i < kLess || c < kAll) {
            const unsigned char *blk = block_at(place(t * kTile + x * kBlockTokens) / kBlockTokens);
            if (40 * D % 1024 == 0 || lane * 16 < 40 * D - at) copy_to_lds(blk + at, slot + x * (40 * D) + at, lane * 16);
          }
        }
      };
      // This wavefront's chunks are there, but those of the `later` tiles that it asked for last.
      const auto arrived = [&](auto later) {
        constexpr int kLater = decltype(later)::value;
        if (kMost == kLess || wave < kAll % WAVES) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kMost * kLater) : "memory");
        else asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLess * kLater) : "memory");
      };
      const auto unpack = [&](int t) {
        const unsigned char *b0 = reinterpret_cast<const unsigned char *>(sh.raw[(uint32_t)(t - t0) % kRing]), *b1 = b0 + (TB == 2 ? 40 * D : 0);
        uint4 *const k = sh.k[(t - t0) & 1], *const v = sh.v[(t - t0) & 1];
        Words<D> words[NP];
        constexpr bool kWhole = 2 * kPairs<D, TB> % kLanes == 0;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          const int u = i * kLanes + threadIdx.x;
          if (kWhole || u < 2 * kPairs<D, TB>) load_words<D, TB>(words[i], u, b0, b1);
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          const int u = i * kLanes + threadIdx.x;
          if (kWhole || u < 2 * kPairs<D, TB>) put_words<D, TB>(words[i], u, k, v);
        }
      };
      for (int i = 0; i < kRing - 1; ++i)
        if (t0 + i < t1) copy(t0 + i);
      if (t0 + kRing - 1 <= t1) arrived(std::integral_constant<int, kRing - 2>());
      else arrived(std::integral_constant<int, 0>());
      meet();
      unpack(t0);
      if (t0 + kRing - 1 < t1) copy(t0 + kRing - 1);
      for (int t = t0; t < t1; ++t) {
        if (t + kRing <= t1) arrived(std::integral_constant<int, kRing - 2>());
        else arrived(std::integral_constant<int, 0>());
        meet();  // (tile t is unpacked, the next one's codes are there, and what this turn writes over has been read)
        if (t + kRing < t1) copy(t + kRing);
        if (t + 1 < t1) unpack(t + 1);
        const int tok0 = place(t * kTile), tok1 = SIGHT && TB == 2 ? place(t * kTile + kBlockTokens) : tok0;
        const auto seen = [&](int tok) { return tok < any_to && (tok + kBlockTokens > any_from || tok < g.sinks); };
        if (SIGHT ? !(seen(tok0) || seen(tok1)) : !(tok0 < any_to && tok0 + kTile > any_from)) continue;
        // (matrix instructions first: the other wavefront of the SIMD has its exponentials beside them)
        __builtin_amdgcn_s_setprio(1);
        scores(sh.k[(t - t0) & 1]);
        __builtin_amdgcn_s_setprio(0);
        probabilities(tok0, tok1);
        __builtin_amdgcn_s_setprio(1);
        weigh(sh.v[(t - t0) & 1]);
        __builtin_amdgcn_s_setprio(0);
      }
    } else {
      Words<D> next[NP];
      constexpr bool kWhole = 2 * kPairs<D, TB> % kLanes == 0;
      const auto load_tile = [&](Words<D> (&to)[NP], int t) {
        const int block = (from + t * kTile) / kBlockTokens;
        const unsigned char *b0 = block_at(block), *b1 = TB == 2 ? block_at(block + 1) : b0;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          const int u = i * kLanes + threadIdx.x;
          if (kWhole || u < 2 * kPairs<D, TB>) load_words<D, TB>(to[i], u, b0, b1);
        }
      };
      const auto put_tile = [&](const Words<D> (&of)[NP], uint4 *k, uint4 *v) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          const int u = i * kLanes + threadIdx.x;
          if (kWhole || u < 2 * kPairs<D, TB>) put_words<D, TB>(of[i], u, k, v);
        }
      };
      {
        Words<D> first[NP];
        load_tile(first, t0);
        if (t0 + 1 < t1) load_tile(next, t0 + 1);
        put_tile(first, sh.k[0], sh.v[0]);
      }
      __syncthreads();
      for (int t = t0; t < t1; ++t) {
        const int tok0 = from + t * kTile, now = (t - t0) & 1;
        const bool some = tok0 < any_to && tok0 + kTile > any_from;
        if (t + 1 < t1) put_tile(next, sh.k[now ^ 1], sh.v[now ^ 1]);
        if (t + 2 < t1) load_tile(next, t + 2);
        if (some) {
          __builtin_amdgcn_s_setprio(1);
          scores(sh.k[now]);
          __builtin_amdgcn_s_setprio(0);
          probabilities(tok0, tok0);
          __builtin_amdgcn_s_setprio(1);
          weigh(sh.v[now]);
          __builtin_amdgcn_s_setprio(0);
        }
        __syncthreads();
      }
    }
  }
  l += __shfl_xor(l, 32);
  m *= rest;

  if (SIGHT && split && threadIdx.x == 0 && pc.nth == 0) d.joins[pc.entry * d.kv_heads + head] = (uint32_t)pc.parts << 16 | (uint32_t)pc.part;
  if (SIGHT && pc.parts > 1) {  // (joined by the next launch)
    float *p = d.part + ((int64_t)(pc.part + pc.nth) * WAVES + wave) * (64 * 16 * NC) + lane * 2;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < 16; e += 2) *reinterpret_cast<float2 *>(p + (c * 8 + e / 2) * 128) = make_float2(o[c][e], o[c][e + 1]);
    *reinterpret_cast<float2 *>(d.part_ml + (((int64_t)(pc.part + pc.nth) * WAVES + wave) * 64 + lane) * 2) = make_float2(m, l);
    return;
  }
  if (!SIGHT && pc.parts > 1) {
    // Parts lie as the lanes hold them, so that stores are whole lines and the last workgroup to arrive joins them in its own registers.
    const auto part_of = [&](int i) { return d.part + ((int64_t)(pc.part + i) * WAVES + wave) * (64 * 16 * NC) + lane * 2; };
    const auto ml_of = [&](int i) { return d.part_ml + (((int64_t)(pc.part + i) * WAVES + wave) * 64 + lane) * 2; };
    {
      float *p = part_of(pc.nth);
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < 16; e += 2) put_pair(p + (c * 8 + e / 2) * 128, o[c][e], o[c][e + 1]);
      put_pair(ml_of(pc.nth), m, l);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wavefront's part is out ...
    __syncthreads();                                  // ... and that of the others
    if (threadIdx.x == 0) {
      uint32_t *there = d.arrived + pc.part;
      flag = __hip_atomic_fetch_add(there, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)pc.parts - 1;
      if (flag) __hip_atomic_store(there, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!flag) return;
    m = -INFINITY;
    for (int i = 0; i < pc.parts; ++i) m = fmaxf(m, get_pair(ml_of(i)).x);
    l = 0.0f;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[c][e] = 0.0f;
    for (int i = 0; i < pc.parts; ++i) {
      const float2 ml = get_pair(ml_of(i));
      const float by = ml.x == -INFINITY && m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ml.x - m), *p = part_of(i);
      l += ml.y * by;
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          const float2 x = get_pair(p + (c * 8 + e / 2) * 128);
          o[c][e] += x.x * by;
          o[c][e + 1] += x.y * by;
        }
    }
  }
  if (!real) return;
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int e = 0; e < 16; e += 4)
      store_row(q, row0 + j, qh, c * 32 + 2 * e + 4 * h, f32x4{o[c][e], o[c][e + 1], o[c][e + 2], o[c][e + 3]}, m, l);
}

template <int D, int WAVES>
__global__ __launch_bounds__(WAVES * 64, D == 256 ? 1 : 2) void k_cache_prompt(CacheDev d, CacheQuery q, int tiles, int tile_rows, int split, uint32_t first) {
  attend_many<D, WAVES, tile_blocks(D), false>(d, q, CacheSight{}, tiles, tile_rows, split, first);
}

template <int D, int WAVES, int TB>
__global__ __launch_bounds__(WAVES * 64, D == 256 ? 1 : 2) void k_cache_prompt_sight(CacheDev d, CacheQuery q, CacheSight g, int tiles, int tile_rows, int split, uint32_t first) {
  attend_many<D, WAVES, TB, true>(d, q, g, tiles, tile_rows, split, first);
}

// Joins what several workgroups have of a row tile: a wavefront has 32 channels of 32 rows, held as they lie in the parts.  (Up to 32 parts of 128 KiB
// are too much for the last workgroup to arrive, as in k_cache_prompt; a few are not.  252 rows of 128 channels, 8 heads, behind one sequence of 32,000, 4 of up to
// 60,063, 16 of up to 6,001, 32 of up to 2,000: 117, 206, 94, 72 us so, without a sight, and 68, 200, 103, 81 here, as a tree that is a chain.)
template <int D, int WAVES>
__global__ __launch_bounds__(256) void k_cache_join_many(CacheDev d, CacheQuery q, CacheSight g, int tiles, int tile_rows) {
  constexpr int NC = D / 32, kUnit = WAVES * NC;
  static_assert(kUnit % 4 == 0, "whole workgroups");
  const int lane = threadIdx.x & 63, col = lane & 31, h = lane >> 5, x = blockIdx.x * 4 + uniform(threadIdx.x >> 6), entry = x / kUnit, wave = x % kUnit / NC, c = x % NC;
  const int head = entry % d.kv_heads, item = entry / d.kv_heads % q.r.n, tile = tiles - 1 - entry / d.kv_heads / q.r.n;
  const Span sp = find_span<true>(d, q, g, item, tile, tile_rows, 32, false);
  if (!sp.count) return;
  const uint32_t join = d.joins[entry], parts = join >> 16, first = join & 0xffff;
  const int row = wave * 32 + col, mine = tile * tile_rows + row;
  if (parts < 2 || !__any(row < min(q.share * sp.count - tile * tile_rows, tile_rows))) return;
  const float *ml = d.part_ml + ((int64_t)first * WAVES + wave) * 128 + lane * 2, *p = d.part + ((int64_t)first * WAVES + wave) * (1024 * NC) + c * 1024 + lane * 2;
  float m = -INFINITY;
#pragma unroll 8
  for (uint32_t i = 0; i < parts; ++i) m = fmaxf(m, ml[i * WAVES * 128]);
  float l = 0.0f;
  f32x16 o;
#pragma unroll
  for (int e = 0; e < 16; ++e) o[e] = 0.0f;
#pragma unroll 4
  for (uint32_t i = 0; i < parts; ++i) {
    const float2 at = *reinterpret_cast<const float2 *>(ml + i * WAVES * 128);
    const float by = at.x == -INFINITY && m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(at.x - m);
    l += at.y * by;
#pragma unroll
    for (int e = 0; e < 16; e += 2) {
      const float2 y = *reinterpret_cast<const float2 *>(p + (int64_t)i * WAVES * (1024 * NC) + e * 64);
      o[e] += y.x * by;
      o[e + 1] += y.y * by;
    }
  }
  if (row >= min(q.share * sp.count - tile * tile_rows, tile_rows)) return;
#pragma unroll
  for (int e = 0; e < 16; e += 4)
    store_row(q, sp.row0 + mine / q.share, head * q.share + mine % q.share, c * 32 + 2 * e + 4 * h, f32x4{o[e], o[e + 1], o[e + 2], o[e + 3]}, m, l);
}

template <int D, int WAVES, int TB>
void launch(const CacheDev &d, const CacheQuery &q, const CacheSight *g, hipStream_t s) {
  constexpr int kWorkers = kUnits * at_once(D, WAVES), kSplits = kSplit * kUnits * at_once(D, 8) / kWorkers;
  const int64_t rows = (int64_t)q.share * q.r.max_new;
  const int tiles = (int)((rows + WAVES * 32 - 1) / (WAVES * 32)), tile_rows = (int)((rows + tiles - 1) / tiles + 31) / 32 * 32;  // (all about as long)
  const int64_t groups = (int64_t)tiles * q.r.n * d.kv_heads;
  static_assert(kSplits >= 1 && kSplits * kWorkers <= kMostEntries, "all row tiles of all items are planned");
  // (steps of all row tiles are counted in 32 bits)
  const bool split = groups < (q.r.n > 1 ? kSplits : 1) * kWorkers && groups * ((int64_t)d.max_pages * d.page_blocks + 1) < (int64_t)1 << 32;
  const int64_t all = split ? groups + kWorkers : groups, most = 1 << 22;  // (of a launch; one that finds no rows takes 10 ns: 512 items of 8 heads, one of 32,768 rows, 28 ms of which it takes 6)
  for (int64_t at = 0; at < all; at += most) {
    const uint32_t grid = (uint32_t)(all - at < most ? all - at : most);
    if (g) k_cache_prompt_sight<D, WAVES, TB><<<grid, WAVES * 64, sizeof(Shared<D, TB, true>), s>>>(d, q, *g, tiles, tile_rows, split, (uint32_t)at);
    else if constexpr (TB == tile_blocks(D) && WAVES == (D == 256 ? 4 : 8)) k_cache_prompt<D, WAVES><<<grid, WAVES * 64, sizeof(Shared<D, TB, by_copies(D, false)>), s>>>(d, q, tiles, tile_rows, split, (uint32_t)at);
  }
  if (g && split) k_cache_join_many<D, WAVES><<<(uint32_t)(groups * WAVES * (D / 32) / 4), 256, 0, s>>>(d, q, *g, tiles, tile_rows);
}

}  // namespace

// Rows of parts: at most two pieces that are parts for each that runs at once.
size_t cache_prompt_part_rows() { return (size_t)2 * kUnits * kRows; }
size_t cache_prompt_groups() { return (size_t)4 * kUnits; }

void launch_cache_prompt(const CacheDev &d, const CacheQuery &q, const CacheSight *g, hipStream_t s) {
  // With a sight 65 to 128 rows have workgroups of 4 wavefronts, two to a unit, against 8: 128 rows of 128 channels, 8 heads, 16 sequences of up to 6,001, 4 of up to 60,063, 32 of up to 2,000,
  // one of 32,000: 67, 148, 56, 67 us and 86, 156, 67, 59; of 64 channels 50, 109, 41, 59 and 67, 121, 52, 49; 252 rows of the first: 120 and 105.  Without a
  // sight they have 8, and the join of k_cache_prompt: the same 128 rows of 128 channels 72, 149, 56, 105 us, as a tree that is a chain 65, 143, 52, 66.
  const bool few = g && (int64_t)q.share * q.r.max_new <= 128;
  switch (d.head_dim) {
    case 64: return few ? launch<64, 4, 1>(d, q, g, s) : launch<64, 8, 2>(d, q, g, s);
    case 96: return few ? launch<96, 4, 1>(d, q, g, s) : launch<96, 8, 2>(d, q, g, s);
    case 128: return few ? launch<128, 4, 1>(d, q, g, s) : launch<128, 8, 2>(d, q, g, s);
    default: return launch<256, 4, 1>(d, q, g, s);
  }
}

hipError_t allow_large_lds_cache_prompt() {
  hipError_t e = hipSuccess;
  const auto allow = [&](auto kernel, size_t bytes) {
    if (e == hipSuccess) e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  };
  allow(k_cache_prompt<96, 8>, sizeof(Shared<96, 2, by_copies(96, false)>));
  allow(k_cache_prompt<128, 8>, sizeof(Shared<128, 2, by_copies(128, false)>));
  allow(k_cache_prompt<256, 4>, sizeof(Shared<256, 1, by_copies(256, false)>));
  allow(k_cache_prompt_sight<96, 8, 2>, sizeof(Shared<96, 2, true>));
  allow(k_cache_prompt_sight<128, 8, 2>, sizeof(Shared<128, 2, true>));
  allow(k_cache_prompt_sight<256, 4, 1>, sizeof(Shared<256, 1, true>));
  return e;
}

}  // namespace rtams
