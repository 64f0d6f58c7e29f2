// Attention of many rows over the cache in 4 bits: prompts, and pieces of prompts behind what the cache already holds.
//
// The formulas are those of cache_attend.hip; here arithmetic bounds: 4 * head_dim flops for a row and token.  A workgroup has
// 32 rows for each wavefront (a row: a token's query head of those that share a kv head) and goes over the tokens that they see
// 64 at a time (32 where head_dim is 256): all its lanes turn their codes into halves in LDS, once for all rows, while the loads of the next
// tokens are under way; two buffers, one barrier.  Scores are S^T = K Q^T with Q in registers; a lane has one row's scores and its
// probabilities are the operand that O^T = V^T P^T takes.  The running maximum enters as the start of the scores' sums and moves
// only where a score has left it far behind (kLag).  LDS holds operands in the order in which the lanes take them, 16 bytes each; the slots are
// swapped so that writing meets no bank twice.  Where rows are too few to fill the chip the tokens are split, and the last
// part of a row to arrive joins them.
//
// The scale's power of two is in the query, exact as an operand; what is left of it multiplies scores in 32 bits (in the query and rounded there:
// 576 us instead of 580, and half outputs 1.6 to 1.8 times as far from 64 bits as their own rounding alone, not 1.5 to 1.6).
//
// Measured: a prompt of 8,192 tokens, 32 heads of 128 over 8: 575 to 640 us from card to card for 550 GFLOP, 860 to 957 TFLOP/s where a plain product
// of 8,192 squared reaches 1,140 in bfloat16 and 1,084 in halves.  Vector instructions (exponentials, masks, codes) take 48 % of the cycles, matrix
// instructions 41 %, and two wavefronts of a SIMD overlap them in part.  Heads of 64, 96, 128, 256 on one card: 455, 551, 640, 2,314 us; 604, 749, 859,
// 475 TFLOP/s: the fewer the channels, the more exponentials for a flop; at 256 one wavefront fits a SIMD.  At 128 channels, on a card of 580 us:
// 4 wavefronts a workgroup 710, wavefronts half a tile apart 610.
#include "../../include/rtams_cache.h"

#include <climits>

#include "cache_mm.h"
#include "rtams_dev.h"

namespace rtams {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int tile_blocks(int head_dim) { return head_dim == 256 ? 1 : 2; }  // of 32 tokens; registers decide
constexpr int kRows = 256;       // of a workgroup's parts at most

// Workgroups that a compute unit runs at once: registers decide.
constexpr int at_once(int head_dim, int waves) { return waves == 8 || head_dim == 256 ? 1 : 2; }

template <int D>
struct Staging {  // tiles in LDS: operands of 16 bytes
  uint4 k[2][tile_blocks(D) * 4 * D];  // [block][word][token]
  uint4 v[2][tile_blocks(D) * 4 * D];  // [block][32 channels][lane group][channel]
};

__device__ inline int key_slot(int word, int token) { return token ^ (((word >> 1) & 7) << 1); }
__device__ inline int value_slot(int tile, int ch) { return ch ^ ((tile & 1) << 3); }

template <int D>
struct Words {  // two words of keys or values with their steps and zeros
  uint2 code;
  HalfWords step, zero;  // keys: w[0] holds both
};

// Pairs of words of a tile whose blocks are at blk0 and blk1: the first kPairs<D> are keys, as many more values.
template <int D>
constexpr int kPairs = tile_blocks(D) * 2 * D;
template <int D>
__device__ inline void load_words(Words<D> &p, int u, const unsigned char *blk0, const unsigned char *blk1) {
  constexpr int WP = D / 16, VC = value_chunk(D);
  if (u < kPairs<D>) {
    const int token = u / WP, wp = u % WP;
    const unsigned char *blk = token < 32 ? blk0 : blk1;
    p.code = *reinterpret_cast<const uint2 *>(blk + (token & 31) * (D / 2) + wp * 8);
    p.step.w[0] = *reinterpret_cast<const uint32_t *>(blk + 16 * D + ((token & 31) * (D / 32) + (wp >> 1)) * 4);
  } else {
    const int x = u - kPairs<D>, idx = x % (2 * D);
    const unsigned char *blk = x < 2 * D ? blk0 : blk1;
    p.code = *reinterpret_cast<const uint2 *>(blk + 20 * D + idx * 8);
    const int group = VC == 4 ? (idx >> 7) * 2 + (idx & 1) : idx >> 6, b = VC == 4 ? (idx >> 5) & 3 : (idx >> 4) & 3;
    const uint4 s = *reinterpret_cast<const uint4 *>(blk + 36 * D + group * 128 + b * 16), z = *reinterpret_cast<const uint4 *>(blk + 36 * D + group * 128 + 64 + b * 16);
    __builtin_memcpy(&p.step, &s, 16);
    __builtin_memcpy(&p.zero, &z, 16);
  }
}

template <int D>
__device__ inline void put_words(const Words<D> &p, int u, uint4 *k, uint4 *v) {
  constexpr int WP = D / 16, VC = value_chunk(D);
  if (u < kPairs<D>) {
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
    const int y = u - kPairs<D>, idx = y % (2 * D), block = y / (2 * D);
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
  int seq, count, length, from, steps;  // from: first position, at a block's begin
};

// Row tile `tile` (of `rows` rows) of an item; count 0: none.
__device__ inline Span find_span(const CacheDev &d, const CacheQuery &q, int item, int tile, int rows, int step_tokens, bool tell) {
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
  const int to = q.causal ? s.length - s.count + last + 1 : s.length;
  s.from = q.causal && q.window ? max(0, s.length - s.count + tile * rows / q.share - q.window + 1) & ~(kBlockTokens - 1) : 0;
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

template <int D>
union Shared {
  Staging<D> tile;
  float steps[kMostEntries];  // in front of them
};

// Which piece is workgroup blockIdx.x's, where tokens are split (find_piece in cache_attend.hip has the same for few rows).  One wavefront's work.
__device__ inline bool find_piece(const CacheDev &d, const CacheQuery &q, int tiles, int rows, int step_tokens, uint32_t workers, float *steps, Piece *piece) {
  const int lane = threadIdx.x & 63, n = q.r.n * tiles;
  uint32_t all = 0;
  float longest = 1.0f;
  for (int base = 0; base < (n + 255) / 256 * 256; base += 64) {
    const int e = base + lane;
    const Span sp = e < n ? find_span(d, q, e % q.r.n, tiles - 1 - e / q.r.n, rows, step_tokens, blockIdx.x == 0) : Span{};
    const int mine = sp.count ? sp.steps : 0;
    steps[e] = (float)mine;
    longest = fmaxf(longest, (float)mine);
    all += last_lane(wave_running_sum((uint32_t)mine));
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) longest = fmaxf(longest, __shfl_xor(longest, o));
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  // (never less than an even share: scratch has room for twice as many parts as there are workers, as in cache_attend.hip)
  const uint32_t share = max(1u, (all * (uint32_t)d.kv_heads + workers - 1) / workers), size = share > 1 ? piece_steps(steps, n, d.kv_heads, share, workers) : 1;
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
  constexpr int kAhead = 6, kRead = 0x100, kMfma = 0x8;
  __builtin_amdgcn_sched_group_barrier(kRead, kAhead, 0);
#pragma unroll
  for (int i = 0; i < N - kAhead; ++i) {
    __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
    __builtin_amdgcn_sched_group_barrier(kRead, 1, 0);
  }
  __builtin_amdgcn_sched_group_barrier(kMfma, kAhead, 0);
}

template <int D, int WAVES>
__global__ __launch_bounds__(WAVES * 64, D == 256 ? 1 : 2) void k_cache_prompt(CacheDev d, CacheQuery q, int tiles, int tile_rows, int split, uint32_t first) {
  constexpr int kLanes = WAVES * 64, NS = D / 16, NC = D / 32, NP = (2 * kPairs<D> + kLanes - 1) / kLanes;
  constexpr int TB = tile_blocks(D), kTile = TB * kBlockTokens;
  extern __shared__ uint4 lds[];
  Shared<D> &shared = *reinterpret_cast<Shared<D> *>(lds);
  Staging<D> &sh = shared.tile;
  __shared__ Piece piece;
  __shared__ int flag;
  Piece pc;
  if (split) {
    if (threadIdx.x < 64) {
      const bool found = find_piece(d, q, tiles, tile_rows, kTile, kUnits * at_once(D, WAVES), shared.steps, &piece);
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
  const Span sp = find_span(d, q, item, tile, tile_rows, kTile, !split && tile == 0 && head == 0 && threadIdx.x == 0);
  const int count = uniform(sp.count);
  if (!count) return;
  const int64_t row0 = sp.row0;
  const int seq = uniform(sp.seq), length = uniform(sp.length), from = uniform(sp.from), steps = uniform(sp.steps), rows = q.share * count - tile * tile_rows;  // rows: from this tile on
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), col = lane & 31, h = lane >> 5;

  // this lane's row
  const int row = wave * 32 + col, mine = tile * tile_rows + row;
  const bool real = row < min(rows, tile_rows);
  const int j = real ? mine / q.share : 0, qh = head * q.share + (real ? mine % q.share : 0);
  const int pos = length - count + j;
  const int see_from = q.causal && q.window ? pos - q.window + 1 : 0;
  const uint32_t sees = !real ? 0 : (uint32_t)max(0, (q.causal ? pos + 1 : length) - see_from);  // positions from see_from on
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
  const int any_to = !busy ? INT_MIN : q.causal ? length - count + j_last + 1 : length, all_to = q.causal ? length - count + j_first + 1 : length;
  const int any_from = q.causal && q.window ? length - count + j_first - q.window + 1 : 0, all_from = q.causal && q.window ? length - count + j_last - q.window + 1 : 0;
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
  Words<D> next[NP];
  const auto load_tile = [&](Words<D> (&to)[NP], int t) {
    const int block = (from + t * kTile) / kBlockTokens;
    const unsigned char *b0 = block_at(block), *b1 = TB == 2 ? block_at(block + 1) : b0;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int u = i * kLanes + threadIdx.x;
      if (2 * kPairs<D> % kLanes == 0 || u < 2 * kPairs<D>) load_words<D>(to[i], u, b0, b1);
    }
  };
  const auto put_tile = [&](const Words<D> (&of)[NP], uint4 *k, uint4 *v) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int u = i * kLanes + threadIdx.x;
      if (2 * kPairs<D> % kLanes == 0 || u < 2 * kPairs<D>) put_words<D>(of[i], u, k, v);
    }
  };
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
  const auto probabilities = [&](int tok0) {
    if (tok0 + kTile > all_to || tok0 < all_from) {
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
        // (matrix instructions first: the other wavefront of the SIMD has its exponentials beside them)
        __builtin_amdgcn_s_setprio(1);
        scores(sh.k[now]);
        __builtin_amdgcn_s_setprio(0);
        probabilities(tok0);
        __builtin_amdgcn_s_setprio(1);
        weigh(sh.v[now]);
        __builtin_amdgcn_s_setprio(0);
      }
      __syncthreads();
    }
  }
  l += __shfl_xor(l, 32);
  m *= rest;

  if (pc.parts > 1) {
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
void launch(const CacheDev &d, const CacheQuery &q, hipStream_t s) {
  constexpr int kWorkers = kUnits * at_once(D, WAVES);
  const int64_t rows = (int64_t)q.share * q.r.max_new;
  const int tiles = (int)((rows + WAVES * 32 - 1) / (WAVES * 32)), tile_rows = (int)((rows + tiles - 1) / tiles + 31) / 32 * 32;  // (all about as long)
  const int64_t groups = (int64_t)tiles * q.r.n * d.kv_heads;
  static_assert(kSplit * kWorkers <= kMostEntries, "all row tiles of all items are planned");
  // (steps of all row tiles are counted in 32 bits)
  const bool split = groups < (q.r.n > 1 ? kSplit : 1) * kWorkers && groups * ((int64_t)d.max_pages * d.page_blocks + 1) < (int64_t)1 << 32;
  const int64_t all = split ? groups + kWorkers : groups, most = 1 << 22;  // (of a launch; one that finds no rows takes 10 ns: 512 items of 8 heads, one of 32,768 rows, 28 ms of which it takes 6)
  for (int64_t at = 0; at < all; at += most)
    k_cache_prompt<D, WAVES><<<(uint32_t)(all - at < most ? all - at : most), WAVES * 64, sizeof(Shared<D>), s>>>(d, q, tiles, tile_rows, split, (uint32_t)at);
}

}  // namespace

// Rows of parts: at most two pieces that are parts for each that runs at once.
size_t cache_prompt_part_rows() { return (size_t)2 * kUnits * kRows; }
size_t cache_prompt_groups() { return (size_t)4 * kUnits; }

void launch_cache_prompt(const CacheDev &d, const CacheQuery &q, hipStream_t s) {
  switch (d.head_dim) {
    case 64: return launch<64, 8>(d, q, s);
    case 96: return launch<96, 8>(d, q, s);
    case 128: return launch<128, 8>(d, q, s);
    default: return launch<256, 4>(d, q, s);
  }
}

hipError_t allow_large_lds_cache_prompt() {
  const auto allow = [](const void *f, size_t bytes) { return hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes); };
  if (const hipError_t e = allow(reinterpret_cast<const void *>(k_cache_prompt<128, 8>), sizeof(Shared<128>))) return e;
  return allow(reinterpret_cast<const void *>(k_cache_prompt<256, 4>), sizeof(Shared<256>));
}

}  // namespace rtams
