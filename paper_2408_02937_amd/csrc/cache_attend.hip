// Attention of few rows over the cache in 4 bits: single tokens and some tokens of each sequence.
//
//   s_t = scale * q . K_t,  o = sum_t exp(s_t - m) V_t / sum_t exp(s_t - m),  m the running maximum
//
// Bound by the bytes of the cache: 1.25 a channel and token for keys and values together.  A step of a workgroup is 128 tokens of
// one kv head, 32 to a wavefront; a workgroup takes a piece of a head's steps, of a size that lets all pieces run at once, so
// that ragged lengths fill the chip alike.  The query heads that share a kv head (times an item's rows) are the 16 columns of
// the matrix instructions, of one tile or two.  A wavefront copies its blocks into LDS of its own, the next one while it works on this one;
// codes become halves in registers.  Scores come out as S^T = K Q^T, tokens down and rows across, which is the operand that O^T = V^T P^T
// takes, so nothing is transposed.  A query is a half as it is, times a power of two; what is left of the scale meets the scores in 32 bits, in the
// same instruction that takes the maximum off.  What a piece leaves of a row goes to scratch; the last piece of it to arrive joins them, in order.
//
// Measured: 8 sequences of 16 to 131 thousand tokens, 8 heads of 128, 32 query heads: 170 us for 874 MB, 5.1 TB/s where a plain read of 4 GiB reaches
// 6.0.  32 of 0.5 to 4 thousand: 26.9 us for 94 MB; of these 3 are the plan, 5 pass until the first blocks are there, 3 are the join.
// One token over 100: 4.8 us.  Heads of 64, 96, 128, 256 channels, 8 times 32,000 tokens each: 4.2, 4.7, 4.7, 5.0 TB/s.
#include "../../include/rtams_cache.h"

#include "cache_mm.h"
#include "rtams_dev.h"

namespace rtams {

namespace {

constexpr int kLanes = 256, kWaves = 4, kStep = kWaves * kBlockTokens;

// Workgroups that a compute unit runs at once: registers decide, and from 128 channels on LDS (40 * D * 8 bytes of blocks).
constexpr int at_once(int head_dim, int tiles) {
  return tiles == 2 ? (head_dim == 64 ? 3 : 2) : head_dim == 64 ? 5 : head_dim == 96 ? 4 : head_dim == 128 ? 3 : 1;
}

struct Span {  // what an item asks for
  int seq, count, length, low;  // low: first position that a row of it sees, rounded down to a block
  int steps;
  int tiles;  // of its rows
  int64_t row0;
};

// Items i + 64 k of the launch, for k of 0 .. N - 1; steps 0 behind the last one.  Loads are asked for together, whatever they find: each is
// a trip to memory, at the beginning of a launch.
template <int N, int ROWS>
__device__ inline void find_spans(const CacheDev &d, const CacheQuery &q, int i, bool tell, Span (&s)[N]) {
  const int n = q.r.n;
  int first[N], past[N], seq[N], length[N];
#pragma unroll
  for (int k = 0; k < N; ++k) first[k] = min(i + 64 * k, n - 1), past[k] = first[k] + 1, seq[k] = first[k];
  if (q.r.seqs)
#pragma unroll
    for (int k = 0; k < N; ++k) seq[k] = q.r.seqs[min(i + 64 * k, n - 1)];
  if (q.r.starts)
#pragma unroll
    for (int k = 0; k < N; ++k) {
      first[k] = q.r.starts[min(i + 64 * k, n - 1)];
      past[k] = q.r.starts[min(i + 64 * k, n - 1) + 1];
    }
#pragma unroll
  for (int k = 0; k < N; ++k) length[k] = d.lengths[(uint32_t)seq[k] < (uint32_t)d.max_seqs ? seq[k] : 0];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const bool there = i + 64 * k < n, known = (uint32_t)seq[k] < (uint32_t)d.max_seqs;
    const bool rows = first[k] >= 0 && past[k] >= first[k] && past[k] <= q.r.rows && past[k] - first[k] <= q.r.max_new;
    const bool ok = rows && known && (!q.causal || past[k] - first[k] <= length[k]);
    s[k].row0 = first[k];
    s[k].seq = seq[k];
    s[k].count = there && ok ? past[k] - first[k] : 0;
    s[k].length = length[k];
    if (tell && there && !ok) cache_raise(d, RTAMS_EINVAL);
    const int low = length[k] - s[k].count - q.window + 1;
    s[k].low = q.window && low > 0 ? low & ~(kBlockTokens - 1) : 0;
    s[k].steps = s[k].count <= 0 ? 0 : length[k] > s[k].low ? (length[k] - s[k].low + kStep - 1) / kStep : 1;
    s[k].tiles = (q.share * s[k].count + ROWS - 1) / ROWS;
  }
}

constexpr int kAhead = 2;   // blocks of a wavefront that are in LDS or on their way

struct Piece {  // steps [sa, sb) of a row tile of an item's head
  Span sp;
  int item, head, tile, sa, sb;
  int parts, nth;  // pieces of the tile; which one this is
  int part;        // where the tile's parts begin, if there are several
};

constexpr int kRound = 256;  // items that the planning wavefront has at a time, four to a lane at most

template <int D, int NR>
struct alignas(16) Shared {
  union {
    unsigned char ring[kWaves][kAhead][40 * D];
    float o[kWaves][16][D + 4];  // when the rings are read: the wavefronts' parts of 16 rows
    float steps[kRound];         // in front of it all: of each item
  };
  float ml[kWaves][16 * NR][2];
  Piece piece;
  int last;
};

// Which piece is workgroup blockIdx.x's: the items' steps, the size of a piece, and the pieces of the items in front.  One wavefront's work, EACH
// items to a lane (lane, lane + 64, ...); false where there is none left.
template <int EACH, int ROWS, class S>
__device__ bool find_piece(const CacheDev &d, const CacheQuery &q, int tiles, uint32_t workers, S &sh) {
  constexpr int kItems = 64 * EACH;
  const int lane = threadIdx.x & 63, n = q.r.n;
  Span sp[EACH];
  uint32_t all = 0;
  for (int base = 0; base < n; base += kItems) {
    find_spans<EACH, ROWS>(d, q, base + lane, blockIdx.x == 0, sp);
    uint32_t sum = 0;
#pragma unroll
    for (int k = 0; k < EACH; ++k) sum += (uint32_t)(sp[k].steps * sp[k].tiles);
    all += last_lane(wave_running_sum(sum));
  }
  all *= (uint32_t)d.kv_heads;
  // Where items are many, pieces are an even share, and long items do not keep the others waiting.  (Never less than an even share: scratch has room
  // for twice as many parts as there are workers.  A head of s steps that is split, s > size, has fewer than 2 s / size parts, all of them fewer than
  // 2 all / size.)
  const uint32_t share = (all + workers - 1) / workers;
  uint32_t size = share > 1 ? share : 1;
  if (share > 1 && n <= kItems && n * d.kv_heads * tiles <= (int)workers / 2) {
#pragma unroll
    for (int k = 0; k < EACH; ++k) sh.steps[64 * k + lane] = (float)sp[k].steps;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    size = piece_steps(sh.steps, n, d.kv_heads * tiles, share, workers);
  }
  const float one_over = 1.0f / (float)size;
  uint32_t before = 0, parts_before = 0;
  for (int base = 0; base < n; base += kItems) {
    if (n > kItems) find_spans<EACH, ROWS>(d, q, base + lane, false, sp);
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      const uint32_t parts = div_up((uint32_t)sp[k].steps, size, one_over), pieces = parts * (uint32_t)(d.kv_heads * sp[k].tiles), shared = parts > 1 ? pieces : 0;
      const uint32_t upto = wave_running_sum(pieces), upto_shared = wave_running_sum(shared), x = blockIdx.x - (before + upto - pieces);
      if (x < pieces) {  // (row tiles fastest: they read the same tokens)
        const uint32_t t = x % (uint32_t)sp[k].tiles, y = x / (uint32_t)sp[k].tiles, head = y / parts;
        sh.piece = Piece{sp[k], base + 64 * k + lane, (int)head, (int)t, 0, 0, (int)parts, (int)(y % parts),
                         (int)(parts_before + upto_shared - shared + (head * sp[k].tiles + t) * parts)};
      }
      if (__any(x < pieces)) return true;
      before += last_lane(upto);
      parts_before += last_lane(upto_shared);
    }
  }
  return false;
}

typedef const __attribute__((address_space(4))) int32_t *ScalarInts;

// The copies of a wavefront's blocks into its ring: its n-th block goes to slot n % kAhead.
template <int D>
struct Copies {
  static constexpr int kCopies = (40 * D + 1023) / 1024;  // loads of a block
  ScalarInts table;
  int head, tok, to;   // next block's first token; end of the piece's tokens
  uint32_t ring, slot;
  uint32_t page, page2;  // of the next block and the one after

  // (pages are looked up by scalar loads, two blocks ahead: a vector load would wait for all copies under way)
  __device__ __forceinline__ uint32_t look(const CacheDev &d, int at) { return (uint32_t)table[cache_page_of(d, (uint32_t)min(at, to - 1) / kBlockTokens)]; }
  __device__ __forceinline__ void begin(const CacheDev &d) {
    if (tok >= to) return;
    page = look(d, tok);
    page2 = look(d, tok + kStep);
  }
  __device__ __forceinline__ void one(const CacheDev &d, int layer, int lane) {
    if (tok >= to) return;
    const uint32_t block = (uint32_t)tok / kBlockTokens;
    const unsigned char *blk = cache_block(d, layer, (int)page, head, block - cache_page_of(d, block) * d.page_blocks);
#pragma unroll
    for (int i = 0; i < kCopies; ++i)
      if (40 * D - i * 1024 >= 1024 || lane * 16 < 40 * D - i * 1024) copy_to_lds(blk + i * 1024, ring + slot * (40 * D) + i * 1024, lane * 16);
    slot ^= 1;
    tok += kStep;
    page = page2;
    page2 = look(d, tok + kStep);
  }
};

template <int D, int NR>
__global__ __launch_bounds__(kLanes, at_once(D, NR)) void k_cache_attend(CacheDev d, CacheQuery q, int tiles) {
  constexpr int NJ = D / 32, NT = D / 16;
  extern __shared__ uint4 lds[];
  Shared<D, NR> &sh = *reinterpret_cast<Shared<D, NR> *>(lds);
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), col = lane & 15, b = lane >> 4;

  if (wave == 0) {
    const bool found = q.r.n <= 64 ? find_piece<1, 16 * NR>(d, q, tiles, kUnits * at_once(D, NR), sh) : find_piece<kRound / 64, 16 * NR>(d, q, tiles, kUnits * at_once(D, NR), sh);
    if (lane == 0) sh.last = found;
  }
  __syncthreads();
  if (!sh.last) return;
  Piece pc = sh.piece;
  const Span sp{uniform(pc.sp.seq), uniform(pc.sp.count), uniform(pc.sp.length), uniform(pc.sp.low), uniform(pc.sp.steps), uniform(pc.sp.tiles),
                (int64_t)uniform((int)((uint64_t)pc.sp.row0 >> 32)) << 32 | (uint32_t)uniform((int)pc.sp.row0)};
  pc = Piece{sp, uniform(pc.item), uniform(pc.head), uniform(pc.tile), 0, 0, uniform(pc.parts), uniform(pc.nth), uniform(pc.part)};
  {  // steps in as many equal pieces, the first ones one longer
    const int each = sp.steps / pc.parts, longer = sp.steps - each * pc.parts;
    pc.sa = each * pc.nth + min(pc.nth, longer);
    pc.sb = pc.sa + each + (pc.nth < longer);
  }
  const int row_first = pc.tile * 16 * NR, rows = min(16 * NR, q.share * sp.count - row_first), head = pc.head, first_tok = sp.low + pc.sa * kStep + wave * kBlockTokens;
  Copies<D> cp;
  cp.table = (ScalarInts)(uintptr_t)(d.table + (int64_t)sp.seq * d.max_pages);
  cp.head = head;
  cp.tok = first_tok;
  cp.to = min(sp.low + pc.sb * kStep, sp.length);
  cp.ring = (uint32_t)uniform((int)lds_address(sh.ring[wave][0]));
  cp.slot = 0;
  cp.begin(d);
#pragma unroll
  for (int i = 0; i < kAhead; ++i) cp.one(d, q.layer, lane);

  half8 qf[NR][NJ];
  int see_to[NR], see_from[NR];
#pragma unroll
  for (int t = 0; t < NR; ++t) {
    const int row = t * 16 + col;
    const bool real = row < rows;
    const int j = real ? (row_first + row) / q.share : 0, h = real ? (row_first + row) % q.share : 0;
    const int pos = sp.length - sp.count + j;
    see_to[t] = q.causal ? pos + 1 : sp.length;
    see_from[t] = q.window ? pos - q.window + 1 : 0;
    const uint16_t *p = q.q + (sp.row0 + j) * q.q_row + (int64_t)(head * q.share + h) * q.q_head + b * (D / 4);
#pragma unroll
    for (int x = 0; x < NJ; ++x) qf[t][x] = real ? load_query(p + 8 * x, q.half_type, q.vec, q.scale_two) : half8{};
  }
  const int all_to = q.causal ? sp.length - sp.count + 1 : sp.length;     // every row sees [all_from, all_to)
  const int all_from = q.window ? sp.length - q.window : 0;

  f32x4 o[NR][NT];
  float m[NR], l[NR];
#pragma unroll
  for (int t = 0; t < NR; ++t) {
    m[t] = -INFINITY;
    l[t] = 0.0f;
#pragma unroll
    for (int n = 0; n < NT; ++n) o[t][n] = f32x4{0, 0, 0, 0};
  }
  const int to = cp.to;
  uint32_t slot = 0;
  for (int tok0 = first_tok; tok0 < to; tok0 += kStep) {
    static_assert(kAhead == 2, "one block behind this one");
    if (tok0 + kStep < to) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(Copies<D>::kCopies) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    const unsigned char *blk = sh.ring[wave][slot];
    KeyTile<D> kt[2];
    kt[0].load(blk, 0, lane);
    kt[1].load(blk, 1, lane);
    ValueBlock<D> vb;
    vb.load(blk, lane);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the slot has been read
    slot ^= 1;
    cp.one(d, q.layer, lane);
    f32x4 sc[NR][2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
      for (int t = 0; t < NR; ++t) sc[t][x] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const half8 a = kt[x].values(j);
#pragma unroll
        for (int t = 0; t < NR; ++t) sc[t][x] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, qf[t][j], sc[t][x], 0, 0, 0);
      }
    }
    if (tok0 + kBlockTokens > all_to || tok0 < all_from) {
      const int first = tok0 + 16 * (b >> 1) + 4 * (b & 1);
#pragma unroll
      for (int t = 0; t < NR; ++t)
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int at = first + 8 * x + r;
            if (at >= see_to[t] || at < see_from[t]) sc[t][x][r] = -INFINITY;
          }
    }
    half8 pf[NR];
#pragma unroll
    for (int t = 0; t < NR; ++t) {
      float top = fmaxf(fmaxf(fmaxf(sc[t][0][0], sc[t][0][1]), fmaxf(sc[t][0][2], sc[t][0][3])),
                        fmaxf(fmaxf(sc[t][1][0], sc[t][1][1]), fmaxf(sc[t][1][2], sc[t][1][3])));
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32)) * q.scale_rest;
      if (__any(top > m[t] + (kTop + kLag))) {
        const float now = fmaxf(m[t], top - kTop), by = m[t] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m[t] - now);
        m[t] = now;
        l[t] *= by;
#pragma unroll
        for (int n = 0; n < NT; ++n) o[t][n] *= by;
      }
      const float base = m[t] == -INFINITY ? 0.0f : m[t];
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = __builtin_amdgcn_exp2f(fmaf(sc[t][e / 4][e % 4], q.scale_rest, -base));
      pf[t] = to_half8(p);
      l[t] += add_up(0.0f, pf[t]);
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const half8 v = vb.values(n);
#pragma unroll
      for (int t = 0; t < NR; ++t) o[t][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pf[t], o[t][n], 0, 0, 0);
    }
  }

  // The wavefronts' parts of each row.
#pragma unroll
  for (int t = 0; t < NR; ++t) {
    l[t] += __shfl_xor(l[t], 16);
    l[t] += __shfl_xor(l[t], 32);
    if (b == 0) {
      sh.ml[wave][t * 16 + col][0] = m[t];
      sh.ml[wave][t * 16 + col][1] = l[t];
    }
  }
  __syncthreads();  // (and the rings are read)
  float *part = d.part + (int64_t)(pc.part + pc.nth) * (16 * NR) * D, *part_ml = d.part_ml + (int64_t)(pc.part + pc.nth) * (16 * NR) * 2;
#pragma unroll
  for (int t = 0; t < NR; ++t) {
    float most = -INFINITY;
    for (int w = 0; w < kWaves; ++w) most = fmaxf(most, sh.ml[w][t * 16 + col][0]);
    const float by = m[t] == -INFINITY && most == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[t] - most);
    if (t * 16 + col < rows)
#pragma unroll
      for (int n = 0; n < NT; ++n) *reinterpret_cast<f32x4 *>(&sh.o[wave][col][n * 16 + b * 4]) = o[t][n] * by;
    __syncthreads();
    for (int u = threadIdx.x; u < min(16, rows - t * 16) * (D / 4); u += kLanes) {
      const int r = u / (D / 4), c = u % (D / 4) * 4, row = t * 16 + r;
      float top = -INFINITY, sum = 0.0f;
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sh.ml[w][row][0]);
      f32x4 v{0, 0, 0, 0};
      for (int w = 0; w < kWaves; ++w) {
        const float mw = sh.ml[w][row][0];
        sum += sh.ml[w][row][1] * (mw == -INFINITY && top == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(mw - top));
        v += *reinterpret_cast<const f32x4 *>(&sh.o[w][r][c]);
      }
      if (pc.parts == 1) {
        store_row(q, sp.row0 + (row_first + row) / q.share, head * q.share + (row_first + row) % q.share, c, v, top, sum);
      } else {
        put_pair(part + row * D + c, v[0], v[1]);
        put_pair(part + row * D + c + 2, v[2], v[3]);
        if (c == 0) put_pair(part_ml + row * 2, top, sum);
      }
    }
    if (t + 1 < NR) __syncthreads();
  }
  if (pc.parts == 1) return;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wavefront's part is out ...
  __syncthreads();                                  // ... and that of the others
  if (threadIdx.x == 0) {
    uint32_t *there = d.arrived + ((int64_t)pc.item * d.kv_heads + head) * tiles + pc.tile;
    const bool last = __hip_atomic_fetch_add(there, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)pc.parts - 1;
    if (last) __hip_atomic_store(there, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    sh.last = last;
  }
  __syncthreads();
  if (!sh.last) return;
  part = d.part + (int64_t)pc.part * (16 * NR) * D;
  part_ml = d.part_ml + (int64_t)pc.part * (16 * NR) * 2;
  for (int u = threadIdx.x; u < rows * (D / 4); u += kLanes) {
    const int row = u / (D / 4), c = u % (D / 4) * 4;
    join_parts(q, sp.row0 + (row_first + row) / q.share, head * q.share + (row_first + row) % q.share, c, pc.parts, part + row * D + c, part_ml + row * 2, D, 16 * NR);
  }
}

// (an even share makes no more pieces than run at once, and one more for each row tile of a head)
template <int D, int NR>
void launch(const CacheDev &d, const CacheQuery &q, int tiles, hipStream_t s) {
  k_cache_attend<D, NR><<<(uint32_t)(kUnits * at_once(D, NR) + q.r.n * d.kv_heads * tiles), kLanes, sizeof(Shared<D, NR>), s>>>(d, q, tiles);
}

// Up to 64 rows; a head's row tiles read its cache one beside the other, and the second finds it in the last-level cache.
constexpr int kTiles = 4;  // of 16 or 32 rows, at most

}  // namespace

// Rows of parts: of the pieces that are parts there are at most two for each that runs at once, a long head's last being short.
static size_t part_rows(int head_dim) {
  const size_t few = (size_t)kUnits * 2 * (head_dim == 256 ? 16 * at_once(256, 1) : head_dim == 128 ? 32 * at_once(128, 2) : head_dim == 96 ? 32 * at_once(96, 2) : 32 * at_once(64, 2));
  const size_t many = cache_prompt_part_rows();
  return few > many ? few : many;
}
size_t cache_part_floats(int head_dim) { return part_rows(head_dim) * head_dim; }
size_t cache_part_ml_floats(int head_dim) { return part_rows(head_dim) * 4; }  // (of many rows two lanes have a pair each)
size_t cache_arrived_words(int max_seqs, int kv_heads) {
  const size_t few = (size_t)max_seqs * kv_heads * kTiles, many = cache_prompt_groups();
  return few > many ? few : many;
}

void launch_cache_attend(const CacheDev &d, const CacheQuery &q, hipStream_t s) {
  // Against the kernel for many rows, 8 sequences of up to 32,000 tokens and 8 heads: of 128 channels 32, 40, 64, 96, 128 rows take 69, 111, 108, 159,
  // 186 us here and 144 to 152 there; of 256 channels 24, 32, 40, 48, 64 rows 200, 201, 368, 369, 421 us and 420 to 433.  64 rows of 64, 96, 256 channels:
  // one sequence of 32,000 34, 42, 71 us and 66, 86, 160; 8 of up to 8,000 28, 36, 122 and 41, 49, 129; 32 of up to 2,000 29, 34, 105 and 44, 51, 153,
  // of 128 channels 50 and 51.
  const int64_t rows = (int64_t)q.share * q.r.max_new;
  const int each = d.head_dim == 256 || rows <= 16 ? 16 : 32;
  const int64_t tiles = (rows + each - 1) / each;
  // (steps of all row tiles are counted in 32 bits, and they are one launch)
  const int64_t heads = q.r.n * (int64_t)d.kv_heads * tiles;
  if (rows > 64 || (tiles > 1 && (heads >= 1 << 22 || heads * ((int64_t)d.max_pages * d.page_blocks / kWaves + 1) >= (int64_t)1 << 32))) return launch_cache_prompt(d, q, s);
  switch (d.head_dim) {
    case 64: return each == 16 ? launch<64, 1>(d, q, 1, s) : launch<64, 2>(d, q, (int)tiles, s);
    case 96: return each == 16 ? launch<96, 1>(d, q, 1, s) : launch<96, 2>(d, q, (int)tiles, s);
    case 128: return each == 16 ? launch<128, 1>(d, q, 1, s) : launch<128, 2>(d, q, (int)tiles, s);
    default: return launch<256, 1>(d, q, (int)tiles, s);
  }
}

hipError_t allow_large_lds_cache_attend() {
  return hipFuncSetAttribute(reinterpret_cast<const void *>(k_cache_attend<256, 1>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Shared<256, 1>));
}

}  // namespace rtams
