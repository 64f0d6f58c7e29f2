// Attention of few rows over the cache in 4 bits: single tokens and some tokens of each sequence.
//
//   s_t = scale * q . K_t,  o = sum_t exp(s_t - m) V_t / sum_t exp(s_t - m),  m the running maximum
//
// Bound by the bytes of the cache: 1.25 a channel and token for keys and values together.  A step of a workgroup is 128 tokens of
// one kv head, 32 to a wavefront; the steps of all sequences and heads lie on one line, which is cut into equal pieces, so
// that ragged lengths fill the chip alike.  The query heads that share a kv head (times an item's rows) are the 16 columns of
// the matrix instructions.  Codes become halves in registers, straight from the loads: scores come out as S^T = K Q^T,
// tokens down and rows across, which is the operand that O^T = V^T P^T takes, so nothing is transposed and LDS only joins
// the wavefronts.  What a piece leaves of a row goes to scratch; the last piece of it to arrive joins them, in order.
#include "../../include/rtams_cache.h"

#include "cache_mm.h"

namespace rtams {

namespace {

constexpr int kLanes = 256, kWaves = 4, kStep = kWaves * kBlockTokens;
constexpr int kWorkers = 768;    // workgroups of a launch: three to a compute unit
constexpr int kScan = 256;       // items that are numbered at a time

struct Span {  // what an item asks for
  int seq, count, length, low;  // low: first position that a row of it sees, rounded down to a block
  int steps;
  int64_t row0;
};

__device__ inline Span find_span(const CacheDev &d, const CacheQuery &q, int i, bool tell) {
  Span s{};
  if (i >= q.r.n) return s;
  const bool ok = cache_item_rows(q.r, i, &s.row0, &s.count);
  s.seq = cache_item_seq(q.r, i);
  if (!ok || (uint32_t)s.seq >= (uint32_t)d.max_seqs) {
    if (tell) cache_raise(d, RTAMS_EINVAL);
    s.count = 0;
    return s;
  }
  s.length = d.lengths[s.seq];
  if (tell && q.causal && s.count > s.length) cache_raise(d, RTAMS_EINVAL);
  if (q.causal && q.window) {
    const int low = s.length - s.count - q.window + 1;
    s.low = low > 0 ? low & ~(kBlockTokens - 1) : 0;
  }
  if (s.count > 0) s.steps = s.length > s.low ? (s.length - s.low + kStep - 1) / kStep : 1;
  return s;
}

// Channels that the wavefronts join at a time: 32 KiB of LDS.
constexpr int joined(int head_dim) { return head_dim < 128 ? head_dim : 128; }

template <int D, int NR>
struct Shared {
  uint32_t before[kScan + 1];
  uint32_t waves[kWaves];
  int last;
  float ml[kWaves][16 * NR][2];
  float o[kWaves][16][joined(D) + 4];
};

// Numbers of the steps of items base .. base + 255 (times kv heads), from `at` on; returns the first number behind them.
template <int D, int NR>
__device__ uint32_t number_steps(const CacheDev &d, const CacheQuery &q, int base, uint32_t at, Shared<D, NR> &sh, bool tell) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t mine = (uint32_t)find_span(d, q, base + threadIdx.x, tell).steps * (uint32_t)d.kv_heads;
  uint32_t inc = mine;
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t x = __shfl_up(inc, o);
    if (lane >= o) inc += x;
  }
  __syncthreads();
  if (lane == 63) sh.waves[wave] = inc;
  __syncthreads();
  uint32_t lower = at, all = at;
  for (int w = 0; w < kWaves; ++w) {
    lower += w < wave ? sh.waves[w] : 0;
    all += sh.waves[w];
  }
  sh.before[threadIdx.x] = lower + inc - mine;
  if (threadIdx.x == 0) sh.before[kScan] = all;
  __syncthreads();
  return all;
}

// The worker that step u falls to: worker w has the steps [all * w / workers, all * (w + 1) / workers).
__device__ inline uint32_t worker_of(uint32_t u, uint32_t all, uint32_t workers) {
  return (uint32_t)((((uint64_t)u + 1) * workers - 1) / all);
}

// Steps [sa, sb) of an item's head; first_unit: the number of its step 0.
template <int D, int NR>
__device__ void attend_piece(const CacheDev &d, const CacheQuery &q, const Span &sp, int item, int head, int sa, int sb, uint32_t first_unit,
                             uint32_t all, uint32_t workers, uint32_t worker, Shared<D, NR> &sh) {
  constexpr int NJ = D / 32, NT = D / 16, CH = joined(D);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, b = lane >> 4;
  const int rows = q.share * sp.count;

  half8 qf[NR][NJ];
  int see_to[NR], see_from[NR];
#pragma unroll
  for (int t = 0; t < NR; ++t) {
    const int row = t * 16 + col;
    const bool real = row < rows;
    const int j = real ? row / q.share : 0, h = real ? row % q.share : 0;
    const int pos = sp.length - sp.count + j;
    see_to[t] = q.causal ? pos + 1 : sp.length;
    see_from[t] = q.window ? pos - q.window + 1 : 0;
    const uint16_t *p = q.q + (sp.row0 + j) * q.q_row + (int64_t)(head * q.share + h) * q.q_head + b * (D / 4);
#pragma unroll
    for (int x = 0; x < NJ; ++x) qf[t][x] = real ? load_query(p + 8 * x, q.half_type, q.vec, q.scale_log2) : half8{};
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
  const int32_t *table = d.table + (int64_t)sp.seq * d.max_pages;
  for (int s = sa; s < sb; ++s) {
    const int tok0 = __builtin_amdgcn_readfirstlane(sp.low + s * kStep + wave * kBlockTokens);
    if (tok0 >= sp.length) break;
    const uint32_t block = (uint32_t)tok0 / kBlockTokens, pg = cache_page_of(d, block);
    const unsigned char *blk = cache_block(d, q.layer, table[pg], head, block - pg * d.page_blocks);
    KeyTile<D> kt[2];
    kt[0].load(blk, 0, lane);
    kt[1].load(blk, 1, lane);
    ValueBlock<D> vb;
    vb.load(blk, lane);
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
      top = fmaxf(top, __shfl_xor(top, 32));
      // The maximum follows only where a score has left it 8 behind: probabilities stay below 2^8, far inside a half.
      if (__any(top > m[t] + 8.0f)) {
        const float now = fmaxf(m[t], top), by = m[t] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m[t] - now);
        m[t] = now;
        l[t] *= by;
#pragma unroll
        for (int n = 0; n < NT; ++n) o[t][n] *= by;
      }
      const float base = m[t] == -INFINITY ? 0.0f : m[t];
      float p[8], sum = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = __builtin_amdgcn_exp2f(sc[t][e / 4][e % 4] - base);
        sum += p[e];
      }
      l[t] += sum;
      pf[t] = to_half8(p);
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
  __syncthreads();
  const bool whole = sa == 0 && sb == sp.steps;
  const uint32_t slot = worker * 2 + (sa == 0 ? 1 : 0);
#pragma unroll
  for (int t = 0; t < NR; ++t) {
    float most = -INFINITY;
    for (int w = 0; w < kWaves; ++w) most = fmaxf(most, sh.ml[w][t * 16 + col][0]);
    const float by = m[t] == -INFINITY && most == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[t] - most);
#pragma unroll
    for (int c0 = 0; c0 < D; c0 += CH) {
#pragma unroll
      for (int n = 0; n < CH / 16; ++n) *reinterpret_cast<f32x4 *>(&sh.o[wave][col][n * 16 + b * 4]) = o[t][c0 / 16 + n] * by;
      __syncthreads();
      for (int u = threadIdx.x; u < 16 * (CH / 4); u += kLanes) {
        const int r = u / (CH / 4), c = u % (CH / 4) * 4, row = t * 16 + r;
        if (row >= rows) continue;
        float top = -INFINITY, sum = 0.0f;
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sh.ml[w][row][0]);
        f32x4 v{0, 0, 0, 0};
        for (int w = 0; w < kWaves; ++w) {
          const float mw = sh.ml[w][row][0];
          sum += sh.ml[w][row][1] * (mw == -INFINITY && top == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(mw - top));
          v += *reinterpret_cast<const f32x4 *>(&sh.o[w][r][c]);
        }
        if (whole) {
          store_row(q, sp.row0 + row / q.share, head * q.share + row % q.share, c0 + c, v, top, sum);
        } else {
          float *part = d.part + ((int64_t)slot * (16 * NR) + row) * D + c0 + c;
          put_pair(part, v[0], v[1]);
          put_pair(part + 2, v[2], v[3]);
          if (c0 + c == 0) put_pair(d.part_ml + ((int64_t)slot * (16 * NR) + row) * 2, top, sum);
        }
      }
      __syncthreads();
    }
  }
  if (whole) return;
  const uint32_t w0 = worker_of(first_unit, all, workers), w1 = worker_of(first_unit + sp.steps - 1, all, workers);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wavefront's part is out ...
  __syncthreads();                                  // ... and that of the others
  if (threadIdx.x == 0) {
    uint32_t *there = d.arrived + (int64_t)item * d.kv_heads + head;
    const bool last = __hip_atomic_fetch_add(there, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == w1 - w0;
    if (last) __hip_atomic_store(there, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    sh.last = last;
  }
  __syncthreads();
  if (sh.last) {
    // (slot 2 w + 1 has what worker w began and did not end, slot 2 w what it found begun)
    for (int u = threadIdx.x; u < rows * (D / 4); u += kLanes) {
      const int row = u / (D / 4), c = u % (D / 4) * 4;
      const int64_t at = (int64_t)(w0 * 2 + 1) * (16 * NR) + row;
      join_parts(q, sp.row0 + row / q.share, head * q.share + row % q.share, c, (int)(w1 - w0 + 1), d.part + at * D + c, d.part_ml + at * 2,
                 D, 16 * NR, 32 * NR);
    }
  }
  __syncthreads();
}

template <int D, int NR>
__global__ __launch_bounds__(kLanes) void k_cache_attend(CacheDev d, CacheQuery q) {
  __shared__ Shared<D, NR> sh;
  const bool tell = blockIdx.x == 0;
  uint32_t all = 0;
  for (int base = 0; base < q.r.n; base += kScan) all = number_steps<D, NR>(d, q, base, all, sh, tell);
  if (all == 0) return;
  const uint32_t workers = all < gridDim.x ? all : gridDim.x, worker = blockIdx.x;
  if (worker >= workers) return;
  uint32_t u = (uint32_t)((uint64_t)all * worker / workers);
  const uint32_t end = (uint32_t)((uint64_t)all * (worker + 1) / workers);
  uint32_t at = 0;
  for (int base = 0; base < q.r.n && u < end; base += kScan) {
    if (q.r.n > kScan) at = number_steps<D, NR>(d, q, base, at, sh, false);
    while (u < end && u < sh.before[kScan]) {
      int lo = 0, hi = kScan - 1;  // the last item whose steps begin at u or before
      while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (sh.before[mid] <= u) lo = mid;
        else hi = mid - 1;
      }
      const int item = base + lo;
      const Span sp = find_span(d, q, item, false);
      const uint32_t within = u - sh.before[lo];
      const int head = (int)(within / (uint32_t)sp.steps), sa = (int)(within % (uint32_t)sp.steps);
      const uint32_t left = end - u, rest = (uint32_t)(sp.steps - sa), take = left < rest ? left : rest;
      attend_piece<D, NR>(d, q, sp, item, head, sa, sa + (int)take, u - (uint32_t)sa, all, workers, worker, sh);
      u += take;
    }
  }
}

}  // namespace

size_t cache_part_floats(int head_dim) {
  const size_t few = (size_t)kWorkers * 2 * 32 * head_dim, many = cache_prompt_part_floats(head_dim);
  return few > many ? few : many;
}
size_t cache_part_ml_floats(int) {
  const size_t few = (size_t)kWorkers * 2 * 32 * 2, many = cache_prompt_part_ml_floats();
  return few > many ? few : many;
}
size_t cache_arrived_words(int max_seqs, int kv_heads) {
  const size_t few = (size_t)max_seqs * kv_heads, many = cache_prompt_groups();
  return few > many ? few : many;
}

void launch_cache_attend(const CacheDev &d, const CacheQuery &q, hipStream_t s) {
  const int64_t rows = (int64_t)q.share * q.r.max_new;
  const auto go = [&](auto kernel) { kernel<<<kWorkers, kLanes, 0, s>>>(d, q); };
  if (rows > (d.head_dim == 256 ? 16 : 32)) return launch_cache_prompt(d, q, s);
  switch (d.head_dim) {
    case 64: return rows <= 16 ? go(k_cache_attend<64, 1>) : go(k_cache_attend<64, 2>);
    case 96: return rows <= 16 ? go(k_cache_attend<96, 1>) : go(k_cache_attend<96, 2>);
    case 128: return rows <= 16 ? go(k_cache_attend<128, 1>) : go(k_cache_attend<128, 2>);
    default: return go(k_cache_attend<256, 1>);
  }
}

}  // namespace rtams
