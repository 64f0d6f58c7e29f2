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
#include "rtams_dev.h"

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

constexpr int kAhead = 2;   // blocks of a wavefront that are in LDS or on their way
constexpr int kJoin = 32;   // channels that the wavefronts join at a time

__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

template <int D, int NR>
struct alignas(16) Shared {
  unsigned char ring[kWaves][kAhead][40 * D];
  uint32_t before[kScan + 1];
  uint32_t waves[kWaves];
  int last;
  float ml[kWaves][16 * NR][2];
  alignas(16) float o[kWaves][16][kJoin + 4];
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

struct Run {  // steps [sa, sb) of an item's head
  Span sp;
  int item, head, sa, sb;
  uint32_t first_unit;  // the number of its step 0
};

typedef const __attribute__((address_space(4))) int32_t *ScalarInts;

// The copies of a wavefront's blocks into its ring: block n of the run goes to slot n % kAhead.
template <int D>
struct Copies {
  static constexpr int kCopies = (40 * D + 1023) / 1024;  // loads of a block
  ScalarInts table;
  int head, tok, to;   // next block's first token; end of the run's tokens
  uint32_t ring, slot;
  uint32_t page;       // of the next block

  // (pages are looked up by scalar loads, a block ahead: a vector load would wait for all copies under way)
  __device__ __forceinline__ void look(const CacheDev &d) {
    if (tok < to) page = (uint32_t)table[cache_page_of(d, (uint32_t)tok / kBlockTokens)];
  }
  __device__ __forceinline__ void begin(const CacheDev &d, const Run &r, int wave, uint32_t ring_at) {
    table = (ScalarInts)(uintptr_t)(d.table + (int64_t)r.sp.seq * d.max_pages);
    head = r.head;
    tok = r.sp.low + r.sa * kStep + wave * kBlockTokens;
    to = min(r.sp.low + r.sb * kStep, r.sp.length);
    ring = ring_at;
    slot = 0;
    look(d);
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
    look(d);
  }
};

// The copies of the run's first blocks are under way; those of `next`, if there is one, are when it returns.
template <int D, int NR>
__device__ void attend_run(const CacheDev &d, const CacheQuery &q, const Run &run, bool more, const Run &next, uint32_t all, uint32_t workers, uint32_t worker, Copies<D> &cp,
                           Shared<D, NR> &sh) {
  constexpr int NJ = D / 32, NT = D / 16;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, b = lane >> 4;
  const Span &sp = run.sp;
  const int rows = q.share * sp.count, head = run.head;

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
  const int to = cp.to;
  uint32_t slot = 0;
  for (int tok0 = sp.low + run.sa * kStep + wave * kBlockTokens; tok0 < to; tok0 += kStep) {
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
  if (more) {  // (this wavefront has read its ring)
    cp.begin(d, next, wave, cp.ring);
    for (int i = 0; i < kAhead; ++i) cp.one(d, q.layer, lane);
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
  const bool whole = run.sa == 0 && run.sb == sp.steps;
  const uint32_t slot_at = worker * 2 + (run.sa == 0 ? 1 : 0);
#pragma unroll
  for (int t = 0; t < NR; ++t) {
    float most = -INFINITY;
    for (int w = 0; w < kWaves; ++w) most = fmaxf(most, sh.ml[w][t * 16 + col][0]);
    const float by = m[t] == -INFINITY && most == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[t] - most);
#pragma unroll
    for (int c0 = 0; c0 < D; c0 += kJoin) {
#pragma unroll
      for (int n = 0; n < kJoin / 16; ++n) *reinterpret_cast<f32x4 *>(&sh.o[wave][col][n * 16 + b * 4]) = o[t][c0 / 16 + n] * by;
      __syncthreads();
      if (threadIdx.x < 16 * (kJoin / 4)) {
        const int r = threadIdx.x / (kJoin / 4), c = threadIdx.x % (kJoin / 4) * 4, row = t * 16 + r;
        if (row < rows) {
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
            float *part = d.part + ((int64_t)slot_at * (16 * NR) + row) * D + c0 + c;
            put_pair(part, v[0], v[1]);
            put_pair(part + 2, v[2], v[3]);
            if (c0 + c == 0) put_pair(d.part_ml + ((int64_t)slot_at * (16 * NR) + row) * 2, top, sum);
          }
        }
      }
      __syncthreads();
    }
  }
  if (whole) return;
  const uint32_t w0 = worker_of(run.first_unit, all, workers), w1 = worker_of(run.first_unit + sp.steps - 1, all, workers);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wavefront's part is out ...
  __syncthreads();                                  // ... and that of the others
  if (threadIdx.x == 0) {
    uint32_t *there = d.arrived + (int64_t)run.item * d.kv_heads + head;
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
__global__ __launch_bounds__(kLanes, NR == 1 && D <= 128 ? 3 : 1) void k_cache_attend(CacheDev d, CacheQuery q) {
  extern __shared__ uint4 lds[];
  Shared<D, NR> &sh = *reinterpret_cast<Shared<D, NR> *>(lds);
  const bool tell = blockIdx.x == 0;
  uint32_t all = 0;
  for (int base = 0; base < q.r.n; base += kScan) all = number_steps<D, NR>(d, q, base, all, sh, tell);
  if (all == 0) return;
  const uint32_t workers = all < gridDim.x ? all : gridDim.x, worker = blockIdx.x;
  if (worker >= workers) return;
  uint32_t u = (uint32_t)((uint64_t)all * worker / workers);
  const uint32_t end = (uint32_t)((uint64_t)all * (worker + 1) / workers);
  int base = 0;
  if (q.r.n > kScan) {
    uint32_t at = number_steps<D, NR>(d, q, 0, 0, sh, false);
    while (at <= u) at = number_steps<D, NR>(d, q, base += kScan, at, sh, false);
  }
  // The run that step u begins or goes on with; u moves behind it.
  const auto find_run = [&]() {
    while (u >= sh.before[kScan]) number_steps<D, NR>(d, q, base += kScan, sh.before[kScan], sh, false);
    int lo = 0, hi = kScan - 1;  // the last item whose steps begin at u or before
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (sh.before[mid] <= u) lo = mid;
      else hi = mid - 1;
    }
    Run r;
    r.item = base + lo;
    r.sp = find_span(d, q, r.item, false);
    const uint32_t within = u - sh.before[lo], steps = (uint32_t)r.sp.steps, take = min(end - u, steps - within % steps);
    r.head = (int)(within / steps);
    r.sa = (int)(within % steps);
    r.sb = r.sa + (int)take;
    r.first_unit = u - (uint32_t)r.sa;
    u += take;
    r.sp.row0 = (int64_t)uniform((int)((uint64_t)r.sp.row0 >> 32)) << 32 | (uint32_t)uniform((int)r.sp.row0);
    r.sp = Span{uniform(r.sp.seq), uniform(r.sp.count), uniform(r.sp.length), uniform(r.sp.low), uniform(r.sp.steps), r.sp.row0};
    return Run{r.sp, uniform(r.item), uniform(r.head), uniform(r.sa), uniform(r.sb), (uint32_t)uniform((int)r.first_unit)};
  };
  Run run = find_run();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  Copies<D> cp;
  cp.begin(d, run, wave, (uint32_t)uniform((int)lds_address(sh.ring[wave][0])));
  for (int i = 0; i < kAhead; ++i) cp.one(d, q.layer, lane);
  for (;;) {
    const bool more = u < end;
    const Run next = more ? find_run() : run;
    attend_run<D, NR>(d, q, run, more, next, all, workers, worker, cp, sh);
    if (!more) return;
    run = next;
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
  const auto go = [&](auto kernel, size_t lds) { kernel<<<kWorkers, kLanes, lds, s>>>(d, q); };
  if (rows > (d.head_dim == 256 ? 16 : 32)) return launch_cache_prompt(d, q, s);
  switch (d.head_dim) {
    case 64: return rows <= 16 ? go(k_cache_attend<64, 1>, sizeof(Shared<64, 1>)) : go(k_cache_attend<64, 2>, sizeof(Shared<64, 2>));
    case 96: return rows <= 16 ? go(k_cache_attend<96, 1>, sizeof(Shared<96, 1>)) : go(k_cache_attend<96, 2>, sizeof(Shared<96, 2>));
    case 128: return rows <= 16 ? go(k_cache_attend<128, 1>, sizeof(Shared<128, 1>)) : go(k_cache_attend<128, 2>, sizeof(Shared<128, 2>));
    default: return go(k_cache_attend<256, 1>, sizeof(Shared<256, 1>));
  }
}

hipError_t allow_large_lds_cache_attend() {
  return hipFuncSetAttribute(reinterpret_cast<const void *>(k_cache_attend<256, 1>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Shared<256, 1>));
}

}  // namespace rtams
