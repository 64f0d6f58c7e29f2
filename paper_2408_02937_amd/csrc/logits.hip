// Log probabilities of given tokens, entropy and the most likely tokens of rows of logits (include/rtams_logits.h).
//
//   1 + R = sum 2^(c (x - m)),  T = sum 2^(c (x - m)) c (x - m),  c = scale * log2 e, m the row's largest, whose own 1 is not in R
//   lse = scale m + log(1 + R),  entropy = log(1 + R) - ln 2 T / (1 + R),  log probability = scale (x - m) - log(1 + R)
//
// (Of a peaked row R is far below 1, and log(1 + R) and the entropy are as exact as R.)
//
// Bound by reading the logits once.  A workgroup takes a row, or where rows are few a piece of one, in panels that its lanes hold in registers, 256
// bytes each: all of a panel's loads go out before the first is needed, and a lane's largest is known before its first power, so that sums are scaled
// once a panel.  The most likely tokens: of the first panel the k-th largest of the lanes' largest is a bound that the k largest of all reach, and few
// others do; the lanes that have some are listed, all lanes look through their vectors, and what reaches the bound goes to LDS and is ranked there.  Later
// panels are held against the k-th so far.  Where too many reach the bound, those above it are taken and of those equal to it the lowest tokens counted off;
// where too many are above it (a few lanes have them all) a better one is found by bisection.
#include "../../include/rtams_logits.h"

#include "host.h"
#include "rtams_dev.h"

using namespace rtams;

namespace rtams {

namespace {

constexpr int kLanes = 256, kWaves = kLanes / 64;
constexpr int kVectors = 16;      // of 16 bytes, that a lane holds
constexpr int kMostTop = 64;
constexpr int kRoom = 512;        // tokens that are ranked with the best so far
constexpr int kMostPieces = 64;   // of a row
constexpr int kSplitBelow = 1024; // rows: from so many on none is split
constexpr float kFar = -1024.0f;  // powers of less are 0

struct LogitsDev {
  int64_t rows, row_stride;
  int32_t vocab, top, tokens, pieces;
  int32_t panels;  // of a piece
  float scale, c;
  const void *logits;
  const int32_t *given;
  float *lse, *entropy, *logprobs;
  int32_t *best;
  float *best_logprobs;
  float4 *part;          // [rows][pieces]: m, S, T
  uint64_t *part_best;   // [rows][pieces][top]
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <int TYPE>
constexpr int each_of() { return TYPE == RTAMS_TYPE_F32 ? 4 : 8; }  // logits of a vector

template <int TYPE>
__device__ __forceinline__ float logit(const u32x4 &w, int e) {
  if (TYPE == RTAMS_TYPE_F32) return __uint_as_float(w[e]);
  if (TYPE == RTAMS_TYPE_BF16) return __uint_as_float(e % 2 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
  const uint16_t u = (uint16_t)(e % 2 ? w[e / 2] >> 16 : w[e / 2]);
  _Float16 h;
  __builtin_memcpy(&h, &u, 2);
  return (float)h;
}

template <int TYPE>
__device__ inline float logit_at(const void *row, int i) {
  if (TYPE == RTAMS_TYPE_F32) return static_cast<const float *>(row)[i];
  const uint16_t u = static_cast<const uint16_t *>(row)[i];
  if (TYPE == RTAMS_TYPE_BF16) return __uint_as_float((uint32_t)u << 16);
  _Float16 h;
  __builtin_memcpy(&h, &u, 2);
  return (float)h;
}

// Logits as whole numbers in the same order (0 and -0 alike), and back.
__device__ inline uint32_t ordered(float x) {
  const int32_t i = (int32_t)__float_as_uint(x + 0.0f);
  return (uint32_t)(i ^ ((i >> 31) & 0x7fffffff)) ^ 0x80000000u;
}
__device__ inline float unordered(uint32_t u) {
  const int32_t i = (int32_t)(u ^ 0x80000000u);
  return __uint_as_float((uint32_t)(i ^ ((i >> 31) & 0x7fffffff)));
}
__device__ inline uint64_t key_of(float x, int token) { return (uint64_t)ordered(x) << 32 | (uint32_t)~token; }

struct Sums {
  float m, s, t;  // of a lane: largest, as it is; the sums relative to it.  Of lanes together: s is R, or -1 where there are no logits
};

// A lane's sums relative to another largest, which is no smaller.
__device__ inline void move_to(Sums &a, float m, float c) {
  const float by = a.m == -INFINITY ? kFar : (a.m - m) * c, shrink = __builtin_amdgcn_exp2f(by);
  a.t = shrink * fmaf(a.s, fmaxf(by, kFar), a.t);
  a.s *= shrink;
  a.m = m;
}

__device__ inline float wave_sum(float x) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) x += __shfl_xor(x, o);
  return x;
}

__device__ inline float wave_largest(float x) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) x = fmaxf(x, __shfl_xor(x, o));
  return x;
}

struct Shared {
  uint64_t best[kMostTop + kRoom];  // the best so far, then what is ranked with them
  uint64_t sorted[kMostTop];
  alignas(16) uint32_t most[kLanes];
  uint16_t listed[kLanes];          // lanes whose vectors are looked through
  uint32_t waves[kWaves];
  float largest[kWaves], sums[kWaves], weighted[kWaves];
  float2 rest;
  uint32_t count, lanes, near, have;
  float bound;
};

// The logit of the i-th token given for a row.
template <int TYPE>
__device__ inline float given_logit(const LogitsDev &q, int64_t row, int i) {
  if (i >= q.tokens) return -INFINITY;
  const int t = q.given[row * q.tokens + i];
  return (uint32_t)t < (uint32_t)q.vocab ? logit_at<TYPE>(static_cast<const char *>(q.logits) + row * q.row_stride * (TYPE == RTAMS_TYPE_F32 ? 4 : 2), t) : -INFINITY;
}

// The numbers of a row, by `lanes` lanes; given: the logit of token number `lane`, asked for ahead.
template <int TYPE>
__device__ void put_row(const LogitsDev &q, int64_t row, const Sums &a, const uint64_t *best, int have, int lane, int lanes, float given) {
  const bool wrong = a.s != a.s, none = !wrong && a.m == -INFINITY;
  const float log_s = log1pf(a.s), nan = __uint_as_float(0x7fc00000u);
  if (lane == 0) {
    if (q.lse) q.lse[row] = wrong ? nan : none ? -INFINITY : fmaf(a.m, q.scale, log_s);
    if (q.entropy) q.entropy[row] = wrong ? nan : none ? 0.0f : fmaf(-0.6931471805599453f, a.t / (1.0f + a.s), log_s);
  }
  const auto log_probability = [&](float x) { return wrong ? nan : x == -INFINITY ? -INFINITY : fmaf(x - a.m, q.scale, -log_s); };
  for (int i = lane; i < q.tokens; i += lanes) q.logprobs[row * q.tokens + i] = log_probability(i == lane ? given : given_logit<TYPE>(q, row, i));
  for (int i = lane; i < q.top; i += lanes) {
    const bool there = i < have && !wrong;
    q.best[row * q.top + i] = there ? (int32_t)~(uint32_t)best[i] : -1;
    if (q.best_logprobs) q.best_logprobs[row * q.top + i] = log_probability(there ? unordered((uint32_t)(best[i] >> 32)) : -INFINITY);
  }
}

// Logits at .. at + E - 1 of a row, 16 bytes that lie at whole 16; -inf where the row has none.
template <int TYPE>
__device__ __forceinline__ u32x4 load_vector(const char *x, int at, int vocab) {
  constexpr int E = each_of<TYPE>(), kSize = 16 / E;
  constexpr uint32_t kNone = TYPE == RTAMS_TYPE_F32 ? 0xff800000u : TYPE == RTAMS_TYPE_BF16 ? 0xff80ff80u : 0xfc00fc00u;
  if (at >= 0 && at + E <= vocab) return *reinterpret_cast<const u32x4 *>(x + (int64_t)at * kSize);
  uint32_t w[4] = {kNone, kNone, kNone, kNone};
  if (at + E > 0 && at < vocab)
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (at + e >= 0 && at + e < vocab) {
        if (E == 4) w[e] = reinterpret_cast<const uint32_t *>(x)[at + e];
        else w[e / 2] = (e % 2 ? w[e / 2] & 0xffffu : w[e / 2] & 0xffff0000u) | (uint32_t)reinterpret_cast<const uint16_t *>(x)[at + e] << (e % 2 * 16);
      }
  return u32x4{w[0], w[1], w[2], w[3]};
}

// Sum over the workgroup, to every lane.
__device__ inline uint32_t sum_lanes(uint32_t v, Shared &sh) {
  v = last_lane(wave_running_sum(v));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.waves[threadIdx.x >> 6] = v;
  __syncthreads();
  return sh.waves[0] + sh.waves[1] + sh.waves[2] + sh.waves[3];
}

// Ranks the first `n` of sh.best; the best of them are in sh.sorted and again in sh.best.
__device__ inline void rank(int n, int top, Shared &sh) {
  for (int i = threadIdx.x; i < n; i += kLanes) {
    const uint64_t mine = sh.best[i];
    int above = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) above += sh.best[j] > mine;
    if (above < top) sh.sorted[above] = mine;
  }
  __syncthreads();
  const int have = min(n, top);
  for (int i = threadIdx.x; i < have; i += kLanes) sh.best[i] = sh.sorted[i];
  if (threadIdx.x == 0) {
    sh.have = have;
    // what a token must exceed, which comes behind all of these
    sh.bound = have == top ? unordered((uint32_t)(sh.sorted[top - 1] >> 32)) : -INFINITY;
  }
  __syncthreads();
}

// Takes a panel's most likely tokens to those so far.  panel: token of the panel's first logit; most: the lane's largest.  (Logits are read again: out of
// registers every look is 128 steps of code, and registers spill.)
template <int TYPE>
__device__ void take_best(const char *x, int vocab, int panel, float most, int top, Shared &sh) {
  constexpr int E = each_of<TYPE>();
  const float bound = sh.bound;
  const int lanes = __syncthreads_count(most > bound);
  if (!lanes) return;
  const int have = sh.have;
  // Those that reach `least` go behind the best so far, as far as there is room; how many they are (where there is none left, more than kRoom).
  const auto collect = [&](float least) {
    if (threadIdx.x == 0) sh.count = sh.lanes = 0;
    __syncthreads();
    if (most >= least) sh.listed[atomicAdd(&sh.lanes, 1u)] = (uint16_t)threadIdx.x;
    __syncthreads();
    const uint32_t all = sh.lanes * kVectors;
    const bool crowded = all > kLanes / 2 * kVectors;  // (32,768 equal ones one after the other take 15 us)
    for (uint32_t u = threadIdx.x; u < all; u += kLanes) {
      if (crowded && __hip_atomic_load(&sh.count, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) > kRoom) break;
      const int at = panel + ((int)(u % kVectors) * kLanes + sh.listed[u / kVectors]) * E;
      const u32x4 raw = load_vector<TYPE>(x, at, vocab);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float l = logit<TYPE>(raw, e);
        if (l >= least) {
          const uint32_t slot = atomicAdd(&sh.count, 1u);
          if (slot < kRoom) sh.best[have + slot] = key_of(l, at + e);
        }
      }
    }
    __syncthreads();
    return sh.count;
  };
  // The top-th largest of the lanes' largest; own: of few, the largest that a wavefront's own lanes have there (if they are as many), which some more reach.
  const auto near = [&](bool own) {
    const uint32_t mine = most > bound ? ordered(most) : 0;
    if (own) {
      int above = 0;
#pragma unroll
      for (int j = 0; j < 64; ++j) above += (uint32_t)__builtin_amdgcn_readlane((int)mine, j) > mine;
      const uint32_t reach = above >= top - 1 && mine ? mine : 0;  // (as many reach these)
      const uint32_t best = last_lane(wave_reduce_last(reach, [](uint32_t a, uint32_t b) { return a > b ? a : b; }));
      if ((threadIdx.x & 63) == 0) sh.waves[threadIdx.x >> 6] = best;
      __syncthreads();
      const uint32_t most_of = max(max(sh.waves[0], sh.waves[1]), max(sh.waves[2], sh.waves[3]));
      if (most_of) return unordered(most_of);
    }
    sh.most[threadIdx.x] = mine;
    if (threadIdx.x == 0) sh.near = ~0u;
    __syncthreads();
    int above = 0;
#pragma unroll 8
    for (int j = 0; j < kLanes / 4; ++j) {
      const uint4 y = reinterpret_cast<const uint4 *>(sh.most)[j];
      above += (int)(y.x > mine) + (int)(y.y > mine) + (int)(y.z > mine) + (int)(y.w > mine);
    }
    if (mine && above < top) atomicMin(&sh.near, mine);
    __syncthreads();
    return unordered(sh.near);
  };
  float from = unordered(ordered(bound) + 1);  // the least that exceeds it (of -inf the least number)
  const bool many = lanes >= top, own = top <= 32;
  if (have < top && many) from = near(own);
  uint32_t all = collect(from);
  if (all > kRoom && many && (have == top || own)) {
    from = near(own && have == top);
    all = collect(from);
  }
  if (all <= kRoom) return rank(have + (int)all, top, sh);
  // Of a row that is masked with a number (its type's lowest) and allows less than that many tokens, `from` is that number, which nearly all are
  // equal to: those above it come first.  (1,000 rows of 32,768 halves, 19 tokens allowed, the best 20: 38 us, where a
  // mask of -inf takes 19 and a search for `from` bit by bit 260.)
  float over = unordered(ordered(from) + 1);
  __syncthreads();  // (the count has been read)
  all = collect(over);
  if (all >= (uint32_t)top && all <= kRoom) return rank(have + (int)all, top, sh);
  const int first = panel + (int)threadIdx.x * E;
  const auto reaching = [&](float least) {  // how many do, in all lanes
    uint32_t n = 0;
    if (most >= least) {
#pragma unroll 1
      for (int v = 0; v < kVectors; ++v) {
        const u32x4 raw = load_vector<TYPE>(x, first + v * kLanes * E, vocab);
#pragma unroll
        for (int e = 0; e < E; ++e) n += logit<TYPE>(raw, e) >= least;
      }
    }
    return sum_lanes(n, sh);
  };
  if (all > kRoom) {
    // the top-th largest, exactly: the highest that as many reach
    const uint32_t highest = last_lane(wave_reduce_last(most > over ? ordered(most) : 0, [](uint32_t a, uint32_t b) { return a > b ? a : b; }));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.waves[threadIdx.x >> 6] = highest;
    __syncthreads();
    uint32_t low = ordered(over), high = max(max(sh.waves[0], sh.waves[1]), max(sh.waves[2], sh.waves[3]));
    while (low < high) {
      const uint32_t mid = low + (high - low + 1) / 2;
      if (reaching(unordered(mid)) >= (uint32_t)top) low = mid;
      else high = mid - 1;
    }
    from = unordered(low);
    over = unordered(low + 1);
    all = collect(over);
  }
  const float equal = from;
  uint32_t filled = have + all, need = top - all;
#pragma unroll 1
  for (int v = 0; v < kVectors && need; ++v) {  // in the order of the tokens
    const int at = first + v * kLanes * E;
    const u32x4 raw = load_vector<TYPE>(x, at, vocab);
    uint32_t n = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) n += logit<TYPE>(raw, e) == equal;
    const uint32_t upto = wave_running_sum(n);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) sh.waves[threadIdx.x >> 6] = upto;
    __syncthreads();
    uint32_t place = upto - n, total = 0;
    for (int w = 0; w < kWaves; ++w) {
      place += w < (int)(threadIdx.x >> 6) ? sh.waves[w] : 0;
      total += sh.waves[w];
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (logit<TYPE>(raw, e) == equal) {
        if (place < need) sh.best[filled + place] = key_of(equal, at + e);
        ++place;
      }
    const uint32_t taken = min(total, need);
    filled += taken;
    need -= taken;
  }
  __syncthreads();
  rank((int)filled, top, sh);
}

// A lane's largest logit, of its first `some` vectors.
template <int TYPE>
__device__ __forceinline__ float largest_of(const u32x4 (&raw)[kVectors], int some) {
  if constexpr (TYPE == RTAMS_TYPE_F32) {
    float most = -INFINITY;
#pragma unroll
    for (int v = 0; v < kVectors; ++v)
      if (v < some)
        most = fmaxf(fmaxf(fmaxf(most, __uint_as_float(raw[v].x)), __uint_as_float(raw[v].y)), fmaxf(__uint_as_float(raw[v].z), __uint_as_float(raw[v].w)));
    return most;
  } else if constexpr (TYPE == RTAMS_TYPE_F16) {
    typedef _Float16 half2v __attribute__((ext_vector_type(2)));
    half2v most = {(_Float16)-INFINITY, (_Float16)-INFINITY};
#pragma unroll
    for (int v = 0; v < kVectors; ++v)
      if (v < some)
#pragma unroll
        for (int j = 0; j < 4; ++j) most = __builtin_elementwise_max(most, __builtin_bit_cast(half2v, (uint32_t)raw[v][j]));
    return fmaxf((float)most[0], (float)most[1]);
  } else {
    // as whole numbers two at a time: the largest of them if one is not negative, of negative numbers the least
    typedef int16_t short2v __attribute__((ext_vector_type(2)));
    short2v most = {-32768, -32768}, least = {32767, 32767};
#pragma unroll
    for (int v = 0; v < kVectors; ++v)
      if (v < some)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          most = __builtin_elementwise_max(most, __builtin_bit_cast(short2v, (uint32_t)raw[v][j]));
          least = __builtin_elementwise_min(least, __builtin_bit_cast(short2v, (uint32_t)raw[v][j]));
        }
    const int high = max(most[0], most[1]), low = min(least[0], least[1]);
    return __uint_as_float((uint32_t)(uint16_t)(high >= 0 ? high : low) << 16);
  }
}

template <int TYPE>
__global__ __launch_bounds__(kLanes, 4) void k_logits(LogitsDev q, int64_t first_unit) {
  constexpr int E = each_of<TYPE>(), kPanel = kLanes * kVectors * E, kSize = 16 / E;
  constexpr uint32_t kNone = TYPE == RTAMS_TYPE_F32 ? 0xff800000u : TYPE == RTAMS_TYPE_BF16 ? 0xff80ff80u : 0xfc00fc00u;  // -inf
  __shared__ Shared sh;
  const int64_t unit = first_unit + blockIdx.x, row = unit / q.pieces;
  const int piece = (int)(unit % q.pieces), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const char *const x = static_cast<const char *>(q.logits) + row * q.row_stride * kSize;
  // vectors lie at whole 16 bytes: the first may begin in front of the row
  const int ahead = (int)(((uintptr_t)x & 15) / kSize);
  if (threadIdx.x == 0) {
    sh.have = 0;
    sh.bound = -INFINITY;
  }
  const float given = q.pieces == 1 ? given_logit<TYPE>(q, row, threadIdx.x) : 0.0f;
  Sums a{-INFINITY, 0.0f, 0.0f};
  const int panel0 = piece * q.panels * kPanel - ahead;  // (below 2^30 and a panel)
  for (int p = 0; p < q.panels; ++p) {
    const int panel = panel0 + p * kPanel, first = panel + (int)threadIdx.x * E;  // tokens of the panel's first logit and of the lane's
    if (panel >= q.vocab) break;
    u32x4 raw[kVectors];
    const char *const from = x + (int64_t)panel * kSize;
    const uint32_t own = threadIdx.x * 16;
    if (panel + kPanel <= q.vocab) {
      // (the first lane's first vector may begin in front of the row: it has another one until it is put together below)
#pragma unroll
      for (int v = 0; v < kVectors; ++v) raw[v] = *reinterpret_cast<const u32x4 *>(from + v * kLanes * 16 + (v == 0 && first < 0 ? 16 : own));
    } else {
#pragma unroll
      for (int v = 0; v < kVectors; ++v) {
        const int at = first + v * kLanes * E;
        raw[v] = u32x4{kNone, kNone, kNone, kNone};
        if (at >= 0 && at + E <= q.vocab) raw[v] = *reinterpret_cast<const u32x4 *>(from + v * kLanes * 16 + own);
      }
      const int last = (q.vocab - panel) / E;  // the panel's vector that the row's end is in
      if (last % kLanes == (int)threadIdx.x && (q.vocab - panel) % E && last < kVectors * kLanes) {
        const u32x4 end = load_vector<TYPE>(x, panel + last * E, q.vocab);
#pragma unroll
        for (int v = 0; v < kVectors; ++v)
          if (v == last / kLanes) raw[v] = end;
      }
    }
    if (first < 0) raw[0] = load_vector<TYPE>(x, first, q.vocab);
    const int some = min(kVectors, (q.vocab - panel + kLanes * E - 1) / (kLanes * E));  // vectors that hold some: the others cost nothing
    const float most = largest_of<TYPE>(raw, some);
    move_to(a, fmaxf(a.m, most), q.c);
    const float m = a.m == -INFINITY ? 0.0f : a.m, mc = m * q.c;
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f}, t[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    // (NaN, and +inf less +inf, are NaN in the sums; -inf is 0 in both.  One vector after the other: registers hold the logits as they came, not
    // all of them turned into 32 bits.)
    const auto add_up = [&](auto power) {
#pragma unroll
      for (int v = 0; v < kVectors; ++v) {
        if (v >= some) break;
        asm("" : "+v"(raw[v]));
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float z = power(logit<TYPE>(raw[v], e)), y = __builtin_amdgcn_exp2f(z);
          s[e % 4] += y;
          t[e % 4] = fmaf(y, fmaxf(z, kFar), t[e % 4]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    float off = 0.0f;
    if (!__any(!(fabsf(mc) < 1048576.0f))) {
      add_up([&](float l) { return fmaf(l, q.c, -mc); });
      off = fmaf(m, q.c, -mc);  // what the product's rounding left in every power
    } else {  // (masks of the type's lowest number: c times it may be none, differences come first)
      add_up([&](float l) { return (l - m) * q.c; });
    }
    const float by = __builtin_amdgcn_exp2f(-off), sum = (s[0] + s[1]) + (s[2] + s[3]), weighted = (t[0] + t[1]) + (t[2] + t[3]);
    a.s = fmaf(sum, by, a.s);
    a.t = fmaf(fmaf(-off, sum, weighted), by, a.t);
    if (q.top) {
      if (p == 0) __syncthreads();
      take_best<TYPE>(x, q.vocab, panel, most, q.top, sh);
    }
  }
  // The lanes' sums, without the 1 of the first that has the largest.
  float m = wave_largest(a.m);
  if (lane == 0) sh.largest[wave] = m;
  __syncthreads();
  m = fmaxf(fmaxf(sh.largest[0], sh.largest[1]), fmaxf(sh.largest[2], sh.largest[3]));
  const uint64_t who = __ballot(a.m == m);
  int owner = kLanes;
  for (int w = kWaves - 1; w >= 0; --w)
    if (sh.largest[w] == m) owner = w * 64;
  const bool mine = wave * 64 == owner && lane == __ffsll((unsigned long long)who) - 1;
  move_to(a, m, q.c);
  const auto together = [&](float s) {
    const float ws = wave_sum(s), wt = wave_sum(a.t);
    __syncthreads();
    if (lane == 0) {
      sh.sums[wave] = ws;
      sh.weighted[wave] = wt;
    }
    __syncthreads();
    return Sums{m, (sh.sums[0] + sh.sums[1]) + (sh.sums[2] + sh.sums[3]), (sh.weighted[0] + sh.weighted[1]) + (sh.weighted[2] + sh.weighted[3])};
  };
  Sums all = together(mine ? a.s - 1.0f : a.s);
  if (all.s > -0.5f && all.s < 0.0625f) {  // (-1: no logits)
    // A peaked row: what that lane has beside the 1, and the weighted sum, in which the largest's roundings stand, are summed once more, by the first wavefront.
    if (mine) sh.listed[0] = (uint16_t)threadIdx.x;
    __syncthreads();
    if (wave == 0) {
      float rest = 0.0f, weighted = 0.0f;
      for (int u = lane; u < q.panels * kVectors; u += 64) {
        const int at = panel0 + (u * kLanes + sh.listed[0]) * E;
        if (at >= q.vocab) break;
        const u32x4 raw = load_vector<TYPE>(x, at, q.vocab);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float l = logit<TYPE>(raw, e);
          const float z = (l - m) * q.c, y = l == m ? 0.0f : __builtin_amdgcn_exp2f(z);  // (a second one would make R 1)
          rest += y;
          weighted = fmaf(y, fmaxf(z, kFar), weighted);
        }
      }
      rest = wave_sum(rest);
      weighted = wave_sum(weighted);
      if (lane == 0) sh.rest = make_float2(rest, weighted);
    }
    __syncthreads();
    if (mine) a.t = sh.rest.y;
    all = together(mine ? sh.rest.x : a.s);
  }
  const int have = q.top ? (int)sh.have : 0;
  if (q.pieces == 1) {
    put_row<TYPE>(q, row, all, sh.sorted, have, threadIdx.x, kLanes, given);
  } else {
    if (threadIdx.x == 0) q.part[unit] = make_float4(all.m, all.s, all.t, 0.0f);
    for (int i = threadIdx.x; i < q.top; i += kLanes) q.part_best[unit * q.top + i] = i < have ? sh.sorted[i] : 0;
  }
}

// Joins the pieces of a row: sums, and the pieces' lists, which are in order.  A token's place is how many of each list are in front of it.  (Four lists are
// searched side by side, since a search is a chain of reads of LDS: 64 rows of 8 lists of 20 in a recorded graph 23.5 us one by one, 22.9 so; eight at a time
// 22.7, but of 4 lists 20.0 for 18.6.)
constexpr int kSideBySide = 4;

template <int TYPE>
__global__ __launch_bounds__(kLanes) void k_logits_join(LogitsDev q, int64_t first_row) {
  __shared__ uint64_t lists[kMostPieces * kMostTop], best[kMostTop];
  __shared__ uint32_t count;
  const int64_t row = first_row + blockIdx.x;
  const int lane = threadIdx.x & 63, n = q.pieces * q.top, first_step = q.top ? 1 << (31 - __clz(q.top)) : 0;
  const float given = given_logit<TYPE>(q, row, threadIdx.x);
  if (threadIdx.x == 0) count = 0;
  for (int i = threadIdx.x; i < n; i += kLanes) lists[i] = q.part_best[row * n + i];
  Sums a{-INFINITY, -1.0f, 0.0f};
  if (lane < q.pieces) {
    const float4 p = q.part[row * q.pieces + lane];
    a = Sums{p.x, p.y, p.z};
  }
  const float m = wave_largest(a.m);
  const bool mine = lane == __ffsll((unsigned long long)__ballot(a.m == m)) - 1;
  const float rest = a.s;
  a.s += 1.0f;
  move_to(a, m, q.c);
  a.s = wave_sum(mine ? rest : a.s);
  a.t = wave_sum(a.t);
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kLanes) {
    const uint64_t key = lists[i];
    if (!key) continue;
    atomicAdd(&count, 1u);
    int place = i % q.top;
    const int own = i / q.top;
    for (int b = 0; b < q.pieces && place < q.top; b += kSideBySide) {
      int in_front[kSideBySide] = {};
      for (int step = first_step; step; step >>= 1)
#pragma unroll
        for (int e = 0; e < kSideBySide; ++e) {
          const int at = in_front[e] + step, list = min(b + e, q.pieces - 1);
          if (at <= q.top && lists[list * q.top + at - 1] > key) in_front[e] = at;
        }
#pragma unroll
      for (int e = 0; e < kSideBySide; ++e) place += b + e < q.pieces && b + e != own ? in_front[e] : 0;
    }
    if (place < q.top) best[place] = key;
  }
  __syncthreads();
  put_row<TYPE>(q, row, a, best, min((int)count, q.top), threadIdx.x, kLanes, given);
}

constexpr int panel_of(int type) { return kLanes * kVectors * (type == RTAMS_TYPE_F32 ? 4 : 8); }

// Pieces of a row, and the panels of a piece.
void split(const rtams_logits_query *q, int *pieces, int *panels) {
  // (a row that does not begin at whole 16 bytes has some logits less in its first panel)
  const int size = q->type == RTAMS_TYPE_F32 ? 4 : 2, each = 16 / size;
  const bool whole = (uintptr_t)q->d_logits % 16 == 0 && (q->rows == 1 || q->row_stride % each == 0);
  const int64_t all = ((int64_t)q->vocab + (whole ? 0 : each - 1) + panel_of(q->type) - 1) / panel_of(q->type);
  int64_t want = q->rows < kSplitBelow ? (kSplitBelow + q->rows - 1) / q->rows : 1;
  if (want > kMostPieces) want = kMostPieces;
  if (want > all) want = all;
  *panels = (int)((all + want - 1) / want);
  *pieces = (int)((all + *panels - 1) / *panels);
}

bool query_ok(const rtams_logits_query *q) {
  if (!q) return fail(RTAMS_EINVAL, "query is NULL"), false;
  if (q->rows < 0 || q->rows > 0x7fffffff) return fail(RTAMS_EINVAL, "rows must be in 0..2^31 - 1, got %lld", (long long)q->rows), false;
  if (q->vocab < 1 || q->vocab >= 1 << 30) return fail(RTAMS_EINVAL, "vocab must be in 1..2^30 - 1, got %d", q->vocab), false;
  if (q->type < RTAMS_TYPE_BF16 || q->type > RTAMS_TYPE_F32) return fail(RTAMS_EINVAL, "unknown type %d", q->type), false;
  if (q->top < 0 || q->top > kMostTop) return fail(RTAMS_EINVAL, "top must be in 0..%d, got %d", kMostTop, q->top), false;
  if (q->tokens < 0) return fail(RTAMS_EINVAL, "tokens must not be negative, got %d", q->tokens), false;
  if (!(q->scale > 0.0f) || !(q->scale <= 1e30f)) return fail(RTAMS_EINVAL, "scale must be positive and at most 1e30"), false;
  if (q->row_stride < 0 || q->row_stride >= (int64_t)1 << 40) return fail(RTAMS_EINVAL, "row_stride must be in 0..2^40 - 1, got %lld", (long long)q->row_stride), false;
  return true;
}

size_t scratch_for(const rtams_logits_query *q) {
  int pieces, panels;
  if (q->rows == 0) return 0;
  split(q, &pieces, &panels);
  return pieces == 1 ? 0 : (size_t)q->rows * pieces * (16 + 8 * (size_t)q->top);
}

}  // namespace

}  // namespace rtams

extern "C" {

size_t rtams_logits_scratch_bytes_for(const rtams_logits_query *q) { return query_ok(q) ? scratch_for(q) : (size_t)-1; }

int rtams_logits_score(const rtams_logits_query *q, void *hip_stream) {
  if (!query_ok(q)) return RTAMS_EINVAL;
  if (q->rows == 0) return RTAMS_OK;
  const uintptr_t size = q->type == RTAMS_TYPE_F32 ? 4 : 2;
  if (!q->d_logits || (q->tokens && (!q->d_tokens || !q->d_logprobs)) || (q->top && !q->d_top)) return fail(RTAMS_EINVAL, "logits, tokens or an output asked for are NULL");
  if ((uintptr_t)q->d_logits % size) return fail(RTAMS_EINVAL, "logits are not aligned to their type");
  if (((uintptr_t)q->d_tokens | (uintptr_t)q->d_lse | (uintptr_t)q->d_entropy | (uintptr_t)q->d_logprobs | (uintptr_t)q->d_top | (uintptr_t)q->d_top_logprobs) % 4)
    return fail(RTAMS_EINVAL, "tokens or outputs are not aligned to their type");
  const size_t scratch = scratch_for(q);
  if (scratch && (!q->d_scratch || q->scratch_bytes < scratch)) return fail(RTAMS_EINVAL, "scratch_bytes %zu, %zu are needed", q->d_scratch ? q->scratch_bytes : 0, scratch);
  if (scratch && (uintptr_t)q->d_scratch % 16) return fail(RTAMS_EINVAL, "scratch must be 16-byte aligned");
  LogitsDev d{};
  d.rows = q->rows;
  d.row_stride = q->rows == 1 ? 0 : q->row_stride;
  d.vocab = q->vocab;
  d.top = q->top;
  d.tokens = q->tokens;
  split(q, &d.pieces, &d.panels);
  d.scale = q->scale;
  d.c = (float)((double)q->scale * 1.4426950408889634);
  d.logits = q->d_logits;
  d.given = q->d_tokens;
  d.lse = q->d_lse;
  d.entropy = q->d_entropy;
  d.logprobs = q->d_logprobs;
  d.best = q->d_top;
  d.best_logprobs = q->top ? q->d_top_logprobs : nullptr;
  d.part = static_cast<float4 *>(q->d_scratch);
  d.part_best = reinterpret_cast<uint64_t *>(d.part + q->rows * d.pieces);
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const auto go = [&](auto kernel, auto joiner) {
    const int64_t units = q->rows * d.pieces, most = 1 << 22;
    for (int64_t at = 0; at < units; at += most) kernel<<<(uint32_t)(units - at < most ? units - at : most), kLanes, 0, s>>>(d, at);
    if (d.pieces > 1) joiner<<<(uint32_t)q->rows, kLanes, 0, s>>>(d, 0);
  };
  switch (q->type) {
    case RTAMS_TYPE_BF16: go(k_logits<RTAMS_TYPE_BF16>, k_logits_join<RTAMS_TYPE_BF16>); break;
    case RTAMS_TYPE_F16: go(k_logits<RTAMS_TYPE_F16>, k_logits_join<RTAMS_TYPE_F16>); break;
    default: go(k_logits<RTAMS_TYPE_F32>, k_logits_join<RTAMS_TYPE_F32>); break;
  }
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? RTAMS_OK : fail(RTAMS_EHIP, "score launch failed: %s", hipGetErrorString(e));
}

}  // extern "C"
