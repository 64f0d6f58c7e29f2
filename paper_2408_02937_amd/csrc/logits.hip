// Log probabilities of given tokens, entropy and the most likely tokens of rows of logits (include/rtams_logits.h).
//
//   S = sum 2^(c (x - m)),  T = sum 2^(c (x - m)) c (x - m),  c = scale * log2 e, m the largest so far
//   lse = scale m + ln 2 log2 S,  entropy = ln 2 (log2 S - T / S),  log probability = scale (x - m) - ln 2 log2 S
//
// (Differences are taken first: rows masked with the type's lowest number have that as their largest, and c times it is none.)
//
// Bound by reading the logits once.  A workgroup takes a row, or where rows are few a piece of one, in panels that its lanes hold in registers, 256
// bytes each: all of a panel's loads go out before the first is needed, and its largest is known before the first power, so that sums are scaled
// once a panel.  The most likely tokens: of the first panel the k-th largest of the lanes' largest is a bound that the k largest of all reach, and few
// others do; what reaches it goes to LDS and is ranked there.  Later panels are held against the k-th so far.  Where too many reach the
// bound (one lane has them all, or they are equal) it is found by bisection, and of those equal to it the lowest tokens are counted off.
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

template <int TYPE>
constexpr int each_of() { return TYPE == RTAMS_TYPE_F32 ? 4 : 8; }  // logits of a vector

template <int TYPE>
__device__ inline float logit(const uint4 &v, int e) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
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
  float m, s, t;  // largest, as it is; the sums relative to it
};

// Sums relative to another largest, which is no smaller.
__device__ inline void move_to(Sums &a, float m, float c) {
  if (a.m == m) return;
  const float by = a.m == -INFINITY ? kFar : (a.m - m) * c, shrink = __builtin_amdgcn_exp2f(by);
  a.t = shrink * fmaf(a.s, fmaxf(by, kFar), a.t);
  a.s *= shrink;
  a.m = m;
}

__device__ inline void join(Sums &a, Sums b, float c) {
  const float m = fmaxf(a.m, b.m);
  move_to(a, m, c);
  move_to(b, m, c);
  a.s += b.s;
  a.t += b.t;
}

struct Shared {
  uint64_t best[kMostTop + kRoom];  // the best so far, then what is ranked with them
  uint64_t sorted[kMostTop];
  uint32_t most[kLanes];
  uint32_t waves[kWaves];
  Sums sums[kWaves];
  uint32_t count, have;
  float bound;
};

// The numbers of a row, one workgroup or wavefront of `lanes` lanes.
template <int TYPE>
__device__ void put_row(const LogitsDev &q, int64_t row, const Sums &a, const uint64_t *best, int have, int lane, int lanes) {
  constexpr float kLn2 = 0.6931471805599453f;
  const bool none = a.m == -INFINITY && a.s == 0.0f, wrong = !(a.s >= 0.0f) || a.m == INFINITY;
  const float log_s = __builtin_amdgcn_logf(a.s), nan = __uint_as_float(0x7fc00000u);
  if (lane == 0) {
    if (q.lse) q.lse[row] = wrong ? nan : none ? -INFINITY : fmaf(a.m, q.scale, kLn2 * log_s);
    if (q.entropy) q.entropy[row] = wrong ? nan : none ? 0.0f : kLn2 * (log_s - a.t / a.s);
  }
  const auto log_probability = [&](float x) { return wrong ? nan : x == -INFINITY ? -INFINITY : fmaf(x - a.m, q.scale, -kLn2 * log_s); };
  const char *x = static_cast<const char *>(q.logits) + row * q.row_stride * (TYPE == RTAMS_TYPE_F32 ? 4 : 2);
  for (int i = lane; i < q.tokens; i += lanes) {
    const int t = q.given[row * q.tokens + i];
    q.logprobs[row * q.tokens + i] = log_probability((uint32_t)t < (uint32_t)q.vocab ? logit_at<TYPE>(x, t) : -INFINITY);
  }
  for (int i = lane; i < q.top; i += lanes) {
    const bool there = i < have && !wrong;
    q.best[row * q.top + i] = there ? (int32_t)~(uint32_t)best[i] : -1;
    if (q.best_logprobs) q.best_logprobs[row * q.top + i] = log_probability(there ? unordered((uint32_t)(best[i] >> 32)) : -INFINITY);
  }
}

// Logits at .. at + E - 1 of a row, 16 bytes that lie at whole 16; -inf where the row has none.
template <int TYPE>
__device__ __forceinline__ uint4 load_vector(const char *x, int at, int vocab) {
  constexpr int E = each_of<TYPE>(), kSize = 16 / E;
  constexpr uint32_t kNone = TYPE == RTAMS_TYPE_F32 ? 0xff800000u : TYPE == RTAMS_TYPE_BF16 ? 0xff80ff80u : 0xfc00fc00u;
  if (at >= 0 && at + E <= vocab) return *reinterpret_cast<const uint4 *>(x + (int64_t)at * kSize);
  uint32_t w[4] = {kNone, kNone, kNone, kNone};
  if (at + E > 0 && at < vocab)
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (at + e >= 0 && at + e < vocab) {
        if (E == 4) w[e] = reinterpret_cast<const uint32_t *>(x)[at + e];
        else w[e / 2] = (e % 2 ? w[e / 2] & 0xffffu : w[e / 2] & 0xffff0000u) | (uint32_t)reinterpret_cast<const uint16_t *>(x)[at + e] << (e % 2 * 16);
      }
  return make_uint4(w[0], w[1], w[2], w[3]);
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

// Takes a panel's most likely tokens to those so far.  first: token of the lane's first logit; most: the lane's largest.  (Few lanes look at their
// logits again, most of them once in a row: they read them again.  Out of registers every look is 128 steps of code, and registers spill.)
template <int TYPE>
__device__ void take_best(const char *x, int vocab, int first, float most, int top, Shared &sh) {
  constexpr int E = each_of<TYPE>();
  if (!__syncthreads_or(most > sh.bound)) return;
  const float bound = sh.bound;
  const int have = sh.have;
  const auto each = [&](float least, auto f) {  // f(token, logit) in the order of the lane's tokens
    if (!(most >= least)) return;
#pragma unroll 2
    for (int v = 0; v < kVectors; ++v) {
      const int at = first + v * kLanes * E;
      const uint4 raw = load_vector<TYPE>(x, at, vocab);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float l = logit<TYPE>(raw, e);
        if (l >= least) f(at + e, l);
      }
    }
  };
  const auto reaching = [&](float least, uint32_t *mine) {  // how many do, in all lanes
    uint32_t n = 0;
    each(least, [&](int, float) { ++n; });
    *mine = n;
    return sum_lanes(n, sh);
  };
  const auto append = [&](float least, uint32_t n) {  // n in this lane
    if (threadIdx.x == 0) sh.count = have;
    __syncthreads();
    uint32_t at = n ? atomicAdd(&sh.count, n) : 0;
    if (n) each(least, [&](int token, float l) { sh.best[at++] = key_of(l, token); });
    __syncthreads();
  };
  float from = unordered(ordered(bound) + 1);  // the least that exceeds it (of -inf the least number)
  uint32_t mine = 0, all = kRoom + 1;
  if (have == top) all = reaching(from, &mine);
  if (all > kRoom) {
    // the top-th largest of the lanes' largest
    const uint32_t largest = most > bound ? ordered(most) : 0;
    sh.most[threadIdx.x] = largest;
    __syncthreads();
    int above = 0;
    for (int j = 0; j < kLanes; ++j) above += sh.most[j] > largest || (sh.most[j] == largest && j < (int)threadIdx.x);
    if (above == top - 1) sh.count = largest;
    __syncthreads();
    if (sh.count) from = unordered(sh.count);
    all = reaching(from, &mine);
  }
  if (all <= kRoom) {
    append(from, mine);
    return rank(have + (int)all, top, sh);
  }
  // the top-th largest, exactly: the highest that as many reach
  uint32_t low = ordered(from), high = ordered(INFINITY);
  while (low < high) {
    const uint32_t mid = low + (high - low + 1) / 2;
    uint32_t n;
    if (reaching(unordered(mid), &n) >= (uint32_t)top) low = mid;
    else high = mid - 1;
  }
  const float equal = unordered(low), over = unordered(low + 1);
  all = reaching(over, &mine);
  append(over, mine);
  uint32_t filled = have + all, need = top - all;
  for (int v = 0; v < kVectors && need; ++v) {  // in the order of the tokens
    const int at = first + v * kLanes * E;
    const uint4 raw = load_vector<TYPE>(x, at, vocab);
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

template <int TYPE>
__global__ __launch_bounds__(kLanes, 4) void k_logits(LogitsDev q, int64_t first_unit) {
  constexpr int E = each_of<TYPE>(), kPanel = kLanes * kVectors * E, kSize = 16 / E;
  __shared__ Shared sh;
  const int64_t unit = first_unit + blockIdx.x, row = unit / q.pieces;
  const int piece = (int)(unit % q.pieces), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const char *const x = static_cast<const char *>(q.logits) + row * q.row_stride * kSize;
  // vectors begin at whole 16 bytes: the first may begin in front of the row
  const int ahead = (int)(((uintptr_t)x & 15) / kSize);
  const char *const x16 = x - ahead * kSize;
  if (threadIdx.x == 0) {
    sh.have = 0;
    sh.bound = -INFINITY;
  }
  Sums a{-INFINITY, 0.0f, 0.0f};
  for (int p = 0; p < q.panels; ++p) {
    const int64_t begin = ((int64_t)piece * q.panels + p) * kPanel;  // counted from x16
    if (begin >= (int64_t)q.vocab + ahead) break;
    const int first = (int)(begin - ahead) + (int)threadIdx.x * E;  // token of this lane's first logit
    uint4 raw[kVectors];
    if (first - (int)threadIdx.x * E >= 0 && begin - ahead + kPanel <= q.vocab) {
#pragma unroll
      for (int v = 0; v < kVectors; ++v) raw[v] = *reinterpret_cast<const uint4 *>(x16 + begin * kSize + (v * kLanes + threadIdx.x) * 16);
    } else {
#pragma unroll
      for (int v = 0; v < kVectors; ++v) {
        raw[v] = load_vector<TYPE>(x, first + v * kLanes * E, q.vocab);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    // (one vector after the other: registers hold the logits as they came, not all of them turned into 32 bits)
    const auto each = [&](auto f) {
#pragma unroll
      for (int v = 0; v < kVectors; ++v) {
        asm("" : "+v"(raw[v].x), "+v"(raw[v].y), "+v"(raw[v].z), "+v"(raw[v].w));
#pragma unroll
        for (int e = 0; e < E; ++e) f(e, logit<TYPE>(raw[v], e));
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    float most = -INFINITY;
    each([&](int, float l) { most = fmaxf(most, l); });
    move_to(a, fmaxf(a.m, most), q.c);
    const float m = a.m == -INFINITY ? 0.0f : a.m;
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f}, t[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    each([&](int e, float l) {
      // (NaN, and +inf less +inf, are NaN in the sums; -inf is 0 in both)
      const float z = (l - m) * q.c, y = __builtin_amdgcn_exp2f(z);
      s[e % 4] += y;
      t[e % 4] = fmaf(y, fmaxf(z, kFar), t[e % 4]);
    });
    a.s += (s[0] + s[1]) + (s[2] + s[3]);
    a.t += (t[0] + t[1]) + (t[2] + t[3]);
    if (q.top) {
      if (p == 0) __syncthreads();
      take_best<TYPE>(x, q.vocab, first, most, q.top, sh);
    }
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) join(a, Sums{__shfl_xor(a.m, o), __shfl_xor(a.s, o), __shfl_xor(a.t, o)}, q.c);
  if (lane == 0) sh.sums[wave] = a;
  __syncthreads();
  a = sh.sums[0];
  for (int w = 1; w < kWaves; ++w) join(a, sh.sums[w], q.c);
  const int have = q.top ? (int)sh.have : 0;
  if (q.pieces == 1) {
    put_row<TYPE>(q, row, a, sh.sorted, have, threadIdx.x, kLanes);
  } else {
    if (threadIdx.x == 0) q.part[unit] = make_float4(a.m, a.s, a.t, 0.0f);
    for (int i = threadIdx.x; i < q.top; i += kLanes) q.part_best[unit * q.top + i] = i < have ? sh.sorted[i] : 0;
  }
}

// A wavefront joins the pieces of a row: sums, and the heads of the pieces' lists, which are in order.
template <int TYPE>
__global__ __launch_bounds__(64) void k_logits_join(LogitsDev q, int64_t first_row) {
  __shared__ uint64_t best[kMostTop];
  const int64_t row = first_row + blockIdx.x;
  const int lane = threadIdx.x;
  Sums a{-INFINITY, 0.0f, 0.0f};
  if (lane < q.pieces) {
    const float4 p = q.part[row * q.pieces + lane];
    a = Sums{p.x, p.y, p.z};
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) join(a, Sums{__shfl_xor(a.m, o), __shfl_xor(a.s, o), __shfl_xor(a.t, o)}, q.c);
  const uint64_t *list = q.part_best + (row * q.pieces + min(lane, q.pieces - 1)) * q.top;
  int at = 0, have = 0;
  uint64_t head = lane < q.pieces && q.top ? list[0] : 0;
  for (; have < q.top; ++have) {
    uint64_t most = head;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint64_t other = (uint64_t)__shfl_xor((unsigned long long)most, o);
      most = other > most ? other : most;
    }
    if (most == 0) break;
    if (lane == 0) best[have] = most;
    if (head == most) head = ++at < q.top ? list[at] : 0;  // (keys differ: one lane)
  }
  __syncthreads();
  put_row<TYPE>(q, row, a, best, have, lane, 64);
}

constexpr int panel_of(int type) { return kLanes * kVectors * (type == RTAMS_TYPE_F32 ? 4 : 8); }

// Pieces of a row, and the panels of a piece.
void split(const rtams_logits_query *q, int *pieces, int *panels) {
  const int64_t all = ((int64_t)q->vocab + 7 + panel_of(q->type) - 1) / panel_of(q->type);
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
    if (d.pieces > 1) joiner<<<(uint32_t)q->rows, 64, 0, s>>>(d, 0);
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
