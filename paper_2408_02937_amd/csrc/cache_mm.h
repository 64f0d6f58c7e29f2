// Codes of the cache as operands of the matrix instructions, and what the attention kernels share.
#pragma once
#include "cache.h"

namespace rtams {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

union HalfWords {
  half8 h;
  half2v p[4];
  uint32_t w[4];
};

// The eight codes of a word as halves.  Or'ed into the low bits of 1024 a code c is 1024 + c, four bits further up 1024 + 16 c: exact, and
// so is what is taken off again.
__device__ inline HalfWords codes_of(uint32_t w) {
  HalfWords x;
  const uint32_t w8 = w >> 8;
  // (in registers, where the compiler does not see them, so that and and or are one instruction, which takes no constants)
  uint32_t low = 0x000f000fu, high = 0x00f000f0u, base = 0x64006400u;
  asm("" : "+s"(low), "+s"(high), "+v"(base));
  x.w[0] = (w & low) | base;
  x.w[1] = (w & high) | base;
  x.w[2] = (w8 & low) | base;
  x.w[3] = (w8 & high) | base;
  const half2v k1024 = {(_Float16)1024.0f, (_Float16)1024.0f}, k16 = {(_Float16)0.0625f, (_Float16)0.0625f}, k64 = {(_Float16)-64.0f, (_Float16)-64.0f};
  x.p[0] = x.p[0] - k1024;
  x.p[1] = __builtin_elementwise_fma(x.p[1], k16, k64);
  x.p[2] = x.p[2] - k1024;
  x.p[3] = __builtin_elementwise_fma(x.p[3], k16, k64);
  return x;
}

__device__ inline _Float16 half_at(uint32_t w, int high) {
  const uint16_t u = (uint16_t)(high ? w >> 16 : w);
  _Float16 h;
  __builtin_memcpy(&h, &u, 2);
  return h;
}

// 16 tokens of a block's keys, 16 (i / 8) + i % 8 + 8 tile for i of 0..15, as the left operand: lane i + 16 b holds the b-th quarter of
// token i's channels.
template <int D>
struct KeyTile {
  static constexpr int NJ = D / 32;
  uint32_t code[NJ];
  uint32_t meta[D == 96 ? 3 : (NJ + 3) / 4];

  __device__ void load(const unsigned char *blk, int tile, int lane) {
    const int i = lane & 15, b = lane >> 4, token = 16 * (i >> 3) + (i & 7) + 8 * tile;
    const uint32_t *p = reinterpret_cast<const uint32_t *>(blk + token * (D / 2)) + b * NJ;
    const uint32_t *mp = reinterpret_cast<const uint32_t *>(blk + 16 * D) + token * (D / 32);
    if constexpr (D == 96) {  // three words, a group each
#pragma unroll
      for (int j = 0; j < 3; ++j) {
        code[j] = p[j];
        meta[j] = mp[(3 * b + j) >> 2];
      }
    } else if constexpr (D == 64) {
      const uint2 x = *reinterpret_cast<const uint2 *>(p);
      code[0] = x.x;
      code[1] = x.y;
      meta[0] = mp[b >> 1];
    } else {
#pragma unroll
      for (int j = 0; j < NJ; j += 4) {
        const uint4 x = *reinterpret_cast<const uint4 *>(p + j);
        code[j] = x.x;
        code[j + 1] = x.y;
        code[j + 2] = x.z;
        code[j + 3] = x.w;
        meta[j / 4] = mp[b * (NJ / 4) + j / 4];
      }
    }
  }
  // Eight channels, rounded once to a half, as the matrix instructions take them: by 2^-11 of a value at most, half a unit in the last place of a half and
  // less of a bfloat16 that was written, but more than a step of the codes where a group's zero is above 2^11 steps; reading back has the values in 32
  // bits.  (Exact, zeros would be products of their own beside those of the codes.)
  __device__ half8 values(int j) const {
    HalfWords x = codes_of(code[j]);
    const uint32_t mt = meta[D == 96 ? j : j / 4];
    const half2v step = {half_at(mt, 0), half_at(mt, 0)}, zero = {half_at(mt, 1), half_at(mt, 1)};
#pragma unroll
    for (int i = 0; i < 4; ++i) x.p[i] = __builtin_elementwise_fma(x.p[i], step, zero);
    return x.h;
  }
};

// A block's values as the left operand V^T: lane ch % 16 + 16 b holds 8 tokens of a channel (value_word).
template <int D>
struct ValueBlock {
  static constexpr int NT = D / 16, VC = value_chunk(D);
  uint32_t code[NT];
  HalfWords step[D / 32], zero[D / 32];

  __device__ void load(const unsigned char *blk, int lane) {
    const uint32_t *p = reinterpret_cast<const uint32_t *>(blk + 20 * D);
#pragma unroll
    for (int q = 0; q < NT / VC; ++q) {
      if constexpr (VC == 4) {
        const uint4 x = reinterpret_cast<const uint4 *>(p)[q * 64 + lane];
        code[4 * q] = x.x;
        code[4 * q + 1] = x.y;
        code[4 * q + 2] = x.z;
        code[4 * q + 3] = x.w;
      } else {
        const uint2 x = reinterpret_cast<const uint2 *>(p)[q * 64 + lane];
        code[2 * q] = x.x;
        code[2 * q + 1] = x.y;
      }
    }
    const uint4 *mp = reinterpret_cast<const uint4 *>(blk + 36 * D) + (lane >> 4);
#pragma unroll
    for (int g = 0; g < D / 32; ++g) {
      const uint4 x = mp[g * 8], y = mp[g * 8 + 4];
      __builtin_memcpy(&step[g], &x, 16);
      __builtin_memcpy(&zero[g], &y, 16);
    }
  }
  __device__ half8 values(int n) const {
    HalfWords x = codes_of(code[n]);
#pragma unroll
    for (int i = 0; i < 4; ++i) x.p[i] = __builtin_elementwise_fma(x.p[i], step[n / 2].p[i], zero[n / 2].p[i]);
    return x.h;
  }
};

// A probability is the half exp2(score - m) that its product takes, and it is these halves that are summed, so that what rounding takes from the
// values it takes from their weights too.  m is set kTop below the largest score and follows once a score is kTop + kLag over it, still inside a half:
// the largest probability of a row is between 2^kTop and 2^15, one 2^-(kTop + 14) of it has all its bits and one 2^-(kTop + 25) some.  A lag of 4
// and a top of 11 reach further down and cost prompts a tenth (583 and 641 us), a lag of 1 a fifth (701); single tokens take the same with each.
constexpr float kTop = 7.0f, kLag = 8.0f;
static_assert(kTop + kLag <= 15.0f, "a half ends at 65504");

__device__ inline float add_up(float sum, const half8 &p) {
  const half2v ones = {(_Float16)1.0f, (_Float16)1.0f};
  HalfWords w;
  w.h = p;
#pragma unroll
  for (int i = 0; i < 4; ++i) sum = __builtin_amdgcn_fdot2(w.p[i], ones, sum, false);
  return sum;
}

__device__ inline half8 to_half8(const float p[8]) {
  half8 h;
#pragma unroll
  for (int e = 0; e < 8; ++e) h[e] = (_Float16)p[e];
  return h;
}

// Eight channels of a row of q, times the scale in 32 bits, rounded to halves: to a bit or none where the scale is a power of two.
__device__ inline half8 load_query(const uint16_t *p, bool half_type, bool vec, float scale) {
  uint16_t raw[8];
  if (vec) {
    const uint4 x = *reinterpret_cast<const uint4 *>(p);
    __builtin_memcpy(raw, &x, 16);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) raw[e] = p[e];
  }
  half8 h;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    _Float16 x;
    __builtin_memcpy(&x, &raw[e], 2);
    h[e] = (_Float16)((half_type ? (float)x : __uint_as_float((uint32_t)raw[e] << 16)) * scale);
  }
  return h;
}

// Channels c .. c + 3 of an output row: sums over the tokens, relative to the maximum `top` of the scores in powers of two.
__device__ inline void store_row(const CacheQuery &q, int64_t row, int head, int c, f32x4 v, float top, float sum) {
  const float by = sum == 0.0f ? 0.0f : 1.0f / sum;  // (a row that sees nothing: zeros)
  uint16_t h[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float x = v[e] * by;
    if (q.half_type) {
      const _Float16 y = (_Float16)x;
      __builtin_memcpy(&h[e], &y, 2);
    } else {
      const __bf16 y = (__bf16)x;
      __builtin_memcpy(&h[e], &y, 2);
    }
  }
  uint16_t *p = q.out + row * q.out_row + (int64_t)head * q.out_head + c;
  if (q.vec) {
    *reinterpret_cast<uint2 *>(p) = make_uint2((uint32_t)h[0] | (uint32_t)h[1] << 16, (uint32_t)h[2] | (uint32_t)h[3] << 16);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) p[e] = h[e];
  }
  if (q.lse && c == 0) q.lse[row * q.q_heads + head] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
}

// Parts of rows pass between workgroups on different dies: stores that go through to where all dies read, and loads that look
// there.  (Fences would write back and drop a whole L2 each time: 0.25 ms for 768 workgroups.)
__device__ inline void put_pair(float *p, float x, float y) {
  const uint64_t v = (uint64_t)__float_as_uint(y) << 32 | __float_as_uint(x);
  __hip_atomic_store(reinterpret_cast<uint64_t *>(p), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ inline float2 get_pair(const float *p) {
  const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t *>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}

__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// a / b rounded up, a below 2^24
__device__ inline uint32_t div_up(uint32_t a, uint32_t b, float one_over_b) {
  uint32_t q = (uint32_t)((float)a * one_over_b), r = a - q * b;  // off by one at most
  if ((int32_t)r < 0) { --q; r += b; }
  if (r >= b) { ++q; r -= b; }
  return q + (r > 0);
}

// What rows see (CacheSight), 32 tokens at a time as the bits of a word.
__device__ inline uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; }
// Bits from number `at` on, -31 or more; those that are not there are 0.
__device__ inline uint32_t bits_at(uint64_t x, int at) { return at >= 64 ? 0u : at >= 0 ? (uint32_t)(x >> at) : (uint32_t)x << -at; }
// Positions that the sinks take, in whole blocks.
__device__ inline int sink_blocks(const CacheSight &g) { return (g.sinks + kBlockTokens - 1) & ~(kBlockTokens - 1); }

constexpr int kUnits = 256;  // compute units

// Steps of a piece, of n items' steps.  Pieces are to run all at once, `workers` of them, and to leave the compute units alike much to do:
// of sixteen sizes from an even share up to twice that, a quarter of the items to a lane, the one with the least steps for a
// compute unit, which has pieces / 256 rounded up.
// beside: what a unit's first piece costs beyond the others that run beside it.
__device__ inline uint32_t piece_steps(const float *steps, int n, int kv_heads, uint32_t share, uint32_t workers, uint32_t beside = 0) {
  const int lane = threadIdx.x & 63;
  const uint32_t more = (share + 15) / 16, size = share + (lane & 15) * more;
  const float one_over = __builtin_amdgcn_rcpf((float)size);
  float pieces = 0.0f;
  for (int i = (lane >> 4) * 4; i < n; i += 16) {
    const f32x4 x = *reinterpret_cast<const f32x4 *>(steps + i) * one_over;  // (no steps behind the last item)
    pieces += ceilf(x[0]) + ceilf(x[1]) + ceilf(x[2]) + ceilf(x[3]);
  }
  pieces += __shfl_xor(pieces, 16);
  pieces += __shfl_xor(pieces, 32);
  const uint32_t all = (uint32_t)pieces * (uint32_t)kv_heads;
  float cost = all <= workers ? (float)((all + kUnits - 1) / kUnits + beside) * (float)size : 3e38f;
  const float mine = cost;
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) cost = fminf(cost, __shfl_xor(cost, o));
  const uint64_t best = __ballot(mine == cost && cost < 3e38f) & 0xffff;
  return best ? share + (uint32_t)(__ffsll((unsigned long long)best) - 1) * more : 2 * share;
}

// Channels c .. c + 3 of a row of n parts, `stride` rows apart, joined in order.  before: an earlier launch wrote them.
template <bool BEFORE>
__device__ inline void join_parts(const CacheQuery &q, int64_t row, int head, int c, int n, const float *part, const float *ml, int head_dim, int stride) {
  constexpr int kRun = BEFORE ? 16 : 8;  // parts that are asked for at a time
  float top = -INFINITY, sum = 0.0f;
  f32x4 v{0, 0, 0, 0};
  for (int i0 = 0; i0 < n; i0 += kRun) {
    float2 x[kRun], a[kRun], b[kRun];
#pragma unroll
    for (int k = 0; k < kRun; ++k) {
      const int64_t i = min(i0 + k, n - 1) * (int64_t)stride;
      if constexpr (BEFORE) {
        const f32x4 y = *reinterpret_cast<const f32x4 *>(part + i * head_dim);
        x[k] = *reinterpret_cast<const float2 *>(ml + i * 2);
        a[k] = make_float2(y[0], y[1]);
        b[k] = make_float2(y[2], y[3]);
      } else {
        x[k] = get_pair(ml + i * 2);
        a[k] = get_pair(part + i * head_dim);
        b[k] = get_pair(part + i * head_dim + 2);
      }
    }
    float now = top;
#pragma unroll
    for (int k = 0; k < kRun; ++k) now = fmaxf(now, x[k].x);
    const float shrink = top == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(top - now);
    sum *= shrink;
    v *= shrink;
    top = now;
#pragma unroll
    for (int k = 0; k < kRun; ++k)
      if (i0 + k < n) {
        const float by = x[k].x == -INFINITY && top == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(x[k].x - top);
        sum += x[k].y * by;
        v += f32x4{a[k].x, a[k].y, b[k].x, b[k].y} * by;
      }
  }
  store_row(q, row, head, c, v, top, sum);
}

}  // namespace rtams
