// Writing keys and values into the cache in 4 bits and reading them back (the format: include/rtams_cache.h).
//
// A workgroup owns 32 tokens of one head.  A lane has 8 channels of a token, 16 bytes and a word of codes; the four lanes of a group of 32 find
// its least and largest among themselves.  A word of value codes holds 8 tokens of a channel: the tokens' words meet in LDS, where a lane
// takes 8 tokens by 2 channels and turns them round; tokens already there keep their bits.  Both directions are bound by memory: 4 bytes a
// channel on the side of the rows, 1.25 on that of the cache.  Of single tokens they are a chain of loads (length, page, count), so the
// rows are asked for before the page is known.
//
// Measured: 34,439 rows of 8 heads of 128 channels, keys and values: read back in 31 us for 185 MB, 5.9 TB/s; written in 56 us, 3.3 TB/s: vector
// instructions take 62 % of the cycles.
// 64 single rows: 5 us written, 4 read.  Four heads a workgroup took 72 us (half as many run at once), 8 workgroups a unit forced 92 (registers spill).
#include "../../include/rtams_cache.h"

#include "cache_mm.h"

namespace rtams {

namespace {

constexpr int kLanes = 256;

template <bool HALF>
__device__ inline float from_bits(uint16_t x) {
  if (!HALF) return __uint_as_float((uint32_t)x << 16);
  _Float16 h;
  __builtin_memcpy(&h, &x, 2);
  return (float)h;
}

__device__ inline uint16_t half_bits(_Float16 h) {
  uint16_t u;
  __builtin_memcpy(&u, &h, 2);
  return u;
}

__device__ inline _Float16 half_of(uint16_t u) {
  _Float16 h;
  __builtin_memcpy(&h, &u, 2);
  return h;
}

// The other lanes of four: a move between lanes inside the vector unit.
template <int CTRL>
__device__ inline float quad(float x) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xf, 0xf, false));
}

// Step and zero of a group of 32 channels of which four lanes have 8 each, and this lane's word of codes.
template <bool HALF>
__device__ inline uint32_t quantise(const uint4 &in, uint32_t *code) {
  const uint32_t raw[4] = {in.x, in.y, in.z, in.w};
  float f[8];
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  u16x2 top = {0, 0};  // magnitudes as whole numbers: in both types larger ones, and NaN behind them all, are larger
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, raw[j] & 0x7fff7fffu));
    f[2 * j] = from_bits<HALF>((uint16_t)raw[j]);
    f[2 * j + 1] = from_bits<HALF>((uint16_t)(raw[j] >> 16));
  }
  if (max(top[0], top[1]) > (HALF ? 0x7b53 : 0x476a))  // more than 60000 or not a number
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = f[e] != f[e] ? 0.0f : fminf(fmaxf(f[e], -kCacheMost), kCacheMost);
  float lo = f[0], hi = f[0];
#pragma unroll
  for (int e = 1; e < 8; ++e) {
    lo = fminf(lo, f[e]);
    hi = fmaxf(hi, f[e]);
  }
  lo = fminf(lo, quad<0xb1>(lo));  // lanes 1, 0, 3, 2
  hi = fmaxf(hi, quad<0xb1>(hi));
  lo = fminf(lo, quad<0x4e>(lo));  // lanes 2, 3, 0, 1
  hi = fmaxf(hi, quad<0x4e>(hi));
  // (a fifteenth and a reciprocal with a step of correction each: what a division gives, in a quarter of its operations)
  const float fifteenth = (hi - lo) * (1.0f / 15.0f);
  const _Float16 step = (_Float16)fmaf(fmaf(-15.0f, fifteenth, hi - lo), 1.0f / 15.0f, fifteenth), zero = (_Float16)lo;
  const float z = (float)zero, s = (float)step, near = __builtin_amdgcn_rcpf(s), inv = s > 0.0f ? fmaf(fmaf(-s, near, 1.0f), near, near) : 0.0f;
  // Added to 1.5 * 2^23 a number below 16 is rounded to the nearest whole one, ties to even, and is in the low bits; what the upper bits add up to
  // over the word is taken off at its start.
  constexpr uint32_t kMagic = 0x4b400000u;
  uint32_t word = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) word -= kMagic << element_shift(e);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float c = __builtin_amdgcn_fmed3f(__fmul_rn(f[e] - z, inv), 0.0f, 15.0f);
    word += __float_as_uint(c + 12582912.0f) << element_shift(e);
  }
  *code = word;
  return (uint32_t)half_bits(step) | (uint32_t)half_bits(zero) << 16;
}

// Eight words w, of 8 elements each: elements 2 i and 2 i + 1 of all of them, as words a and b (a lane's part of an 8 by 8 transposition).
__device__ inline void turn_round(const uint32_t w[8], int i, uint32_t *a, uint32_t *b) {
  uint32_t even = 0, odd = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    even |= ((w[2 * k] >> (4 * i)) & 0x000f000fu) << (4 * k);
    odd |= ((w[2 * k + 1] >> (4 * i)) & 0x000f000fu) << (4 * k);
  }
  *a = (even & 0xffffu) | odd << 16;
  *b = even >> 16 | (odd & 0xffff0000u);
}

// Value codes on their way: as words of a token, as words of a channel, and their steps and zeros.
template <int D>
struct Turn {
  uint32_t in[kBlockTokens * (D / 8 + 1)];
  alignas(16) uint32_t out[4 * D];
  alignas(16) uint16_t meta[2 * D];
};

struct BlockRows {  // the rows of the call that lie in one block of 32 tokens
  int64_t row0;     // of token 0 of the block (the rows before `from` are not the call's)
  int from, to;     // its tokens
  int page;
  uint32_t block_in_page;
};

// Block number b of the item's rows; false where there is none.  *bad: the item is not what the call asks for.
__device__ inline bool find_block(const CacheDev &d, const CacheRows &r, int item, int b, BlockRows *out, bool *bad) {
  int64_t first;
  int count;
  const int seq = uniform(cache_item_seq(r, item));
  const bool rows = cache_item_rows(r, item, &first, &count);
  const bool known = (uint32_t)seq < (uint32_t)d.max_seqs;
  const int length = uniform(d.lengths[known ? seq : 0]), from = uniform((int)first);
  count = uniform(count);
  *bad = uniform(!rows || !known || count > length);
  if (*bad) return false;
  const int start = length - count, block = start / kBlockTokens + b;
  if (count == 0 || block * kBlockTokens >= length) return false;
  out->from = start > block * kBlockTokens ? start - block * kBlockTokens : 0;
  out->to = length - block * kBlockTokens < kBlockTokens ? length - block * kBlockTokens : kBlockTokens;
  out->row0 = (int64_t)from + (int64_t)block * kBlockTokens - start;
  const uint32_t p = cache_page_of(d, (uint32_t)block);
  out->page = uniform(d.table[(int64_t)seq * d.max_pages + p]);
  out->block_in_page = (uint32_t)block - p * d.page_blocks;
  return true;
}

template <int D>
struct Rows {  // keys first, then values: 8 channels of a token to a lane
  static constexpr int W = D / 8, kEach = 2 * kBlockTokens * W / kLanes;
  static_assert(2 * kBlockTokens * W % kLanes == 0, "whole rounds");
  uint4 raw[kEach];

  __device__ void load(const uint16_t *k, const uint16_t *v, const BlockRows &t, int head, int64_t row_stride, int64_t head_stride, int vec) {
    const uint16_t *k0 = k + t.row0 * row_stride + head * head_stride, *v0 = v + t.row0 * row_stride + head * head_stride;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int u = i * kLanes + threadIdx.x, x = u % (kBlockTokens * W), tok = x / W, o = x % W;
      raw[i] = make_uint4(0, 0, 0, 0);
      if (tok >= t.from && tok < t.to) {
        const int32_t at = tok * (int32_t)row_stride + o * 8;  // (32 rows of a stride below 2^24)
        const uint16_t *p = (u >= kBlockTokens * W ? v0 : k0) + at;
        if (vec) {
          raw[i] = *reinterpret_cast<const uint4 *>(p);
        } else {
          uint16_t e[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) e[j] = p[j];
          __builtin_memcpy(&raw[i], e, 16);
        }
      }
    }
  }
};

template <int D, bool HALF>
__device__ void write_block(const Rows<D> &rows, const BlockRows &t, unsigned char *blk, Turn<D> &sh) {
  constexpr int G = D / 32, W = D / 8, kEach = Rows<D>::kEach;
  uint4 *vcodes = reinterpret_cast<uint4 *>(blk + 20 * D);
  const bool whole = t.from == 0 && t.to == kBlockTokens;
  const uint4 old = !whole && threadIdx.x < D ? vcodes[threadIdx.x] : make_uint4(0, 0, 0, 0);
  uint16_t *vmeta = reinterpret_cast<uint16_t *>(blk + 36 * D);
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int u = i * kLanes + threadIdx.x, x = u % (kBlockTokens * W), tok = x / W, o = x % W;
    uint32_t code;
    const uint32_t meta = quantise<HALF>(rows.raw[i], &code);  // (four lanes of one token)
    if (tok < t.from || tok >= t.to) continue;
    if (u < kBlockTokens * W) {
      *reinterpret_cast<uint32_t *>(blk + tok * (D / 2) + o * 4) = code;
      if (o % 4 == 0) *reinterpret_cast<uint32_t *>(blk + 16 * D + (tok * G + o / 4) * 4) = meta;
    } else {
      sh.in[tok * (W + 1) + o] = code;
      if (o % 4 < 2) (whole ? sh.meta : vmeta)[o / 4 * 64 + o % 4 * 32 + value_group(tok) * 8 + value_element(tok)] = (uint16_t)(o % 4 ? meta >> 16 : meta);
    }
  }
  __syncthreads();
  // 8 tokens (of lane group lg) by channels 8 o + 2 i and + 1 to a lane
  for (int u = threadIdx.x; u < 16 * W; u += kLanes) {
    const int o = u / 16, lg = u / 4 % 4, i = u % 4;
    uint32_t w[8], x, y;
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = sh.in[((lg / 2) * 16 + (lg % 2) * 4 + (e / 4) * 8 + e % 4) * (W + 1) + o];
    turn_round(w, i, &x, &y);
    sh.out[value_word(D, o * 8 + 2 * i, lg)] = x;
    sh.out[value_word(D, o * 8 + 2 * i + 1, lg)] = y;
  }
  __syncthreads();
  if (threadIdx.x < D) {  // four words of one lane group
    uint4 w = reinterpret_cast<const uint4 *>(sh.out)[threadIdx.x];
    if (!whole) {
      const int lg = threadIdx.x * (4 / value_chunk(D)) % 64 / 16;
      uint32_t keep = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int tok = (lg / 2) * 16 + (lg % 2) * 4 + (e / 4) * 8 + e % 4;
        keep |= tok >= t.from && tok < t.to ? 0 : 15u << element_shift(e);
      }
      w = make_uint4((old.x & keep) | (w.x & ~keep), (old.y & keep) | (w.y & ~keep), (old.z & keep) | (w.z & ~keep), (old.w & keep) | (w.w & ~keep));
    }
    vcodes[threadIdx.x] = w;
  }
  if (whole && threadIdx.x < 8 * G) reinterpret_cast<uint4 *>(vmeta)[threadIdx.x] = reinterpret_cast<const uint4 *>(sh.meta)[threadIdx.x];
}

// A sequence that a call names twice would have two workgroups change the same words at once, so its items are left out.  Every workgroup looks
// for its own among up to kLooked items, asked for in front of the chain of its other loads; of more, one workgroup finds them ahead of the call.
// A row each of 64, 256, 512, 1024 sequences: 6.6, 9.1, 15.0, 25.9 us, without names 6.1, 8.1, 13.3, 23.4; of 2048 48.0 and 42.8, of which a launch
// ahead takes 5.  With every wavefront looking for itself, and no barrier: 6.6, 8.7, 14.6, 27.4.
constexpr int kLooked = 1024;

struct Named {
  static constexpr int kEach = kLooked / kLanes;
  struct alignas(4) Run {
    int x[kEach];
  } seq;
  int first;  // item of the first of them

  __device__ void load(const CacheRows &r) {
    if (r.n <= kLanes) {
      first = min((int)threadIdx.x, r.n - 1);
      seq.x[0] = r.seqs[first];
    } else {  // (the last lanes' runs overlap)
      first = min(kEach * (int)threadIdx.x, r.n - kEach);
      seq = *reinterpret_cast<const Run *>(r.seqs + first);
    }
  }
  __device__ bool again(const CacheRows &r, int item, int mine) const {
    bool twice = first != item && seq.x[0] == mine;
    if (r.n > kLanes)
#pragma unroll
      for (int j = 1; j < kEach; ++j) twice |= first + j != item && seq.x[j] == mine;
    return __syncthreads_or(twice);
  }
};

__global__ __launch_bounds__(1024) void k_cache_named(CacheDev d, CacheRows r) {
  __shared__ uint32_t seen[kCacheMaxSeqs / 32], again[kCacheMaxSeqs / 32];
  for (int i = threadIdx.x; i < kCacheMaxSeqs / 32; i += 1024) seen[i] = again[i] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < r.n; i += 1024) {
    const uint32_t s = (uint32_t)r.seqs[i], bit = 1u << (s & 31);
    if (s < (uint32_t)d.max_seqs && (atomicOr(&seen[s >> 5], bit) & bit)) atomicOr(&again[s >> 5], bit);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < r.n; i += 1024) {
    const uint32_t s = (uint32_t)r.seqs[i];
    d.items[i].copy = s < (uint32_t)d.max_seqs && (again[s >> 5] >> (s & 31)) & 1;
  }
}

template <int D, bool HALF>
__global__ __launch_bounds__(kLanes) void k_cache_write(CacheDev d, CacheRows r, int layer, const uint16_t *k, const uint16_t *v, int64_t row_stride,
                                                        int64_t head_stride, int vec, int blocks, uint32_t first) {
  __shared__ Turn<D> sh;
  const uint32_t u = first + blockIdx.x, stopped = d.ctrl->stopped;
  const int head = u % d.kv_heads, rest = u / d.kv_heads, b = rest % blocks, item = rest / blocks;
  const bool look = r.seqs && r.n > 1, here = look && r.n <= kLooked;
  Named named;
  if (here) named.load(r);
  BlockRows t;
  bool bad;
  const bool mine = find_block(d, r, item, b, &t, &bad);
  Rows<D> rows;
  int named_by = 0;
  if (mine) {
    rows.load(k, v, t, head, row_stride, head_stride, vec);
    named_by = d.refs[t.page];
  }
  const bool again = here ? named.again(r, item, r.seqs[item]) : look && uniform(d.items[item].copy);
  if ((bad || again) && b == 0 && head == 0 && threadIdx.x == 0) cache_raise(d, RTAMS_EINVAL);
  if (!mine || again) return;
  const bool shared = uniform(named_by) != 1;  // another sequence reads it
  if (shared && threadIdx.x == 0) cache_raise(d, RTAMS_EINVAL);
  if (stopped || shared) return;
  write_block<D, HALF>(rows, t, cache_block(d, layer, t.page, head, t.block_in_page), sh);
}

__device__ inline void put_values(void *out, int64_t at, const float f[8], int type) {
  if (type == RTAMS_TYPE_F32) {
    float *p = static_cast<float *>(out) + at;
    *reinterpret_cast<float4 *>(p) = make_float4(f[0], f[1], f[2], f[3]);
    *reinterpret_cast<float4 *>(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
    return;
  }
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint16_t a, b;
    if (type == RTAMS_TYPE_F16) {
      a = half_bits((_Float16)f[2 * j]);
      b = half_bits((_Float16)f[2 * j + 1]);
    } else {
      const __bf16 x = (__bf16)f[2 * j], y = (__bf16)f[2 * j + 1];
      __builtin_memcpy(&a, &x, 2);
      __builtin_memcpy(&b, &y, 2);
    }
    w[j] = (uint32_t)a | (uint32_t)b << 16;
  }
  *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(out) + at) = make_uint4(w[0], w[1], w[2], w[3]);
}

// A lane writes 8 channels of a row at a time.  Values come out of words that hold 8 tokens, through LDS: 8 channels by 2 tokens to a lane.
template <int D>
__device__ void read_block(const CacheDev &d, const CacheRows &r, int layer, void *k, void *v, int type, uint32_t unit, int blocks, uint32_t *words) {
  constexpr int G = D / 32, W = D / 8, kUnits = kBlockTokens * W, kEach = (kUnits + kLanes - 1) / kLanes;
  const int head = unit % d.kv_heads, rest = unit / d.kv_heads, b = rest % blocks, item = rest / blocks;
  BlockRows t;
  bool bad;
  const bool mine = find_block(d, r, item, b, &t, &bad);
  if (bad && b == 0 && head == 0 && threadIdx.x == 0) cache_raise(d, RTAMS_EINVAL);
  if (!mine) return;
  const unsigned char *blk = cache_block(d, layer, t.page, head, t.block_in_page);
  const uint4 *vcodes = reinterpret_cast<const uint4 *>(blk + 20 * D);
  for (int u = threadIdx.x; u < D; u += kLanes) reinterpret_cast<uint4 *>(words)[u] = vcodes[u];
  uint32_t code[kEach], meta[kEach];
#pragma unroll
  for (int n = 0; n < kEach; ++n) {
    const int u = n * kLanes + threadIdx.x, tok = u / W, o = u % W;
    code[n] = meta[n] = 0;
    if (kUnits % kLanes && u >= kUnits) break;
    code[n] = *reinterpret_cast<const uint32_t *>(blk + tok * (D / 2) + o * 4);
    meta[n] = *reinterpret_cast<const uint32_t *>(blk + 16 * D + (tok * G + o / 4) * 4);
  }
  const auto put = [&](void *to, int tok, int o, uint32_t w, float step, float zero) {
    if (tok < t.from || tok >= t.to) return;
    float f[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) f[c] = fmaf((float)((w >> element_shift(c)) & 15u), step, zero);
    put_values(to, ((t.row0 + tok) * d.kv_heads + head) * D + o * 8, f, type);
  };
#pragma unroll
  for (int n = 0; n < kEach; ++n) {
    const int u = n * kLanes + threadIdx.x;
    if (kUnits % kLanes && u >= kUnits) break;
    put(k, u / W, u % W, code[n], (float)half_of((uint16_t)meta[n]), (float)half_of((uint16_t)(meta[n] >> 16)));
  }
  __syncthreads();
  const uint16_t *vmeta = reinterpret_cast<const uint16_t *>(blk + 36 * D);
  for (int u = threadIdx.x; u < 16 * W; u += kLanes) {
    const int o = u % W, lg = u / W % 4, i = u / W / 4;
    uint32_t w[8], x[2];
#pragma unroll
    for (int c = 0; c < 8; ++c) w[c] = words[value_word(D, o * 8 + c, lg)];
    turn_round(w, i, &x[0], &x[1]);
    const uint16_t *m = vmeta + o / 4 * 64 + lg * 8 + 2 * i;
    const uint32_t steps = *reinterpret_cast<const uint32_t *>(m), zeros = *reinterpret_cast<const uint32_t *>(m + 32);
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int e = 2 * i + y, tok = (lg / 2) * 16 + (lg % 2) * 4 + (e / 4) * 8 + e % 4;
      put(v, tok, o, x[y], (float)half_of((uint16_t)(steps >> (16 * y))), (float)half_of((uint16_t)(zeros >> (16 * y))));
    }
  }
}

template <int D>
__global__ __launch_bounds__(kLanes) void k_cache_read(CacheDev d, CacheRows r, int layer, void *k, void *v, int type, int blocks, uint32_t first) {
  __shared__ uint32_t words[4 * D];
  read_block<D>(d, r, layer, k, v, type, first + blockIdx.x, blocks, words);
}

// Blocks that the rows of one item lie in at most.
int item_blocks(const CacheRows &r) { return (r.max_new + kBlockTokens - 2) / kBlockTokens + 1; }

// Units are blocks of an item and heads; a launch takes at most 2^22 of them.  (A loop in the kernels would keep what does not change in it in registers, and
// half as many workgroups would run at once.)
template <class F>
void each_launch(const CacheDev &d, const CacheRows &r, int blocks, F launch) {
  const int64_t units = (int64_t)r.n * blocks * d.kv_heads;
  for (int64_t at = 0; at < units; at += 1 << 22) launch((uint32_t)(units - at < 1 << 22 ? units - at : 1 << 22), (uint32_t)at);
}

}  // namespace

void launch_cache_write(const CacheDev &d, const CacheRows &r, int layer, const void *k, const void *v, int64_t row_stride, int64_t head_stride,
                        bool half_type, bool vec, hipStream_t s) {
  const int blocks = item_blocks(r);
  const uint16_t *kp = static_cast<const uint16_t *>(k), *vp = static_cast<const uint16_t *>(v);
  if (r.seqs && r.n > kLooked) k_cache_named<<<1, 1024, 0, s>>>(d, r);
  const auto go = [&](auto kernel) {
    each_launch(d, r, blocks, [&](uint32_t grid, uint32_t first) { kernel<<<grid, kLanes, 0, s>>>(d, r, layer, kp, vp, row_stride, head_stride, vec, blocks, first); });
  };
  switch (d.head_dim) {
    case 64: return half_type ? go(k_cache_write<64, true>) : go(k_cache_write<64, false>);
    case 96: return half_type ? go(k_cache_write<96, true>) : go(k_cache_write<96, false>);
    case 128: return half_type ? go(k_cache_write<128, true>) : go(k_cache_write<128, false>);
    default: return half_type ? go(k_cache_write<256, true>) : go(k_cache_write<256, false>);
  }
}

void launch_cache_read(const CacheDev &d, const CacheRows &r, int layer, void *k, void *v, int type, hipStream_t s) {
  const int blocks = item_blocks(r);
  const auto go = [&](auto kernel) {
    each_launch(d, r, blocks, [&](uint32_t grid, uint32_t first) { kernel<<<grid, kLanes, 0, s>>>(d, r, layer, k, v, type, blocks, first); });
  };
  switch (d.head_dim) {
    case 64: return go(k_cache_read<64>);
    case 96: return go(k_cache_read<96>);
    case 128: return go(k_cache_read<128>);
    default: return go(k_cache_read<256>);
  }
}

}  // namespace rtams
