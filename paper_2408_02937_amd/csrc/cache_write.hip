// Writing keys and values into the cache in 4 bits and reading them back (the format: include/rtams_cache.h).
//
// A workgroup owns 32 tokens of one head: half its lanes quantise keys, half values, a lane a group of 32 channels of one token, so that
// least and largest need no other lane.  A word of value codes holds 8 tokens of a channel: the tokens' words meet in LDS, where a lane takes 8 tokens
// by 8 channels and turns them round; tokens already there keep their bits.  Both directions are bound by memory: 4 bytes a channel on the
// side of the rows, 1.25 on that of the cache.
#include "../../include/rtams_cache.h"

#include "cache.h"

namespace rtams {

namespace {

constexpr int kLanes = 256;

__device__ inline float from_bits(uint16_t x, bool half_type) {
  if (!half_type) return __uint_as_float((uint32_t)x << 16);
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

// Step, zero and the codes of 32 channels (word w: channels 8 w .. 8 w + 7).
__device__ inline uint32_t quantise(const uint16_t *p, bool half_type, bool vec, uint32_t code[4]) {
  uint16_t raw[32];
  if (vec) {
    uint4 x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = reinterpret_cast<const uint4 *>(p)[j];
    __builtin_memcpy(raw, x, 64);
  } else {
#pragma unroll
    for (int j = 0; j < 32; ++j) raw[j] = p[j];
  }
  float f[32], lo, hi;
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    const float x = from_bits(raw[j], half_type);
    f[j] = x != x ? 0.0f : fminf(fmaxf(x, -kCacheMost), kCacheMost);
    lo = j ? fminf(lo, f[j]) : f[0];
    hi = j ? fmaxf(hi, f[j]) : f[0];
  }
  const _Float16 step = (_Float16)((hi - lo) / 15.0f), zero = (_Float16)lo;
  const float z = (float)zero, inv = (float)step > 0.0f ? 1.0f / (float)step : 0.0f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    uint32_t bits = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float c = fminf(fmaxf(rintf(__fmul_rn(f[8 * w + e] - z, inv)), 0.0f), 15.0f);
      bits |= (uint32_t)c << element_shift(e);
    }
    code[w] = bits;
  }
  return (uint32_t)half_bits(step) | (uint32_t)half_bits(zero) << 16;
}

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
  const int seq = cache_item_seq(r, item);
  *bad = !cache_item_rows(r, item, &first, &count) || (uint32_t)seq >= (uint32_t)d.max_seqs || count > d.lengths[(uint32_t)seq < (uint32_t)d.max_seqs ? seq : 0];
  if (*bad) return false;
  const int length = d.lengths[seq], start = length - count;
  const int block = start / kBlockTokens + b;
  if (count == 0 || block * kBlockTokens >= length) return false;
  out->from = start > block * kBlockTokens ? start - block * kBlockTokens : 0;
  out->to = length - block * kBlockTokens < kBlockTokens ? length - block * kBlockTokens : kBlockTokens;
  out->row0 = first + (int64_t)block * kBlockTokens - start;
  const uint32_t p = cache_page_of(d, (uint32_t)block);
  out->page = d.table[(int64_t)seq * d.max_pages + p];
  out->block_in_page = (uint32_t)block - p * d.page_blocks;
  return true;
}

template <int D>
__device__ void write_block(const CacheDev &d, const CacheRows &r, int layer, const uint16_t *k, const uint16_t *v, int64_t row_stride, int64_t head_stride,
                            int half_type, int vec, uint32_t unit, int blocks, uint32_t *words) {
  constexpr int G = D / 32, W = D / 8;
  const int head = unit % d.kv_heads, rest = unit / d.kv_heads, b = rest % blocks, item = rest / blocks;
  BlockRows t;
  bool bad;
  const bool mine = find_block(d, r, item, b, &t, &bad);
  if (bad && b == 0 && head == 0 && threadIdx.x == 0) cache_raise(d, RTAMS_EINVAL);
  if (!mine) return;
  if (d.refs[t.page] != 1) {  // another sequence reads it
    if (threadIdx.x == 0) cache_raise(d, RTAMS_EINVAL);
    return;
  }
  unsigned char *blk = cache_block(d, layer, t.page, head, t.block_in_page);
  uint16_t *vmeta = reinterpret_cast<uint16_t *>(blk + 36 * D);
  // (row0 may lie before the call's rows: only tokens of the call are addressed)
  for (int u = threadIdx.x; u < 2 * kBlockTokens * G; u += kLanes) {
    const bool value = u >= kBlockTokens * G;
    const int x = value ? u - kBlockTokens * G : u, tok = x / G, g = x % G;
    if (tok < t.from || tok >= t.to) continue;
    const uint16_t *p = (value ? v : k) + (t.row0 + tok) * row_stride + head * head_stride + g * 32;
    uint32_t code[4];
    const uint32_t meta = quantise(p, half_type, vec, code);
    if (!value) {
      *reinterpret_cast<uint4 *>(blk + tok * (D / 2) + g * 16) = make_uint4(code[0], code[1], code[2], code[3]);
      *reinterpret_cast<uint32_t *>(blk + 16 * D + (tok * G + g) * 4) = meta;
    } else {
#pragma unroll
      for (int w = 0; w < 4; ++w) words[tok * (W + 1) + g * 4 + w] = code[w];
      uint16_t *m = vmeta + g * 64 + value_group(tok) * 8 + value_element(tok);
      m[0] = (uint16_t)meta;
      m[32] = (uint16_t)(meta >> 16);
    }
  }
  __syncthreads();
  // 8 tokens (of lane group lg) by 8 channels (of octet o) to a lane: a word of each channel
  uint32_t *vcodes = reinterpret_cast<uint32_t *>(blk + 20 * D);
  for (int u = threadIdx.x; u < 4 * W; u += kLanes) {
    const int lg = u % 4, o = u / 4;
    uint32_t out[8] = {0, 0, 0, 0, 0, 0, 0, 0}, keep = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int tok = (lg / 2) * 16 + (lg % 2) * 4 + (e / 4) * 8 + e % 4;
      if (tok < t.from || tok >= t.to) {
        keep |= 15u << element_shift(e);
        continue;
      }
      const uint32_t w = words[tok * (W + 1) + o];
#pragma unroll
      for (int c = 0; c < 8; ++c) out[c] |= ((w >> element_shift(c)) & 15u) << element_shift(e);
    }
    if (keep == ~0u) continue;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      uint32_t *at = vcodes + value_word(D, o * 8 + c, lg);
      *at = keep ? (*at & keep) | out[c] : out[c];
    }
  }
}

template <int D>
__global__ __launch_bounds__(kLanes) void k_cache_write(CacheDev d, CacheRows r, int layer, const uint16_t *k, const uint16_t *v, int64_t row_stride,
                                                        int64_t head_stride, int half_type, int vec, int blocks) {
  __shared__ uint32_t words[kBlockTokens * (D / 8 + 1)];
  if (d.ctrl->stopped) return;
  for (uint32_t u = blockIdx.x; u < (uint32_t)r.n * blocks * d.kv_heads; u += gridDim.x) {
    write_block<D>(d, r, layer, k, v, row_stride, head_stride, half_type, vec, u, blocks, words);
    __syncthreads();
  }
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

// A lane writes 8 channels of a row; values come out of words that hold 8 tokens, through LDS.
template <int D>
__device__ void read_block(const CacheDev &d, const CacheRows &r, int layer, void *k, void *v, int type, uint32_t unit, int blocks, uint32_t *words) {
  constexpr int G = D / 32, W = D / 8;
  const int head = unit % d.kv_heads, rest = unit / d.kv_heads, b = rest % blocks, item = rest / blocks;
  BlockRows t;
  bool bad;
  const bool mine = find_block(d, r, item, b, &t, &bad);
  if (bad && b == 0 && head == 0 && threadIdx.x == 0) cache_raise(d, RTAMS_EINVAL);
  if (!mine) return;
  const unsigned char *blk = cache_block(d, layer, t.page, head, t.block_in_page);
  const uint32_t *vcodes = reinterpret_cast<const uint32_t *>(blk + 20 * D);
  for (int u = threadIdx.x; u < D; u += kLanes) reinterpret_cast<uint4 *>(words)[u] = reinterpret_cast<const uint4 *>(vcodes)[u];
  __syncthreads();
  const uint16_t *vmeta = reinterpret_cast<const uint16_t *>(blk + 36 * D);
  for (int u = threadIdx.x; u < 2 * kBlockTokens * W; u += kLanes) {
    const bool value = u >= kBlockTokens * W;
    const int x = value ? u - kBlockTokens * W : u, tok = x / W, o = x % W, g = o / 4;
    if (tok < t.from || tok >= t.to) continue;
    uint32_t w = 0;
    float step, zero;
    if (!value) {
      w = *reinterpret_cast<const uint32_t *>(blk + tok * (D / 2) + o * 4);
      const uint32_t meta = *reinterpret_cast<const uint32_t *>(blk + 16 * D + (tok * G + g) * 4);
      step = (float)half_of((uint16_t)meta);
      zero = (float)half_of((uint16_t)(meta >> 16));
    } else {
      const int lg = value_group(tok), sh = element_shift(value_element(tok));
#pragma unroll
      for (int c = 0; c < 8; ++c) w |= ((words[value_word(D, o * 8 + c, lg)] >> sh) & 15u) << element_shift(c);
      const uint16_t *m = vmeta + g * 64 + lg * 8 + value_element(tok);
      step = (float)half_of(m[0]);
      zero = (float)half_of(m[32]);
    }
    float f[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) f[c] = fmaf((float)((w >> element_shift(c)) & 15u), step, zero);
    put_values(value ? v : k, ((t.row0 + tok) * d.kv_heads + head) * D + o * 8, f, type);
  }
}

template <int D>
__global__ __launch_bounds__(kLanes) void k_cache_read(CacheDev d, CacheRows r, int layer, void *k, void *v, int type, int blocks) {
  __shared__ uint32_t words[4 * D];
  for (uint32_t u = blockIdx.x; u < (uint32_t)r.n * blocks * d.kv_heads; u += gridDim.x) {
    read_block<D>(d, r, layer, k, v, type, u, blocks, words);
    __syncthreads();
  }
}

// Blocks that the rows of one item lie in at most.
int item_blocks(const CacheRows &r) { return (r.max_new + kBlockTokens - 2) / kBlockTokens + 1; }

uint32_t groups_for(const CacheDev &d, const CacheRows &r, int blocks) {
  const int64_t units = (int64_t)r.n * blocks * d.kv_heads;
  return (uint32_t)(units < (1 << 20) ? units : 1 << 20);
}

}  // namespace

void launch_cache_write(const CacheDev &d, const CacheRows &r, int layer, const void *k, const void *v, int64_t row_stride, int64_t head_stride,
                        bool half_type, bool vec, hipStream_t s) {
  const int blocks = item_blocks(r);
  const uint32_t grid = groups_for(d, r, blocks);
  const uint16_t *kp = static_cast<const uint16_t *>(k), *vp = static_cast<const uint16_t *>(v);
  auto go = [&](auto kernel) { kernel<<<grid, kLanes, 0, s>>>(d, r, layer, kp, vp, row_stride, head_stride, half_type, vec, blocks); };
  switch (d.head_dim) {
    case 64: return go(k_cache_write<64>);
    case 96: return go(k_cache_write<96>);
    case 128: return go(k_cache_write<128>);
    default: return go(k_cache_write<256>);
  }
}

void launch_cache_read(const CacheDev &d, const CacheRows &r, int layer, void *k, void *v, int type, hipStream_t s) {
  const int blocks = item_blocks(r);
  const uint32_t grid = groups_for(d, r, blocks);
  auto go = [&](auto kernel) { kernel<<<grid, kLanes, 0, s>>>(d, r, layer, k, v, type, blocks); };
  switch (d.head_dim) {
    case 64: return go(k_cache_read<64>);
    case 96: return go(k_cache_read<96>);
    case 128: return go(k_cache_read<128>);
    default: return go(k_cache_read<256>);
  }
}

}  // namespace rtams
