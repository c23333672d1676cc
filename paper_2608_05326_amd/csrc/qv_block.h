// Device helpers of the 8-bit block cache's kernels: scale and codes of a block (decided
// exactly), closing a block into its page, pages of a table.
#pragma once
#include "qv_device.h"

namespace qv {

constexpr int kBlk = kBlockTokens;
constexpr int kCodes = kBlk * kHeadDim;      // codes of a page's keys (or values), one KV head
constexpr float kMinScale = 0x1p-100f;
constexpr int kThreads = 256;

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

__device__ __forceinline__ float lo_f32(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float hi_f32(uint32_t x) { return __uint_as_float(x & 0xFFFF0000u); }

// A store of rows or codes that no one reads soon, past the caches: with ordinary stores
// two 64K sequences are fetched in 167 us, with these in 120, two 32K prompts stored in 94
// and 81 (805 and 403 MB).
template <class T>
__device__ __forceinline__ void put(T x, void* p) {
  __builtin_nontemporal_store(x, (T*)p);
}
// 16 bytes of codes; PAST: past the caches
template <bool PAST>
__device__ __forceinline__ u32x4 get(const int8_t* p) {
  if constexpr (PAST) return __builtin_nontemporal_load((const u32x4*)p);
  else return *(const u32x4*)p;
}

// Scale of a block whose largest magnitude is amax (bits of a non-negative float, NaN and
// infinity above all others): NaN when amax is not finite.
__device__ __forceinline__ float block_scale(uint32_t amax) {
  if (amax >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
  return fmaxf(__fdiv_rn(__uint_as_float(amax), 127.f), kMinScale);
}

// round-half-even(x / s) for finite x.  The product with the rounded reciprocal is within
// 2^-15 of x / s, so its nearest integer c is right or off by one.  The rest r = x - c s is
// exact: c s and x are multiples of the last place of s (a smaller x has c = 0 and r = x)
// and |r| <= s.  c moves towards r where |r| > s / 2, and an odd c where |r| = s / 2: at
// s / 2 or at the float after it, compared as integers.  inv = 1 / s (s >= 2^-100: no
// overflow), half = the bits of s / 2.
__device__ __forceinline__ uint32_t code_byte(float x, float s, float inv, uint32_t half) {
  const float c = rintf(x * inv), r = fmaf(-c, s, x);
  const int ci = (int)c;
  const uint32_t rb = __float_as_uint(r), from = half + (~ci & 1);
  return (uint32_t)(ci + ((rb & 0x7FFFFFFFu) >= from ? (int)rb >> 31 | 1 : 0)) & 0xFFu;
}

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
// bf16 magnitudes as integers (NaN and infinity above all others), two at once
__device__ __forceinline__ uint32_t amax_pair(u32x4 x, uint32_t m) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
    m = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, m),
                                                              __builtin_bit_cast(u16x2, x[j] & 0x7FFF7FFFu)));
  return m;
}
__device__ __forceinline__ uint32_t amax_bits(uint32_t pair) { return max(pair << 16, pair & 0xFFFF0000u); }

// Quantizes the keys (VALUES: the values) of one complete block of one KV head into its
// page (all 256 threads): thread (m, c) = (tid / 16, tid % 16) holds channels 8 c .. + 7 of
// tokens 4 m .. + 3.
struct CloseLds {
  uint32_t amax[kThreads / 64];
  uint32_t vt[kHeadDim][kBlk / 4 + 1];   // value codes, four tokens a word (keys: not used)
};
template <bool VALUES>
__device__ __forceinline__ void close_rows(const u32x4 (&x)[4], int8_t* codes, float* scale, CloseLds& sm) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int c = tid & 15, m = tid >> 4;   // 8-channel chunk, group of four tokens
  uint32_t am = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) am = amax_pair(x[i], am);
  am = amax_bits(am);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) am = max(am, (uint32_t)__shfl_xor((int)am, d, 64));
  if (lane == 0) sm.amax[wave] = am;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) am = max(am, sm.amax[w]);
  const float s = block_scale(am), inv = 1.f / s;
  const uint32_t half = __float_as_uint(0.5f * s);
  const bool finite = s == s;
  if (tid == 0) *scale = s;
  if constexpr (!VALUES) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t w[2] = {0, 0};
      if (finite) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          w[j >> 1] |= code_byte(lo_f32(x[i][j]), s, inv, half) << (16 * (j & 1));
          w[j >> 1] |= code_byte(hi_f32(x[i][j]), s, inv, half) << (16 * (j & 1) + 8);
        }
      }
      put((u32x2){w[0], w[1]}, codes + (4 * m + i) * kHeadDim + 8 * c);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t w = 0;
      if (finite) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t y = x[i][j >> 1];
          w |= code_byte(j & 1 ? hi_f32(y) : lo_f32(y), s, inv, half) << (8 * i);
        }
      }
      sm.vt[8 * c + j][m] = w;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {   // 16 bytes a thread: channel e / 4, tokens 16 (e % 4) ..
      const int e = tid + kThreads * i;
      u32x4 y;
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] = sm.vt[e >> 2][4 * (e & 3) + j];
      put(y, codes + 16 * e);
    }
  }
}

// The same of rows in memory: row(t) is the address of token t's channels.
template <bool VALUES, class Row>
__device__ __forceinline__ void close_block(Row row, int8_t* codes, float* scale, CloseLds& sm) {
  const int c = threadIdx.x & 15, m = threadIdx.x >> 4;
  u32x4 x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = *(const u32x4*)(row(4 * m + i) + 8 * c);
  close_rows<VALUES>(x, codes, scale, sm);
}

// Page of a sequence's block; -1 when the table holds none (dropped, or out of range).
__device__ __forceinline__ int page_of(const BlockArgs& a, int seq, int blk) {
  if (blk >= a.n_cols) return -1;
  const int p = a.table[(int64_t)seq * a.n_cols + blk];
  return (uint32_t)p < (uint32_t)a.n_pages ? p : -1;
}

}  // namespace qv
