// The 8-bit block cache: sequences that keep every token (nothing is ranked or evicted),
// at half the bytes of bf16.  Tokens are grouped in blocks of 64; a complete block of one
// KV head is a page entry of int8 codes with one fp32 scale for its keys and one for its
// values, the open block of a sequence stays in bf16 (its tail).  A block is quantized
// once, when its last token arrives (Sec. 4.3, write-once codes):
//   s = max(fl32(max|x| / 127), 2^-100),   c = round-half-even(x / s), decided exactly,
// so |x - s c| <= s / 2.  A block with a value that is not finite gets the scale NaN (all
// its values read as NaN).
//
//   k_block_store   packed prompts -> pages and tails
//   k_block_fetch   pages and tails -> packed bf16 rows
//   k_block_attend, k_block_merge  one decode token per sequence: append, attend, close a
//                   full block
//
// Page layout, one KV head: keys [64][128] (a token's channels together), values [128][64]
// (a channel's tokens together): each is the order in which the matrix instruction of its
// product reads it, 16 bytes a lane.
#include "qv_device.h"
#include "qv_parts.h"

namespace qv {

namespace {
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
// page (all 256 threads).  row(t) is the address of token t's channels.
struct CloseLds {
  uint32_t vt[kHeadDim][kBlk / 4 + 1];   // value codes, four tokens a word
  uint32_t amax[kThreads / 64];
};
template <bool VALUES, class Row>
__device__ __forceinline__ void close_block(Row row, int8_t* codes, float* scale, CloseLds& sm) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int c = tid & 15, m = tid >> 4;   // 8-channel chunk, group of four tokens
  u32x4 x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = *(const u32x4*)(row(4 * m + i) + 8 * c);
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

// Page of a sequence's block; -1 when the table holds none (dropped, or out of range).
__device__ __forceinline__ int page_of(const BlockArgs& a, int seq, int blk) {
  if (blk >= a.n_cols) return -1;
  const int p = a.table[(int64_t)seq * a.n_cols + blk];
  return (uint32_t)p < (uint32_t)a.n_pages ? p : -1;
}
}  // namespace

// Packed prompts into the cache, one workgroup per (block, KV head, keys or values).
__global__ __launch_bounds__(kThreads) void k_block_store(BlockArgs a, PackedRows r) {
  __shared__ CloseLds sm;
  const bool values = blockIdx.x & 1;
  const int g = (blockIdx.x >> 1) % a.H_kv;
  PackedTile w;
  if (!find_tile(r.cu, a.B, r.total, 1, kBlk, (blockIdx.x >> 1) / a.H_kv, &w)) return;
  const int t0 = w.tile * kBlk, n = min(kBlk, min(w.len, a.max_context) - t0);
  if (n <= 0) return;
  const int64_t st = values ? r.v_st : r.k_st;
  const uint16_t* x = (values ? r.v + g * r.v_sh : r.k + g * r.k_sh) + (int64_t)(w.start + t0) * st;
  if (n == kBlk) {
    const int page = page_of(a, w.seq, w.tile);
    if (page < 0) return;
    const int64_t e = (int64_t)page * a.H_kv + g;
    auto row = [&](int t) { return x + t * st; };
    if (values) close_block<true>(row, a.v_codes + e * kCodes, a.v_scale + e, sm);
    else close_block<false>(row, a.k_codes + e * kCodes, a.k_scale + e, sm);
    return;
  }
  uint16_t* tail = (values ? a.v_tail : a.k_tail) + ((int64_t)w.seq * a.H_kv + g) * kCodes;
  for (int e = threadIdx.x; e < n * 16; e += kThreads)
    *(u32x4*)(tail + 8 * e) = *(const u32x4*)(x + (e >> 4) * st + 8 * (e & 15));
}

// The cache back into packed bf16 rows: a token of a complete block is bf16(fl32(c s)), a
// token of a block without a page is zero, a token of the tail is copied.  Rows past a
// sequence's length are not written.
__global__ __launch_bounds__(kThreads) void k_block_fetch(BlockArgs a, PackedRows r) {
  __shared__ uint32_t vt[kHeadDim][kBlk / 4 + 1];
  const int g = blockIdx.x % a.H_kv, tid = threadIdx.x;
  PackedTile w;
  if (!find_tile(r.cu, a.B, r.total, 1, kBlk, blockIdx.x / a.H_kv, &w)) return;
  const int held = max(min(a.lens[w.seq], a.max_context), 0);
  const int t0 = w.tile * kBlk, n = min(min(kBlk, w.len - t0), held - t0);
  if (n <= 0) return;
  uint16_t* k = r.k_out + (int64_t)(w.start + t0) * r.k_st + g * r.k_sh;
  uint16_t* v = r.v_out + (int64_t)(w.start + t0) * r.v_st + g * r.v_sh;
  if (w.tile >= held / kBlk) {
    const int64_t tail = ((int64_t)w.seq * a.H_kv + g) * kCodes;
    for (int e = tid; e < n * 16; e += kThreads) {
      const int t = e >> 4, c = 8 * (e & 15);
      *(u32x4*)(k + t * r.k_st + c) = *(const u32x4*)(a.k_tail + tail + t * kHeadDim + c);
      *(u32x4*)(v + t * r.v_st + c) = *(const u32x4*)(a.v_tail + tail + t * kHeadDim + c);
    }
    return;
  }
  const int page = page_of(a, w.seq, w.tile);
  const int64_t e0 = (int64_t)max(page, 0) * a.H_kv + g;
  const int c = tid & 15, m = tid >> 4;
  float sk = 0.f, sv = 0.f;
  u32x2 kc[4] = {};
  if (page >= 0) {
    sk = a.k_scale[e0];
    sv = a.v_scale[e0];
#pragma unroll
    for (int i = 0; i < 4; ++i) kc[i] = *(const u32x2*)(a.k_codes + e0 * kCodes + (4 * m + i) * kHeadDim + 8 * c);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int e = tid + kThreads * i;
      const u32x4 x = *(const u32x4*)(a.v_codes + e0 * kCodes + 16 * e);
#pragma unroll
      for (int j = 0; j < 4; ++j) vt[e >> 2][4 * (e & 3) + j] = x[j];
    }
  }
  __syncthreads();
  auto val = [](uint32_t word, int byte, float s) { return (float)(int8_t)(word >> (8 * byte)) * s; };
  auto pack = [](float lo, float hi) {
    const bf16x2 p = {(__bf16)lo, (__bf16)hi};
    return __builtin_bit_cast(uint32_t, p);
  };
  uint32_t vw[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) vw[j] = page >= 0 ? vt[8 * c + j][m] : 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int t = 4 * m + i;
    if (t >= n) break;
    u32x4 x, y;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[j] = pack(val(kc[i][j >> 1], 2 * (j & 1), sk), val(kc[i][j >> 1], 2 * (j & 1) + 1, sk));
      y[j] = pack(val(vw[2 * j], i, sv), val(vw[2 * j + 1], i, sv));
    }
    put(x, k + t * r.k_st + 8 * c);
    put(y, v + t * r.v_st + 8 * c);
  }
}

// ------------------------------------------------------------------ decode attention
// One token per sequence, in two launches.  In the first, one workgroup per (sequence, KV
// head) pair takes the open block, and a pair's complete blocks too if they are few; the
// blocks of all other pairs, in pair order, are cut into equal parts, one per further
// workgroup, whatever the lengths are (they are read on the device).  Such a workgroup goes
// through the pairs its part touches (segments); the four waves of a workgroup take a
// segment's blocks in turn and are joined in LDS.  A pair that one workgroup served is
// written out; the others leave (maximum, sum, output) rows that k_block_merge joins.
//
// A wave's products, by 16x16x32 MFMAs with the G query heads of the KV head as columns
// (padded to 16):
//   S^T = K q^T   (A = 16 keys; a lane holds 4 keys of ONE head per tile)
//   O^T = V^T P^T (A = 16 channels; the same lane owns 32 channels of that head)
// Row r of key tile tt is token 16 (r / 4) + 4 tt + r % 4 of the block, so that lane group
// qd holds the logits of tokens 16 qd .. + 15: the 16 codes that one 16-byte load of a
// value channel gives it.  Codes become fp16 integers (exact): byte + 128 placed below
// 0x64 is 1152 + c, minus 1152.  A head's query is scaled by a power of two into fp16, its
// largest entry to [2^14, 2^15): exact (bf16 has 8 bits) down to entries 2^-31 of that;
// smaller ones are off by at most 2^-39 of it.  P is rounded beside codes to fp16: by 2^-11
// of itself, below 2^-14 of the head's reference by 2^-25 of that; beside the open block's
// values to bf16 (2^-8 of itself).  The sum takes P unrounded; logits, maximum, sum and
// output are held in 32 bits, a block's value scale is applied to its products' fp32 sum.
//
// Bound by the pages' bytes: eight 8B sequences (401 MB) take 76 us, 32 ragged 70B places
// (985 MB) 189 us, 5.3 and 5.2 TB/s where a large copy reaches 5.2; one sequence of 32K
// (67 MB) 21 us, of which 3 go by before the first page is asked for and 5 in the join.
namespace {
constexpr float kLazyD = 8.f;

__device__ __forceinline__ f32x4 mfma_f16(f16x8 x, f16x8 y, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma_bf(u32x4 x, u32x4 y, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0,
                                                 0, 0);
}
// eight codes (two words) as fp16 integers
__device__ __forceinline__ f16x8 codes_f16(uint32_t w0, uint32_t w1) {
  const f16x2 bias = {(_Float16)1152.f, (_Float16)1152.f};
  union {
    f16x2 h[4];
    f16x8 v;
  } r;
  w0 ^= 0x80808080u;
  w1 ^= 0x80808080u;
  r.h[0] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w0, 0x04010400u)) - bias;
  r.h[1] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w0, 0x04030402u)) - bias;
  r.h[2] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w1, 0x04010400u)) - bias;
  r.h[3] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w1, 0x04030402u)) - bias;
  return r.v;
}

struct Running {     // of one head (column): reference maximum (log2 units), sum, output
  float m, l;
  f32x4 o[8];        // channel 16 ct + 4 qd + i
};

// Raises the reference to mt where a head exceeds it by more than 2^kLazyD (for all heads
// of the wave at once), and rescales.
__device__ __forceinline__ void raise(Running& st, float mt) {
  if (__any(mt > st.m + kLazyD)) {
    const float mn = fmaxf(st.m, mt);
    const float al = st.m == mn ? 1.f : __builtin_amdgcn_exp2f(st.m - mn);
    st.m = mn;
    st.l *= al;
#pragma unroll
    for (int ct = 0; ct < 8; ++ct)
#pragma unroll
      for (int i = 0; i < 4; ++i) st.o[ct][i] *= al;
  }
}

// inclusive sum over the wave's lanes: within rows of 16, then across them
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);   // from 1, 2, 4, 8 lanes below
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);   // last lane of rows 0, 2 to rows 1, 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);   // lane 31 to rows 2, 3
  return x;
}

// Page of block blk0 + 4 lane, -1 past `end` or without one.
__device__ __forceinline__ int lane_page(const BlockArgs& a, int b, int blk0, int end) {
  const int blk = blk0 + 4 * (threadIdx.x & 63);
  return blk < end ? page_of(a, b, blk) : -1;
}

// Length in place s0 + lane (-1 past the last).
__device__ __forceinline__ int lane_len(const BlockArgs& a, int s0) {
  const int s = s0 + (threadIdx.x & 63);
  return s < a.B ? a.lens[s] : -1;
}

// Items of the places past the first 64 (of one KV head), and those of them before `place`.
__device__ __forceinline__ int items_past_64(const BlockArgs& a, int place, int* before) {
  const int lane = threadIdx.x & 63;
  int sum = 0, pre = 0;
#pragma unroll 4
  for (int s0 = 64; s0 < a.B; s0 += 64) {
    const int n = items_of(lane_len(a, s0), a.max_context);
    sum += n;
    pre += s0 + lane < place ? n : 0;
  }
  *before = __builtin_amdgcn_readlane(wave_scan(pre), 63);
  return __builtin_amdgcn_readlane(wave_scan(sum), 63);
}

constexpr int kTailRow = 2 * kHeadDim;
constexpr int kJoinRow = kHeadDim + 4;
}  // namespace

template <bool PAST>
__global__ __launch_bounds__(kThreads, 2) void k_block_attend(BlockArgs a, BlockStep s) {
  __shared__ __attribute__((aligned(16))) uint8_t stail[kBlk * kTailRow];   // the open block's values
  __shared__ float sml[4][16][2];
  extern __shared__ __attribute__((aligned(16))) float so[];                // [4][gqa][kJoinRow]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, qd = lane >> 4;
  const int n_pairs = a.B * a.H_kv;

  // One segment: blocks [i0, i1) of pair (b, g), and the open block with n_tail > 0 tokens
  // (the new one included); `whole` when that is all of the pair.
  auto segment = [&](int b, int g, int i0, int i1, int n_tail, bool whole, int64_t slot) {
    const int hr = min(r, a.gqa - 1);   // columns past the last head repeat it
    const uint16_t* qp = s.q + ((int64_t)b * a.H_q + g * a.gqa + hr) * kHeadDim;
    Running st;
    st.m = -INFINITY;
    st.l = 0.f;
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) st.o[ct] = (f32x4){0.f, 0.f, 0.f, 0.f};

    if (16 * wave < n_tail) {
      // tokens 16 wave .. + 15 of the open block, in bf16 (16x16x16 MFMA for the values: a
      // lane's four logits are the four tokens it wants); the new token is the last, and
      // the wave that meets it stores it
      const int64_t tail = ((int64_t)b * a.H_kv + g) * kCodes;
      const uint16_t* kn = s.k_new + ((int64_t)b * a.H_kv + g) * kHeadDim;
      const uint16_t* vn = s.v_new + ((int64_t)b * a.H_kv + g) * kHeadDim;
      const int t0 = 16 * wave, last = n_tail - 1;
      u32x4 qw[4], kk[4], vv[4];
      const uint16_t* krow = t0 + r < last ? a.k_tail + tail + (t0 + r) * kHeadDim : kn;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        qw[i] = *(const u32x4*)(qp + 32 * i + 8 * qd);
        kk[i] = *(const u32x4*)(krow + 32 * i + 8 * qd);
        const int t = t0 + 4 * i + qd;
        vv[i] = *(const u32x4*)((t < last ? a.v_tail + tail + t * kHeadDim : vn) + 8 * r);
        if (t > last) vv[i] = (u32x4){0, 0, 0, 0};
      }
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        acc = mfma_bf(kk[i], qw[i], acc);
        *(u32x4*)(stail + (t0 + 4 * i + qd) * kTailRow + 16 * r) = vv[i];
        if (t0 + 4 * i + qd == last) *(u32x4*)(a.v_tail + tail + last * kHeadDim + 8 * r) = vv[i];
        if (t0 + r == last) *(u32x4*)(a.k_tail + tail + last * kHeadDim + 32 * i + 8 * qd) = kk[i];
      }
      float mt = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        acc[i] = t0 + 4 * qd + i <= last ? acc[i] * a.scale_log2 : -INFINITY;
        mt = fmaxf(mt, acc[i]);
      }
      st.m = rows_max(mt);
      const float mu = st.m > -INFINITY ? st.m : 0.f;
      s16x4 p;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = __builtin_amdgcn_exp2f(acc[i] - mu);
        st.l += x;
        p[i] = __builtin_bit_cast(short, (__bf16)x);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // this wave's rows are in LDS
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) {
        const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_s16x4*)(stail + (t0 + 4 * qd + (r >> 2)) * kTailRow + 32 * ct + 8 * (r & 3)));
        st.o[ct] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(x, p, st.o[ct], 0, 0, 0);
      }
    }

    if (i0 + wave < i1) {
      // pages and scales of the wave's next 64 blocks, one per lane (a dropped block's
      // tokens take no part), then the first one's keys: the query is read and scaled
      // while they are on their way
      int page = lane_page(a, b, i0 + wave, i1);
      u32x4 qw[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) qw[i] = *(const u32x4*)(qp + 64 * (i >> 1) + 16 * qd + 8 * (i & 1));
      const int row = (16 * (r >> 2) + (r & 3)) * kHeadDim + 16 * qd;   // + 4 tt rows
      u32x4 kb[8], vb[8];
      float ks_l, vs_l;
      uint64_t live;
      auto entry = [&](int j) { return ((int64_t)__builtin_amdgcn_readlane(page, j) * a.H_kv + g) * kCodes; };
      auto load_k = [&](int j) {
        const int8_t* kc = a.k_codes + entry(j) + row;
#pragma unroll
        for (int i = 0; i < 8; ++i) kb[i] = get<PAST>(kc + 4 * (i >> 1) * kHeadDim + 64 * (i & 1));
      };
      auto start = [&]() {
        live = __ballot(page >= 0);
        if (live) load_k(__builtin_ctzll(live));
        const int64_t e = (int64_t)max(page, 0) * a.H_kv + g;
        ks_l = vs_l = 0.f;
        if (page >= 0) {
          ks_l = a.k_scale[e];
          vs_l = a.v_scale[e];
        }
      };
      start();
      // query operand: k-step (p, e) covers channels 64 p + 16 qd + 8 e + j
      uint32_t am = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) am = amax_pair(qw[i], am);
      am = amax_bits(am);
      am = max(am, (uint32_t)__shfl_xor((int)am, 16, 64));
      am = max(am, (uint32_t)__shfl_xor((int)am, 32, 64));
      // 2^(14 - ex) for a largest magnitude in [2^ex, 2^(ex + 1))
      const int ex = (int)(am >> 23) - 127;
      f16x8 qf[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          qf[i][2 * j] = (_Float16)ldexpf(lo_f32(qw[i][j]), 14 - ex);
          qf[i][2 * j + 1] = (_Float16)ldexpf(hi_f32(qw[i][j]), 14 - ex);
        }
      // log2 units per (q' c s): scale_log2 2^(ex - 14) = qm 2^qe.  For small queries that is
      // below 2^-126, where it would lose bits, though logits need not be small (large keys):
      // the power of two is applied last, to qm times a block's scale (2^-100 or more).
      const float qm = __builtin_amdgcn_frexp_mantf(a.scale_log2);
      const int qe = __builtin_amdgcn_frexp_expf(a.scale_log2) + ex - 14;

      for (int blk0 = i0 + wave;;) {
        while (live) {
          const int j = __builtin_ctzll(live);
          live &= live - 1;
          const int8_t* vc = a.v_codes + entry(j) + r * kBlk + 16 * qd;
#pragma unroll
          for (int ct = 0; ct < 8; ++ct) vb[ct] = get<PAST>(vc + 16 * ct * kBlk);
          float sc = ldexpf(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ks_l), j)) * qm, qe);
          if (sc == INFINITY) sc = __FLT_MAX__;   // (a product of zero is a logit of zero)
          const float vs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vs_l), j));
          f32x4 acc[4];
#pragma unroll
          for (int tt = 0; tt < 4; ++tt) {
            acc[tt] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int p = 0; p < 2; ++p) {
              const u32x4 x = kb[2 * tt + p];
              acc[tt] = mfma_f16(codes_f16(x[0], x[1]), qf[2 * p], acc[tt]);
              acc[tt] = mfma_f16(codes_f16(x[2], x[3]), qf[2 * p + 1], acc[tt]);
            }
          }
          if (live) load_k(__builtin_ctzll(live));
          float mt = -INFINITY;
#pragma unroll
          for (int tt = 0; tt < 4; ++tt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              acc[tt][i] *= sc;
              mt = fmaxf(mt, acc[tt][i]);
            }
          raise(st, rows_max(mt));
          const float mu = st.m > -INFINITY ? st.m : 0.f;
          f16x8 p[2];
#pragma unroll
          for (int tt = 0; tt < 4; ++tt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float x = __builtin_amdgcn_exp2f(acc[tt][i] - mu);
              st.l += x;
              p[tt >> 1][4 * (tt & 1) + i] = (_Float16)x;
            }
#pragma unroll
          for (int ct = 0; ct < 8; ++ct) {
            const u32x4 x = vb[ct];
            f32x4 y = {0.f, 0.f, 0.f, 0.f};
            y = mfma_f16(codes_f16(x[0], x[1]), p[0], y);
            y = mfma_f16(codes_f16(x[2], x[3]), p[1], y);
#pragma unroll
            for (int i = 0; i < 4; ++i) st.o[ct][i] = fmaf(y[i], vs, st.o[ct][i]);
          }
        }
        blk0 += 256;
        if (blk0 >= i1) break;
        page = lane_page(a, b, blk0, i1);
        start();
      }
    }

    // ---- join the four waves
    const float l = rows_sum(st.l);
    if (r < a.gqa) {
      if (qd == 0) {
        sml[wave][r][0] = st.m;
        sml[wave][r][1] = l;
      }
      float* row = so + (wave * a.gqa + r) * kJoinRow + 4 * qd;
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) *(f32x4*)(row + 16 * ct) = st.o[ct];
    }
    __syncthreads();
    for (int e = tid; e < a.gqa * (kHeadDim / 4); e += kThreads) {
      const int h = e / (kHeadDim / 4), c = 4 * (e % (kHeadDim / 4));
      float M = -INFINITY;
#pragma unroll
      for (int v = 0; v < 4; ++v) M = fmaxf(M, sml[v][h][0]);
      const float mu = M > -INFINITY ? M : 0.f;
      float L = 0.f;
      f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const float f = __builtin_amdgcn_exp2f(sml[v][h][0] - mu);
        L = fmaf(f, sml[v][h][1], L);
        const f32x4 y = *(const f32x4*)(so + (v * a.gqa + h) * kJoinRow + c);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = fmaf(f, y[i], x[i]);
      }
      if (whole) {
        const bf16x2 v0 = {(__bf16)(x[0] / L), (__bf16)(x[1] / L)}, v1 = {(__bf16)(x[2] / L), (__bf16)(x[3] / L)};
        *(u32x2*)(s.out + ((int64_t)b * a.H_q + g * a.gqa + h) * kHeadDim + c) =
            (u32x2){__builtin_bit_cast(uint32_t, v0), __builtin_bit_cast(uint32_t, v1)};
      } else {
        *(f32x4*)(s.part_o + (slot * a.gqa + h) * kHeadDim + c) = x;
        if (c == 0) s.part_ml[slot * a.gqa + h] = make_float2(M, L);
      }
    }
    __syncthreads();
  };

  // ---- this workgroup's pair, or its part of the items
  const bool own_pair = (int)blockIdx.x < n_pairs;
  const int part = blockIdx.x - n_pairs;
  int s_begin = 0, s_end = a.B;
  Span items = {0, 1};   // of the part (a pair's own workgroup has none: the loop's one round)
  if (own_pair) {
    s_begin = (int)(blockIdx.x / a.H_kv) & ~63;
    s_end = s_begin + 1;
  }
  const int len0 = lane_len(a, s_begin + touch_kernargs<sizeof(BlockArgs) + sizeof(BlockStep)>());
  int incl0 = 0;
  if (!own_pair) {
    incl0 = wave_scan(items_of(len0, a.max_context) * a.H_kv);
    int total = __builtin_amdgcn_readlane(incl0, 63), before;   // at most 2^30 (checked on the host)
    if (a.B > 64) total += items_past_64(a, 0, &before) * a.H_kv;
    const int size = part_items(total);
    if ((int64_t)part * size >= total) return;
    items = {part * size, min(part * size + size, total)};
  }
  int base = 0;   // items before the 64 places of this round
  for (int s0 = s_begin; s0 < s_end && base < items.end; s0 += 64) {
    const int len = s0 == s_begin ? len0 : lane_len(a, s0);
    const int n = items_of(len, a.max_context) * a.H_kv;
    const int incl = s0 == s_begin ? incl0 : base + wave_scan(n);
    // places of the round that the workgroup serves
    uint64_t mine = own_pair ? (uint64_t)1 << ((blockIdx.x / a.H_kv) & 63)
                             : __ballot(n > 0 && incl > items.begin && incl - n < items.end);
    base = __builtin_amdgcn_readlane(incl, 63);
    for (; mine; mine &= mine - 1) {
      const int w = __builtin_ctzll(mine), b = s0 + w;
      const int pos = __builtin_amdgcn_readlane(len, w);   // position of the new token
      const int n_blk = blocks_of(pos, a.max_context), per = n_blk + kSegCost;
      if (n_blk < 0) return;
      const int first = __builtin_amdgcn_readlane(incl, w) - per * a.H_kv;
      const bool small = n_blk <= kSmall;
      Span pairs = {(int)(blockIdx.x % a.H_kv), (int)(blockIdx.x % a.H_kv) + 1};
      if (!own_pair) pairs = pairs_of(items, first, per, a.H_kv);
      for (int g = pairs.begin; g < pairs.end; ++g) {
        Span blks = {0, small ? n_blk : 0};
        if (!own_pair) {
          blks = blocks_in(items, first, per, g);
          if (blks.begin >= blks.end) continue;
        }
        // (part and pair grow together: no two segments share a slot)
        const int64_t slot = own_pair ? (int64_t)blockIdx.x : (int64_t)n_pairs + part + b * a.H_kv + g;
        segment(b, g, blks.begin, blks.end, own_pair ? pos % kBlk + 1 : 0, own_pair && small, slot);
      }
    }
  }
}

// Joins the parts of the pairs that more than one workgroup served, one workgroup per
// (place, query head): eight groups of 32 lanes take the parts in turn.  The workgroups
// before those quantize the blocks that the step's token filled, one per (place, KV head,
// keys or values).
__global__ __launch_bounds__(kThreads) void k_block_merge(BlockArgs a, BlockStep s) {
  __shared__ f32x4 sx[8][kHeadDim / 4];
  __shared__ float2 sml[8];
  const int tid = threadIdx.x;
  const int n_close = 2 * a.B * a.H_kv;
  if ((int)blockIdx.x < n_close) {
    __shared__ CloseLds sm;
    const int pair = blockIdx.x >> 1, b = pair / a.H_kv, g = pair % a.H_kv;
    const int pos = a.lens[b];
    if (pos < 0 || pos >= a.max_context || pos % kBlk != kBlk - 1) return;
    const int page = page_of(a, b, pos / kBlk);
    if (page < 0) return;
    const uint16_t* x = (blockIdx.x & 1 ? a.v_tail : a.k_tail) + (int64_t)pair * kCodes;
    const int64_t e = (int64_t)page * a.H_kv + g;
    auto row = [&](int t) { return x + t * kHeadDim; };
    if (blockIdx.x & 1) close_block<true>(row, a.v_codes + e * kCodes, a.v_scale + e, sm);
    else close_block<false>(row, a.k_codes + e * kCodes, a.k_scale + e, sm);
    return;
  }
  const int b = (blockIdx.x - n_close) / a.H_q, head = (blockIdx.x - n_close) % a.H_q, g = head / a.gqa;
  const int per = items_of(a.lens[b + touch_kernargs<sizeof(BlockArgs) + sizeof(BlockStep)>()], a.max_context);
  if (per == 0) return;   // no sequence, or written by the attention pass
  const int incl0 = wave_scan(items_of(lane_len(a, 0), a.max_context));
  int all = __builtin_amdgcn_readlane(incl0, 63), before;
  if (b < 64) before = __builtin_amdgcn_readlane(incl0, b) - per;
  if (a.B > 64) {
    int more;
    const int past = items_past_64(a, b, &more);
    if (b >= 64) before = all + more;
    all += past;
  }
  const int total = all * a.H_kv, size = part_items(total);
  const int first = before * a.H_kv + g * per;
  const Span parts = parts_of(first, per, size);
  const int pair = b * a.H_kv + g, h = head % a.gqa;
  // row 0 is the open block's, the others the parts'
  const int64_t row0 = (int64_t)pair * a.gqa + h, row1 = ((int64_t)a.B * a.H_kv + parts.begin + pair - 1) * a.gqa + h;
  const int n = parts.end - parts.begin + 1, grp = tid >> 5, c = tid & 31;
  float M = -INFINITY, L = 0.f;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = grp; i0 < n; i0 += 64) {
    // a round of eight rows, all loads first (rows past the last repeat it, with no weight)
    float2 ml[8];
    f32x4 y[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int i = min(i0 + 8 * k, n - 1);
      const int64_t row = i ? row1 + (int64_t)i * a.gqa : row0;
      ml[k] = s.part_ml[row];
      y[k] = *(const f32x4*)(s.part_o + row * kHeadDim + 4 * c);
    }
    float mn = M;
#pragma unroll
    for (int k = 0; k < 8; ++k) mn = fmaxf(mn, ml[k].x);
    const float mu = mn > -INFINITY ? mn : 0.f;
    const float f0 = __builtin_amdgcn_exp2f(M - mu);
    M = mn;
    L *= f0;
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] *= f0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (i0 + 8 * k >= n) break;
      const float f = __builtin_amdgcn_exp2f(ml[k].x - mu);
      L = fmaf(f, ml[k].y, L);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = fmaf(f, y[k][j], x[j]);
    }
  }
  sx[grp][c] = x;
  if (c == 0) sml[grp] = make_float2(M, L);
  __syncthreads();
  if (grp) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) M = fmaxf(M, sml[i].x);
  const float mu = M > -INFINITY ? M : 0.f;
  L = 0.f;
  x = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float f = __builtin_amdgcn_exp2f(sml[i].x - mu);
    L = fmaf(f, sml[i].y, L);
    const f32x4 y = sx[i][c];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = fmaf(f, y[j], x[j]);
  }
  const bf16x2 v0 = {(__bf16)(x[0] / L), (__bf16)(x[1] / L)}, v1 = {(__bf16)(x[2] / L), (__bf16)(x[3] / L)};
  *(u32x2*)(s.out + ((int64_t)b * a.H_q + head) * kHeadDim + 4 * c) =
      (u32x2){__builtin_bit_cast(uint32_t, v0), __builtin_bit_cast(uint32_t, v1)};
}

// Workgroups of the packed kernels (an upper bound: every sequence may end inside a block).
int64_t block_packed_groups(int64_t total, int n_seqs, int H_kv) { return (total / kBlk + n_seqs) * H_kv; }

hipError_t launch_block_store(const BlockArgs& a, const PackedRows& r, hipStream_t st) {
  const int64_t n = block_packed_groups(r.total, a.B, a.H_kv);
  k_block_store<<<dim3((uint32_t)(2 * n)), kThreads, 0, st>>>(a, r);
  return hipGetLastError();
}
hipError_t launch_block_fetch(const BlockArgs& a, const PackedRows& r, hipStream_t st) {
  const int64_t n = block_packed_groups(r.total, a.B, a.H_kv);
  k_block_fetch<<<dim3((uint32_t)n), kThreads, 0, st>>>(a, r);
  return hipGetLastError();
}

// Partial rows of a step: one segment per pair, and one per step from (part, pair) to the
// next in item order.
static int64_t part_rows(int64_t B, int H_kv, int gqa) { return (kParts + 2 * B * H_kv) * gqa; }
int64_t block_workspace_bytes(int64_t B, int H_kv, int gqa) {
  return part_rows(B, H_kv, gqa) * (int64_t)(sizeof(float2) + kHeadDim * sizeof(float));
}

hipError_t launch_block_attend(const BlockArgs& a, BlockStep s, void* workspace, hipStream_t st) {
  s.part_o = (float*)workspace;
  s.part_ml = (float2*)(s.part_o + part_rows(a.B, a.H_kv, a.gqa) * kHeadDim);
  const size_t lds = (size_t)4 * a.gqa * kJoinRow * sizeof(float);
  const dim3 grid(a.B * a.H_kv + kParts);
  // Pages are read past the caches where the layer's pool (the host does not know the
  // lengths) is more than half the 256 MB Infinity Cache: the same eight 8B sequences, 401 MB,
  // again and again 85 -> 78 us, 32 ragged places, 985 MB, 188 -> 174.  Below, the two are
  // within 1 us: one 32K sequence, 67 MB, in turn over 8 layers 24.0 us through the caches and
  // 23.2 past them, the same layer again and again 21.7 and 21.8; a 2K sequence, 4 MB, in turn
  // over 32 layers 11.2 and (in a large pool) 12.1.
  const bool past = (int64_t)a.n_pages * a.H_kv * (2 * kCodes) > (128 << 20);
  if (past) k_block_attend<true><<<grid, kThreads, lds, st>>>(a, s);
  else k_block_attend<false><<<grid, kThreads, lds, st>>>(a, s);
  if (hipError_t e = hipGetLastError()) return e;
  k_block_merge<<<dim3(a.B * (a.H_q + 2 * a.H_kv)), kThreads, 0, st>>>(a, s);
  return hipGetLastError();
}

}  // namespace qv
