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
#include <algorithm>

#include "qv_device.h"

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

// Scale of a block whose largest magnitude is amax (bits of a non-negative float, NaN and
// infinity above all others): NaN when amax is not finite.
__device__ __forceinline__ float block_scale(uint32_t amax) {
  if (amax >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
  return fmaxf(__fdiv_rn(__uint_as_float(amax), 127.f), kMinScale);
}

// round-half-even(x / s) for finite x: the product with the rounded reciprocal is within
// one of it, and the signs of x - (c + 1/2) s and x - (c - 1/2) s (one fused operation
// each, so exact) decide.  inv = 1 / s (s >= 2^-100: no overflow).
__device__ __forceinline__ int code_of(float x, float s, float inv) {
  float c = rintf(x * inv);
  const float up = fmaf(-(c + 0.5f), s, x), dn = fmaf(-(c - 0.5f), s, x);
  const bool odd = ((int)c & 1) != 0;
  if (up > 0.f || (up == 0.f && odd)) c += 1.f;
  else if (dn < 0.f || (dn == 0.f && odd)) c -= 1.f;
  return (int)c;
}

__device__ __forceinline__ uint32_t amax_bits(u32x4 x, uint32_t m) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    m = max(m, (x[j] << 16) & 0x7FFF0000u);
    m = max(m, x[j] & 0x7FFF0000u);
  }
  return m;
}

// Quantizes one complete block of one KV head into its page (all 256 threads).  row(r) is
// the address of token r's keys (values: vrow).  sm: 8 KiB + 512 B of LDS + 8 words.
struct CloseLds {
  uint32_t vt[kHeadDim][kBlk / 4 + 1];   // value codes, four tokens a word
  uint32_t amax[2][kThreads / 64];
};
template <class KRow, class VRow>
__device__ __forceinline__ void close_block(KRow krow, VRow vrow, int8_t* kc, int8_t* vc, float* ks, float* vs,
                                            CloseLds& sm) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int c = tid & 15, m = tid >> 4;   // 8-channel chunk, group of four tokens
  u32x4 xk[4], xv[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    xk[i] = *(const u32x4*)(krow(4 * m + i) + 8 * c);
    xv[i] = *(const u32x4*)(vrow(4 * m + i) + 8 * c);
  }
  uint32_t ak = 0, av = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    ak = amax_bits(xk[i], ak);
    av = amax_bits(xv[i], av);
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    ak = max(ak, (uint32_t)__shfl_xor((int)ak, d, 64));
    av = max(av, (uint32_t)__shfl_xor((int)av, d, 64));
  }
  if (lane == 0) {
    sm.amax[0][wave] = ak;
    sm.amax[1][wave] = av;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    ak = max(ak, sm.amax[0][w]);
    av = max(av, sm.amax[1][w]);
  }
  const float sk = block_scale(ak), sv = block_scale(av);
  const bool fk = sk == sk, fv = sv == sv;
  const float ik = 1.f / sk, iv = 1.f / sv;
  if (tid == 0) {
    *ks = sk;
    *vs = sv;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t w[2] = {0, 0};
    if (fk) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        w[j >> 1] |= (uint32_t)(uint8_t)code_of(lo_f32(xk[i][j]), sk, ik) << (16 * (j & 1));
        w[j >> 1] |= (uint32_t)(uint8_t)code_of(hi_f32(xk[i][j]), sk, ik) << (16 * (j & 1) + 8);
      }
    }
    *(u32x2*)(kc + (4 * m + i) * kHeadDim + 8 * c) = (u32x2){w[0], w[1]};
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    uint32_t w = 0;
    if (fv) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t x = xv[i][j >> 1];
        w |= (uint32_t)(uint8_t)code_of(j & 1 ? hi_f32(x) : lo_f32(x), sv, iv) << (8 * i);
      }
    }
    sm.vt[8 * c + j][m] = w;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {   // 16 bytes a thread: channel e / 4, tokens 16 (e % 4) ..
    const int e = tid + kThreads * i;
    u32x4 x;
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = sm.vt[e >> 2][4 * (e & 3) + j];
    *(u32x4*)(vc + 16 * e) = x;
  }
}

// Where a workgroup of the packed kernels works: block `blk` of sequence `seq`, whose rows
// start at `start` in the packed order and number `len`.
struct PackedBlock {
  int seq, blk, start, len;
};
// The idx-th block of the packed sequences (every sequence has ceil(len / 64)); false past
// the last.  The same in every lane of every wave.
__device__ __forceinline__ bool find_block(const int32_t* cu, int n_seqs, int total, int idx, PackedBlock* out) {
  const int lane = threadIdx.x & 63;
  for (int s0 = 0; s0 < n_seqs; s0 += 64) {
    const int s = s0 + lane;
    int b = 0, n = 0;
    if (s < n_seqs) {
      b = min(max(cu[s], 0), total);
      n = min(max(cu[s + 1], b), total) - b;
    }
    const int blocks = n / kBlk + (n % kBlk != 0);
    int incl = blocks;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(incl, d, 64);
      if (lane >= d) incl += o;
    }
    const uint64_t past = __ballot(incl > idx);
    if (past) {
      const int w = __builtin_ctzll(past);
      out->seq = s0 + w;
      out->start = __builtin_amdgcn_readlane(b, w);
      out->len = __builtin_amdgcn_readlane(n, w);
      out->blk = idx - (__builtin_amdgcn_readlane(incl, w) - __builtin_amdgcn_readlane(blocks, w));
      return true;
    }
    idx -= __builtin_amdgcn_readlane(incl, 63);
  }
  return false;
}

// Page of a sequence's block; -1 when the table holds none (dropped, or out of range).
__device__ __forceinline__ int page_of(const BlockArgs& a, int seq, int blk) {
  if (blk >= a.n_cols) return -1;
  const int p = a.table[(int64_t)seq * a.n_cols + blk];
  return (uint32_t)p < (uint32_t)a.n_pages ? p : -1;
}
}  // namespace

// Packed prompts into the cache, one workgroup per (block, KV head).
__global__ __launch_bounds__(kThreads) void k_block_store(BlockArgs a, PackedRows r) {
  __shared__ CloseLds sm;
  const int g = blockIdx.x % a.H_kv;
  PackedBlock w;
  if (!find_block(r.cu, a.B, r.total, blockIdx.x / a.H_kv, &w)) return;
  const int t0 = w.blk * kBlk, n = min(kBlk, min(w.len, a.max_context) - t0);
  if (n <= 0) return;
  const uint16_t* k = r.k + (int64_t)(w.start + t0) * r.k_st + g * r.k_sh;
  const uint16_t* v = r.v + (int64_t)(w.start + t0) * r.v_st + g * r.v_sh;
  if (n == kBlk) {
    const int page = page_of(a, w.seq, w.blk);
    if (page < 0) return;
    const int64_t e = (int64_t)page * a.H_kv + g;
    close_block([&](int t) { return k + t * r.k_st; }, [&](int t) { return v + t * r.v_st; },
                a.k_codes + e * kCodes, a.v_codes + e * kCodes, a.k_scale + e, a.v_scale + e, sm);
    return;
  }
  const int64_t tail = ((int64_t)w.seq * a.H_kv + g) * kCodes;
  for (int e = threadIdx.x; e < n * 16; e += kThreads) {
    const int t = e >> 4, c = 8 * (e & 15);
    *(u32x4*)(a.k_tail + tail + t * kHeadDim + c) = *(const u32x4*)(k + t * r.k_st + c);
    *(u32x4*)(a.v_tail + tail + t * kHeadDim + c) = *(const u32x4*)(v + t * r.v_st + c);
  }
}

// The cache back into packed bf16 rows: a token of a complete block is bf16(fl32(c s)), a
// token of a block without a page is zero, a token of the tail is copied.  Rows past a
// sequence's length are not written.
__global__ __launch_bounds__(kThreads) void k_block_fetch(BlockArgs a, PackedRows r) {
  __shared__ uint32_t vt[kHeadDim][kBlk / 4 + 1];
  const int g = blockIdx.x % a.H_kv, tid = threadIdx.x;
  PackedBlock w;
  if (!find_block(r.cu, a.B, r.total, blockIdx.x / a.H_kv, &w)) return;
  const int held = min(a.lens[w.seq], a.max_context);
  const int t0 = w.blk * kBlk, n = min(min(kBlk, w.len - t0), held - t0);
  if (n <= 0) return;
  uint16_t* k = r.k_out + (int64_t)(w.start + t0) * r.k_st + g * r.k_sh;
  uint16_t* v = r.v_out + (int64_t)(w.start + t0) * r.v_st + g * r.v_sh;
  if (w.blk >= held / kBlk) {
    const int64_t tail = ((int64_t)w.seq * a.H_kv + g) * kCodes;
    for (int e = tid; e < n * 16; e += kThreads) {
      const int t = e >> 4, c = 8 * (e & 15);
      *(u32x4*)(k + t * r.k_st + c) = *(const u32x4*)(a.k_tail + tail + t * kHeadDim + c);
      *(u32x4*)(v + t * r.v_st + c) = *(const u32x4*)(a.v_tail + tail + t * kHeadDim + c);
    }
    return;
  }
  const int page = page_of(a, w.seq, w.blk);
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
    *(u32x4*)(k + t * r.k_st + 8 * c) = x;
    *(u32x4*)(v + t * r.v_st + 8 * c) = y;
  }
}

// ------------------------------------------------------------------ decode attention
// One token per sequence, in two launches.  The items of a (sequence, KV head) pair are
// its complete blocks, then its open block; the items of all pairs, in pair order, are cut
// into equal parts, one per workgroup, whatever the lengths are (they are read on the
// device).  A workgroup goes through the pairs its part touches (segments); its four waves
// take a segment's items in turn and are joined in LDS.  A segment that is a whole pair is
// written out; the others leave (maximum, sum, output) rows that k_block_merge joins.
//
// A wave's products, by 16x16x32 MFMAs with the G query heads of the KV head as columns
// (padded to 16):
//   S^T = K q^T   (A = 16 keys; a lane holds 4 keys of ONE head per tile)
//   O^T = V^T P^T (A = 16 channels; the same lane owns 32 channels of that head)
// Row r of key tile tt is token 16 (r / 4) + 4 tt + r % 4 of the block, so that lane group
// qd holds the logits of tokens 16 qd .. + 15: the 16 codes that one 16-byte load of a
// value channel gives it.  Codes become fp16 integers (exact): byte + 128 placed below
// 0x64 is 1152 + c, minus 1152.  A head's query is scaled by a power of two into fp16
// (exact: bf16 has 8 bits; entries 2^-38 below the head's largest round).
namespace {
constexpr float kLazyD = 8.f;
constexpr int kParts = 512;      // workgroups of a step: two per compute unit

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

// Items of a place: its complete blocks and the open one; none without a sequence or room.
__device__ __forceinline__ int items_of(int len, int max_context) {
  return len < 0 || len >= max_context ? 0 : len / kBlk + 1;
}

// inclusive sum over the wave's lanes
__device__ __forceinline__ int wave_scan(int x, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(x, d, 64);
    if (lane >= d) x += o;
  }
  return x;
}

// Items of all places (of one KV head); with a place, *before receives those of the places
// before it.  At most 2^31 / H_kv (checked on the host).
__device__ __forceinline__ int count_items(const BlockArgs& a, int place, int* before) {
  const int lane = threadIdx.x & 63;
  int sum = 0;
  for (int s0 = 0; s0 < a.B; s0 += 64) {
    const int n = s0 + lane < a.B ? items_of(a.lens[s0 + lane], a.max_context) : 0;
    const int incl = wave_scan(n, lane);
    if (place >= s0 && place < s0 + 64)
      *before = sum + __builtin_amdgcn_readlane(incl, place - s0) - __builtin_amdgcn_readlane(n, place - s0);
    sum += __builtin_amdgcn_readlane(incl, 63);
  }
  return sum;
}

constexpr int kTailRow = 2 * kHeadDim;
constexpr int kJoinRow = kHeadDim + 4;
}  // namespace

__global__ __launch_bounds__(kThreads, 2) void k_block_attend(BlockArgs a, BlockStep s) {
  __shared__ __attribute__((aligned(16))) uint8_t stail[kBlk * kTailRow];   // the open block's values
  __shared__ float sml[4][16][2];
  extern __shared__ __attribute__((aligned(16))) float so[];                // [4][gqa][kJoinRow]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, qd = lane >> 4;

  // ---- this workgroup's part of the items
  const int64_t total = (int64_t)count_items(a, -1, nullptr) * a.H_kv;
  const int parts = (int)min((int64_t)gridDim.x, total), part = blockIdx.x;
  if (part >= parts) return;
  const int begin = (int)(total * part / parts), end = (int)(total * (part + 1) / parts);

  int base = 0;   // items before the 64 places of this round
  for (int s0 = 0; s0 < a.B && base < end; s0 += 64) {
    const int len = s0 + lane < a.B ? a.lens[s0 + lane] : -1;
    const int n = items_of(len, a.max_context) * a.H_kv;
    const int incl = base + wave_scan(n, lane);
    // places of the round that the part touches
    uint64_t mine = __ballot(n > 0 && incl > begin && incl - n < end);
    base = __builtin_amdgcn_readlane(incl, 63);
    for (; mine; mine &= mine - 1) {
      const int w = __builtin_ctzll(mine), b = s0 + w;
      const int pos = __builtin_amdgcn_readlane(len, w);   // position of the new token
      const int n_blk = pos / kBlk, n_tail = pos % kBlk + 1, per = n_blk + 1;
      const int first = __builtin_amdgcn_readlane(incl, w) - per * a.H_kv;
      const int lo = max(begin - first, 0), hi = min(end - first, per * a.H_kv);
      for (int g = lo / per; g * per < hi; ++g) {
        // ---- segment: items [i0, i1) of pair (b, g)
        const int i0 = max(lo - g * per, 0), i1 = min(hi - g * per, per);
        const int hr = min(r, a.gqa - 1);   // columns past the last head repeat it
        const uint16_t* qp = s.q + ((int64_t)b * a.H_q + g * a.gqa + hr) * kHeadDim;
        Running st;
        st.m = -INFINITY;
        st.l = 0.f;
#pragma unroll
        for (int ct = 0; ct < 8; ++ct) st.o[ct] = (f32x4){0.f, 0.f, 0.f, 0.f};

        const int b_end = min(i1, n_blk);
        if (i0 + wave < b_end) {
          // query operand: k-step (p, e) covers channels 64 p + 16 qd + 8 e + j
          u32x4 qw[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) qw[i] = *(const u32x4*)(qp + 64 * (i >> 1) + 16 * qd + 8 * (i & 1));
          uint32_t am = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) am = amax_bits(qw[i], am);
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
          const float qs = ldexpf(a.scale_log2, ex - 14);   // log2 units per (q' c s)

          for (int blk0 = i0 + wave; blk0 < b_end; blk0 += 256) {
            // pages and scales of the wave's next 64 blocks, one per lane; a dropped block's
            // tokens take no part
            const int blk = blk0 + 4 * lane;
            const int page = blk < b_end ? page_of(a, b, blk) : -1;
            const int64_t e = (int64_t)max(page, 0) * a.H_kv + g;
            float ks_l = 0.f, vs_l = 0.f;
            if (page >= 0) {
              ks_l = a.k_scale[e];
              vs_l = a.v_scale[e];
            }
            uint64_t live = __ballot(page >= 0);
            if (!live) continue;
            const int row = (16 * (r >> 2) + (r & 3)) * kHeadDim + 16 * qd;   // + 4 tt rows
            u32x4 kb[8], vb[8];
            auto entry = [&](int j) { return ((int64_t)__builtin_amdgcn_readlane(page, j) * a.H_kv + g) * kCodes; };
            auto load_k = [&](int j) {
              const int8_t* kc = a.k_codes + entry(j) + row;
#pragma unroll
              for (int i = 0; i < 8; ++i) kb[i] = *(const u32x4*)(kc + 4 * (i >> 1) * kHeadDim + 64 * (i & 1));
            };
            load_k(__builtin_ctzll(live));
            while (live) {
              const int j = __builtin_ctzll(live);
              live &= live - 1;
              const int8_t* vc = a.v_codes + entry(j) + r * kBlk + 16 * qd;
#pragma unroll
              for (int ct = 0; ct < 8; ++ct) vb[ct] = *(const u32x4*)(vc + 16 * ct * kBlk);
              const float sc = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ks_l), j)) * qs;
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
          }
        }

        if (i1 == per && wave == ((n_blk - i0) & 3)) {
          // the open block, in bf16: row n_tail - 1 is the new token, which this wave stores
          const uint16_t* kn = s.k_new + ((int64_t)b * a.H_kv + g) * kHeadDim;
          const uint16_t* vn = s.v_new + ((int64_t)b * a.H_kv + g) * kHeadDim;
          uint16_t* kt = a.k_tail + ((int64_t)b * a.H_kv + g) * kCodes;
          uint16_t* vt = a.v_tail + ((int64_t)b * a.H_kv + g) * kCodes;
          const u32x4 z = {0, 0, 0, 0};
          if (lane < 32) {
            const uint16_t* src = lane < 16 ? kn : vn;
            uint16_t* dst = (lane < 16 ? kt : vt) + (n_tail - 1) * kHeadDim;
            *(u32x4*)(dst + 8 * r) = *(const u32x4*)(src + 8 * r);
          }
#pragma unroll 4
          for (int i = 0; i < 16; ++i) {
            const int t = 4 * i + qd;
            const u32x4 x = t < n_tail - 1 ? *(const u32x4*)(vt + t * kHeadDim + 8 * r)
                                           : (t == n_tail - 1 ? *(const u32x4*)(vn + 8 * r) : z);
            *(u32x4*)(stail + t * kTailRow + 16 * r) = x;
          }
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          u32x4 qw[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) qw[i] = *(const u32x4*)(qp + 32 * i + 8 * qd);
          f32x4 acc[4];
          float mt = -INFINITY;
#pragma unroll
          for (int tt = 0; tt < 4; ++tt) {
            acc[tt] = (f32x4){0.f, 0.f, 0.f, 0.f};
            const int t = 16 * (r >> 2) + 4 * tt + (r & 3);
            const uint16_t* row = t < n_tail - 1 ? kt + t * kHeadDim : kn;
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[tt] = mfma_bf(*(const u32x4*)(row + 32 * i + 8 * qd), qw[i], acc[tt]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              acc[tt][i] = 16 * qd + 4 * tt + i < n_tail ? acc[tt][i] * a.scale_log2 : -INFINITY;
              mt = fmaxf(mt, acc[tt][i]);
            }
          }
          raise(st, rows_max(mt));
          const float mu = st.m > -INFINITY ? st.m : 0.f;
          u32x4 p[2];
#pragma unroll
          for (int tt = 0; tt < 4; ++tt)
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
              const float x = __builtin_amdgcn_exp2f(acc[tt][i] - mu), y = __builtin_amdgcn_exp2f(acc[tt][i + 1] - mu);
              st.l += x + y;
              const bf16x2 h = {(__bf16)x, (__bf16)y};
              p[tt >> 1][2 * (tt & 1) + (i >> 1)] = __builtin_bit_cast(uint32_t, h);
            }
#pragma unroll
          for (int ct = 0; ct < 8; ++ct)
#pragma unroll
            for (int e = 0; e < 2; ++e) {   // tokens 16 qd + 8 e + j
              const uint8_t* src = stail + (16 * qd + 8 * e + (r >> 2)) * kTailRow + 32 * ct + 8 * (r & 3);
              const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)src));
              const u32x2 y =
                  __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(src + 4 * kTailRow)));
              st.o[ct] = mfma_bf((u32x4){x[0], x[1], y[0], y[1]}, p[e], st.o[ct]);
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
        const bool whole = i0 == 0 && i1 == per;
        const int64_t slot = (int64_t)part + (int64_t)b * a.H_kv + g;   // both grow: no two segments share one
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
      }
    }
  }
}

// Joins the parts of the pairs that more than one workgroup served, one workgroup per
// (place, query head): eight groups of 32 lanes take the parts in turn.  The workgroups past
// those quantize the blocks that the step's token filled, one per (place, KV head).
__global__ __launch_bounds__(kThreads) void k_block_merge(BlockArgs a, BlockStep s, int n_parts) {
  __shared__ f32x4 sx[8][kHeadDim / 4];
  __shared__ float2 sml[8];
  const int tid = threadIdx.x;
  if (blockIdx.x >= a.B * a.H_q) {
    __shared__ CloseLds sm;
    const int pair = blockIdx.x - a.B * a.H_q, b = pair / a.H_kv, g = pair % a.H_kv;
    const int pos = a.lens[b];
    if (pos < 0 || pos >= a.max_context || pos % kBlk != kBlk - 1) return;
    const int page = page_of(a, b, pos / kBlk);
    if (page < 0) return;
    const uint16_t* kt = a.k_tail + (int64_t)pair * kCodes;
    const uint16_t* vt = a.v_tail + (int64_t)pair * kCodes;
    const int64_t e = (int64_t)page * a.H_kv + g;
    close_block([&](int t) { return kt + t * kHeadDim; }, [&](int t) { return vt + t * kHeadDim; },
                a.k_codes + e * kCodes, a.v_codes + e * kCodes, a.k_scale + e, a.v_scale + e, sm);
    return;
  }
  const int b = blockIdx.x / a.H_q, head = blockIdx.x % a.H_q, g = head / a.gqa;
  const int per = items_of(a.lens[b], a.max_context);
  if (per == 0) return;
  int before;
  const int64_t total = (int64_t)count_items(a, b, &before) * a.H_kv;
  const int64_t parts = min((int64_t)n_parts, total);
  const int64_t first = (int64_t)before * a.H_kv + (int64_t)g * per;
  // the part of item i is the largest p with floor(total p / parts) <= i
  const int p0 = (int)(((first + 1) * parts - 1) / total), p1 = (int)(((first + per) * parts - 1) / total);
  if (p0 == p1) return;   // written by the attention pass
  const int64_t row0 = ((int64_t)p0 + (int64_t)b * a.H_kv + g) * a.gqa + head % a.gqa;
  const int n = p1 - p0 + 1, grp = tid >> 5, c = tid & 31;
  float M = -INFINITY, L = 0.f;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  for (int i = grp; i < n; i += 8) {
    const int64_t row = row0 + (int64_t)i * a.gqa;
    const float2 ml = s.part_ml[row];
    const f32x4 y = *(const f32x4*)(s.part_o + row * kHeadDim + 4 * c);
    const float mn = fmaxf(M, ml.x), mu = mn > -INFINITY ? mn : 0.f;
    const float f0 = __builtin_amdgcn_exp2f(M - mu), f1 = __builtin_amdgcn_exp2f(ml.x - mu);
    M = mn;
    L = fmaf(f1, ml.y, f0 * L);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = fmaf(f1, y[j], f0 * x[j]);
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
  k_block_store<<<dim3((uint32_t)n), kThreads, 0, st>>>(a, r);
  return hipGetLastError();
}
hipError_t launch_block_fetch(const BlockArgs& a, const PackedRows& r, hipStream_t st) {
  const int64_t n = block_packed_groups(r.total, a.B, a.H_kv);
  k_block_fetch<<<dim3((uint32_t)n), kThreads, 0, st>>>(a, r);
  return hipGetLastError();
}

// Partial rows of a step: at most one segment per (workgroup, pair) step in item order.
static int64_t part_rows(int64_t B, int H_kv, int gqa) { return (kParts + B * H_kv) * gqa; }
int64_t block_workspace_bytes(int64_t B, int H_kv, int gqa) {
  return part_rows(B, H_kv, gqa) * (int64_t)(sizeof(float2) + kHeadDim * sizeof(float));
}

hipError_t launch_block_attend(const BlockArgs& a, BlockStep s, void* workspace, hipStream_t st) {
  s.part_o = (float*)workspace;
  s.part_ml = (float2*)(s.part_o + part_rows(a.B, a.H_kv, a.gqa) * kHeadDim);
  k_block_attend<<<dim3(kParts), kThreads, (size_t)4 * a.gqa * kJoinRow * sizeof(float), st>>>(a, s);
  if (hipError_t e = hipGetLastError()) return e;
  k_block_merge<<<dim3(a.B * (a.H_q + a.H_kv)), kThreads, 0, st>>>(a, s, kParts);
  return hipGetLastError();
}

}  // namespace qv
