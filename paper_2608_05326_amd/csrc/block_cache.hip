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
//   k_block_attend  one decode token per sequence: append, attend, close a full block
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
// One token per sequence.  A workgroup of four waves takes one (sequence, KV head): wave w
// takes blocks w, w + 4, ..., the tail is wave 0's last one.  With 16x16x32 MFMAs, the G
// query heads of the KV head as columns (padded to 16):
//   S^T = K q^T   (A = 16 keys; a lane holds 4 keys of ONE head per tile)
//   O^T = V^T P^T (A = 16 channels; the same lane owns 32 channels of that head)
// Row r of key tile tt is token 16 (r / 4) + 4 tt + r % 4 of the block, so that lane group
// qd holds the logits of tokens 16 qd .. + 15: the 16 codes that one 16-byte load of a
// value channel gives it.  Codes become fp16 integers (exact): byte + 128 placed below
// 0x64 is 1152 + c, minus 1152.  A head's query is scaled by a power of two into fp16
// (exact: bf16 has 8 bits; entries 2^-38 below the head's largest round).
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

constexpr int kTailRow = 2 * kHeadDim;
}  // namespace

__global__ __launch_bounds__(kThreads, 2) void k_block_attend(BlockArgs a, BlockStep s) {
  __shared__ __attribute__((aligned(16))) uint8_t stail[kBlk * kTailRow];   // the tail's values
  __shared__ __attribute__((aligned(16))) float so[4][16][kHeadDim + 4];
  __shared__ float sml[4][16][2];
  __shared__ CloseLds sm;
  const int g = blockIdx.x, b = blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, qd = lane >> 4;
  const int pos = a.lens[b];                     // position of the new token
  if (pos < 0 || pos >= a.max_context) return;   // no sequence in this place
  const int n_blk = pos / kBlk, n_tail = pos % kBlk + 1;

  const int hr = min(r, a.gqa - 1);   // columns past the last head repeat it
  const uint16_t* qp = s.q + ((int64_t)b * a.H_q + g * a.gqa + hr) * kHeadDim;
  const uint16_t* kn = s.k_new + ((int64_t)b * a.H_kv + g) * kHeadDim;
  const uint16_t* vn = s.v_new + ((int64_t)b * a.H_kv + g) * kHeadDim;
  uint16_t* kt = a.k_tail + ((int64_t)b * a.H_kv + g) * kCodes;
  uint16_t* vt = a.v_tail + ((int64_t)b * a.H_kv + g) * kCodes;

  Running st;
  st.m = -INFINITY;
  st.l = 0.f;
#pragma unroll
  for (int ct = 0; ct < 8; ++ct) st.o[ct] = (f32x4){0.f, 0.f, 0.f, 0.f};

  if (wave < n_blk) {
    // query operand: k-step (p, e) covers channels 64 p + 16 qd + 8 e + j
    u32x4 qw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) qw[i] = *(const u32x4*)(qp + 64 * (i >> 1) + 16 * qd + 8 * (i & 1));
    uint32_t am = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) am = amax_bits(qw[i], am);
    am = max(am, (uint32_t)__shfl_xor((int)am, 16, 64));
    am = max(am, (uint32_t)__shfl_xor((int)am, 32, 64));
    // 2^(14 - e) for a largest magnitude in [2^e, 2^(e + 1)); ldexp takes what its factors
    // cannot hold in one
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

    for (int blk = wave; blk < n_blk; blk += 4) {
      const int page = page_of(a, b, blk);
      if (page < 0) continue;   // dropped: its tokens take no part
      const int64_t e = (int64_t)page * a.H_kv + g;
      const int8_t* kc = a.k_codes + e * kCodes;
      const int8_t* vc = a.v_codes + e * kCodes;
      const float sc = a.k_scale[e] * qs, vs = a.v_scale[e];
      f32x4 acc[4];
#pragma unroll
      for (int tt = 0; tt < 4; ++tt) {
        acc[tt] = (f32x4){0.f, 0.f, 0.f, 0.f};
        const int8_t* row = kc + (16 * (r >> 2) + 4 * tt + (r & 3)) * kHeadDim + 16 * qd;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          const u32x4 x = *(const u32x4*)(row + 64 * p);
          acc[tt] = mfma_f16(codes_f16(x[0], x[1]), qf[2 * p], acc[tt]);
          acc[tt] = mfma_f16(codes_f16(x[2], x[3]), qf[2 * p + 1], acc[tt]);
        }
      }
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
        const u32x4 x = *(const u32x4*)(vc + (16 * ct + r) * kBlk + 16 * qd);
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
        y = mfma_f16(codes_f16(x[0], x[1]), p[0], y);
        y = mfma_f16(codes_f16(x[2], x[3]), p[1], y);
#pragma unroll
        for (int i = 0; i < 4; ++i) st.o[ct][i] = fmaf(y[i], vs, st.o[ct][i]);
      }
    }
  }

  if (wave == 0) {
    // the tail, in bf16: row n_tail - 1 is the new token, which this wave stores
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
  if (qd == 0) {
    sml[wave][r][0] = st.m;
    sml[wave][r][1] = l;
  }
#pragma unroll
  for (int ct = 0; ct < 8; ++ct) *(f32x4*)&so[wave][r][16 * ct + 4 * qd] = st.o[ct];
  __syncthreads();
  for (int e = tid; e < a.gqa * (kHeadDim / 2); e += kThreads) {
    const int h = e / (kHeadDim / 2), c = 2 * (e % (kHeadDim / 2));
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) M = fmaxf(M, sml[w][h][0]);
    const float mu = M > -INFINITY ? M : 0.f;
    float L = 0.f, x = 0.f, y = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = __builtin_amdgcn_exp2f(sml[w][h][0] - mu);
      L = fmaf(f, sml[w][h][1], L);
      x = fmaf(f, so[w][h][c], x);
      y = fmaf(f, so[w][h][c + 1], y);
    }
    const bf16x2 v = {(__bf16)(x / L), (__bf16)(y / L)};
    *(bf16x2*)(s.out + ((int64_t)b * a.H_q + g * a.gqa + h) * kHeadDim + c) = v;
  }

  if (n_tail == kBlk) {   // the token filled its block
    const int page = page_of(a, b, n_blk);
    if (page < 0) return;
    const int64_t e = (int64_t)page * a.H_kv + g;
    close_block([&](int t) { return t < kBlk - 1 ? kt + t * kHeadDim : kn; },
                [&](int t) { return t < kBlk - 1 ? vt + t * kHeadDim : vn; }, a.k_codes + e * kCodes,
                a.v_codes + e * kCodes, a.k_scale + e, a.v_scale + e, sm);
  }
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
hipError_t launch_block_attend(const BlockArgs& a, const BlockStep& s, hipStream_t st) {
  k_block_attend<<<dim3(a.H_kv, a.B), kThreads, 0, st>>>(a, s);
  return hipGetLastError();
}

}  // namespace qv
