// Causal attention of whole prompts, packed one behind the other (the prompt pass that
// precedes the tier assignment: Sec. 4.1 attention, a query per token).
//
//   out_i = sum_{j <= i} softmax_j(scale q_i . k_j) v_j      inside each prompt,
//
// query head h on KV head h / G, G = H_q / H_kv.  The G heads of a KV head share its keys,
// so the rows of one (prompt, KV head) pair are its (position, head) pairs, row = position
// * G + head: a workgroup of four waves takes 128 consecutive rows, 32 a wave, over the
// keys 0 .. its last position, 64 keys a tile.  One pass with the running maximum and sum
// of the softmax; the products are 32x32x16 bf16 MFMAs:
//   S^T = K Q^T   (A = keys, B = rows): a lane holds 16 of a tile's 32 keys of ONE row, so
//                 maximum and sum are in-lane but for one exchange of the two lane halves
//   O^T = V^T P^T (A = channels, B = rows): the same lane owns the row's output channels
// The keys of the A operand are permuted so that a lane's logits 8 s .. 8 s + 7 of a tile
// are the eight consecutive keys the second product wants from it (acc_key): P goes from
// the first product's result to the second's operand without moving between lanes.
// P enters the second product in bf16 (off by at most 2^-8 of itself, the size of the
// output's own rounding); logits, maximum, sum and output are held in 32 bits.
#include <algorithm>

#include "qv_device.h"

namespace qv {

namespace {
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr int kRows = 128;      // (position, head) rows per workgroup
constexpr int kKeys = 64;       // keys per tile
constexpr int kThreads = 256;
constexpr int kRowBytes = 2 * kHeadDim;
// the running maximum is raised (and the output rescaled) only when a tile exceeds it by
// this many powers of two: P stays below 256
constexpr float kLazy = 8.f;

__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                 0, 0, 0);
}

__device__ __forceinline__ float half_max(float x) {
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const uint32_t s0 = s[0], s1 = s[1];
  return fmaxf(__uint_as_float(s0), __uint_as_float(s1));
}
__device__ __forceinline__ float half_sum(float x) {
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const uint32_t s0 = s[0], s1 = s[1];
  return __uint_as_float(s0) + __uint_as_float(s1);
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const bf16x2 p = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, p);
}

// 16-byte chunks of a staged row are stored at chunk ^ swizzle(key), so that the reads of
// either product meet all banks: 16 rows at one chunk (keys), 4 rows at two chunks (values)
__device__ __forceinline__ int swz_k(int key) { return key & 15; }
__device__ __forceinline__ int swz_v(int key) { return ((key & 3) << 2) | ((key >> 2) & 3); }

// 16 bytes a lane from global memory to LDS, in lane order from a row that is uniform
__device__ __forceinline__ void dma16(const void* g, uint8_t* lds_row) {
  __builtin_amdgcn_global_load_lds(g, (__attribute__((address_space(3))) void*)lds_row, 16, 0, 0);
}

__device__ __forceinline__ bool nonfinite_pair(uint32_t x) {
  return (x & 0x7F80u) == 0x7F80u || (x & 0x7F800000u) == 0x7F800000u;
}
}  // namespace

__global__ __launch_bounds__(kThreads, 2) void k_prompt_attend(PromptArgs a) {
  // two tiles of keys and values, in four arrays: reads of one tile do not wait for the
  // loads of the next (the compiler tells arrays apart, not parts of one)
  __shared__ __attribute__((aligned(16))) uint8_t sk0[kKeys * kRowBytes];
  __shared__ __attribute__((aligned(16))) uint8_t sv0[kKeys * kRowBytes];
  __shared__ __attribute__((aligned(16))) uint8_t sk1[kKeys * kRowBytes];
  __shared__ __attribute__((aligned(16))) uint8_t sv1[kKeys * kRowBytes];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, lh = lane >> 5;

  // ---- this workgroup's KV head, prompt and rows: tiles of all prompts are numbered in
  // prompt order, the longest tile of a prompt first
  const int g = blockIdx.x % a.H_kv;
  int tile = blockIdx.x / a.H_kv;
  int start = 0, len = 0;
  bool found = false;
  for (int s0 = 0; s0 < a.n_seqs && !found; s0 += 64) {
    const int s = s0 + lane;
    int b = 0, n = 0;
    if (s < a.n_seqs) {
      b = min(max(a.cu[s], 0), a.total);
      n = min(max(a.cu[s + 1], b), a.total) - b;
    }
    const int tiles = (int)(((int64_t)n * a.gqa + kRows - 1) / kRows);
    int incl = tiles;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(incl, d, 64);
      if (lane >= d) incl += o;
    }
    const uint64_t past = __ballot(incl > tile);
    if (past) {
      const int w = __builtin_ctzll(past);
      start = __builtin_amdgcn_readlane(b, w);
      len = __builtin_amdgcn_readlane(n, w);
      // the tile's number inside its prompt, counted from the prompt's end
      tile = __builtin_amdgcn_readlane(incl, w) - 1 - tile;
      found = true;
    } else {
      tile -= __builtin_amdgcn_readlane(incl, 63);
    }
  }
  if (!found) return;
  const int64_t n_rows = (int64_t)len * a.gqa;
  const int64_t row0 = (int64_t)tile * kRows;

  // this lane's row (rows past the prompt's last repeat it and are not stored)
  const int64_t row = row0 + wave * 32 + lr;
  const int64_t rowc = min(row, n_rows - 1);
  const int pos = (int)(rowc / a.gqa), head = g * a.gqa + (int)(rowc % a.gqa);
  const int pos_first = (int)(row0 / a.gqa);   // of the workgroup
  const int pos_last = (int)(min(row0 + kRows - 1, n_rows - 1) / a.gqa);

  u32x4 q[8];
  {
    const uint16_t* p = a.q + (start + pos) * a.q_st + head * a.q_sh + 8 * lh;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) q[ks] = *(const u32x4*)(p + 16 * ks);
  }
  f32x16 o[4];
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[c][i] = 0.f;
  float m = -INFINITY, l = 0.f;
  const float sc = a.scale_log2;

  const uint16_t* kp = a.k + (int64_t)start * a.k_st + g * a.k_sh;
  const uint16_t* vp = a.v + (int64_t)start * a.v_st + g * a.v_sh;
  // LDS addresses: A operand row lr of a 32-key tile is key krow of it
  const int krow = 16 * (lr >> 4) + 8 * ((lr >> 2) & 1) + 4 * ((lr >> 3) & 1) + (lr & 3);
  const int vkey = 8 * lh + ((lane >> 2) & 3);                 // + 4 j
  const int vchunk = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);   // + 4 c
  const int vsub = 8 * (lane & 1);

  const int n_tiles = pos_last / kKeys + 1;
  // Starts the loads of tile t straight into LDS: a wave's instruction fills four rows, its
  // lanes in order, so the swizzle is applied to the chunk a lane fetches.
  auto fetch = [&](int t, uint8_t* sk, uint8_t* sv) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 16 * wave + 4 * i + (lane >> 4);
      const int64_t key = min(t * kKeys + r, len - 1);   // keys past the prompt are masked
      dma16(kp + key * a.k_st + 8 * ((lane & 15) ^ swz_k(r)), sk + (16 * wave + 4 * i) * kRowBytes);
      dma16(vp + key * a.v_st + 8 * ((lane & 15) ^ swz_v(r)), sv + (16 * wave + 4 * i) * kRowBytes);
    }
  };
  auto compute = [&](int t, uint8_t* sk, uint8_t* sv) {
    const int key0 = t * kKeys;
    // only tiles that reach past the workgroup's first position mask keys
    const bool edge = key0 + kKeys - 1 > pos_first;
    bool odd_values = false;
    if (edge) {
      // a masked key's value must not reach a row through 0 * infinity: values that are
      // not finite leave the tile here and are added to the rows that see them below
      for (int i = 0; i < 4; ++i) {
        u32x4* p = (u32x4*)sv + tid + kThreads * i;
        u32x4 x = *p;
        bool bad = false;
#pragma unroll
        for (int j = 0; j < 4; ++j) bad |= nonfinite_pair(x[j]);
        if (bad) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if ((x[j] & 0x7F80u) == 0x7F80u) x[j] &= 0xFFFF0000u;
            if ((x[j] & 0x7F800000u) == 0x7F800000u) x[j] &= 0xFFFFu;
          }
          *p = x;
        }
        odd_values |= bad;
      }
      odd_values = __syncthreads_or(odd_values);
    }

    f32x16 s[2];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[kt][i] = 0.f;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks)
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const int key = 32 * kt + krow;
        const u32x4 kk = *(const u32x4*)(sk + key * kRowBytes + 16 * ((2 * ks + lh) ^ swz_k(key)));
        s[kt] = mfma32(kk, q[ks], s[kt]);
      }
    // s[kt][i]: raw logit of key key0 + 32 kt + 16 (i / 8) + 8 lh + i % 8 for this lane's row
    if (edge) {
      const int rel = pos - key0 - 8 * lh;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (32 * kt + 16 * (i >> 3) + (i & 7) > rel) s[kt][i] = -INFINITY;
    }
    float mt = -INFINITY;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) mt = fmaxf(mt, s[kt][i]);
    mt = half_max(mt) * sc;
    if (__any(mt > m + kLazy)) {
      const float mn = fmaxf(m, mt);
      const float al = m == mn ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= al;
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[c][i] *= al;
    }
    const float mu = m > -INFINITY ? m : 0.f;
    u32x4 p[4];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        const float e0 = __builtin_amdgcn_exp2f(fmaf(s[kt][i], sc, -mu));
        const float e1 = __builtin_amdgcn_exp2f(fmaf(s[kt][i + 1], sc, -mu));
        l += e0 + e1;
        p[2 * kt + (i >> 3)][(i & 7) >> 1] = pack_bf16(e0, e1);
      }
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int k0 = 16 * ks + vkey;
        const s16x4 x0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_s16x4*)(sv + k0 * kRowBytes + 16 * ((4 * c + vchunk) ^ swz_v(k0)) + vsub));
        const s16x4 x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_s16x4*)(sv + (k0 + 4) * kRowBytes + 16 * ((4 * c + vchunk) ^ swz_v(k0 + 4)) + vsub));
        const u32x2 y0 = __builtin_bit_cast(u32x2, x0), y1 = __builtin_bit_cast(u32x2, x1);
        o[c] = mfma32((u32x4){y0[0], y0[1], y1[0], y1[1]}, p[ks], o[c]);
      }
    // o[c][i]: channel 32 c + 8 (i / 4) + 4 lh + i % 4 of this lane's row
    if (odd_values) {
      for (int r = 0; r < kKeys && key0 + r <= pos; ++r) {
        const uint16_t* vr = vp + (int64_t)(key0 + r) * a.v_st + 4 * lh;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const uint16_t x = vr[32 * c + 8 * (i >> 2) + (i & 3)];
            if ((x & 0x7F80u) == 0x7F80u) o[c][i] += bf16_to_f32(x);
          }
      }
    }
  };
  fetch(0, sk0, sv0);
  for (int t = 0; t < n_tiles; t += 2) {
    // a tile's loads have landed and the tile before is consumed: its arrays are free
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (t + 1 < n_tiles) fetch(t + 1, sk1, sv1);
    compute(t, sk0, sv0);
    if (t + 1 == n_tiles) break;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (t + 2 < n_tiles) fetch(t + 2, sk0, sv0);
    compute(t + 1, sk1, sv1);
  }

  const float inv = 1.f / half_sum(l);
  uint16_t* op = a.out + (start + pos) * a.o_st + head * a.o_sh;
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int e = 0; e < 4; e += 2) {   // channels 32 c + 8 e .. + 15: eight to each lane half
      uint32_t x[2], y[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const auto sw = __builtin_amdgcn_permlane32_swap(
            pack_bf16(o[c][4 * e + 2 * j] * inv, o[c][4 * e + 2 * j + 1] * inv),
            pack_bf16(o[c][4 * e + 4 + 2 * j] * inv, o[c][4 * e + 5 + 2 * j] * inv), false, false);
        x[j] = sw[0];
        y[j] = sw[1];
      }
      if (row < n_rows) *(u32x4*)(op + 32 * c + 8 * (e + lh)) = (u32x4){x[0], x[1], y[0], y[1]};
    }
}

// Workgroups of a launch (an upper bound: every prompt's last tile may be a partial one).
int64_t prompt_attend_groups(int64_t total, int n_seqs, int gqa, int H_kv) {
  return (total * gqa / kRows + n_seqs) * H_kv;
}

hipError_t launch_prompt_attend(const PromptArgs& a, hipStream_t st) {
  const int64_t n = prompt_attend_groups(a.total, a.n_seqs, a.gqa, a.H_kv);
  if (n == 0) return hipSuccess;
  k_prompt_attend<<<dim3((uint32_t)n), kThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace qv
