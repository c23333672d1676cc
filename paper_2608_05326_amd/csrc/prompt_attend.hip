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
// are the eight consecutive keys the second product wants from it: P goes from the first
// product's result to the second's operand without moving between lanes.
// P enters the second product in bf16 (off by at most 2^-8 of itself, the size of the
// output's own rounding; against 64 bits the output is off by 0.0018 to 0.0022 of its norm,
// 0.0016 where only the output is rounded), the sum takes it unrounded; logits, maximum, sum
// and output are held in 32 bits.
//
// Per 32 rows and 64 keys a wave issues 32 products (1024 cycles), 32 exponentials and
// about 120 other vector instructions (some 730 cycles) and reads 32 KB of LDS; two waves
// share a SIMD so that one's products run beside the other's exponentials.  A 32K prompt of
// 32/8 heads takes 7.7 ms (1145 TFLOP/s, a large bf16 matrix product reaches 1260 on such a
// card); with all inputs zero the same instructions run at 1430, so at that size the
// clock under load bounds it: orders of the loads, priorities and a barrier that keeps
// the two waves half a tile apart moved it by 4% at most.
#include <algorithm>

#include "qv_device.h"

namespace qv {

namespace {
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr int kRowBytes = 2 * kHeadDim;
constexpr int kAhead = 3;       // steps that key operands are read ahead
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

// RS row sets of 32 rows, KG waves a row set: with one, a wave takes all keys of a 64-key
// tile; with more, each takes 32 keys of a tile of 32 KG (they are joined at the end).
template <int RS, int KG>
__global__ __launch_bounds__(64 * RS * KG, 2) void k_prompt_attend(PromptArgs a) {
  constexpr int kWaves = RS * KG;
  constexpr int kRows = 32 * RS;                 // (position, head) rows of the workgroup
  constexpr int kKeys = KG == 1 ? 64 : 32 * KG;  // keys per tile
  constexpr int KT = KG == 1 ? 2 : 1;            // 32-key tiles of a wave in it
  // two tiles of keys and values, in four arrays: reads of one tile do not wait for the
  // loads of the next (the compiler tells arrays apart, not parts of one)
  __shared__ __attribute__((aligned(16))) uint8_t sk0[kKeys * kRowBytes];
  __shared__ __attribute__((aligned(16))) uint8_t sv0[kKeys * kRowBytes];
  __shared__ __attribute__((aligned(16))) uint8_t sk1[kKeys * kRowBytes];
  __shared__ __attribute__((aligned(16))) uint8_t sv1[kKeys * kRowBytes];
  __shared__ int sodd[2][kWaves];   // a tile held values that are not finite
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, lh = lane >> 5;

  // ---- this workgroup's KV head, prompt and rows, the longest tile of a prompt first
  const int g = (int)(blockIdx.x % a.H_kv) + touch_kernargs<sizeof(PromptArgs)>();
  PackedTile pt;
  int slot = blockIdx.x / a.H_kv;
  if (slot >= a.fold && slot < a.fold_end) slot = a.fold + a.fold_end - 1 - slot;
  if (!find_tile(a.cu, a.n_seqs, a.total, a.gqa, kRows, slot, &pt)) return;
  const int start = pt.start, len = pt.len, tile = pt.n_tiles - 1 - pt.tile;
  const int n_rows = len * a.gqa, row0 = tile * kRows;   // at most 2^30 (checked on the host)
  const int rw = wave % RS, kg = wave / RS, kw = 32 * kg;   // the wave's row set and first key
  const int pos_first = row0 / a.gqa, pos_last = min(row0 + kRows - 1, n_rows - 1) / a.gqa;   // of the workgroup
  const int n_tiles = pos_last / kKeys + 1;

  const uint16_t* kp = a.k + (int64_t)start * a.k_st + g * a.k_sh;
  const uint16_t* vp = a.v + (int64_t)start * a.v_st + g * a.v_sh;
  // Starts the loads of a tile straight into LDS: a wave's instruction fills four rows, its
  // lanes in order, so the swizzle is applied to the chunk a lane fetches.  Byte offsets in
  // a tile fit 32 bits (checked on the host).
  constexpr int kLoads = kKeys / 4 / kWaves;
  const int fr0 = kKeys / kWaves * wave, fr = fr0 + (lane >> 4);
  uint32_t koff[kLoads], voff[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int r = fr + 4 * i;
    koff[i] = (uint32_t)r * (uint32_t)(2 * a.k_st) + 16 * ((lane & 15) ^ swz_k(r));
    voff[i] = (uint32_t)r * (uint32_t)(2 * a.v_st) + 16 * ((lane & 15) ^ swz_v(r));
  }
  // Keys past the prompt repeat its last (they are masked): the offsets of the last tile,
  // which is the last to be loaded.
  auto clamp = [&](int t, int64_t stride, uint32_t (&off)[kLoads]) __attribute__((always_inline)) {
    const int past = t * kKeys + kKeys - len;
    if (past <= 0) return;
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      off[i] -= (uint32_t)max(fr + 4 * i - (kKeys - 1 - past), 0) * (uint32_t)(2 * stride);
  };
  auto fetch = [&](int t, const uint16_t* base, int64_t stride, const uint32_t (&off)[kLoads], uint8_t* tile,
                   int i) __attribute__((always_inline)) {
    if (t < n_tiles)
      dma16((const uint8_t*)(base + (int64_t)t * kKeys * stride) + off[i], tile + (fr0 + 4 * i) * kRowBytes);
  };
  clamp(0, a.k_st, koff);
#pragma unroll
  for (int i = 0; i < kLoads; ++i) fetch(0, kp, a.k_st, koff, sk0, i);

  // this lane's row (rows past the prompt's last repeat it and are not stored)
  const int row = row0 + rw * 32 + lr;
  const int rowc = min(row, n_rows - 1);
  const int pos = rowc / a.gqa, head = g * a.gqa + rowc % a.gqa;
  // first and last position of the wave's rows, and the tiles in which it has keys to see
  const int wpos0 = (row0 + rw * 32) / a.gqa, wpos1 = min(row0 + rw * 32 + 31, n_rows - 1) / a.gqa;
  const int n_mine = row0 + rw * 32 < n_rows && wpos1 >= kw ? (wpos1 - kw) / kKeys + 1 : 0;
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

  // LDS offsets: A operand row lr of a 32-key tile is key krow of it; the swizzles leave
  // k-step ks at kbase ^ 32 ks (keys) and channels 32 c .. at vbase[] ^ 64 c (values of keys
  // 8 lh .. + 3 and + 4 .. + 7)
  const int krow = kw + 16 * (lr >> 4) + 8 * ((lr >> 2) & 1) + 4 * ((lr >> 3) & 1) + (lr & 3);
  const int kbase = krow * kRowBytes + 16 * (lh ^ swz_k(krow));
  int vbase[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int key = kw + 8 * lh + 4 * j + ((lane >> 2) & 3);
    vbase[j] = key * kRowBytes + 16 * ((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ swz_v(key)) + 8 * (lane & 1);
  }

  // only tiles that reach past the workgroup's first position hold masked keys
  auto edge = [&](int t) { return t * kKeys + kKeys - 1 > pos_first; };
  f32x16 s[KT];
  u32x4 p[2 * KT];

  // o += V^T P^T of tile t.  Operands are read ahead of their products: a read takes longer
  // than the products of one step.  `beside` goes with each step's.
  auto values = [&](int t, const uint8_t* sv, auto beside) __attribute__((always_inline)) {
    u32x4 vv[2][4];
    auto read_v = [&](int ks) {
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(
                                                      sv + (vbase[0] ^ (64 * c)) + 16 * ks * kRowBytes)));
        const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(
                                                      sv + (vbase[1] ^ (64 * c)) + 16 * ks * kRowBytes)));
        vv[ks & 1][c] = (u32x4){x[0], x[1], y[0], y[1]};
      }
    };
    read_v(0);
#pragma unroll
    for (int ks = 0; ks < 2 * KT; ++ks) {
      if (ks + 1 < 2 * KT) read_v(ks + 1);
      beside(ks);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int c = 0; c < 4; ++c) o[c] = mfma32(vv[ks & 1][c], p[ks], o[c]);
      __builtin_amdgcn_sched_barrier(0);
    }
    // o[c][i]: channel 32 c + 8 (i / 4) + 4 lh + i % 4 of this lane's row
    if (edge(t)) {
      int odd = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) odd |= sodd[t & 1][w];
      if (__builtin_amdgcn_readfirstlane(odd)) {   // the values left out of the tile
        for (int r = kw; r < kw + 32 * KT && t * kKeys + r <= pos; ++r) {
          const uint16_t* vr = vp + (int64_t)(t * kKeys + r) * a.v_st + 4 * lh;
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const uint16_t x = vr[32 * c + 8 * (i >> 2) + (i & 3)];
              if ((x & 0x7F80u) == 0x7F80u) o[c][i] += bf16_to_f32(x);
            }
        }
      }
    }
  };
  // s = K Q^T of tile t
  auto logits = [&](const uint8_t* sk, auto beside) __attribute__((always_inline)) {
    u32x4 kk[kAhead][KT];
    auto read_k = [&](int ks) {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
        kk[ks % kAhead][kt] = *(const u32x4*)(sk + (kbase ^ (32 * ks)) + 32 * kt * kRowBytes);
    };
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[kt][i] = 0.f;
#pragma unroll
    for (int ks = 0; ks < kAhead; ++ks) read_k(ks);
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      beside(ks);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) s[kt] = mfma32(kk[ks % kAhead][kt], q[ks], s[kt]);
      __builtin_amdgcn_sched_barrier(0);
      if (ks + kAhead < 8) read_k(ks + kAhead);
    }
  };
  // p = exp2(s - m), l and o kept relative to m
  auto weights = [&](int t) __attribute__((always_inline)) {
    // s[kt][i]: raw logit of key t kKeys + kw + 32 kt + 16 (i / 8) + 8 lh + i % 8 for this lane's row
    if (t * kKeys + kw + 32 * KT - 1 > wpos0) {
      const int rel = pos - t * kKeys - kw - 8 * lh;
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (32 * kt + 16 * (i >> 3) + (i & 7) > rel) s[kt][i] = -INFINITY;
    }
    float mt = -INFINITY;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
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
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        const float e0 = __builtin_amdgcn_exp2f(fmaf(s[kt][i], sc, -mu));
        const float e1 = __builtin_amdgcn_exp2f(fmaf(s[kt][i + 1], sc, -mu));
        l += e0 + e1;
        p[2 * kt + (i >> 3)][(i & 7) >> 1] = pack_bf16(e0, e1);
      }
  };
  // A masked key's value must not reach a row through 0 * infinity: values that are not
  // finite leave an edge tile, in the rows this wave has loaded, and are added to the rows
  // that see them after its products.
  auto clean = [&](int t, uint8_t* sv) __attribute__((always_inline)) {
    int odd = 0;
#pragma unroll 1
    for (int i = 0; i < kLoads; ++i) {
      u32x4* const at = (u32x4*)(sv + (fr0 + 4 * i) * kRowBytes) + lane;
      u32x4 x = *at;
      bool bad = false;
#pragma unroll
      for (int j = 0; j < 4; ++j) bad |= nonfinite_pair(x[j]);
      if (bad) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if ((x[j] & 0x7F80u) == 0x7F80u) x[j] &= 0xFFFF0000u;
          if ((x[j] & 0x7F800000u) == 0x7F800000u) x[j] &= 0xFFFFu;
        }
        *at = x;
        odd = 1;
      }
    }
    odd = __any(odd);
    if (lane == 0) sodd[t & 1][wave] = odd;
  };
  // loads landed and LDS writes done, for all waves
  auto landed = [&]() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  // Tile t: the products of the values of the tile before and of its own keys, then its
  // weights.  Meanwhile the next tile's keys and its own values arrive; the arrays they
  // fill were last read in the products of the tile before.  Eight loads in a row hold a
  // wave for 500 to 800 cycles (a unit takes 64 bytes a cycle from all its waves).  Two
  // workgroups a unit fill that with each other's work; a lone one issues them one at a time
  // beside its products (one prompt of 2067 tokens and 8 heads 30 -> 28 us, but 8192 with
  // four waves 193 -> 211).
  auto step = [&](int t, uint8_t* sk, uint8_t* sv_before, uint8_t* sk_next,
                  uint8_t* sv) __attribute__((always_inline)) {
    if (t + 1 < n_tiles) clamp(t + 1, a.k_st, koff);
    clamp(t, a.v_st, voff);
    constexpr bool kSpread = KG > 1;
    auto next_keys = [&](int ks) __attribute__((always_inline)) {
      if constexpr (kSpread) {
#pragma unroll
        for (int i = ks * kLoads / (2 * KT); i < (ks + 1) * kLoads / (2 * KT); ++i)
          fetch(t + 1, kp, a.k_st, koff, sk_next, i);
      }
    };
    auto own_values = [&](int ks) __attribute__((always_inline)) {
      if constexpr (kSpread) {
        if (ks < kLoads) fetch(t, vp, a.v_st, voff, sv, ks);
      }
    };
    if constexpr (!kSpread) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) fetch(t + 1, kp, a.k_st, koff, sk_next, i);
#pragma unroll
      for (int i = 0; i < kLoads; ++i) fetch(t, vp, a.v_st, voff, sv, i);
    }
    if (t > 0 && t - 1 < n_mine) {
      values(t - 1, sv_before, next_keys);
    } else {
#pragma unroll
      for (int ks = 0; ks < 2 * KT; ++ks) next_keys(ks);
    }
    if (t < n_mine) {
      logits(sk, own_values);
    } else {
#pragma unroll
      for (int ks = 0; ks < 8; ++ks) own_values(ks);
    }
    if (t < n_mine) weights(t);
    if (edge(t)) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      clean(t, sv);
    }
    landed();
  };
  landed();
  for (int t = 0; t < n_tiles; t += 2) {
    step(t, sk0, sv1, sk1, sv0);
    if (t + 1 < n_tiles) step(t + 1, sk1, sv0, sk0, sv1);
  }
  if (n_tiles - 1 < n_mine) {
    if (n_tiles & 1) values(n_tiles - 1, sv0, [](int) {});
    else values(n_tiles - 1, sv1, [](int) {});
  }

  l = half_sum(l);
  // channels 32 c .. + 31 of the row, from the 16 of each lane half
  auto store = [&](int c, const f32x16& x, float inv) __attribute__((always_inline)) {
    uint16_t* op = a.out + (start + pos) * a.o_st + head * a.o_sh + 32 * c + 8 * lh;
#pragma unroll
    for (int e = 0; e < 4; e += 2) {   // channels 8 e .. 8 e + 15: eight to each lane half
      uint32_t y[2], z[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const auto sw = __builtin_amdgcn_permlane32_swap(
            pack_bf16(x[4 * e + 2 * j] * inv, x[4 * e + 2 * j + 1] * inv),
            pack_bf16(x[4 * e + 4 + 2 * j] * inv, x[4 * e + 5 + 2 * j] * inv), false, false);
        y[j] = sw[0];
        z[j] = sw[1];
      }
      if (row < n_rows) *(u32x4*)(op + 8 * e) = (u32x4){y[0], y[1], z[0], z[1]};
    }
  };
  if constexpr (KG == 1) {
    const float inv = 1.f / l;
#pragma unroll
    for (int c = 0; c < 4; ++c) store(c, o[c], inv);
  } else {
    // the waves of a row set put their maxima, sums and outputs (16 KB a wave) in the
    // tiles' arrays, and each joins 32 of the channels
    static_assert(KG == 4, "a wave for each 32 channels");
    __shared__ float2 sml[kWaves][64];
    constexpr int kPer = kKeys * kRowBytes / 16384;   // waves per array
    static_assert(kWaves == 4 * kPer, "room for the waves' outputs");
    auto rows_of = [&](int w) {
      uint8_t* const arr = w / kPer == 0 ? sk0 : w / kPer == 1 ? sv0 : w / kPer == 2 ? sk1 : sv1;
      return (float*)(arr + w % kPer * 16384) + lane;
    };
    __syncthreads();   // the tiles are consumed
    sml[wave][lane] = make_float2(m, l);
    float* mine = rows_of(wave);
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) mine[64 * (16 * c + i)] = o[c][i];
    __syncthreads();
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int j = 0; j < KG; ++j) M = fmaxf(M, sml[rw + j * RS][lane].x);
    const float mu = M > -INFINITY ? M : 0.f;
    f32x16 x;
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = 0.f;
#pragma unroll
    for (int j = 0; j < KG; ++j) {
      const float2 ml = sml[rw + j * RS][lane];
      const float f = __builtin_amdgcn_exp2f(ml.x - mu);
      L = fmaf(f, ml.y, L);
      const float* from = rows_of(rw + j * RS) + 64 * 16 * kg;
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = fmaf(f, from[64 * i], x[i]);
    }
    store(kg, x, 1.f / L);
  }
}

// Workgroups of a launch (an upper bound: every prompt's last tile may be a partial one).
static int64_t groups_of(int64_t total, int n_seqs, int gqa, int H_kv, int rows) {
  return (total * gqa / rows + n_seqs) * H_kv;
}
int64_t prompt_attend_groups(int64_t total, int n_seqs, int gqa, int H_kv) {
  return groups_of(total, n_seqs, gqa, H_kv, 64);
}

constexpr int kUnits = 256;   // compute units

// Which form: 128 rows and four waves that take all keys, two such workgroups to a compute
// unit, or 64 rows and eight waves, four to a row set, one to a unit.  The second ends its
// longest row sooner but pays its start and join for half as many rows.  Estimated from the
// prompts' mean length t, a launch takes the larger of its longest workgroup and its sum
// over the chip, in microseconds (measured: one prompt of 8 heads and 2067 tokens 47 and
// 28, 4096 89 and 60, 8192 192 and 218; 32/8 heads and 512 tokens 17 and 13, 2048 54 and
// 72; 32 prompts of 100 tokens 23 and 54).  The host sees the rows and the number of prompts
// only: one long prompt among short or empty ones, or beside rows outside all prompts, is
// taken for short ones (2067 tokens, 8 heads, beside 31 empty prompts 45 us instead of 27;
// 4000 beside fifteen of 16 tokens 82 instead of 56).
static bool eight_waves(const PromptArgs& a, int64_t n128, int64_t n64) {
  const float t = (float)a.total / a.n_seqs;
  const float four = std::max(t / 64 * 1.3f + 5.f, n128 * (t / 128 * 1.6f + 5.f) / (2 * kUnits));
  const float eight = std::max(t / 128 * 1.28f + 7.f, n64 * (t / 256 * 1.28f + 7.f) / kUnits);
  return n64 < 4096 && eight < four;
}

hipError_t launch_prompt_attend(PromptArgs a, hipStream_t st) {
  const int64_t n128 = groups_of(a.total, a.n_seqs, a.gqa, a.H_kv, 128);
  const int64_t n64 = groups_of(a.total, a.n_seqs, a.gqa, a.H_kv, 64);
  const bool eight = eight_waves(a, n128, n64);
  // Workgroups are dealt round the units, the longest first.  Where they fill the chip about
  // once (two to a unit), the second of each unit comes in reverse, the shortest beside the
  // longest: 8 heads of 8192 tokens 204 -> 194 us, 64/8 heads of 1024 35 -> 33.
  const int64_t slots = n128 / a.H_kv, first = kUnits / a.H_kv;
  a.fold = (int)std::min(first, slots);
  a.fold_end = (int)(eight || slots >= 4 * first ? a.fold : std::min(slots, 2 * first));
  if (eight) k_prompt_attend<2, 4><<<dim3((uint32_t)n64), 512, 0, st>>>(a);
  else k_prompt_attend<4, 1><<<dim3((uint32_t)n128), 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace qv
