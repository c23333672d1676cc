// Rotary positions: pair i of a head's channels is turned by the angle p f_i, p the token's
// position along the axis that the pair follows.  Angles are held in turns of 2^-64: with
// F_i = f_i / 2 pi 2^64 the product p F_i, modulo 2^64, is the angle modulo a turn, for
// every 32-bit position and with an error of |p| 2^-65 turns (the rounding of F_i): no
// table, and far positions are as exact as near ones.
#pragma once
#include "qv_device.h"

namespace qv {

constexpr int kMaxPairs = kHeadDim / 2, kMaxAxes = 4;

struct RotaryArgs {
  uint64_t turns[kMaxPairs];   // F_i (the inverse rotation: -F_i)
  uint32_t axis[kMaxPairs / 4];   // four pairs a word
  int32_t n_pairs;             // a multiple of 8; channels past 2 n_pairs are left as they are
  int32_t n_axes;
  int32_t interleaved;         // pairs (2 i, 2 i + 1), else (i, i + n_pairs)
  const int32_t* pos;          // position of row r along axis a: pos[r p_st + a p_sa]
  int64_t p_st, p_sa;
};

// cos and sin of u 2^-32 turns, to 2^-23.4 (the largest error over the range; a product with a
// bf16 value is rounded by 2^-8 in the end).  The nearest quarter turn is taken off, the
// rest (at most pi / 4) goes into the Taylor series, whose first terms left out are
// x^11 / 11! < 2^-29 and x^10 / 10! < 2^-25.
__device__ __forceinline__ float2 cos_sin(uint32_t u) {
  const uint32_t quarter = (u + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(u - (quarter << 30)) * 0x1.921fb6p-30f;   // 2 pi 2^-32
  const float z = x * x;
  float s = fmaf(z, 1.f / 362880.f, -1.f / 5040.f);
  s = fmaf(z, s, 1.f / 120.f);
  s = fmaf(z, s, -1.f / 6.f);
  s = fmaf(z * x, s, x);
  float c = fmaf(z, 1.f / 40320.f, -1.f / 720.f);
  c = fmaf(z, c, 1.f / 24.f);
  c = fmaf(z, c, -0.5f);
  c = fmaf(z, c, 1.f);
  const bool swap = quarter & 1;
  const float a = swap ? s : c, b = swap ? c : s;
  // quarter 1: (-s, c), 2: (-c, -s), 3: (s, -c)
  return make_float2(__uint_as_float(__float_as_uint(a) ^ ((quarter + 1) << 30 & 0x80000000u)),
                     __uint_as_float(__float_as_uint(b) ^ (quarter << 30 & 0x80000000u)));
}

// The angle at position p of a pair with F = turns, in 2^-32 turns (rounded).
__device__ __forceinline__ uint32_t turned(uint64_t turns, int32_t p) {
  return (uint32_t)(((uint64_t)(int64_t)p * turns + 0x80000000u) >> 32);
}

// The pairs' tables in LDS, staged by 256 threads (a barrier follows).  Scalar loads: a launch's
// arguments are in memory that vector loads read anew for every wave.
struct alignas(16) RotaryLds {
  uint64_t turns[kMaxPairs];
  uint32_t axis[kMaxPairs / 4];
};
__device__ __forceinline__ void stage_rotary(const RotaryArgs& r, RotaryLds& t) {
  static_assert(kMaxPairs % 16 == 0);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (w >= kMaxPairs / 16) return;
  uint64_t f[16];
  uint32_t ax[4];
#pragma unroll
  for (int i = 0; i < 16; ++i) f[i] = r.turns[16 * w + i];
#pragma unroll
  for (int i = 0; i < 4; ++i) ax[i] = r.axis[4 * w + i];
  if (threadIdx.x & 63) return;
#pragma unroll
  for (int i = 0; i < 16; ++i) t.turns[16 * w + i] = f[i];
#pragma unroll
  for (int i = 0; i < 4; ++i) t.axis[4 * w + i] = ax[i];
}

// cos and sin of pair i for a token with the positions p[axis]
__device__ __forceinline__ float2 pair_cos_sin(const RotaryLds& r, int i, const int32_t (&p)[kMaxAxes]) {
  const int a = r.axis[i >> 2] >> 8 * (i & 3) & 0xFF;
  const int32_t at = a < 2 ? (a ? p[1] : p[0]) : (a == 2 ? p[2] : p[3]);
  return cos_sin(turned(r.turns[i], at));
}

__device__ __forceinline__ void row_positions(const RotaryArgs& r, int64_t row, int32_t (&p)[kMaxAxes]) {
#pragma unroll
  for (int a = 0; a < kMaxAxes; ++a) p[a] = a < r.n_axes ? r.pos[row * r.p_st + a * r.p_sa] : 0;
}

__device__ __forceinline__ uint32_t pack_rne(float lo, float hi) {
  const bf16x2 p = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, p);
}
// (x, y) turned by the angle of cs
__device__ __forceinline__ float turn_x(float x, float y, float2 cs) { return fmaf(x, cs.x, -(y * cs.y)); }
__device__ __forceinline__ float turn_y(float x, float y, float2 cs) { return fmaf(y, cs.x, x * cs.y); }

// Two channels of a word that are a pair
__device__ __forceinline__ uint32_t turn_word(uint32_t w, float c, float s) {
  const float x = __uint_as_float(w << 16), y = __uint_as_float(w & 0xFFFF0000u);
  return pack_rne(turn_x(x, y, make_float2(c, s)), turn_y(x, y, make_float2(c, s)));
}
// Two channels whose other channels are in another word: the second (turn_y) or first (turn_x)
// of their pairs; cs the two angles.
__device__ __forceinline__ uint32_t turn_halves(uint32_t own, uint32_t other, f32x4 cs, bool second) {
  const uint32_t flip = second ? 0 : 0x80000000u;
  auto f = [&](uint32_t x, uint32_t y, float c, float s) {
    const float b = __uint_as_float(y) * s;
    return fmaf(__uint_as_float(x), c, __uint_as_float(__float_as_uint(b) ^ flip));
  };
  return pack_rne(f(own << 16, other << 16, cs[0], cs[1]), f(own & 0xFFFF0000u, other & 0xFFFF0000u, cs[2], cs[3]));
}

// Eight pairs: x, y are their channels in bf16, eight and eight (apart) or in turn
// (interleaved: x the first four pairs, y the others).
__device__ __forceinline__ void rotate_pairs(u32x4& x, u32x4& y, const float2 (&cs)[8], bool interleaved) {
  auto lo = [](uint32_t w) { return __uint_as_float(w << 16); };
  auto hi = [](uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); };
  u32x4 u, v;
  if (interleaved) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t a = x[j], b = y[j];
      u[j] = pack_rne(turn_x(lo(a), hi(a), cs[j]), turn_y(lo(a), hi(a), cs[j]));
      v[j] = pack_rne(turn_x(lo(b), hi(b), cs[j + 4]), turn_y(lo(b), hi(b), cs[j + 4]));
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t a = x[j], b = y[j];
      u[j] = pack_rne(turn_x(lo(a), lo(b), cs[2 * j]), turn_x(hi(a), hi(b), cs[2 * j + 1]));
      v[j] = pack_rne(turn_y(lo(a), lo(b), cs[2 * j]), turn_y(hi(a), hi(b), cs[2 * j + 1]));
    }
  }
  x = u;
  y = v;
}

}  // namespace qv
