// Rotary positions on packed queries and keys (Sec. 4.3, the rotation that attention's keys
// and queries carry), with one to four axes: text, or time, height and width of images and
// video.
#include <algorithm>

#include "qv_rotary.h"

namespace qv {

// Every value is read and written once, 3 flops each: bound by memory (32K tokens of 32 + 8 heads
// 127 us, 5.3 TB/s, where a copy of as many bytes takes as long and an elementwise one of 4 GB
// reaches 6.27; 5000 of 64 + 8 heads 42 us).  A thread computes the angles of
// eight pairs of one token once and takes them through up to eight heads (two loads of 16
// bytes a head); eight threads a token.  The workgroups of a token's heads are neighbours, so
// that their rows, which are, are read at about the same time (tokens as neighbours: 160 us).
namespace {
constexpr int kRotThreads = 256, kTokens = kRotThreads / 8;
}

__global__ __launch_bounds__(kRotThreads) void k_rotate(RotateArgs a, RotaryArgs r) {
  __shared__ RotaryLds tables;
  stage_rotary(r, tables);
  __syncthreads();
  const int j = threadIdx.x & 7;
  const int sets = (a.H_q + a.H_k + a.heads - 1) / a.heads;
  const int64_t row = (int64_t)(blockIdx.x / sets) * kTokens + (threadIdx.x >> 3);
  if (row >= a.total) return;
  int32_t p[kMaxAxes];
  row_positions(r, row, p);
  const bool turned = 8 * j < r.n_pairs;
  float2 cs[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) cs[i] = turned ? pair_cos_sin(tables, 8 * j + i, p) : make_float2(1.f, 0.f);
  const bool apart = turned && !r.interleaved;
  const int cx = apart ? 8 * j : 16 * j, cy = apart ? 8 * j + r.n_pairs : 16 * j + 8;
  const int h0 = blockIdx.x % sets * a.heads, h1 = min(h0 + a.heads, a.H_q + a.H_k);
  for (int h = h0; h < h1; ++h) {
    const bool q = h < a.H_q;
    const uint16_t* x = q ? a.q + row * a.q_st + h * a.q_sh : a.k + row * a.k_st + (h - a.H_q) * a.k_sh;
    uint16_t* y = q ? a.q_out + row * a.qo_st + h * a.qo_sh : a.k_out + row * a.ko_st + (h - a.H_q) * a.ko_sh;
    u32x4 u = *(const u32x4*)(x + cx), v = *(const u32x4*)(x + cy);
    if (turned) rotate_pairs(u, v, cs, r.interleaved);
    *(u32x4*)(y + cx) = u;
    *(u32x4*)(y + cy) = v;
  }
}

hipError_t launch_rotate(RotateArgs a, const RotaryArgs& r, hipStream_t st) {
  const int64_t n = (a.total + kTokens - 1) / kTokens;
  const int H = a.H_q + a.H_k;
  // few tokens: fewer heads, down to one, while the workgroups are few (512 tokens 5.9 us; with
  // eight heads always 9.0; from 2048 tokens on both are the same)
  a.heads = 8;
  while (a.heads > 1 && n * H < 512 * a.heads) a.heads /= 2;
  k_rotate<<<(uint32_t)(n * ((H + a.heads - 1) / a.heads)), kRotThreads, 0, st>>>(a, r);
  return hipGetLastError();
}

}  // namespace qv
