// New tokens of many sequences behind the tokens a block cache holds, the keys with their
// rotation on the way: row i of place s becomes token lens[s] + i.  A block that is complete
// by them is quantized from the old open block's bf16 rows and the new ones (as k_block_store
// does, write-once codes), the rows behind the last complete block become the open block.
#include "qv_block.h"
#include "qv_rotary.h"

namespace qv {

// One workgroup per (block that the new tokens touch, KV head, keys or values); keys that are
// rotated may take two heads, one behind the other.  The angles of a block's rows and pairs
// are computed once, by all threads, and kept in LDS: a pair's cosine and sine cost some 30
// vector instructions.  The first head's rows are on their way meanwhile.  A channel then is one
// product and one fused product, with the same roundings as k_rotate's.  The place's last, open
// block is written by the workgroup of the first one, after it has read the old open block: both
// are in the same rows.
// A token and head is 512 bytes read and 256 written.  Not yet bound by memory: 11770 tokens of 8
// heads 28.5 us (25 without the rotation), 18503 45.5 us, 2.5 TB/s.  What a workgroup does one after
// the other (place, positions, angles, rows, largest magnitude, codes) is hidden by four waves a
// SIMD only: 126 registers and 33 KB of LDS, which the angles need and which the workgroups that
// rotate nothing have, too.  (k_block_store, the same without angles at 47 registers and eight
// waves a SIMD, moves 5.2 TB/s.)
namespace {
// The angles (cosine and sine of pair i at angle_at(row, i)) are in the place of the values'
// codes: four workgroups a compute unit.
union AppendLds {
  CloseLds close;
  struct {
    uint32_t amax[kThreads / 64];   // as in CloseLds
    alignas(16) float2 cs[kBlk][kMaxPairs];
  } keys;
};
__device__ __forceinline__ int angle_at(int row, int pair) { return pair ^ (row & 7) << 1; }
}  // namespace
__global__ __launch_bounds__(kThreads, 4) void k_block_append(BlockArgs a, AppendRows r, RotaryArgs rot) {
  __shared__ AppendLds sm;
  __shared__ RotaryLds tables;
  const bool values = (int)blockIdx.x >= r.key_groups;
  const int heads = values ? 1 : r.heads, sets = (a.H_kv + heads - 1) / heads;
  const int idx = values ? blockIdx.x - r.key_groups : blockIdx.x;
  const int g0 = idx % sets * heads, g1 = min(g0 + heads, a.H_kv);
  PackedTile w;
  // (n rows touch at most floor(n / 64) + 2 blocks: the numbers of sequence s begin at
  // floor(cu[s] / 64) + 2 s)
  if (!find_tile(r.cu, a.B, r.total, 1, kBlk, idx / sets, &w, 2)) return;
  const int held = a.lens[w.seq];
  if (held < 0 || held >= a.max_context) return;
  int n = min(w.len, a.max_context - held);
  if (r.counts) n = min(n, r.counts[w.seq]);
  if (n <= 0) return;
  const int first = held / kBlk, last = (held + n - 1) / kBlk, blk = first + w.tile;
  if (blk > last) return;
  const int64_t st = values ? r.v_st : r.k_st, sh = values ? r.v_sh : r.k_sh;
  const uint16_t* rows = (values ? r.v : r.k) + ((int64_t)w.start - held) * st;   // of position 0
  uint16_t* tails = (values ? a.v_tail : a.k_tail) + (int64_t)w.seq * a.H_kv * kCodes;
  const int c = threadIdx.x & 15, m = threadIdx.x >> 4;   // channels 8 c .. + 7
  const bool rotate = r.rotate && !values && 16 * c < 4 * rot.n_pairs;
  // where this chunk's pairs are, and the chunk with their other channels
  const int half = rot.n_pairs >> 3;
  const bool second = c >= half;
  const int other = second ? c - half : c + half, pair0 = 8 * (second ? c - half : c);

  // the angles of positions p0 .. p0 + 63 that are new: a wave has a row at a time, a lane a pair
  auto find_angles = [&](int p0) {
    const int i = threadIdx.x & 63;
    if (i >= rot.n_pairs) return;
    const uint64_t turns = tables.turns[i];
    const int axis = tables.axis[i >> 2] >> 8 * (i & 3) & 0xFF;
    const int32_t* pos = rot.pos + ((int64_t)w.start - held) * rot.p_st + axis * rot.p_sa;
#pragma unroll 4
    for (int k = 0; k < kBlk; k += kThreads / 64) {
      const int t = k + (threadIdx.x >> 6), p = p0 + t;
      if (p >= held && p < held + n) sm.keys.cs[t][angle_at(t, i)] = cos_sin(turned(turns, pos[p * rot.p_st]));
    }
  };
  // chunk c of the token at position p in KV head g, as it is in memory
  auto row = [&](int p, int g) -> u32x4 {
    return *(const u32x4*)((p < held ? tails + g * kCodes + p % kBlk * kHeadDim : rows + p * st + g * sh) + 8 * c);
  };
  // u, chunk c of the new token at position p, turned; all lanes that have the token's chunks call it
  auto turn = [&](int p, u32x4 u) -> u32x4 {
    auto cs = [&](int i) { return *(const f32x4*)&sm.keys.cs[p % kBlk][angle_at(p % kBlk, i)]; };
    if (rot.interleaved) {
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        const f32x4 t = cs(4 * c + i);
        u[i] = turn_word(u[i], t[0], t[1]);
        u[i + 1] = turn_word(u[i + 1], t[2], t[3]);
      }
    } else {
      u32x4 v;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = __shfl((int)u[i], other, 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) u[i] = turn_halves(u[i], v[i], cs(pair0 + 2 * i), second);
    }
    return u;
  };

  if (r.rotate && !values) {
    stage_rotary(rot, tables);
    __syncthreads();
  }
  const bool whole = held + n >= (blk + 1) * kBlk;
  const int page = whole ? page_of(a, w.seq, blk) : -1;
  if (page >= 0) {
    const int p0 = blk * kBlk + 4 * m;
    u32x4 x[4], y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = row(p0 + i, g0);
    if (r.rotate && !values) {
      find_angles(blk * kBlk);
      __syncthreads();
    }
    for (int g = g0; g < g1; ++g) {
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = rotate && p0 + i >= held ? turn(p0 + i, x[i]) : x[i];
      if (g + 1 < g1)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = row(p0 + i, g + 1);
      const int64_t e = (int64_t)page * a.H_kv + g;
      if (values) close_rows<true>(y, a.v_codes + e * kCodes, a.v_scale + e, sm.close);
      else close_rows<false>(y, a.k_codes + e * kCodes, a.k_scale + e, sm.close);
      if (g + 1 < g1) __syncthreads();   // sm is read
    }
  }
  // the rows of the block that stays open; the old ones have been read
  if (blk != first || (held + n) % kBlk == 0) return;
  if (whole) __syncthreads();
  if (r.rotate && !values) {
    find_angles(last * kBlk);
    __syncthreads();
  }
  for (int p = max(held, last * kBlk) + m; p < held + n; p += kThreads / 16)
    for (int g = g0; g < g1; ++g) {
      const u32x4 u = row(p, g);
      *(u32x4*)(tails + g * kCodes + p % kBlk * kHeadDim + 8 * c) = rotate ? turn(p, u) : u;
    }
}

// Blocks that a call may touch (an upper bound), and workgroups.
static int64_t touched(int64_t total, int n_seqs) { return total / kBlk + 2 * (int64_t)n_seqs; }
int64_t block_append_groups(int64_t total, int n_seqs, int H_kv) { return 2 * touched(total, n_seqs) * H_kv; }

hipError_t launch_block_append(const BlockArgs& a, AppendRows r, const RotaryArgs& rot, hipStream_t st) {
  const int64_t n = touched(r.total, a.B);
  // two heads where the workgroups are many all the same (18503 tokens: one head 58 us, two 49,
  // four 54)
  r.heads = 1;
  if (r.rotate)
    while (r.heads < 2 && r.heads < a.H_kv && n * a.H_kv / (2 * r.heads) >= 512) r.heads *= 2;
  r.key_groups = (int32_t)(n * ((a.H_kv + r.heads - 1) / r.heads));
  k_block_append<<<dim3((uint32_t)(r.key_groups + n * a.H_kv)), kThreads, 0, st>>>(a, r, rot);
  return hipGetLastError();
}

}  // namespace qv
