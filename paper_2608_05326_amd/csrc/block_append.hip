// New tokens of many sequences behind the tokens a block cache holds, the keys with their
// rotation on the way: row i of place s becomes token lens[s] + i.  A block that is complete
// by them is quantized from the old open block's bf16 rows and the new ones (as k_block_store
// does, write-once codes), the rows behind the last complete block become the open block.
#include "qv_block.h"
#include "qv_rotary.h"

namespace qv {

// One workgroup per (block that the new tokens touch, KV head, keys or values).  The place's
// last, open block is written by the workgroup of the first one, after it has read the old
// open block: both are in the same rows.
__global__ __launch_bounds__(kThreads) void k_block_append(BlockArgs a, AppendRows r, RotaryArgs rot) {
  __shared__ CloseLds sm;
  const bool values = blockIdx.x & 1;
  const int g = (blockIdx.x >> 1) % a.H_kv;
  PackedTile w;
  // (n rows touch at most floor(n / 64) + 2 blocks: the numbers of sequence s begin at
  // floor(cu[s] / 64) + 2 s)
  if (!find_tile(r.cu, a.B, r.total, 1, kBlk, (blockIdx.x >> 1) / a.H_kv, &w, 2)) return;
  const int held = a.lens[w.seq];
  if (held < 0 || held >= a.max_context) return;
  int n = min(w.len, a.max_context - held);
  if (r.counts) n = min(n, r.counts[w.seq]);
  if (n <= 0) return;
  const int first = held / kBlk, last = (held + n - 1) / kBlk, blk = first + w.tile;
  if (blk > last) return;
  const int64_t st = values ? r.v_st : r.k_st;
  const uint16_t* x = values ? r.v + g * r.v_sh : r.k + g * r.k_sh;
  uint16_t* tail = (values ? a.v_tail : a.k_tail) + ((int64_t)w.seq * a.H_kv + g) * kCodes;
  const int c = threadIdx.x & 15, m = threadIdx.x >> 4;   // channels 8 c .. + 7
  const bool rotate = r.rotate && !values && 16 * c < 4 * rot.n_pairs;
  // where this chunk's pairs are, and the chunk with their other channels
  const int half = rot.n_pairs >> 3;
  const bool second = rot.interleaved ? c & 1 : c >= half;
  const int other = rot.interleaved ? c ^ 1 : second ? c - half : c + half;
  const int pair0 = rot.interleaved ? 8 * (c >> 1) : 8 * (second ? c - half : c);

  // chunk c of the place's token at position p (a new one), rotated
  auto new_row = [&](int p) -> u32x4 {
    const int64_t row = w.start + (p - held);
    u32x4 u = *(const u32x4*)(x + row * st + 8 * c);
    if (rotate) {
      u32x4 v = *(const u32x4*)(x + row * st + 8 * other);
      int32_t at[kMaxAxes];
      row_positions(rot, row, at);
      float2 cs[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) cs[i] = pair_cos_sin(rot, pair0 + i, at);
      if (second) {
        rotate_pairs(v, u, cs, rot.interleaved);
      } else {
        rotate_pairs(u, v, cs, rot.interleaved);
      }
    }
    return u;
  };

  if (held + n >= (blk + 1) * kBlk) {
    u32x4 y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = blk * kBlk + 4 * m + i;
      y[i] = p < held ? *(const u32x4*)(tail + (p % kBlk) * kHeadDim + 8 * c) : new_row(p);
    }
    const int page = page_of(a, w.seq, blk);
    if (page >= 0) {
      const int64_t e = (int64_t)page * a.H_kv + g;
      if (values) close_rows<true>(y, a.v_codes + e * kCodes, a.v_scale + e, sm);
      else close_rows<false>(y, a.k_codes + e * kCodes, a.k_scale + e, sm);
    }
    // rows of the block that stays open; the old ones have been read (a block without a page
    // reads none that matter)
    if (blk != first || (held + n) % kBlk == 0) return;
    __syncthreads();
    for (int p = last * kBlk + m; p < held + n; p += kThreads / 16)
      *(u32x4*)(tail + (p % kBlk) * kHeadDim + 8 * c) = new_row(p);
  } else if (blk == first) {
    for (int p = held + m; p < held + n; p += kThreads / 16)
      *(u32x4*)(tail + (p % kBlk) * kHeadDim + 8 * c) = new_row(p);
  }
}

// Workgroups (an upper bound).
int64_t block_append_groups(int64_t total, int n_seqs, int H_kv) {
  return 2 * (total / kBlk + 2 * (int64_t)n_seqs) * H_kv;
}

hipError_t launch_block_append(const BlockArgs& a, const AppendRows& r, const RotaryArgs& rot, hipStream_t st) {
  const int64_t n = block_append_groups(r.total, a.B, a.H_kv);
  k_block_append<<<dim3((uint32_t)n), kThreads, 0, st>>>(a, r, rot);
  return hipGetLastError();
}

}  // namespace qv
