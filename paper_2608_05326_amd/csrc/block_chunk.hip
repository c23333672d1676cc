// Attention of a chunk of new tokens of many sequences over the 8-bit block cache and the
// chunk itself: a piece of a prompt, drafted tokens to verify, or one token.
//
//   out_i = sum_j softmax_j(scale q_i . k_j) v_j,   j over the tokens held and the chunk's
//                                                   up to i
//
// The keys of a sequence are its tiles of 64 positions: complete blocks are pages (int8 codes
// with a scale), the others are rows in bf16, of the open block and then of the chunk.
#include <algorithm>

#include "qv_block.h"
#include "qv_chunk.h"

namespace qv {

namespace {
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kChunkThreads = 512, kWaves = 8;
constexpr int kRowBytes = 2 * kHeadDim;
// the running maximum is raised (and the output rescaled) only when a tile exceeds it by
// this many powers of two: P stays below 256
constexpr float kLazy = 8.f;
// a row's query is scaled by a power of two that takes its largest entry to [2^-20, 2^-19):
// products with the largest keys, of codes or bf16, and their sums stay in range
constexpr int kQueryExp = -20;

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
__device__ __forceinline__ bool nonfinite(uint32_t x) {   // of two bf16
  return (x & 0x7F80u) == 0x7F80u || (x & 0x7F800000u) == 0x7F800000u;
}
// four codes in bf16, where they are exact
__device__ __forceinline__ u32x2 codes_bf16(uint32_t w) {
  float f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = (float)(int8_t)(w >> (8 * i));
  return (u32x2){__builtin_amdgcn_perm(__float_as_uint(f[1]), __float_as_uint(f[0]), 0x07060302u),
                 __builtin_amdgcn_perm(__float_as_uint(f[3]), __float_as_uint(f[2]), 0x07060302u)};
}
__device__ __forceinline__ u32x4 codes_bf16(uint32_t w0, uint32_t w1) {
  const u32x2 a = codes_bf16(w0), b = codes_bf16(w1);
  return (u32x4){a[0], a[1], b[0], b[1]};
}

// The place in lane, with its length on the line.
__device__ __forceinline__ ChunkPlace lane_place(const BlockArgs& a, const ChunkStep& s, int place, int* start) {
  const int i = min(place, a.B - 1);
  const int b = min(max(s.cu[i], 0), s.total), e = min(max(s.cu[i + 1], b), s.total);
  *start = b;
  return chunk_place(place < a.B ? a.lens[i] : -1, e - b, a.gqa, a.max_context);
}
__device__ __forceinline__ int64_t wave_scan(int64_t x) {   // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t y = __shfl_up(x, d, 64);
    if (lane >= d) x += y;
  }
  return x;
}
__device__ __forceinline__ int64_t lane_of(int64_t x, int lane) {
  return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)x, lane) |
                   (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32);
}

// The line: walks over the row tiles that hold points of [x, end), one segment [from, to) of
// a row tile (points counted from its start) at a time.  The same in every lane.
struct Segment {
  ChunkPlace p;
  int seq, start, g, tile;   // start: the place's first row
  int64_t at;                // the row tile's start on the line
  int64_t from, to;
};
// Up to 64 places of the line, in LDS (registers are the products').
struct LinePlaces {
  int64_t incl[64];          // the line up to the end of the place
  int held[64], n[64], start[64];
};
__device__ __forceinline__ void put_places(const BlockArgs& a, const ChunkStep& s, int s0, int64_t base,
                                           LinePlaces& lp) {
  const int lane = threadIdx.x & 63;
  int start;
  const ChunkPlace p = lane_place(a, s, s0 + lane, &start);
  lp.incl[lane] = base + wave_scan(chunk_pair_cost(p) * a.H_kv);
  lp.held[lane] = p.held;
  lp.n[lane] = p.n;
  lp.start[lane] = start;
}
template <class F>
__device__ __forceinline__ void walk(const BlockArgs& a, int64_t x, int64_t end, const ChunkStep& s, LinePlaces& lp,
                                     F&& f) {
  const int lane = threadIdx.x & 63;
  int64_t base = 0;
  for (int s0 = 0; x < end; s0 += 64) {
    if (s0) {   // (the first 64 are there)
      if (s0 >= a.B) return;
      __syncthreads();
      if (threadIdx.x < 64) put_places(a, s, s0, base, lp);
      __syncthreads();
    }
    base = lane_of(lp.incl[63], 0);
    while (x < end && x < base) {
      const int w = __builtin_ctzll(__ballot(lp.incl[lane] > x));
      Segment g;
      g.seq = s0 + w;
      g.start = __builtin_amdgcn_readfirstlane(lp.start[w]);
      const int held = __builtin_amdgcn_readfirstlane(lp.held[w]), n = __builtin_amdgcn_readfirstlane(lp.n[w]);
      g.p = chunk_place(held, n, a.gqa, a.max_context);
      g.p.per = __builtin_amdgcn_readfirstlane(g.p.per);       // (divisions leave them in vector registers)
      g.p.tiles = __builtin_amdgcn_readfirstlane(g.p.tiles);
      const int64_t pair = chunk_pair_cost(g.p), last = lane_of(lp.incl[w], 0);
      const int64_t first = last - pair * a.H_kv;
      for (g.g = __builtin_amdgcn_readfirstlane((int)((x - first) / pair)); g.g < a.H_kv && x < end; ++g.g) {
        const int64_t at = first + g.g * pair;
        for (g.tile = __builtin_amdgcn_readfirstlane(chunk_tile_at(g.p, x - at)); g.tile < g.p.tiles && x < end; ++g.tile) {
          g.at = at + chunk_before(g.p, g.tile);
          const int64_t stop = min(end, g.at + chunk_cost(g.p, g.tile));
          g.from = x - g.at;
          g.to = stop - g.at;
          f(g);
          x = stop;
        }
      }
    }
  }
}
// The line's length; the first 64 places are put in lp (the whole workgroup).
__device__ __forceinline__ int64_t line_total(const BlockArgs& a, const ChunkStep& s, LinePlaces& lp) {
  if (threadIdx.x < 64) put_places(a, s, 0, 0, lp);
  __syncthreads();
  int64_t total = lane_of(lp.incl[63], 0);
  if (a.B > 64) {
    int64_t sum = 0;
    for (int s0 = 64; s0 < a.B; s0 += 64) {
      int start;
      sum += chunk_pair_cost(lane_place(a, s, s0 + (threadIdx.x & 63), &start));
    }
    total += lane_of(wave_scan(sum * a.H_kv), 63);
  }
  return total;
}

// Bytes between the rows of a wave's staged values, and of joined outputs (floats).
constexpr int kJoin = kHeadDim + 4;
constexpr int kLds = std::max(kWaves * kBlk * kRowBytes, kWaves * 32 * kJoin * (int)sizeof(float));
}  // namespace

__global__ __launch_bounds__(kChunkThreads, 2) void k_chunk_attend(BlockArgs a, ChunkStep s) {
  // 64 value rows of each wave; later the waves' outputs
  __shared__ __attribute__((aligned(16))) uint8_t lds[kLds];
  __shared__ float2 sml[kWaves][32];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, lh = lane >> 5;
  // parts of one KV head on one XCD (workgroup i runs on XCD i % 8)
  const int part = (blockIdx.x & 7) * (kChunkParts / 8) + (blockIdx.x >> 3);

  __shared__ LinePlaces lp;
  const int64_t total = line_total(a, s, lp), size = lane_of(chunk_part(total), 0);
  const int64_t begin = part * size, end = min(begin + size, total);

  const float qm = __builtin_amdgcn_frexp_mantf(a.scale_log2);
  const int qe0 = __builtin_amdgcn_frexp_expf(a.scale_log2);

  auto segment = [&](const Segment& sg) {
    const ChunkPlace& p = sg.p;
    const int v_all = chunk_key_tiles(p, sg.tile);
    const int lo = chunk_key_tile(sg.from), hi = chunk_key_tile(sg.to);
    if (lo >= hi) return;
    const int pos0 = sg.tile * p.per, n_rows = (chunk_end(p, sg.tile) - pos0) * a.gqa;
    const int row = min(lr, n_rows - 1), i_row = pos0 + row / a.gqa, head = sg.g * a.gqa + row % a.gqa;
    const int pos = p.held + i_row;                  // this lane's position
    const int last = p.held + p.n - 1;               // the place's last position
    // query: k-step 2 j + e covers channels 32 j + 16 lh + 8 e + 0 .. 7
    u32x4 q[8];
    const uint16_t* qp = s.q + (sg.start + i_row) * s.q_st + head * s.q_sh + 16 * lh;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) q[ks] = *(const u32x4*)(qp + 32 * (ks >> 1) + 8 * (ks & 1));
    uint32_t am = 0;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) am = amax_pair(q[ks], am);
    am = amax_bits(am);
    am = max(am, (uint32_t)__shfl_xor((int)am, 32, 64));
    const int ex = max((int)(am >> 23), 1) - 127;    // (a row of subnormals keeps its scale)
#pragma unroll
    for (int ks = 0; ks < 8; ++ks)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t w = q[ks][j];
        q[ks][j] = pack_bf16(ldexpf(lo_f32(w), kQueryExp - ex), ldexpf(hi_f32(w), kQueryExp - ex));
      }
    const int qe = qe0 + ex - kQueryExp;

    f32x16 o[4];
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[c][i] = 0.f;
    float m = -INFINITY, l = 0.f;
    f32x16 st[2];
    u32x4 pw[4];
    // weights from the raw logits st[kt][i] of keys 32 kt + 16 lh + i: exp2(st sc - m + ve),
    // with the sum l that leaves the values' scale 2^ve out
    auto weights = [&](float sc, float vs) __attribute__((always_inline)) {
      float mt = -INFINITY;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i) mt = fmaxf(mt, st[kt][i]);
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
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
          const float e0 = __builtin_amdgcn_exp2f(fmaf(st[kt][i], sc, -mu));
          const float e1 = __builtin_amdgcn_exp2f(fmaf(st[kt][i + 1], sc, -mu));
          l += e0 + e1;
          pw[2 * kt + (i >> 3)][(i & 7) >> 1] = pack_bf16(e0 * vs, e1 * vs);
        }
    };
    // row lr of an A operand is this key of 32
    const int krow = 16 * ((lr >> 2) & 1) + 4 * (lr >> 3) + (lr & 3);
    const int n_blk = p.held / kBlk;

    for (int t = lo + wave; t < hi; t += kWaves) {
      if (t < n_blk) {
        const int page = page_of(a, sg.seq, t);
        if (page < 0) continue;
        const int64_t e = (int64_t)page * a.H_kv + sg.g;
        const int8_t* kc = a.k_codes + e * kCodes + krow * kHeadDim + 16 * lh;
        const int8_t* vc = a.v_codes + e * kCodes + lr * kBlk + 16 * lh;
        u32x4 kb[8], vb[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) kb[i] = *(const u32x4*)(kc + 32 * (i >> 2) * kHeadDim + 32 * (i & 3));
        float sc = ldexpf(a.k_scale[e] * qm, qe);
        if (sc == INFINITY) sc = __FLT_MAX__;   // (a product of zero is a logit of zero)
        const float vs = a.v_scale[e];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
          for (int i = 0; i < 16; ++i) st[kt][i] = 0.f;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const u32x4 x = kb[4 * kt + j];
            st[kt] = mfma32(codes_bf16(x[0], x[1]), q[2 * j], st[kt]);
            st[kt] = mfma32(codes_bf16(x[2], x[3]), q[2 * j + 1], st[kt]);
          }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) vb[i] = *(const u32x4*)(vc + 32 * (i >> 1) * kBlk + 32 * (i & 1));
        weights(sc, vs);
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int kt = 0; kt < 2; ++kt) {
            const u32x4 x = vb[2 * c + kt];
            o[c] = mfma32(codes_bf16(x[0], x[1]), pw[2 * kt], o[c]);
            o[c] = mfma32(codes_bf16(x[2], x[3]), pw[2 * kt + 1], o[c]);
          }
      } else {
        // rows in bf16: positions of the open block, then of the chunk (past the last: the
        // last again, masked)
        const int64_t tail = ((int64_t)sg.seq * a.H_kv + sg.g) * kCodes;
        auto k_row = [&](int key) -> const uint16_t* {
          const int pp = min(t * kBlk + key, last);
          return pp < p.held ? a.k_tail + tail + (pp % kBlk) * kHeadDim
                             : s.k + (sg.start + (pp - p.held)) * s.k_st + sg.g * s.k_sh;
        };
        auto v_row = [&](int key) -> const uint16_t* {
          const int pp = min(t * kBlk + key, last);
          return pp < p.held ? a.v_tail + tail + (pp % kBlk) * kHeadDim
                             : s.v + (sg.start + (pp - p.held)) * s.v_st + sg.g * s.v_sh;
        };
        uint8_t* mine = lds + wave * (kBlk * kRowBytes);
        bool odd = false;
#pragma unroll 2
        for (int i = 0; i < 16; ++i) {
          const int key = 4 * i + (lane >> 4);
          u32x4 x = *(const u32x4*)(v_row(key) + 8 * (lane & 15));
          // a masked key's value must not reach a row through 0 * infinity: values that are
          // not finite are left out here and added below to the rows that see them
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (nonfinite(x[j])) {
              odd = true;
              if ((x[j] & 0x7F80u) == 0x7F80u) x[j] &= 0xFFFF0000u;
              if ((x[j] & 0x7F800000u) == 0x7F800000u) x[j] &= 0xFFFFu;
            }
          }
          *(u32x4*)(mine + key * kRowBytes + 16 * (lane & 15)) = x;
        }
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
          const uint16_t* kr = k_row(32 * kt + krow) + 16 * lh;
#pragma unroll
          for (int i = 0; i < 16; ++i) st[kt][i] = 0.f;
#pragma unroll
          for (int ks = 0; ks < 8; ++ks)
            st[kt] = mfma32(*(const u32x4*)(kr + 32 * (ks >> 1) + 8 * (ks & 1)), q[ks], st[kt]);
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (t * kBlk + 32 * kt + 16 * lh + i > pos) st[kt][i] = -INFINITY;
        }
        float sc = ldexpf(qm, qe);
        if (sc == INFINITY) sc = __FLT_MAX__;
        weights(sc, 1.f);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // this wave's rows are in LDS
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            u32x4 x;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const int key = 32 * (ks >> 1) + 16 * lh + 8 * (ks & 1) + 4 * j + ((lane >> 2) & 3);
              const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(
                  mine + key * kRowBytes + 64 * c + 32 * ((lane >> 4) & 1) + 8 * (lane & 3))));
              x[2 * j] = y[0];
              x[2 * j + 1] = y[1];
            }
            o[c] = mfma32(x, pw[ks], o[c]);
          }
        if (__any(odd)) {
          for (int key = 0; key < kBlk && t * kBlk + key <= pos; ++key) {
            const uint16_t* vr = v_row(key) + 4 * lh;
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const uint16_t x = vr[32 * c + 8 * (i >> 2) + (i & 3)];
                if ((x & 0x7F80u) == 0x7F80u) o[c][i] += bf16_to_f32(x);
              }
          }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      }
    }

    // ---- join the waves; o[c][i]: channel 32 c + 8 (i / 4) + 4 lh + i % 4 of row lr
    l = half_sum(l);
    __syncthreads();
    float* so = (float*)lds;
    sml[wave][lr] = make_float2(m, l);
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(f32x4*)(so + (wave * 32 + lr) * kJoin + 32 * c + 8 * i + 4 * lh) =
            (f32x4){o[c][4 * i], o[c][4 * i + 1], o[c][4 * i + 2], o[c][4 * i + 3]};
    __syncthreads();
    const bool whole = lo == 0 && hi == v_all;
    for (int e = tid; e < n_rows * (kHeadDim / 4); e += kChunkThreads) {
      const int r = e / (kHeadDim / 4), c = 4 * (e % (kHeadDim / 4));
      float M = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) M = fmaxf(M, sml[w][r].x);
      const float mu = M > -INFINITY ? M : 0.f;
      float L = 0.f;
      f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(sml[w][r].x - mu);
        L = fmaf(f, sml[w][r].y, L);
        const f32x4 y = *(const f32x4*)(so + (w * 32 + r) * kJoin + c);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = fmaf(f, y[i], x[i]);
      }
      if (whole) {
        uint16_t* op = s.out + (sg.start + pos0 + r / a.gqa) * s.o_st + (sg.g * a.gqa + r % a.gqa) * s.o_sh + c;
        *(u32x2*)op = (u32x2){pack_bf16(x[0] / L, x[1] / L), pack_bf16(x[2] / L, x[3] / L)};
      } else {
        const int64_t slot = (int64_t)chunk_slot(part, lo) * s.slot_rows + r;
        *(f32x4*)(s.part_o + slot * kHeadDim + c) = x;
        if (c == 0) s.part_ml[slot] = make_float2(M, L);
      }
    }
    __syncthreads();
  };
  walk(a, begin, end, s, lp, segment);
}

// Joins the row tiles that more than one part served: workgroup (w, r) takes rows 8 r .. + 7
// of the row tile in which part w begins, if w is the first part that begins inside it.
namespace {
constexpr int kMergeRows = 8;
}
__global__ __launch_bounds__(kThreads) void k_chunk_merge(BlockArgs a, ChunkStep s) {
  const int w = blockIdx.x + 1, r = blockIdx.y * kMergeRows + (threadIdx.x >> 5);
  __shared__ LinePlaces lp;
  const int64_t total = line_total(a, s, lp), size = lane_of(chunk_part(total), 0);
  const int64_t x0 = w * size;
  if (x0 >= total) return;
  walk(a, x0, x0 + 1, s, lp, [&](const Segment& sg) {
    if (sg.from == 0) return;                    // the cut is at its start
    if (x0 - size > sg.at) return;               // an earlier part begins inside it
    const ChunkPlace& p = sg.p;
    const int pos0 = sg.tile * p.per, n_rows = (chunk_end(p, sg.tile) - pos0) * a.gqa;
    if (blockIdx.y * kMergeRows >= n_rows) return;
    const int v_all = chunk_key_tiles(p, sg.tile);
    const int64_t stop = sg.at + chunk_cost(p, sg.tile);
    const int w1 = (int)((stop - 1) / size), c = 4 * (threadIdx.x & 31), rr = min(r, n_rows - 1);
    float M = -INFINITY, L = 0.f;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    for (int i = w - 1; i <= w1; ++i) {
      const int lo = chunk_key_tile(max(i * size - sg.at, (int64_t)0));
      const int hi = chunk_key_tile(min(i * size + size, stop) - sg.at);
      if (lo >= hi) continue;
      if (lo == 0 && hi == v_all) return;        // written by that part
      const int64_t slot = (int64_t)chunk_slot(i, lo) * s.slot_rows + rr;
      const float2 ml = s.part_ml[slot];
      const f32x4 y = *(const f32x4*)(s.part_o + slot * kHeadDim + c);
      const float mn = fmaxf(M, ml.x), mu = mn > -INFINITY ? mn : 0.f;
      const float f0 = __builtin_amdgcn_exp2f(M - mu), f1 = __builtin_amdgcn_exp2f(ml.x - mu);
      M = mn;
      L = fmaf(f1, ml.y, f0 * L);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = fmaf(f1, y[j], f0 * x[j]);
    }
    if (r < n_rows) {
      uint16_t* op = s.out + (sg.start + pos0 + r / a.gqa) * s.o_st + (sg.g * a.gqa + r % a.gqa) * s.o_sh + c;
      *(u32x2*)op = (u32x2){pack_bf16(x[0] / L, x[1] / L), pack_bf16(x[2] / L, x[3] / L)};
    }
  });
}

// Rows of a partial result: those of the largest row tile a call of `total` rows can have.
static int slot_rows(int64_t total, int gqa) { return chunk_rows(total * gqa); }
int64_t block_chunk_workspace_bytes(int64_t total, int gqa) {
  return (int64_t)2 * kChunkParts * slot_rows(total, gqa) * (kHeadDim * sizeof(float) + sizeof(float2));
}

hipError_t launch_chunk_attend(const BlockArgs& a, ChunkStep s, void* workspace, hipStream_t st) {
  s.slot_rows = slot_rows(s.total, a.gqa);
  s.part_o = (float*)workspace;
  s.part_ml = (float2*)(s.part_o + (int64_t)2 * kChunkParts * s.slot_rows * kHeadDim);
  k_chunk_attend<<<dim3(kChunkParts), kChunkThreads, 0, st>>>(a, s);
  if (hipError_t e = hipGetLastError()) return e;
  const int rows = (int)std::min<int64_t>(s.slot_rows, (int64_t)s.total * a.gqa);
  k_chunk_merge<<<dim3(kChunkParts - 1, (rows + kMergeRows - 1) / kMergeRows), kThreads, 0, st>>>(a, s);
  return hipGetLastError();
}

}  // namespace qv
