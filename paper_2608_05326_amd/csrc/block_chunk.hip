// Attention of a chunk of new tokens of many sequences over the 8-bit block cache and the
// chunk itself: a piece of a prompt, drafted tokens to verify, or one token.
//
//   out_i = sum_j softmax_j(scale q_i . k_j) v_j,   j over the tokens held and the chunk's
//                                                   up to i
//
// The keys of a sequence are its tiles of 64 positions: complete blocks are pages (int8 codes
// with a scale), the others are rows in bf16, of the open block and then of the chunk.
//
// One pass with a running maximum and sum, S^T = K Q^T and O^T = V^T P^T by 32x32x16 bf16
// products, in which codes are exact.  256 workgroups take equal parts of all the work (how it is
// cut: qv_chunk.h), partial rows are joined by a second launch.  By the rows (position, head) of
// a place and KV head:
//   to 32 or 64   (drafted tokens) bound by the pages' bytes: a wave has its own pages, straight
//                 from memory to LDS; 28 places, 113 tokens over 966 MB of cache 191 us with
//                 the join's 6 (5.1 TB/s).  64 rows a wave pair cost twice 32.
//   more          (pieces of prompts) bound by the products and the exponentials between them:
//                 eight waves of 32 rows share tiles that are expanded once, into LDS; 4096
//                 tokens of 64 / 8 heads over 61440 take 7.5 to 8.1 ms by card (1.14 to 1.06 PFLOP/s;
//                 a large matrix product reaches 1.45 to 1.35 there), the matrix unit busy 54%.
// The reference of a row's weights is raised by whole powers of two, so that weights in bf16 that
// are in flight scale exactly.
//
// Weights are rounded to bf16 (2^-8 of themselves) and not to fp16 (2^-11), as a single token's
// are beside codes: they carry their block's value scale, which needs bf16's range, so that pages
// and rows in bf16 add to the same 64 sums a lane.  (With the scale left to the products, as there,
// each of the sums takes another fused product a block.)  Logits, maximum, sums and outputs are
// fp32.
#include <algorithm>

#include "qv_block.h"
#include "qv_chunk.h"

namespace qv {

namespace {
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kWaves = kChunkWaves, kChunkThreads = 64 * kWaves;
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

// A value, or threadIdx.x, not to be seen through: what is derived from it is computed where it is
// used (hoisted out of the walk over segments, it would fill the registers that the products need).
__device__ __forceinline__ int here(int x) {
  asm volatile("" : "+v"(x));
  return x;
}
__device__ __forceinline__ int thread_here() { return here(threadIdx.x); }

// The place in lane, with its length on the line.
__device__ __forceinline__ ChunkPlace lane_place(const BlockArgs& a, const ChunkStep& s, int place, int* start) {
  const int i = min(place, a.B - 1);
  const int b = min(max(s.cu[i], 0), s.total), e = min(max(s.cu[i + 1], b), s.total);
  *start = b;
  return chunk_place(place < a.B ? a.lens[i] : -1, e - b, a.gqa, s.gqa_inv, a.H_kv, a.max_context);
}
__device__ __forceinline__ int64_t wave_scan(int64_t x) {   // inclusive
  const int lane = thread_here() & 63;
#pragma unroll 1
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t lo = __builtin_amdgcn_ds_bpermute(4 * (lane - d), (int)x);
    const int hi = __builtin_amdgcn_ds_bpermute(4 * (lane - d), (int)(x >> 32));
    if (lane >= d) x += (int64_t)((uint64_t)lo | (uint64_t)(uint32_t)hi << 32);
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
  int heads;                 // KV heads g .. of a place of solo row tiles (else 1)
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
  const int lane = thread_here() & 63;
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
  int64_t base = 0;
  for (int s0 = 0; x < end; s0 += 64) {
    if (s0) {   // (the first 64 are there)
      if (s0 >= a.B) return;
      __syncthreads();
      if (thread_here() < 64) put_places(a, s, s0, base, lp);
      __syncthreads();
    }
    base = lane_of(lp.incl[63], 0);
    while (x < end && x < base) {
      const int w = __builtin_ctzll(__ballot(lp.incl[thread_here() & 63] > x));
      Segment g;
      g.seq = s0 + w;
      g.start = __builtin_amdgcn_readfirstlane(lp.start[w]);
      const int held = __builtin_amdgcn_readfirstlane(lp.held[w]), n = __builtin_amdgcn_readfirstlane(lp.n[w]);
      g.p = chunk_place(held, n, a.gqa, s.gqa_inv, a.H_kv, a.max_context);
      g.p.per = __builtin_amdgcn_readfirstlane(g.p.per);       // (divisions leave them in vector registers)
      g.p.tiles = __builtin_amdgcn_readfirstlane(g.p.tiles);
      const int64_t pair = chunk_pair_cost(g.p), last = lane_of(lp.incl[w], 0);
      const int64_t first = last - pair * a.H_kv;
      // a KV head at a time; of a place of solo row tiles, up to eight whole ones, one to a wave
      for (g.g = __builtin_amdgcn_readfirstlane(chunk_quotient(x - first, pair)); g.g < a.H_kv && x < end;
           g.g += g.heads) {
        const int64_t at = first + g.g * pair;
        g.heads = 1;
        if (g.p.solo && x == at) {
          const int most = min(kWaves, a.H_kv - g.g);
          while (g.heads < most && end - x >= (g.heads + 1) * pair) ++g.heads;
        }
        for (g.tile = __builtin_amdgcn_readfirstlane(chunk_tile_at(g.p, x - at)); g.tile < g.p.tiles && x < end;
             ++g.tile) {
          g.at = at + chunk_before(g.p, g.tile);
          const int64_t stop = min(end, g.at + chunk_cost(g.p, g.tile));
          g.from = x - g.at;
          g.to = stop - g.at;
          f(g);
          x = g.heads > 1 ? at + g.heads * pair : stop;
        }
      }
    }
  }
}
// The line's length; the first 64 places are put in lp (the whole workgroup).
__device__ __forceinline__ int64_t line_total(const BlockArgs& a, const ChunkStep& s, LinePlaces& lp, int zero) {
  if (threadIdx.x < 64) put_places(a, s, zero, 0, lp);
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

// What a row tile's workgroup needs of a segment, beside the segment.
struct RowTile {
  int lo, hi;                // its tiles of 64 keys
  int pos0, n_rows;          // first new token, (position, head) rows
  bool whole;                // all of the row tile's keys
};

// The query of one row as the B operand of eight k-steps, scaled by a power of two (bf16 stays
// bf16); returns the power of two that takes the products back.  WIDE: k-step ks
// covers channels 16 ks + 8 lh + 0 .. 7, else 32 (ks / 2) + 16 lh + 8 (ks % 2) + 0 .. 7.
template <bool WIDE>
__device__ __forceinline__ int load_query(const BlockArgs& a, const uint16_t* p, int lh, u32x4 (&q)[8]) {
#pragma unroll
  for (int ks = 0; ks < 8; ++ks)
    q[ks] = *(const u32x4*)(p + (WIDE ? 16 * ks + 8 * lh : 32 * (ks >> 1) + 16 * lh + 8 * (ks & 1)));
  uint32_t am = 0;
#pragma unroll
  for (int ks = 0; ks < 8; ++ks) am = amax_pair(q[ks], am);
  am = amax_bits(am);
  const auto swapped = __builtin_amdgcn_permlane32_swap(am, am, false, false);
  const uint32_t am0 = swapped[0], am1 = swapped[1];
  am = max(am0, am1);
  // (a row of subnormals: their scale)
  const int shift = chunk_query_shift(max((int)(am >> 23), 1) - 127, __builtin_amdgcn_frexp_expf(a.scale_log2));
#pragma unroll
  for (int ks = 0; ks < 8; ++ks)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t w = q[ks][j];
      q[ks][j] = pack_bf16(ldexpf(lo_f32(w), -shift), ldexpf(hi_f32(w), -shift));
    }
  return shift;
}
// Log2 units per raw logit of keys with the scale ks: scale_log2 2^shift ks, held as a mantissa
// and a power of two that comes last: products of small queries and large keys are logits of
// ordinary size.
struct LogitScale {
  float m;
  int e;
  __device__ __forceinline__ float operator()(float ks) const {
    const float x = ldexpf(m * ks, e);
    return x == INFINITY ? __FLT_MAX__ : x;   // (a product of zero is a logit of zero)
  }
};
__device__ __forceinline__ LogitScale logit_scale(const BlockArgs& a, int shift) {
  return {__builtin_amdgcn_frexp_mantf(a.scale_log2), __builtin_amdgcn_frexp_expf(a.scale_log2) + shift};
}

// Running maximum (log2 units), sum and output of one row: o[c][i] is channel
// 32 c + 8 (i / 4) + 4 lh + i % 4.
struct Running {
  float m, l;
  f32x16 o[4];
};
__device__ __forceinline__ void clear(Running& r) {
  r.m = -INFINITY;
  r.l = 0.f;
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) r.o[c][i] = 0.f;
}
// The largest of a row's logits, in log2 units.
template <int KT>
__device__ __forceinline__ float largest(const f32x16 (&st)[KT], float sc) {
  float mt = -INFINITY;
#pragma unroll
  for (int kt = 0; kt < KT; ++kt)
#pragma unroll
    for (int i = 0; i < 16; ++i) mt = fmaxf(mt, st[kt][i]);
  return half_max(mt) * sc;
}
__device__ __forceinline__ bool exceeds(const Running& r, float mt) { return __any(mt > r.m + kLazy); }
// Raises the reference above mt (all rows of the wave at once) by a whole power of two, and
// rescales: exact, also of weights in bf16 whose values are still to be added.
template <int N>
__device__ __forceinline__ void raise(Running& r, float mt, u32x4 (&pw)[N]) {
  const float up = fmaxf(ceilf(mt - r.m), 0.f);                   // (infinite from the first: m = mt)
  const float al = __builtin_amdgcn_exp2f(-up);
  r.m = mt > r.m ? (r.m > -INFINITY ? r.m + up : mt) : r.m;
  r.l *= al;
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) r.o[c][i] *= al;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t w = pw[i][j];
      pw[i][j] = pack_bf16(lo_f32(w) * al, hi_f32(w) * al);
    }
}
// Weights exp2(st sc - m) of a k-step, in bf16 with the values' scale vs.
template <int KT>
__device__ __forceinline__ void weigh(Running& r, const f32x16 (&st)[KT], float sc, float vs, int ks, u32x4& pw) {
  const float mu = r.m > -INFINITY ? r.m : 0.f;
  float e[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) e[i] = __builtin_amdgcn_exp2f(fmaf(st[ks >> 1][8 * (ks & 1) + i], sc, -mu));
  r.l += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
#pragma unroll
  for (int i = 0; i < 4; ++i) pw[i] = pack_bf16(e[2 * i] * vs, e[2 * i + 1] * vs);
}
template <int KT>
__device__ __forceinline__ void weigh(Running& r, const f32x16 (&st)[KT], float sc, float vs, u32x4 (&pw)[2 * KT]) {
  const float mt = largest<KT>(st, sc);
  u32x4 none[1] = {};
  if (exceeds(r, mt)) raise(r, mt, none);
#pragma unroll
  for (int ks = 0; ks < 2 * KT; ++ks) weigh<KT>(r, st, sc, vs, ks, pw[ks]);
}

// The same for many rows, with vs in the exponent: w = exp2(st sc - (m - log2 vs)), and the sum of
// weights from the rounded w, as (sum w) / vs: two vector instructions a weight less.  It misses
// weights below 2^-126 / vs, 2^-46 of the largest for scales from kFoldMin on; those of smaller
// ones (inv = 0) are summed by themselves, in unfolded().
constexpr float kFoldMin = 0x1p-80f;
struct ValueScale {
  float log2, inv;
};
__device__ __forceinline__ ValueScale value_scale(float vs) {
  return {__builtin_amdgcn_logf(vs), vs >= kFoldMin ? 1.f / vs : 0.f};
}
__device__ __forceinline__ float reference(const Running& r) { return r.m > -INFINITY ? r.m : 0.f; }
template <int KT>
__device__ __forceinline__ void weigh(Running& r, const f32x16 (&st)[KT], float sc, float mu, float inv, int ks,
                                      u32x4& pw) {
  const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int j = 8 * (ks & 1) + 2 * i;
    const uint32_t w = pack_bf16(__builtin_amdgcn_exp2f(fmaf(st[ks >> 1][j], sc, -mu)),
                                 __builtin_amdgcn_exp2f(fmaf(st[ks >> 1][j + 1], sc, -mu)));
    sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), ones, sum, false);
    pw[i] = w;
  }
  r.l = fmaf(sum, inv, r.l);
}
template <int KT>
__device__ __forceinline__ void unfolded(Running& r, const f32x16 (&st)[KT], float sc, float inv) {
  if (__builtin_amdgcn_readfirstlane(__float_as_uint(inv))) return;
  const float mu = reference(r);
#pragma unroll
  for (int kt = 0; kt < KT; ++kt)
#pragma unroll
    for (int i = 0; i < 16; ++i) r.l += __builtin_amdgcn_exp2f(fmaf(st[kt][i], sc, -mu));
}

// A value that is not finite must not reach a row that its key is masked for, through
// 0 * infinity: such values of rows in bf16 are left out of the products, and added to the
// rows that see them afterwards.
// (take_out: whether any lane of the wave held one.)
__device__ __forceinline__ bool take_out(u32x4& x) {
  // exponents of ones: 0x7F80 + 0x80 in either half
  uint32_t bad = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) bad |= (x[j] & 0x7F807F80u) + 0x00800080u;
  if (!__any(bad & 0x80008000u)) return false;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if ((x[j] & 0x7F80u) == 0x7F80u) x[j] &= 0xFFFF0000u;
    if ((x[j] & 0x7F800000u) == 0x7F800000u) x[j] &= 0xFFFFu;
  }
  return true;
}
template <class Row>
__device__ __forceinline__ void add_odd(Running& r, Row row, int n, int lh) {   // rows 0 .. n - 1 are seen
  for (int key = 0; key < n; ++key) {
    const uint16_t* vr = row(key) + 4 * lh;
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const uint16_t x = vr[32 * c + 8 * (i >> 2) + (i & 3)];
        if ((x & 0x7F80u) == 0x7F80u) r.o[c][i] += bf16_to_f32(x);
      }
  }
}

// Keys (values) of position p of a place, a row in bf16: of the open block or of the chunk.
__device__ __forceinline__ const uint16_t* fresh_row(const BlockArgs& a, const ChunkStep& s, const Segment& sg,
                                                     int g, bool values, int p) {
  if (p < sg.p.held)
    return (values ? a.v_tail : a.k_tail) + ((int64_t)sg.seq * a.H_kv + g) * kCodes + (p % kBlk) * kHeadDim;
  const int64_t row = sg.start + (p - sg.p.held);
  return values ? s.v + row * s.v_st + g * s.v_sh : s.k + row * s.k_st + g * s.k_sh;
}

// A row's output (all lanes, the two halves of a row together; `there`: it is stored).
__device__ __forceinline__ void store_row(const Running& r, uint16_t* row, bool there, int lh) {
  const float inv = 1.f / r.l;
  uint16_t* op = row + 8 * lh;
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int e = 0; e < 4; e += 2) {   // channels 8 e .. 8 e + 15: eight to each lane half
      uint32_t y[2], z[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const auto sw = __builtin_amdgcn_permlane32_swap(
            pack_bf16(r.o[c][4 * e + 2 * j] * inv, r.o[c][4 * e + 2 * j + 1] * inv),
            pack_bf16(r.o[c][4 * e + 4 + 2 * j] * inv, r.o[c][4 * e + 5 + 2 * j] * inv), false, false);
        y[j] = sw[0];
        z[j] = sw[1];
      }
      if (there) *(u32x4*)(op + 32 * c + 8 * e) = (u32x4){y[0], y[1], z[0], z[1]};
    }
}

__device__ __forceinline__ int by_gqa(const ChunkStep& s, int row) { return (uint32_t)row * s.gqa_inv >> 16; }

// Address of a row's output in `out`.
__device__ __forceinline__ uint16_t* out_row(const BlockArgs& a, const ChunkStep& s, const Segment& sg,
                                             const RowTile& rt, int g, int row) {
  const int i = by_gqa(s, row);
  return s.out + (sg.start + rt.pos0 + i) * s.o_st + (g * a.gqa + row - i * a.gqa) * s.o_sh;
}

// LDS of a workgroup, in two arrays: reads of one do not wait for the loads on their way into
// the other (the compiler tells arrays apart, not parts of one).
constexpr int kLds = 64 * 1024;
struct Shared {
  uint8_t* k;
  uint8_t* v;
};
// A wave's output rows for the join, 16 KB: 16-byte chunk c of row r.
__device__ __forceinline__ float* join_at(const Shared& sm, int wave, int r, int c) {
  return (float*)((wave < 4 ? sm.k : sm.v) + (wave & 3) * 16384 + r * 512 + 16 * (c ^ r));
}
// 16 bytes a lane from global memory to LDS, in lane order from an address that is uniform
__device__ __forceinline__ void dma16(const void* g, uint8_t* to) {
  __builtin_amdgcn_global_load_lds(g, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

// ---- few rows: a wave has 32 rows and pages of its own
__device__ __forceinline__ void attend_few(const BlockArgs& a, const ChunkStep& s, const Segment& sg,
                                           const RowTile& rt, int part, const Shared& sm, float2 (*sml)[32]) {
  const int tid = thread_here(), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, lh = lane >> 5;
  // one or two sets of 32 rows; the other waves of a set take the key tiles in turn.  Solo: a
  // KV head to a wave.
  const bool solo = sg.heads > 1;
  const int log_rs = sg.p.c.rows == 32 ? 0 : 1, rs = 1 << log_rs;
  const int rw = wave & (rs - 1), kg = solo ? 0 : wave >> log_rs, n_kg = solo ? 1 : kWaves >> log_rs;
  const bool idle = solo ? wave >= sg.heads : rw * 32 >= rt.n_rows;
  const int g = solo && !idle ? sg.g + wave : sg.g;
  const int row = min(rw * 32 + lr, rt.n_rows - 1), i_row = rt.pos0 + by_gqa(s, row);
  const int head = g * a.gqa + row - (i_row - rt.pos0) * a.gqa;
  const int pos = sg.p.held + i_row;                  // this lane's position
  const int last = sg.p.held + sg.p.n - 1;            // the place's last position
  const int n_blk = sg.p.held / kBlk, page_end = idle ? 0 : min(rt.hi, n_blk);
  // page (-1: none) of block t0 + n_kg lane; the first look-up goes before the query's loads
  auto page_at = [&](int t0) { return t0 + lane * n_kg < page_end ? page_of(a, sg.seq, t0 + lane * n_kg) : -1; };
  int page = page_at(rt.lo + kg);
  u32x4 q[8];
  const int shift = load_query<false>(a, s.q + (sg.start + i_row) * s.q_st + head * s.q_sh, lh, q);
  const LogitScale scale = logit_scale(a, shift);
  Running r;
  clear(r);
  // row lr of an A operand is this key of 32; a lane's logits st[i] are those of keys 16 lh + i
  const int krow = 16 * ((lr >> 2) & 1) + 4 * (lr >> 3) + (lr & 3);

  uint8_t* const sk = sm.k + wave * kCodes;   // a page's keys [64][128] and values [128][64], codes
  uint8_t* const sv = sm.v + wave * kCodes;
  // A wave's load of 1 KB fills LDS in lane order.  16-byte chunks of a row are swizzled
  // through the address that a lane fetches, so that the reads below meet all banks: chunk c
  // of key t is at c ^ ((t / 2) % 4 + 4 ((t / 16) % 2)), of channel h at c ^ ((h / 4) % 4).
  const uint32_t k_from = (lane >> 3) * kHeadDim + 16 * ((lane & 7) ^ ((lane >> 4) & 3));
  const uint32_t v_from = (lane >> 2) * kBlk + 16 * ((lane & 3) ^ ((lane >> 4) & 3));
  const int k_at = krow * kHeadDim + 16 * (lh ^ (((krow >> 1) & 3) | ((krow >> 4) & 1) << 2));
  const int v_at = lr * kBlk + 16 * (lh ^ ((lr >> 2) & 3));
  // (the arrays are at multiples of 128: the address takes the swizzle)
  const uint32_t k_lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)sk + k_at;
  const uint32_t v_lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)sv + v_at;
  for (int t0 = rt.lo + kg; t0 < page_end; t0 += 64 * n_kg) {
    // pages and scales of the wave's next 64 blocks, one per lane (dropped blocks are left out)
    if (t0 != rt.lo + kg) page = page_at(t0);
    float ks_l = 0.f, vs_l = 0.f;
    uint64_t live = __ballot(page >= 0);
    if (!live) continue;
    if (page >= 0) {
      ks_l = a.k_scale[(int64_t)page * a.H_kv + g];
      vs_l = a.v_scale[(int64_t)page * a.H_kv + g];
    }
    auto entry = [&](int j) { return ((int64_t)__builtin_amdgcn_readlane(page, j) * a.H_kv + g) * kCodes; };
    auto load_k = [&](int64_t e) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        dma16(a.k_codes + e + (i & 2 ? k_from ^ 64 : k_from) + 1024 * i, sk + 1024 * i);
    };
    auto load_v = [&](int64_t e) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) dma16(a.v_codes + e + v_from + 1024 * i, sv + 1024 * i);
    };
    int64_t e = entry(__builtin_ctzll(live));
    // (the waits below count loads: the keys' are the older eight, here too)
    load_k(e);
    asm volatile("; values behind keys" ::: "memory");
    load_v(e);
    while (live) {
      const int j = __builtin_ctzll(live);
      live &= live - 1;
      e = entry(live ? __builtin_ctzll(live) : j);     // (after the last: that again)
      const float sc = scale(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ks_l), j)));
      const float vs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vs_l), j));
      f32x16 st[2];
      u32x4 pw[4];
      {
        u32x4 kb[2][4];
        // The keys are there, the values still on their way.  In one block: where the compiler sees
        // reads of LDS behind loads into it, it waits for all of these (197 us instead of 192 for the
        // drafted tokens above, single tokens of 30 places 113 instead of 105).
        asm volatile(
            "s_waitcnt vmcnt(8)\n\t"
            "ds_read_b128 %0, %8\n\t"
            "ds_read_b128 %1, %8 offset:4096\n\t"
            "ds_read_b128 %2, %9\n\t"
            "ds_read_b128 %3, %9 offset:4096\n\t"
            "ds_read_b128 %4, %10\n\t"
            "ds_read_b128 %5, %10 offset:4096\n\t"
            "ds_read_b128 %6, %11\n\t"
            "ds_read_b128 %7, %11 offset:4096\n\t"
            "s_waitcnt lgkmcnt(0)"                           // read, before they are overwritten
            : "=&v"(kb[0][0]), "=&v"(kb[1][0]), "=&v"(kb[0][1]), "=&v"(kb[1][1]), "=&v"(kb[0][2]), "=&v"(kb[1][2]),
              "=&v"(kb[0][3]), "=&v"(kb[1][3])
            : "v"(k_lds), "v"(k_lds ^ 32), "v"(k_lds ^ 64), "v"(k_lds ^ 96)
            : "memory");
        static_assert(32 * kHeadDim == 4096);
        load_k(e);
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int i = 0; i < 16; ++i) st[kt][i] = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int b = 0; b < 4; b += 2)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
              st[kt] = mfma32(codes_bf16(kb[kt][i][b], kb[kt][i][b + 1]), q[2 * i + b / 2], st[kt]);
      }
      weigh<2>(r, st, sc, vs, pw);
      {
        u32x4 vb[2][4];
        asm volatile(
            "s_waitcnt vmcnt(8)\n\t"
            "ds_read_b128 %0, %8\n\t"
            "ds_read_b128 %1, %8 offset:2048\n\t"
            "ds_read_b128 %2, %8 offset:4096\n\t"
            "ds_read_b128 %3, %8 offset:6144\n\t"
            "ds_read_b128 %4, %9\n\t"
            "ds_read_b128 %5, %9 offset:2048\n\t"
            "ds_read_b128 %6, %9 offset:4096\n\t"
            "ds_read_b128 %7, %9 offset:6144\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(vb[0][0]), "=&v"(vb[0][1]), "=&v"(vb[0][2]), "=&v"(vb[0][3]), "=&v"(vb[1][0]), "=&v"(vb[1][1]),
              "=&v"(vb[1][2]), "=&v"(vb[1][3])
            : "v"(v_lds), "v"(v_lds ^ 32)
            : "memory");
        static_assert(32 * kBlk == 2048);
        load_v(e);
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int b = 0; b < 4; b += 2)
#pragma unroll
            for (int c = 0; c < 4; ++c)
              r.o[c] = mfma32(codes_bf16(vb[kt][c][b], vb[kt][c][b + 1]), pw[2 * kt + b / 2], r.o[c]);
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  }

  // tiles of rows in bf16, 32 keys at a time (keys past the place's last are that again, and
  // masked); the values turn in LDS
  const int first = max(rt.lo, n_blk), skip = (first - rt.lo) % n_kg;
  for (int t = first + (kg >= skip ? kg - skip : kg - skip + n_kg); !idle && t < rt.hi; t += n_kg)
#pragma unroll 1
    for (int k0 = t * kBlk; k0 < t * kBlk + kBlk && k0 <= last; k0 += 32) {
      auto at = [&](bool values, int key) { return fresh_row(a, s, sg, g, values, min(k0 + key, last)); };
      uint8_t* mine = sv;   // 32 rows of 256 bytes
      u32x4 vb[8], kb[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) vb[i] = *(const u32x4*)(at(true, 4 * i + (lane >> 4)) + 8 * (lane & 15));
      const uint16_t* kr = at(false, krow) + 16 * lh;
#pragma unroll
      for (int ks = 0; ks < 8; ++ks) kb[ks] = *(const u32x4*)(kr + 32 * (ks >> 1) + 8 * (ks & 1));
      bool odd = false;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        odd |= take_out(vb[i]);
        *(u32x4*)(mine + (4 * i + (lane >> 4)) * kRowBytes + 16 * (lane & 15)) = vb[i];
      }
      f32x16 sr[1];
      u32x4 pr[2];
#pragma unroll
      for (int i = 0; i < 16; ++i) sr[0][i] = 0.f;
#pragma unroll
      for (int ks = 0; ks < 8; ++ks) sr[0] = mfma32(kb[ks], q[ks], sr[0]);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (k0 + 16 * lh + i > pos) sr[0][i] = -INFINITY;
      weigh<1>(r, sr, scale(1.f), 1.f, pr);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // this wave's rows are in LDS
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          u32x4 x;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int key = 16 * lh + 8 * ks + 4 * j + ((lane >> 2) & 3);
            const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(
                mine + key * kRowBytes + 64 * c + 32 * ((lane >> 4) & 1) + 8 * (lane & 3))));
            x[2 * j] = y[0];
            x[2 * j + 1] = y[1];
          }
          r.o[c] = mfma32(x, pr[ks], r.o[c]);
        }
      if (odd) add_odd(r, [&](int key) { return at(true, key); }, min(32, pos - k0 + 1), lh);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }

  r.l = half_sum(r.l);
  if (solo) {
    if (!idle) store_row(r, out_row(a, s, sg, rt, g, row), lr < rt.n_rows, lh);
    __syncthreads();
    return;
  }
  // ---- join the waves of a row set
  __syncthreads();
  sml[wave][lr] = make_float2(r.m, r.l);
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *(f32x4*)join_at(sm, wave, lr, 8 * c + 2 * i + lh) =
          (f32x4){r.o[c][4 * i], r.o[c][4 * i + 1], r.o[c][4 * i + 2], r.o[c][4 * i + 3]};
  __syncthreads();
  for (int e = tid; e < rt.n_rows * (kHeadDim / 4); e += kChunkThreads) {
    const int rr = e / (kHeadDim / 4), c = 4 * (e % (kHeadDim / 4)), w0 = rr >> 5, r32 = rr & 31;
    float M = -INFINITY;
    for (int w = w0; w < kWaves; w += rs) M = fmaxf(M, sml[w][r32].x);
    const float mu = M > -INFINITY ? M : 0.f;
    float L = 0.f;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    for (int w = w0; w < kWaves; w += rs) {
      const float f = __builtin_amdgcn_exp2f(sml[w][r32].x - mu);
      L = fmaf(f, sml[w][r32].y, L);
      const f32x4 y = *(const f32x4*)join_at(sm, w, r32, c / 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = fmaf(f, y[i], x[i]);
    }
    if (rt.whole) {
      *(u32x2*)(out_row(a, s, sg, rt, g, rr) + c) =
          (u32x2){pack_bf16(x[0] / L, x[1] / L), pack_bf16(x[2] / L, x[3] / L)};
    } else {
      const int64_t slot = (int64_t)chunk_slot(part, rt.lo) * s.slot_rows + rr;
      *(f32x4*)(s.part_o + slot * kHeadDim + c) = x;
      if (c == 0) s.part_ml[slot] = make_float2(M, L);
    }
  }
  __syncthreads();
}

// ---- many rows: eight sets of 32 rows share the key tiles, which are expanded into LDS
struct PageRef {
  int page;
  float ks;
  ValueScale vs;
};
constexpr int kList = kChunkThreads;   // pages looked up at once
// bytes of a tile's keys [64][128] or values (of a page [128][64], else [64][128]), bf16
constexpr int kTileBytes = kBlk * kRowBytes;
static_assert(2 * kTileBytes <= kLds && kWaves * kCodes <= kLds && 4 * 16384 <= kLds, "LDS");
// 16-byte chunks of a staged row are stored at chunk ^ swizzle(row), so that the reads of
// either product meet all banks
__device__ __forceinline__ int swz_k(int key) { return key & 15; }
__device__ __forceinline__ int swz_v(int key) { return ((key & 3) << 2) | ((key >> 2) & 3); }
__device__ __forceinline__ int swz_c(int channel) { return (channel >> 1) & 7; }

// Row lr of the A operand of a 32-key tile is this key of it, so that a lane's logits
// st[kt][i] are those of keys 32 kt + 16 (i / 8) + 8 lh + i % 8.
__device__ __forceinline__ int key_of_row(int lr) {
  return 16 * (lr >> 4) + 8 * ((lr >> 2) & 1) + 4 * ((lr >> 3) & 1) + (lr & 3);
}
// The order in which what stands between two scheduling barriers is issued: a product, then
// LDS reads, vector instructions and exponentials beside it, n times over.  A wave issues in
// order, and a product keeps the matrix unit for eight issue slots: what does not stand
// between two products waits for all of them.
template <int N, int READS, int VALU, int TRANS>
__device__ __forceinline__ void interleave() {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    if constexpr (READS) __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
    if constexpr (VALU) __builtin_amdgcn_sched_group_barrier(0x002, VALU, 0);
    if constexpr (TRANS) __builtin_amdgcn_sched_group_barrier(0x400, TRANS, 0);
  }
}
// Operands on their way from LDS: read kAhead ahead of their products, since a read takes longer
// than some products.
constexpr int kAhead = 5;
struct Operands {
  u32x4 x[kAhead + 1];
};
// st = K Q^T of a staged tile; read(n) reads operand n: keys 32 (n % 2) .. of k-step n / 2.
// beside(ks) goes with the products of k-step ks.
template <class Read, class Beside>
__device__ __forceinline__ void wide_logits(const u32x4 (&q)[8], f32x16 (&st)[2], Read read, Beside beside) {
  Operands k;
#pragma unroll
  for (int kt = 0; kt < 2; ++kt)
#pragma unroll
    for (int i = 0; i < 16; ++i) st[kt][i] = 0.f;
#pragma unroll
  for (int n = 0; n < kAhead; ++n) k.x[n] = read(n);
#pragma unroll
  for (int ks = 0; ks < 8; ++ks) {
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const int n = 2 * ks + kt;
      if (n + kAhead < 16) k.x[(n + kAhead) % (kAhead + 1)] = read(n + kAhead);
      st[kt] = mfma32(k.x[n % (kAhead + 1)], q[ks], st[kt]);
    }
    beside(ks);
    interleave<2, 1, 7, 0>();
    __builtin_amdgcn_sched_barrier(0);
  }
}
// o += V^T P^T; read(n) reads operand n: channels 32 (n % 4) .. of k-step n / 4; beside(ks) goes
// with the products of k-step ks and may change pw[ks].
template <class Read, class Beside>
__device__ __forceinline__ void wide_values(Running& r, u32x4 (&pw)[4], Read read, Beside beside) {
  Operands v;
#pragma unroll
  for (int n = 0; n < kAhead; ++n) v.x[n] = read(n);
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int n = 4 * ks + c;
      if (n + kAhead < 16) v.x[(n + kAhead) % (kAhead + 1)] = read(n + kAhead);
      r.o[c] = mfma32(v.x[n % (kAhead + 1)], pw[ks], r.o[c]);
    }
    beside(ks);
    interleave<4, 1, 7, 2>();
    __builtin_amdgcn_sched_barrier(0);
  }
}

// Key tiles 0 .. n - 1 of a source (pages or rows in bf16).  Step e of the loop: the products
// of tile e's keys, and beside them the next tile's keys and its own values are put into the
// arrays that were last read in the step before and the loads of those behind them start; then
// the products of the values of the tile before, and beside them the weights of tile e.  One step
// more ends with the last tile's values.
//   src.peek(e, f), src.look()       starts to read what is known: of tile e for logits(), of f
//                                    for the loads after look(); both come long before their use
//   src.load_k(e), src.load_v(e)     into registers
//   src.put_k(i, to), src.put_v(i, e, to)   half i of it from there into LDS
//   src.sees(n)                      of n tiles, how many hold keys that a row of the wave sees
//   src.logits(e, st, vs)            what is left to do with raw logits; their scale, the values'
//   src.read_v(from, at, ks, c)      an operand of the second product
//   src.after(e, r)                  what is left to do after it
template <class Source>
__device__ __forceinline__ void wide_loop(Source& src, int n, int kbase, const u32x4 (&q)[8], Running& r,
                                          const Shared& sm) {
  src.peek(0, 0);
  src.look();
  src.load_k(0);
  src.load_v(0);
  src.peek(0, min(1, n - 1));
  src.put_k(0, sm.k);
  src.put_k(1, sm.k);
  src.look();
  src.load_k(min(1, n - 1));
  src.peek(0, min(2, n - 1));
  __syncthreads();
  u32x4 pw[4];
  // in six parts (past the last tile: that again, in an array that is not read)
  auto stage = [&](int e, int b, int c, int part) __attribute__((always_inline)) {
    if (part < 2) src.put_k(part, sm.k + c);
    else if (part < 4) src.put_v(part - 2, e, sm.v + b);
    else if (part == 4) src.load_v(min(e + 1, n - 1));
    else if (part == 5) {
      src.look();
      src.load_k(min(e + 2, n - 1));
    }
  };
  auto logits = [&](int e, int b, int c, f32x16 (&st)[2]) __attribute__((always_inline)) {
    const int kb = here(kbase);
    wide_logits(
        q, st,
        [&](int i) __attribute__((always_inline)) {
          return *(const u32x4*)(sm.k + b + (kb ^ (32 * (i >> 1))) + 32 * (i & 1) * kRowBytes);
        },
        [&](int ks) __attribute__((always_inline)) { stage(e, b, c, ks); });
  };
  auto known = [&](int e) __attribute__((always_inline)) { src.peek(min(e + 1, n - 1), min(e + 3, n - 1)); };
  auto stage_all = [&](int e) __attribute__((always_inline)) {
    const int b = (e & 1) * kTileBytes;
#pragma unroll
    for (int part = 0; part < 6; ++part) stage(e, b, b ^ kTileBytes, part);
    known(e);
  };
  auto read_v = [&](int e, int at, int i) __attribute__((always_inline)) {
    return src.read_v(sm.v + (e & 1) * kTileBytes, at, i >> 2, i & 3);
  };
  // Every wave comes to n + 1 barriers: one after each step (the last one before the arrays are
  // written again).
  const int seen = src.sees(n);
  int e = 0;
  if (seen > 0) {
    f32x16 st[2];
    logits(0, 0, kTileBytes, st);
    ValueScale vs;
    {
      const float sc = src.logits(0, st, vs), mt = largest<2>(st, sc);
      known(0);
      u32x4 none[1] = {};
      if (exceeds(r, mt)) raise(r, mt, none);
      unfolded(r, st, sc, vs.inv);
      const float mu = reference(r) - vs.log2;
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) weigh<2>(r, st, sc, mu, vs.inv, ks, pw[ks]);
    }
    __syncthreads();
#pragma unroll 1
    for (e = 1; e < seen; ++e) {
      const int b = (e & 1) * kTileBytes, vb = here(src.vbase);
      logits(e, b, b ^ kTileBytes, st);
      const float sc = src.logits(e, st, vs), mt = largest<2>(st, sc);
      known(e);
      if (exceeds(r, mt)) raise(r, mt, pw);
      unfolded(r, st, sc, vs.inv);
      const float mu = reference(r) - vs.log2;
      wide_values(
          r, pw, [&](int i) __attribute__((always_inline)) { return read_v(e - 1, vb, i); },
          [&](int ks) __attribute__((always_inline)) { weigh<2>(r, st, sc, mu, vs.inv, ks, pw[ks]); });
      src.after(e - 1, r);
      __syncthreads();
    }
    if (e < n) stage_all(e);
    const int vb = here(src.vbase);
    wide_values(
        r, pw, [&](int i) __attribute__((always_inline)) { return read_v(e - 1, vb, i); }, [](int) {});
    src.after(e - 1, r);
    __syncthreads();
    ++e;
  }
#pragma unroll 1
  for (; e <= n; ++e) {
    if (e < n) stage_all(e);
    __syncthreads();
  }
}

struct PageSource {
  const BlockArgs& a;
  const PageRef* list;
  LogitScale scale;
  int g, tid, kput, vput, vbase;
  bool idle;
  int page;                  // of the tile looked at last
  u32x4 kr, vr;
  PageRef known;             // its scales: of the tile whose logits are next
  __device__ __forceinline__ void peek(int e, int f) {
    known.ks = list[e].ks;
    known.vs = list[e].vs;
    known.page = list[f].page;
  }
  __device__ __forceinline__ void look() { page = __builtin_amdgcn_readfirstlane(known.page); }
  __device__ __forceinline__ u32x4 load(const int8_t* codes, int p) const {
    return *(const u32x4*)(codes + ((int64_t)p * a.H_kv + g) * kCodes + (uint32_t)(16 * tid));
  }
  __device__ __forceinline__ void put(const u32x4& x, uint8_t* to, int at, int i) const {
    *(u32x4*)(to + (at ^ (16 * i))) = codes_bf16(x[2 * i], x[2 * i + 1]);
  }
  __device__ __forceinline__ void load_k(int) { kr = load(a.k_codes, page); }
  __device__ __forceinline__ void load_v(int) { vr = load(a.v_codes, page); }
  __device__ __forceinline__ void put_k(int i, uint8_t* to) const { put(kr, to, kput, i); }
  __device__ __forceinline__ void put_v(int i, int, uint8_t* to) const { put(vr, to, vput, i); }
  __device__ __forceinline__ int sees(int n) const { return idle ? 0 : n; }
  __device__ __forceinline__ float logits(int, f32x16 (&)[2], ValueScale& vs) const {
    vs = known.vs;
    return scale(known.ks);
  }
  __device__ __forceinline__ u32x4 read_v(const uint8_t* from, int at, int ks, int c) const {
    return *(const u32x4*)(from + (at ^ (32 * ks)) + c * 32 * 2 * kBlk);
  }
  __device__ __forceinline__ void after(int, Running&) const {}
};

// The pages of tiles [lo, hi), all of whose keys every row sees.
__device__ __forceinline__ void wide_pages(const BlockArgs& a, const Segment& sg, int lo, int hi, bool idle,
                                           int shift, const u32x4 (&q)[8], Running& r, const Shared& sm,
                                           PageRef* list, int* scnt) {
  const int tid = thread_here(), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, lh = lane >> 5, krow = key_of_row(lr);
  PageSource src = {a, list, logit_scale(a, shift), sg.g, tid,
                    (tid >> 3) * kRowBytes + 16 * ((2 * (tid & 7)) ^ swz_k(tid >> 3)),
                    (tid >> 2) * (2 * kBlk) + 16 * ((2 * (tid & 3)) ^ swz_c(tid >> 2)),
                    lr * (2 * kBlk) + 16 * (lh ^ swz_c(lr)), idle};
  for (int t0 = lo; t0 < hi; t0 += kList) {
    // ---- the next pages (blocks without one are left out)
    PageRef x = {-1, 0.f, {0.f, 0.f}};
    if (t0 + tid < hi) x.page = page_of(a, sg.seq, t0 + tid);
    if (x.page >= 0) {
      x.ks = a.k_scale[(int64_t)x.page * a.H_kv + sg.g];
      x.vs = value_scale(a.v_scale[(int64_t)x.page * a.H_kv + sg.g]);
    }
    const uint64_t mask = __ballot(x.page >= 0);
    if (lane == 0) scnt[wave] = __builtin_popcountll(mask);
    __syncthreads();
    int at = __builtin_popcountll(mask & (((uint64_t)1 << lane) - 1)), n = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      at += w < wave ? scnt[w] : 0;
      n += scnt[w];
    }
    n = __builtin_amdgcn_readfirstlane(n);
    if (x.page >= 0) list[at] = x;
    __syncthreads();
    if (n) wide_loop(src, n, krow * kRowBytes + 16 * (lh ^ swz_k(krow)), q, r, sm);
  }
}

// Tiles of rows in bf16, of the open block and of the chunk.  A thread has chunk tid % 16 of
// rows tid / 16 and 32 more; byte offsets in a tile fit 32 bits (checked on the host).
struct RowSource {
  const BlockArgs& a;
  const ChunkStep& s;
  const Segment& sg;
  LogitScale scale;
  int t0, pos, wpos0, wpos1, last;   // last: the place's last position
  int lane, wave, fr, vbase;
  int (*sodd)[2 * kWaves];
  u32x4 kr[2], vr[2];
  __device__ __forceinline__ void load(const uint16_t* tail, const uint16_t* rows, int64_t stride, int e,
                                       u32x4 (&x)[2]) const {
    const int p0 = (t0 + e) * kBlk, c = 16 * (lane & 15);
    const uint8_t* from = (const uint8_t*)(rows + ((int64_t)sg.start + p0 - sg.p.held) * stride);
    if (p0 >= sg.p.held && p0 + kBlk - 1 <= last) {
      const uint32_t off = (uint32_t)fr * (uint32_t)(2 * stride) + c;
      x[0] = *(const u32x4*)(from + off);
      x[1] = *(const u32x4*)(from + 64 * stride + off);
      return;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int key = min(fr + 32 * i, last - p0);         // (past the last: that again, masked)
      const uint8_t* at = from + (uint32_t)((uint32_t)key * (uint32_t)(2 * stride) + c);
      if (p0 + key < sg.p.held) at = (const uint8_t*)tail + key * kRowBytes + c;
      x[i] = *(const u32x4*)at;
    }
  }
  __device__ __forceinline__ int64_t tail() const { return ((int64_t)sg.seq * a.H_kv + sg.g) * kCodes; }
  __device__ __forceinline__ void load_k(int e) { load(a.k_tail + tail(), s.k + sg.g * s.k_sh, s.k_st, e, kr); }
  __device__ __forceinline__ void load_v(int e) { load(a.v_tail + tail(), s.v + sg.g * s.v_sh, s.v_st, e, vr); }
  __device__ __forceinline__ void put_k(int i, uint8_t* to) const {
    *(u32x4*)(to + (fr + 32 * i) * kRowBytes + 16 * ((lane & 15) ^ swz_k(fr))) = kr[i];
  }
  __device__ __forceinline__ void put_v(int i, int e, uint8_t* to) {
    const int odd = take_out(vr[i]);
    *(u32x4*)(to + (fr + 32 * i) * kRowBytes + 16 * ((lane & 15) ^ swz_v(fr))) = vr[i];
    if (lane == 0) sodd[e & 1][2 * wave + i] = odd;
  }
  __device__ __forceinline__ int sees(int n) const { return min(n, max((wpos1 >> 6) - t0 + 1, 0)); }
  __device__ __forceinline__ float logits(int e, f32x16 (&st)[2], ValueScale& vs) const {
    const int p0 = (t0 + e) * kBlk;
    if (p0 + kBlk - 1 > wpos0) {
      const int rel = pos - p0 - 8 * (lane >> 5);
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (32 * kt + 16 * (i >> 3) + (i & 7) > rel) st[kt][i] = -INFINITY;
    }
    vs = {0.f, 1.f};
    return scale(1.f);
  }
  // (chunks of keys 8 lh .. + 3 and of + 4 .. + 7 differ by the bit of 16 bytes in their swizzle)
  __device__ __forceinline__ u32x4 read_v(const uint8_t* from, int at, int ks, int c) const {
    const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(
                                                  from + (at ^ (64 * c)) + 16 * ks * kRowBytes)));
    const u32x2 z = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(
                                                  from + (at ^ (64 * c) ^ 16) + (16 * ks + 4) * kRowBytes)));
    return (u32x4){y[0], y[1], z[0], z[1]};
  }
  __device__ __forceinline__ void peek(int, int) const {}
  __device__ __forceinline__ void look() const {}
  __device__ __forceinline__ void after(int e, Running& r) const {
    if (__any(sodd[e & 1][lane & (2 * kWaves - 1)]))
      add_odd(r, [&](int key) { return fresh_row(a, s, sg, sg.g, true, (t0 + e) * kBlk + key); },
              min(kBlk, pos - (t0 + e) * kBlk + 1), lane >> 5);
  }
};

__device__ __forceinline__ void attend_many(const BlockArgs& a, const ChunkStep& s, const Segment& sg,
                                            const RowTile& rt, int part, const Shared& sm, PageRef* list,
                                            int (*sodd)[2 * kWaves], int* scnt) {
  const int tid = thread_here(), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, lh = lane >> 5;
  const int row = wave * 32 + lr, rowc = min(row, rt.n_rows - 1), i_row = rt.pos0 + by_gqa(s, rowc);
  const int head = sg.g * a.gqa + rowc - (i_row - rt.pos0) * a.gqa;
  const bool idle = wave * 32 >= rt.n_rows;
  u32x4 q[8];
  const int shift = load_query<true>(a, s.q + (sg.start + i_row) * s.q_st + head * s.q_sh, lh, q);
  Running r;
  clear(r);
  const int n_blk = sg.p.held / kBlk;
  if (rt.lo < n_blk) wide_pages(a, sg, rt.lo, min(rt.hi, n_blk), idle, shift, q, r, sm, list, scnt);
  if (rt.hi > n_blk) {
    // first and last position of the wave's rows
    const int wpos0 = sg.p.held + rt.pos0 + by_gqa(s, wave * 32);
    const int wpos1 = idle ? -1 : sg.p.held + rt.pos0 + by_gqa(s, min(wave * 32 + 31, rt.n_rows - 1));
    const int t0 = max(rt.lo, n_blk), krow = key_of_row(lr), vkey = 8 * lh + ((lane >> 2) & 3);
    const int vbase =
        vkey * kRowBytes + 16 * ((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ swz_v(vkey)) + 8 * (lane & 1);
    RowSource src = {a,     s,     sg,                     logit_scale(a, shift), t0,   sg.p.held + i_row,
                     wpos0, wpos1, sg.p.held + sg.p.n - 1, lane,                  wave, tid >> 4,          vbase, sodd};
    wide_loop(src, rt.hi - t0, krow * kRowBytes + 16 * (lh ^ swz_k(krow)), q, r, sm);
  }

  r.l = half_sum(r.l);
  if (rt.whole) {
    store_row(r, out_row(a, s, sg, rt, sg.g, rowc), row < rt.n_rows, lh);
  } else if (row < rt.n_rows) {
    const int64_t slot = (int64_t)chunk_slot(part, rt.lo) * s.slot_rows + row;
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(f32x4*)(s.part_o + slot * kHeadDim + 32 * c + 8 * i + 4 * lh) =
            (f32x4){r.o[c][4 * i], r.o[c][4 * i + 1], r.o[c][4 * i + 2], r.o[c][4 * i + 3]};
    if (lh == 0) s.part_ml[slot] = make_float2(r.m, r.l);
  }
}

// The join's groups of 32 threads that share a row, for a row tile of this many parts: fewer than
// the parts, so that the workgroups of those that begin inside it have room for all rows.
constexpr int kMergeRows = 8, kMergeRound = 4, kMergeGroups = kThreads / 32;
__device__ __forceinline__ int join_groups(int parts) {
  int log_g = 0;
  while (2 * kMergeRound << log_g < parts && 1 << log_g < kMergeGroups) ++log_g;
  return log_g;
}
}  // namespace

// (254 of 256 vector registers, nothing in scratch memory; 188 scalar values of the walk and of the
// arguments are kept in lanes of vector registers.)
__global__ __launch_bounds__(kChunkThreads, 2) void k_chunk_attend(BlockArgs a, ChunkStep s) {
  __shared__ __attribute__((aligned(128))) uint8_t lds_k[kLds], lds_v[kLds];
  const Shared sm = {lds_k, lds_v};
  __shared__ float2 sml[kWaves][32];
  __shared__ PageRef list[kList];
  __shared__ int sodd[2][2 * kWaves], scnt[kWaves];
  __shared__ LinePlaces lp;
  // parts of one KV head on one XCD (workgroup i runs on XCD i % 8)
  const int part = (blockIdx.x & 7) * (kChunkParts / 8) + (blockIdx.x >> 3);
  const int64_t total = line_total(a, s, lp, touch_kernargs<sizeof(BlockArgs) + sizeof(ChunkStep)>());
  const int64_t size = lane_of(chunk_part(total), 0);
  const int64_t begin = part * size, end = min(begin + size, total);
  if (threadIdx.x == 0) s.joins[part].n_rows = 0;
  walk(a, begin, end, s, lp, [&](const Segment& sg) {
    RowTile rt;
    rt.lo = chunk_key_tile(sg.from, sg.p.c);
    rt.hi = chunk_key_tile(sg.to, sg.p.c);
    rt.pos0 = sg.tile * sg.p.per;
    rt.n_rows = (chunk_end(sg.p, sg.tile) - rt.pos0) * a.gqa;
    if (thread_here() == 0 && sg.from > 0) {
      const int64_t stop = sg.at + chunk_cost(sg.p, sg.tile);
      const int col = chunk_quotient(sg.from - 1, size), first = part - col - 1;
      const int last = chunk_quotient(stop - 1, size);
      s.joins[part] = {rt.n_rows, col, join_groups(last - first + 1), first, last, sg.at, stop, size,
                       (int64_t)sg.start + rt.pos0, sg.p.c, chunk_key_tiles(sg.p, sg.tile), sg.g * a.gqa};
    }
    if (rt.lo >= rt.hi) return;
    rt.whole = rt.lo == 0 && rt.hi == chunk_key_tiles(sg.p, sg.tile);
    if (sg.p.c.rows < 256) attend_few(a, s, sg, rt, part, sm, sml);
    else attend_many(a, s, sg, rt, part, sm, list, sodd, scnt);
  });
}

// Joins the row tiles that more than one part served.  The workgroups (w, y) of all parts w that
// begin inside a row tile share its rows.  Two to four parts are the rule, read in one round (67 MB
// of parts 15 us; with rounds of eight 36 us); more than eight are read by up to eight groups of 32
// threads (128 parts of 64 rows 30 -> 6 us; from five parts on, row tiles of four to five took 14
// us instead of 10.5).  Most workgroups find nothing to do: what they read is one record.
namespace {
struct Joined {
  float m, l;
  f32x4 x;
  bool whole;   // one part had all key tiles, and wrote the rows
};
// Parts [i, end) of row rr, channels c .. + 3.
__device__ __forceinline__ Joined join_parts(const ChunkStep& s, const ChunkJoin& jn, int i, int end, int rr, int c) {
  Joined o = {-INFINITY, 0.f, {0.f, 0.f, 0.f, 0.f}, false};
  int lo = chunk_key_tile(max(i * jn.size - jn.at, (int64_t)0), jn.scale);   // first key tile of part i
  while (i < end) {
    // a round of parts, all loads first
    float2 ml[kMergeRound];
    f32x4 y[kMergeRound];
    bool there[kMergeRound];
#pragma unroll
    for (int k = 0; k < kMergeRound; ++k, ++i) {
      there[k] = false;
      if (i >= end) continue;
      const int hi = chunk_key_tile(min((i + 1) * jn.size, jn.stop) - jn.at, jn.scale);
      const bool all = lo == 0 && hi == jn.key_tiles;
      o.whole |= all;
      there[k] = lo < hi && !all;
      if (there[k]) {
        const int64_t slot = (int64_t)chunk_slot(i, lo) * s.slot_rows + rr;
        ml[k] = s.part_ml[slot];
        y[k] = *(const f32x4*)(s.part_o + slot * kHeadDim + c);
      }
      lo = hi;
    }
    float mn = o.m;
#pragma unroll
    for (int k = 0; k < kMergeRound; ++k)
      if (there[k]) mn = fmaxf(mn, ml[k].x);
    const float mu = mn > -INFINITY ? mn : 0.f, f0 = __builtin_amdgcn_exp2f(o.m - mu);
    o.m = mn;
    o.l *= f0;
#pragma unroll
    for (int j = 0; j < 4; ++j) o.x[j] *= f0;
#pragma unroll
    for (int k = 0; k < kMergeRound; ++k) {
      if (!there[k]) continue;
      const float f = __builtin_amdgcn_exp2f(ml[k].x - mu);
      o.l = fmaf(f, ml[k].y, o.l);
#pragma unroll
      for (int j = 0; j < 4; ++j) o.x[j] = fmaf(f, y[k][j], o.x[j]);
    }
  }
  return o;
}
}  // namespace
__global__ __launch_bounds__(kThreads) void k_chunk_merge(int gqa, ChunkStep s) {
  const int w = blockIdx.x + 1;
  const ChunkJoin jn = s.joins[w];
  if (jn.n_rows == 0) return;   // (the rest of the record is not written)
  const int log_g = jn.log_g;
  const int r0 = (jn.col * gridDim.y + blockIdx.y) * (kMergeRows >> log_g);
  if (r0 >= jn.n_rows) return;
  const int group = threadIdx.x >> 5, c = 4 * (threadIdx.x & 31);
  const int r = r0 + (group >> log_g), rr = min(r, jn.n_rows - 1);
  Joined o;
  if (log_g == 0) {
    o = join_parts(s, jn, jn.first, jn.last + 1, rr, c);
  } else {
    __shared__ f32x4 xs[kMergeGroups][32];
    __shared__ float2 mls[kMergeGroups];
    const int g = 1 << log_g, at = group & (g - 1), each = (jn.last - jn.first + g) >> log_g;
    o = join_parts(s, jn, jn.first + at * each, min(jn.first + (at + 1) * each, jn.last + 1), rr, c);
    xs[group][threadIdx.x & 31] = o.x;
    if (c == 0) mls[group] = make_float2(o.m, o.l);
    o.whole = __syncthreads_or(o.whole);
    if (at) return;
    for (int k = 1; k < g; ++k) o.m = fmaxf(o.m, mls[group + k].x);
    const float mu = o.m > -INFINITY ? o.m : 0.f;
    o.l = 0.f;
    o.x = (f32x4){0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < g; ++k) {
      const float f = __builtin_amdgcn_exp2f(mls[group + k].x - mu);
      const f32x4 y = xs[group + k][threadIdx.x & 31];
      o.l = fmaf(f, mls[group + k].y, o.l);
#pragma unroll
      for (int j = 0; j < 4; ++j) o.x[j] = fmaf(f, y[j], o.x[j]);
    }
  }
  if (o.whole || r >= jn.n_rows) return;
  const int i = by_gqa(s, r);
  uint16_t* op = s.out + (jn.row + i) * s.o_st + (jn.head + r - i * gqa) * s.o_sh + c;
  *(u32x2*)op = (u32x2){pack_bf16(o.x[0] / o.l, o.x[1] / o.l), pack_bf16(o.x[2] / o.l, o.x[3] / o.l)};
}

// Rows of a partial result: those of the largest row tile a call of `total` rows can have.
static int slot_rows(int64_t total, int gqa) { return chunk_rows(total * gqa); }
int64_t block_chunk_workspace_bytes(int64_t total, int gqa) {
  return (int64_t)2 * kChunkParts * slot_rows(total, gqa) * (kHeadDim * sizeof(float) + sizeof(float2)) +
         kChunkParts * sizeof(ChunkJoin);
}

hipError_t launch_chunk_attend(const BlockArgs& a, ChunkStep s, void* workspace, hipStream_t st) {
  s.gqa_inv = chunk_inverse(a.gqa);
  s.slot_rows = slot_rows(s.total, a.gqa);
  s.part_o = (float*)workspace;
  s.part_ml = (float2*)(s.part_o + (int64_t)2 * kChunkParts * s.slot_rows * kHeadDim);
  s.joins = (ChunkJoin*)(s.part_ml + (int64_t)2 * kChunkParts * s.slot_rows);
  k_chunk_attend<<<dim3(kChunkParts), kChunkThreads, 0, st>>>(a, s);
  if (hipError_t e = hipGetLastError()) return e;
  const int rows = (int)std::min<int64_t>(s.slot_rows, (int64_t)s.total * a.gqa);
  k_chunk_merge<<<dim3(kChunkParts - 1, (rows + kMergeRows - 1) / kMergeRows), kThreads, 0, st>>>(a.gqa, s);
  return hipGetLastError();
}

}  // namespace qv
