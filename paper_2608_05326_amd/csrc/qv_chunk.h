// How the attention of new tokens over the block cache is cut into parts.  The rows of a
// (place, KV head) pair are its (position, head) pairs, row = position G + head; a row tile
// is as many whole positions as fit the rows that a workgroup holds.  Row tile t of a place
// with L tokens held sees the keys up to its last position, in tiles of 64 keys.  All row
// tiles, in the order place, KV head, tile, are laid on one line, each as long as its time is
// expected to be: a weight for every key that it sees, and what it costs beside them.  The
// line is cut into equal parts, one per workgroup.  Lengths are linear in t, so a place's sum
// has a closed form and nothing is tabulated.  Arithmetic only, so that it also compiles for the
// host.
#pragma once
#include "qv_layout.h"

namespace qv {

constexpr int kChunkParts = 256;    // one workgroup of eight waves to a compute unit
constexpr int kChunkMin = 1024;     // the least a part is
constexpr int kSoloTiles = 16;      // key tiles that a wave takes alone (attend_few)
constexpr int kChunkWaves = 8;

// Rows of a workgroup for a place with this many in all.
QV_HD int chunk_rows(int64_t rows) { return rows <= 32 ? 32 : rows <= 64 ? 64 : 256; }

// How the key tiles of a place's row tiles lie on the line: `extra` first, then the complete
// blocks, then the tiles of rows in bf16.
struct ChunkScale {
  int rows;           // rows of a workgroup
  int extra;          // length beside the keys
  int blocks;         // complete blocks
};
// Length of a key of a complete block, and of one in bf16: many rows at once are bound by their
// products, few by the bytes of the pages (microseconds a tile of 64 keys, over the whole chip:
// 256 rows 1.8 and 2.3, 64 rows 1.1, 32 rows 0.5; a row tile costs 10 to 16 beside them).
QV_HD int chunk_page_key(int rows) { return rows <= 32 ? 2 : rows <= 64 ? 4 : 8; }
QV_HD int chunk_row_key(int rows) { return rows <= 32 ? 2 : rows <= 64 ? 4 : 10; }

struct ChunkPlace {
  int held, n;        // tokens held, new tokens (0: none)
  int per;            // positions of a row tile
  int tiles;          // row tiles of a KV head
  ChunkScale c;
  bool solo;          // a row tile is one wave's: a workgroup takes up to eight KV heads at once
};

// 2^16 / gqa, rounded up: (r * this) >> 16 is r / gqa for r <= 256 and gqa <= 16.
QV_HD uint32_t chunk_inverse(int gqa) { return (65536u + gqa - 1) / gqa; }

// A place with `len` tokens held that is given `rows` new ones; max_context limits both.
QV_HD ChunkPlace chunk_place(int len, int rows, int gqa, uint32_t gqa_inv, int H_kv, int max_context) {
  ChunkPlace p;
  p.held = len;
  p.n = len < 0 || len >= max_context ? 0 : rows < max_context - len ? rows : max_context - len;
  p.c.rows = chunk_rows((int64_t)p.n * gqa);
  p.c.blocks = len < 0 ? 0 : len / kBlockTokens;
  p.per = (int)((uint32_t)p.c.rows * gqa_inv >> 16);
  p.tiles = p.n <= p.per ? p.n > 0 : (p.n + p.per - 1) / p.per;
  p.solo = p.c.rows == 32 && p.tiles == 1 && (int64_t)p.held + p.n <= kSoloTiles * kBlockTokens;
  p.c.extra = p.c.rows > 64 ? (p.c.blocks ? 4480 : 2944)
                            : !p.solo ? 2816 : 1536 / (H_kv < kChunkWaves ? H_kv : kChunkWaves);
  return p;
}

// New tokens up to the end of row tile t.
QV_HD int chunk_end(const ChunkPlace& p, int t) {
  const int64_t e = (int64_t)(t + 1) * p.per;
  return e < p.n ? (int)e : p.n;
}

// Length of row tile t on the line, and of the t row tiles before it.
QV_HD int64_t chunk_held_cost(const ChunkPlace& p) {
  return (int64_t)p.c.blocks * (kBlockTokens * chunk_page_key(p.c.rows)) +
         (p.held - p.c.blocks * kBlockTokens) * chunk_row_key(p.c.rows) + p.c.extra;
}
QV_HD int64_t chunk_cost(const ChunkPlace& p, int t) {
  return chunk_held_cost(p) + (int64_t)chunk_end(p, t) * chunk_row_key(p.c.rows);
}
QV_HD int64_t chunk_before(const ChunkPlace& p, int t) {
  int64_t rows = (int64_t)p.per * t * (t + 1) / 2;
  if (t == p.tiles && t) rows -= (int64_t)p.tiles * p.per - p.n;
  return t * chunk_held_cost(p) + rows * chunk_row_key(p.c.rows);
}
QV_HD int64_t chunk_pair_cost(const ChunkPlace& p) { return chunk_before(p, p.tiles); }

// The row tile of a pair that holds point x of it (0 <= x < its cost).
QV_HD int chunk_tile_at(const ChunkPlace& p, int64_t x) {
  int lo = 0, hi = p.tiles - 1;
  while (lo < hi) {
    const int mid = lo + (hi - lo + 1) / 2;
    if (chunk_before(p, mid) <= x) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// x / y for 0 <= x < 2^62, y > 0 and a quotient below 2^30: a device's 64-bit division is long,
// an fp32 one is right to 2^-22 of it (small quotients: to one).
QV_HD int chunk_quotient(int64_t x, int64_t y) {
  int q = (int)((float)x / (float)y);
  while ((int64_t)q * y > x) --q;
  while ((int64_t)(q + 1) * y <= x) ++q;
  return q;
}

// Tiles of 64 keys that row tile t sees, and the first of them at or past point x of a row
// tile.
QV_HD int chunk_key_tiles(const ChunkPlace& p, int t) {
  return (int)(((int64_t)p.held + chunk_end(p, t) + kBlockTokens - 1) / kBlockTokens);
}
QV_HD int chunk_key_tile(int64_t x, const ChunkScale& c) {
  static_assert(kBlockTokens == 64, "shifts");
  const int64_t y = x - c.extra;
  if (y <= 0) return 0;
  const int shift = c.rows <= 32 ? 7 : c.rows <= 64 ? 8 : 9;        // a tile of a block
  const int64_t z = y - ((int64_t)c.blocks << shift);
  if (z <= 0) return (int)((y + (1 << shift) - 1) >> shift);
  if (c.rows <= 64) return c.blocks + (int)((z + (1 << shift) - 1) >> shift);
  return c.blocks + (int)((uint32_t)((z + 127) >> 7) + 4) / 5;      // 640 a tile
}

// A row's query, its largest magnitude in [2^ex, 2^(ex + 1)), is taken times 2^-shift, which comes
// back with the logits' scale m 2^scale_exp, 1/2 <= m < 1, as 2^shift.  Into [2^-20, 2^-19):
// products with the largest keys, of codes or bf16, and their sums stay in range.  A row of small
// numbers or zeros only so far that the scale of its logits stays a normal number: masked ones
// are -infinity, which times zero were no number.  A row of large numbers only so far that the
// scale stays below 2^100: keys as small as it is large give logits of ordinary size, from
// products that are normal numbers (where products are out of range, their logits are, too).
QV_HD int chunk_query_shift(int ex, int scale_exp) {
  const int s = ex + 20, least = -125 - scale_exp, most = 100 - scale_exp;
  return s < least ? least : s > most ? most : s;
}

// Length of a part, given the line's.
QV_HD int64_t chunk_part(int64_t total) {
  const int64_t s = (total + kChunkParts - 1) / kChunkParts;
  return s > kChunkMin ? s : kChunkMin;
}

// Where part w leaves the partial result of a row tile that it serves from key tile `lo` on,
// not whole: a part has at most one such row tile that it begins and one that it does not.
QV_HD int chunk_slot(int w, int lo) { return 2 * w + (lo == 0); }

}  // namespace qv
