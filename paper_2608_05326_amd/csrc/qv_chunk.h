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

struct ChunkPlace {
  int held, n;        // tokens held, new tokens (0: none)
  int rows, per;      // rows of a workgroup, positions of a row tile
  int tiles;          // row tiles of a KV head
  int extra;          // length of a row tile on the line beside its keys'
  bool solo;          // a row tile is one wave's: a workgroup takes up to eight KV heads at once
};

// A place with `len` tokens held that is given `rows` new ones; max_context limits both.
QV_HD ChunkPlace chunk_place(int len, int rows, int gqa, int H_kv, int max_context) {
  ChunkPlace p;
  p.held = len;
  p.n = len < 0 || len >= max_context ? 0 : rows < max_context - len ? rows : max_context - len;
  p.rows = chunk_rows((int64_t)p.n * gqa);
  p.per = p.rows / gqa;
  p.tiles = (p.n + p.per - 1) / p.per;
  p.solo = p.rows == 32 && p.tiles == 1 && (int64_t)p.held + p.n <= kSoloTiles * kBlockTokens;
  p.extra = p.rows > 64 ? 3072 : !p.solo ? 2304 : 1536 / (H_kv < kChunkWaves ? H_kv : kChunkWaves);
  return p;
}
// log2 of what a key costs on the line, by the rows of its workgroup.
QV_HD int chunk_weight(int rows) { return rows <= 32 ? 1 : rows <= 64 ? 2 : 3; }

// New tokens up to the end of row tile t.
QV_HD int chunk_end(const ChunkPlace& p, int t) {
  const int64_t e = (int64_t)(t + 1) * p.per;
  return e < p.n ? (int)e : p.n;
}

// Length of row tile t on the line, and of the t row tiles before it.
QV_HD int64_t chunk_cost(const ChunkPlace& p, int t) {
  return (((int64_t)p.held + chunk_end(p, t)) << chunk_weight(p.rows)) + p.extra;
}
QV_HD int64_t chunk_before(const ChunkPlace& p, int t) {
  int64_t keys = (int64_t)t * p.held + (int64_t)p.per * t * (t + 1) / 2;
  if (t == p.tiles && t) keys -= (int64_t)p.tiles * p.per - p.n;
  return (keys << chunk_weight(p.rows)) + (int64_t)t * p.extra;
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

// x / y for 0 <= x < 2^62 with a quotient below 2^30 (a device's 64-bit division is long).
QV_HD int chunk_quotient(int64_t x, int64_t y) {
  int q = (int)((double)x / (double)y);
  if ((int64_t)q * y > x) --q;
  if ((int64_t)(q + 1) * y <= x) ++q;
  return q;
}

static_assert(kBlockTokens == 64, "key tiles");
// Tiles of 64 keys that row tile t sees, and the first of them at or past point x of a row
// tile of a place with these rows and extra.
QV_HD int chunk_key_tiles(const ChunkPlace& p, int t) {
  return (int)(((int64_t)p.held + chunk_end(p, t) + kBlockTokens - 1) / kBlockTokens);
}
QV_HD int chunk_key_tile(int64_t x, int rows, int extra) {
  const int64_t y = x - extra;
  const int shift = 6 + chunk_weight(rows);
  return y <= 0 ? 0 : (int)((y + (1 << shift) - 1) >> shift);
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
