// Every part of random chunk steps on the host: each key tile of each row tile served once, a
// place of its own for every partial result, joins that read all of a row tile's.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <vector>

#include "qv_chunk.h"

using namespace qv;

#define CHECK(x)                                                        \
  do {                                                                  \
    if (!(x)) {                                                         \
      printf("line %d: %s (case %d)\n", __LINE__, #x, case_no);         \
      return 1;                                                         \
    }                                                                   \
  } while (0)

struct Tile {
  int s, g, t, v;
  int64_t at, stop;
};
struct Served {
  int part, lo, hi, slot;
};

int main() {
  std::mt19937_64 rng(5);
  auto pick = [&](int64_t lo, int64_t hi) { return lo + (int64_t)(rng() % (uint64_t)(hi - lo + 1)); };
  for (int case_no = 0; case_no < 1500; ++case_no) {
    const int gqa = (int)pick(1, 16), H_kv = (int)pick(1, 8);
    const int B = case_no % 10 == 0 ? (int)pick(65, 200) : (int)pick(1, 20);
    const int max_context = case_no % 7 == 0 ? 1 << 30 : 140000;
    int64_t room = case_no % 50 == 0 ? 60000 : 3000;
    std::vector<ChunkPlace> places;
    int64_t total = 0;
    std::vector<int64_t> before;
    for (int s = 0; s < B; ++s) {
      const int64_t most[4] = {0, 70, 5000, max_context + 5LL};
      const int held = pick(0, 9) == 0 ? -1 : (int)pick(0, most[pick(0, 3)]);
      const int n = (int)std::min<int64_t>(room, pick(0, 1) ? pick(0, 8) : pick(0, 3000));
      room -= n;
      const ChunkPlace p = chunk_place(held, n, gqa, chunk_inverse(gqa), H_kv, max_context);
      CHECK(p.n >= 0 && p.n <= n && (p.n == 0 || (held >= 0 && (int64_t)held + p.n <= max_context)));
      CHECK(p.per >= 1 && p.per * gqa <= p.c.rows && (int64_t)p.tiles * p.per >= p.n);
      CHECK(p.tiles == 0 || (int64_t)(p.tiles - 1) * p.per < p.n);
      CHECK(p.c.extra > 0 && (!p.solo || (p.c.rows == 32 && p.tiles <= 1)));
      for (int r = 0; r <= 256; ++r) CHECK(((uint32_t)r * chunk_inverse(gqa)) >> 16 == (uint32_t)(r / gqa));
      places.push_back(p);
      before.push_back(total);
      total += chunk_pair_cost(p) * H_kv;
    }
    if (total == 0) continue;
    const int64_t size = chunk_part(total);
    CHECK(size > 0 && size * kChunkParts >= total);

    // the row tiles on the line, by their lengths alone
    std::vector<Tile> tiles;
    int64_t at = 0;
    for (int s = 0; s < B; ++s)
      for (int g = 0; g < H_kv; ++g) {
        int64_t in_pair = 0;
        for (int t = 0; t < places[s].tiles; ++t) {
          CHECK(chunk_before(places[s], t) == in_pair);
          const int64_t c = chunk_cost(places[s], t);
          CHECK(c > 0);
          CHECK(chunk_tile_at(places[s], in_pair) == t && chunk_tile_at(places[s], in_pair + c - 1) == t);
          CHECK(chunk_key_tile(c, places[s].c) == chunk_key_tiles(places[s], t));
          tiles.push_back({s, g, t, chunk_key_tiles(places[s], t), at, at + c});
          at += c;
          in_pair += c;
        }
        CHECK(in_pair == chunk_pair_cost(places[s]));
        if (in_pair) CHECK(chunk_quotient((g + 1) * in_pair - 1, in_pair) == g && chunk_quotient(g * in_pair, in_pair) == g);
      }
    CHECK(at == total);

    // what the parts serve
    std::map<size_t, std::vector<Served>> served;
    std::vector<char> slots(2 * kChunkParts, 0);
    size_t i = 0;
    for (int w = 0; w < kChunkParts; ++w) {
      int64_t x = w * size;
      const int64_t end = std::min(x + size, total);
      while (x < end) {
        while (tiles[i].stop <= x) ++i;
        const int64_t stop = std::min(end, tiles[i].stop);
        const ChunkScale& sc = places[tiles[i].s].c;
        const int lo = chunk_key_tile(x - tiles[i].at, sc), hi = chunk_key_tile(stop - tiles[i].at, sc);
        if (lo < hi) {
          int slot = -1;
          if (lo > 0 || hi < tiles[i].v) {
            slot = chunk_slot(w, lo);
            CHECK(slot >= 0 && slot < 2 * kChunkParts && !slots[slot]);
            slots[slot] = 1;
          }
          served[i].push_back({w, lo, hi, slot});
        }
        x = stop;
      }
    }
    for (size_t j = 0; j < tiles.size(); ++j) {
      const Tile& t = tiles[j];
      int next = 0;
      for (const Served& v : served[j]) {
        CHECK(v.lo == next);
        next = v.hi;
      }
      CHECK(next == t.v);
      // the join: every part that begins inside the row tile knows the first one that serves it
      int joins = 0, joined = 0;
      for (int w = 1; w < kChunkParts; ++w) {
        const int64_t x0 = w * size;
        if (x0 >= total || x0 <= t.at || x0 >= t.stop) continue;
        const int col = chunk_quotient(x0 - t.at - 1, size), first = w - col - 1;
        const int last = chunk_quotient(t.stop - 1, size);
        CHECK(first >= 0 && first * size <= t.at && (first + 1) * size > t.at && w <= last && last < kChunkParts);
        CHECK(col == joins);
        ++joins;
        std::vector<Served> got;
        bool whole = false;
        for (int k = first; k <= last; ++k) {
          const int lo = chunk_key_tile(std::max<int64_t>(k * size - t.at, 0), places[t.s].c);
          const int hi = chunk_key_tile(std::min(k * size + size, t.stop) - t.at, places[t.s].c);
          if (lo >= hi) continue;
          if (lo == 0 && hi == t.v) whole = true;
          got.push_back({k, lo, hi, chunk_slot(k, lo)});
        }
        CHECK(got.size() == served[j].size());
        for (size_t k = 0; k < got.size(); ++k) {
          CHECK(got[k].part == served[j][k].part && got[k].lo == served[j][k].lo && got[k].hi == served[j][k].hi);
          CHECK(whole ? served[j][k].slot < 0 : got[k].slot == served[j][k].slot);
        }
        if (col == 0) joined = last - first;
      }
      CHECK(joins == joined);   // parts that share the rows: all but the first
      if (served[j].size() > 1) CHECK(joins > 0);
    }
  }
  printf("ok\n");
  return 0;
}
