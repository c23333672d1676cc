// How the workgroups of a chunk step walk the line, KV heads taken together included: every key
// tile of every row tile served once.  Without arguments random steps; else one step, given as
// H_kv, query heads per KV head, max_context, then tokens held and new tokens of every place: prints
// what its workgroups meet.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "qv_chunk.h"

using namespace qv;

#define CHECK(x)                                          \
  do {                                                    \
    if (!(x)) {                                           \
      printf("line %d: %s (case %d)\n", __LINE__, #x, no); \
      return false;                                       \
    }                                                     \
  } while (0)

struct Met {
  int heads = 0;         // most KV heads of a segment
  int rounds = 0;        // most segments of one place that took several heads, in one workgroup
  int few = 0;           // most pages of a segment of up to 64 rows that are one wave's
  int wide = 0;          // most pages of a segment of 256 rows
  int whole = 0;         // most whole row tiles of 256 rows in a workgroup
  int keys = 0;          // most key tiles of a segment of 256 rows
};

static bool step(int no, int H_kv, int gqa, int max_context, const std::vector<int>& held, const std::vector<int>& lens,
                 Met* met) {
  std::vector<ChunkPlace> places;
  std::vector<int64_t> incl;
  int64_t total = 0;
  for (size_t s = 0; s < held.size(); ++s) {
    places.push_back(chunk_place(held[s], lens[s], gqa, chunk_inverse(gqa), H_kv, max_context));
    total += chunk_pair_cost(places[s]) * H_kv;
    incl.push_back(total);
  }
  if (!total) return true;
  const int64_t size = chunk_part(total);
  std::vector<std::vector<std::vector<int>>> next(held.size());   // key tiles served, in order
  for (size_t s = 0; s < held.size(); ++s)
    next[s].assign(H_kv, std::vector<int>(std::max(places[s].tiles, 1), 0));
  for (int w = 0; w < kChunkParts; ++w) {
    int64_t x = w * size;
    const int64_t end = std::min(x + size, total);
    int whole = 0;
    while (x < end) {
      const size_t s = std::upper_bound(incl.begin(), incl.end(), x) - incl.begin();
      const ChunkPlace& p = places[s];
      const int64_t pair = chunk_pair_cost(p), first = incl[s] - pair * H_kv;
      int heads, rounds = 0;
      for (int g = chunk_quotient(x - first, pair); g < H_kv && x < end; g += heads) {
        const int64_t at = first + g * pair;
        heads = 1;
        if (p.solo && x == at) {
          const int most = std::min(kChunkWaves, H_kv - g);
          while (heads < most && end - x >= (heads + 1) * pair) ++heads;
        }
        for (int t = chunk_tile_at(p, x - at); t < p.tiles && x < end; ++t) {
          const int64_t begin = at + chunk_before(p, t), stop = std::min(end, begin + chunk_cost(p, t));
          const int lo = chunk_key_tile(x - begin, p.c), hi = chunk_key_tile(stop - begin, p.c);
          const int all = chunk_key_tiles(p, t), pages = std::max(std::min(hi, p.c.blocks) - lo, 0);
          if (heads > 1) {
            CHECK(heads <= kChunkWaves && p.tiles == 1 && p.c.rows == 32 && lo == 0 && hi == all);
            CHECK((int64_t)p.held + p.n <= kSoloTiles * kBlockTokens);
            ++rounds;
          }
          for (int h = g; h < g + heads; ++h) {
            CHECK(h < H_kv && next[s][h][t] == lo && (lo < hi || next[s][h][t] == lo));
            next[s][h][t] = hi;
          }
          met->heads = std::max(met->heads, heads);
          if (p.c.rows < 256) {
            const int waves = heads > 1 ? 1 : kChunkWaves >> (p.c.rows == 32 ? 0 : 1);
            met->few = std::max(met->few, (pages + waves - 1) / waves);
          } else {
            met->wide = std::max(met->wide, pages);
            met->keys = std::max(met->keys, hi - lo);
            whole += lo == 0 && hi == all;
          }
          x = heads > 1 ? at + heads * pair : stop;
        }
      }
      met->rounds = std::max(met->rounds, rounds);
    }
    CHECK(x == std::max(end, w * size));
    met->whole = std::max(met->whole, whole);
  }
  for (size_t s = 0; s < held.size(); ++s)
    for (int h = 0; h < H_kv; ++h)
      for (int t = 0; t < places[s].tiles; ++t) CHECK(next[s][h][t] == chunk_key_tiles(places[s], t));
  return true;
}

int main(int argc, char** argv) {
  Met met;
  if (argc > 4) {
    std::vector<int> held, lens;
    for (int i = 4; i + 1 < argc; i += 2) {
      held.push_back(atoi(argv[i]));
      lens.push_back(atoi(argv[i + 1]));
    }
    if (!step(0, atoi(argv[1]), atoi(argv[2]), atoi(argv[3]), held, lens, &met)) return 1;
    printf("%d %d %d %d %d %d\n", met.heads, met.rounds, met.few, met.wide, met.whole, met.keys);
    return 0;
  }
  std::mt19937_64 rng(7);
  auto pick = [&](int64_t lo, int64_t hi) { return lo + (int64_t)(rng() % (uint64_t)(hi - lo + 1)); };
  for (int no = 0; no < 600; ++no) {
    const int gqa = (int)pick(1, 16), H_kv = (int)pick(1, no % 3 ? 16 : 40), B = (int)pick(1, no % 4 ? 300 : 30);
    const int most_held[4] = {0, 70, 1100, 140000}, few = no % 4 ? 2 : 3;
    std::vector<int> held, lens;
    for (int s = 0; s < B; ++s) {
      held.push_back(pick(0, 9) == 0 ? -1 : (int)pick(0, most_held[pick(0, few)]));
      lens.push_back((int)(pick(0, 30) ? pick(0, 8) : pick(0, 1500)));
    }
    if (!step(no, H_kv, gqa, 140000, held, lens, &met)) return 1;
  }
  if (met.heads != kChunkWaves || met.rounds < 2) {
    printf("not reached: %d heads, %d rounds\n", met.heads, met.rounds);
    return 1;
  }
  printf("ok\n");
  return 0;
}
