// Walks every workgroup of block-cache decode steps over random places, with the arithmetic
// of the kernels: each block of a pair that is split is served once, every segment has a
// slot of the workspace to itself, and the join of a pair reads exactly the slots of its
// segments.  Built with checks of undefined behaviour.
#include <algorithm>
#include <cstdio>
#include <map>
#include <random>
#include <vector>

#include "qv_parts.h"

using namespace qv;

static int fail(const char* what, int B, int H) {
  std::printf("%s: %d places, %d KV heads\n", what, B, H);
  return 1;
}

static int step(const std::vector<int>& lens, int max_context, int H, int* largest) {
  const int B = (int)lens.size(), n_pairs = B * H;
  std::vector<int> first(B);
  int total = 0;
  for (int b = 0; b < B; ++b) {
    first[b] = total;
    total += items_of(lens[b], max_context) * H;
  }
  const int size = part_items(total);
  *largest = std::max(*largest, size);
  std::map<int, int> slots;   // slot -> pair
  std::vector<std::vector<char>> served(n_pairs);
  for (int p = 0; p < n_pairs; ++p) {
    const int n = blocks_of(lens[p / H], max_context);
    served[p].assign(std::max(n, 0), 0);
    if (n > kSmall && !slots.emplace(p, p).second) return fail("slot of a pair", B, H);
  }
  for (int part = 0; part < kParts; ++part) {
    if ((int64_t)part * size >= total) break;
    const Span items = {part * size, std::min(part * size + size, total)};
    for (int b = 0; b < B; ++b) {
      const int per = items_of(lens[b], max_context);
      if (!per || first[b] >= items.end || first[b] + per * H <= items.begin) continue;
      const Span pairs = pairs_of(items, first[b], per, H);
      if (pairs.begin < 0 || pairs.end > H) return fail("pairs outside the place", B, H);
      for (int g = pairs.begin; g < pairs.end; ++g) {
        const Span blks = blocks_in(items, first[b], per, g);
        if (blks.begin >= blks.end) continue;
        if (blks.begin < 0 || blks.end > per - kSegCost) return fail("blocks outside the pair", B, H);
        for (int i = blks.begin; i < blks.end; ++i)
          if (served[b * H + g][i]++) return fail("block served twice", B, H);
        const int slot = n_pairs + part + b * H + g;
        if (slot >= kParts + 2 * n_pairs || !slots.emplace(slot, b * H + g).second) return fail("slot", B, H);
      }
    }
  }
  for (int p = 0; p < n_pairs; ++p) {
    const int per = items_of(lens[p / H], max_context);
    if (!per) continue;
    if (std::count(served[p].begin(), served[p].end(), 1) != per - kSegCost) return fail("block not served", B, H);
    const Span parts = parts_of(first[p / H] + p % H * per, per, size);
    for (int part = parts.begin; part < parts.end; ++part) {
      const auto at = slots.find(n_pairs + part + p);
      if (at == slots.end() || at->second != p) return fail("join of a slot that is not the pair's", B, H);
      slots.erase(at);
    }
    if (!slots.erase(p)) return fail("join of the open block", B, H);
  }
  return slots.empty() ? 0 : fail("segment that no join reads", B, H);
}

int main() {
  std::mt19937 rng(1);
  auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
  const int tops[] = {600, 3000, 20000, 140000};
  int largest = 0;
  for (int round = 0; round < 400; ++round) {
    const int B = pick(0, 3) ? pick(1, 40) : pick(60, 200), H = pick(1, 16), top = tops[pick(0, B > 40 ? 2 : 3)];
    std::vector<int> lens(B);
    for (int& t : lens) t = pick(0, 9) ? pick(0, top) : -1;
    if (step(lens, pick(0, 1) ? top + 1 : top, H, &largest)) return 1;
  }
  for (int len : {-1, 0, 575, 576, 577, 1 << 20})
    for (int H : {1, 16})
      if (step({len}, (1 << 20) + 1, H, &largest)) return 1;
  // the most items a call may have (counted in 32 bits)
  if (part_items(1 << 30) != ((1 << 30) + kParts - 1) / kParts) return 1;
  const int per = ((1 << 30) - 8 * kSegCost) / 8 / 64 * 64 + kSegCost, size = part_items(per * 8);
  for (int part = 0; part * (int64_t)size < per * 8; ++part) {
    const Span items = {part * size, std::min(part * size + size, per * 8)};
    const Span pairs = pairs_of(items, 0, per, 8);
    for (int g = pairs.begin; g < pairs.end; ++g) {
      const Span blks = blocks_in(items, 0, per, g);
      if (blks.begin < 0 || blks.end > per - kSegCost) return fail("largest", 1, 8);
    }
  }
  if (largest <= 256) return fail("no part of more than 64 blocks a wave", 0, 0);
  std::printf("ok\n");
  return 0;
}
