// Which blocks of the 8-bit cache a workgroup of a decode step serves.  A (place, KV head)
// pair with more than kSmall complete blocks has an item for each of them and kSegCost more
// (what a segment costs beside its blocks); the items of all pairs, in pair order, are cut
// into kParts equal parts.  Arithmetic only, so that it also compiles for the host.
#pragma once
#include "qv_layout.h"

namespace qv {

// Two workgroups fit a compute unit (214 registers; at 168, for three, the loop spills):
// 480 parts leave room for the pairs' own workgroups of a small batch beside them.  8 KV
// heads: one sequence of 32K 22.2 us a step with 480 parts, 23.1 with 512, 28 with 768.
constexpr int kParts = 480;
// A pair of at most kSmall complete blocks (two rounds of four waves) is one workgroup's,
// and a segment counts as kSegCost blocks beside its own: without either, a part of many
// short sequences outlasts the others (32 ragged places, 985 MB: 329 -> 191 us).
constexpr int kSmall = 8, kSegCost = 4;

// Complete blocks of a place that holds a sequence with room for a token, else -1.
QV_HD int blocks_of(int len, int max_context) { return len < 0 || len >= max_context ? -1 : len / kBlockTokens; }

// Items of one of its pairs.
QV_HD int items_of(int len, int max_context) {
  const int n = blocks_of(len, max_context);
  return n > kSmall ? n + kSegCost : 0;
}

// Items of a part, equal parts but for the last: part p has items [p size, p size + size).
QV_HD int part_items(int total) { return (int)(((uint32_t)total + kParts - 1) / kParts); }

struct Span {
  int begin, end;
};

// Pairs (KV heads) of a place that items [part.begin, part.end) touch; the place's first item
// is `first`, and each of its pairs has `per`.
QV_HD Span pairs_of(Span part, int first, int per, int H_kv) {
  const int lo = part.begin > first ? part.begin - first : 0, all = per * H_kv;
  const int hi = part.end - first < all ? part.end - first : all;
  return {lo / per, (hi + per - 1) / per};
}

// Blocks of pair g of that place in those items (none: end <= begin).
QV_HD Span blocks_in(Span part, int first, int per, int g) {
  const int at = first + g * per, n = per - kSegCost;
  return {part.begin > at ? part.begin - at : 0, part.end - at < n ? part.end - at : n};
}

// Parts that hold blocks of the pair whose first item is `at`: [begin, end).
QV_HD Span parts_of(int at, int per, int size) { return {at / size, (at + per - kSegCost - 1) / size + 1}; }

}  // namespace qv
