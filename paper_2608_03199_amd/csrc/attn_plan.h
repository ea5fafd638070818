// attn_plan.h -- how the packed attention's work is cut into items, and the bias's buckets.
// Host code without HIP: the tests compile it by itself.
//
// Every sequence is cut into row tiles (forward, dQ) and key tiles (dK, dV) for each key
// head; a work-group of a launch takes one item, so ragged batches launch no empty
// work-groups.
#pragma once

#include <math.h>
#include <stdint.h>
#include <stdlib.h>

#include <algorithm>
#include <vector>

namespace sieve {

// One work-group's share.  The rows of a sequence for one key head are its queries
// times the G = heads / kv_heads query heads that read it: row r is query r / G,
// head kvh * G + r % G, so that the heads of a group share every key they load.
struct AttnItem {
  int64_t q0, k0;   // first query and key token of the sequence in the packed batch
  int32_t nq, nk;   // its queries and keys
  int32_t kvh;
  int32_t row;      // first row of the tile (forward, dq), or first key (dk and dv)
  int32_t lo, hi;   // keys to go through (forward, dq), or rows (dk and dv)
  int32_t part;     // forward, dk and dv: slot of a partial result, -1 where the item is its
                    // whole tile; dq: number of the row tile among all sequences
  int32_t tile0, ntiles;  // dk and dv: the sequence's row tiles of the dq pass
  int32_t pad;
};

// One row tile whose keys, or key tile whose rows, several items shared.
struct AttnJoin {
  int64_t t0;                // first query (key) token of the sequence
  int32_t n, kvh, row;       // its queries (keys), the head, the tile's first row (key)
  int32_t part0, parts, pad;
};

constexpr int kAttnPad = 64;      // relative positions past the distance in the bias table
constexpr int kAttnRows = 128;    // rows of a tile: 4 waves of 32
// Rows of a tile whose 4 waves share the keys out, where no sequence has more and one has more
// than kAttnFewKeys keys.  One query over 32 documents of 1,000..30,000 (16 heads over 4 of 128,
// bf16): 227 us, with tiles of 128 rows 247; over 8 documents of 512 10.1, not 14.8; over 512 of
// 2,048 (8 heads over 2 of 128, f32) 532, not 1,176.  Up to 64 keys the waves have nothing to
// share: 512 documents of 4..32 tokens (12 heads of 64, f16) 27 us with tiles of 128 rows, with
// these 55; 512 queries over 64 keys each 10.1 and 18.9 (16 over 4 of 64, f16), 72 and 152 (12 of
// 64, f32), and in no case measured slower by more than 3%.  Between, it depends on the type and
// how many there are: 512 queries over 512 keys each 108 and 137 (16 over 4 of 128, bf16), 309
// and 169 (8 over 2 of 128, f32).
constexpr int kAttnFewRows = 32;
constexpr int kAttnFewKeys = 64;
constexpr int kAttnKeys = 128;    // keys of a dk and dv tile

constexpr int kXcds = 8;
constexpr int64_t kMaxRows = (int64_t(1) << 31) - (int64_t(1) << 16);  // of a sequence
constexpr int64_t kMaxTokens = int64_t(1) << 40;                       // of a batch
// Items of a list: work-groups of a launch, which may have fewer than 2^32 threads.
constexpr int kAttnThreads = 256;
constexpr int64_t kMaxItems = ((int64_t(1) << 32) - 1) / kAttnThreads;
// A forward pass with fewer items than this shares the keys of its row tiles out, at least
// kMinKeys to an item (below that the joining costs more than the reading).  bf16, 16 heads
// over 4 of 128: one query over 20,000 keys 31 us, not shared out 207; one query over 32
// documents of 1,000..30,000 227, not 498; with 2,048 items 257.  Two causal documents of
// 5,000..6,100 310, with 2,048 items 344, with 512 305; 12,007 causal tokens 670, with 2,048
// items 644.  At least 256 keys: the 20,000 take 39 us; 1,024 keys: 30, but 1,000 tokens of
// 12 heads of 64 25.0 instead of 22.7.
constexpr int kWantItems = 1024;
constexpr int kMinKeys = 512;
// The same for dK and dV, whose items are tiles of keys and share out their rows.  More items
// than the GPU holds at once (two to each of 256 CUs) also even out the causal tiles, the
// first of which are seen by every row and the last by few.  Backward pass of the two causal
// documents: 965 us, not shared out 1,571, with 512 items 1,048, with 2,048 998.  Rows of at
// least 512: 969; 4,096: 948, but 4,096 tokens of 4 heads of 64 take 184 instead of 136.
constexpr int kWantKvItems = 1024;
constexpr int kMinRows = 1024;

// Bucket of a relative position (key minus query).  The logarithm's edges are decided in
// 80-bit arithmetic with room for its rounding: where the exact value is a whole number the
// result is that number.
inline int bucket_of(int rel, int buckets, int distance, bool causal) {
  const int side = causal ? buckets : buckets / 2;
  const int base = rel > 0 && !causal ? side : 0;
  const int m = causal ? std::max(-rel, 0) : std::abs(rel);
  const int exact = side / 2;
  if (m < exact) return base + m;
  if (m >= distance) return base + side - 1;
  const long double x = (side - exact) * (logl((long double)m / exact) /
                                          logl((long double)distance / exact));
  return base + std::min(exact + (int)floorl(x + 1e-12L), side - 1);
}

// The order of a list of items: those of a sequence and key head follow one another, the list
// is cut into eight runs of equal cost, one for each XCD (consecutive work-groups go to
// consecutive XCDs), so that an L2 reads a sequence's keys once, and in a run the longest items
// come first, so that no long one is left at the end.
inline void order_items(std::vector<AttnItem>& items) {
  const int64_t n = (int64_t)items.size();
  if (n < 2) return;
  // an item's cost: its rows or keys to go through, and a fixed part for its start and end
  auto cost = [](const AttnItem& x) { return (int64_t)(x.hi - x.lo) + 256; };
  int64_t total = 0;
  for (const auto& x : items) total += cost(x);
  std::vector<AttnItem> runs[kXcds];
  int64_t sum = 0;
  for (const auto& x : items) {
    runs[std::min<int64_t>(sum * kXcds / total, kXcds - 1)].push_back(x);
    sum += cost(x);
  }
  for (auto& r : runs)
    std::stable_sort(r.begin(), r.end(),
                     [&](const AttnItem& p, const AttnItem& q) { return cost(p) > cost(q); });
  size_t at = 0;
  for (size_t i = 0; at < (size_t)n; ++i)
    for (int x = 0; x < kXcds; ++x)
      if (i < runs[x].size()) items[at++] = runs[x][i];
}

// Cuts the ranges of a list that is too short for the GPU into shares of about the same
// length, a multiple of 128 and at least `least`; join_of(item) starts the record that brings
// an item's shares together.
template <typename F>
void share_out(std::vector<AttnItem>& items, std::vector<AttnJoin>& joins, int want, int least,
               int32_t& parts, F join_of) {
  if (items.empty() || (int64_t)items.size() >= 2 * (int64_t)want) return;
  int64_t total = 0;
  for (const auto& x : items) total += x.hi - x.lo;
  const int64_t share = std::max<int64_t>(least, (total / want + 127) / 128 * 128);
  std::vector<AttnItem> cut;
  for (const auto& x : items) {
    const int64_t length = (int64_t)x.hi - x.lo, n = (length + share / 2) / share;
    if (n < 2) {
      cut.push_back(x);
      continue;
    }
    const int64_t each = ((length + n - 1) / n + 127) / 128 * 128;
    AttnJoin j = join_of(x);
    j.part0 = parts;
    for (int64_t at = x.lo; at < x.hi; at += each) {
      AttnItem y = x;
      y.lo = (int32_t)at;
      y.hi = (int32_t)std::min<int64_t>(at + each, x.hi);
      y.part = parts++;
      ++j.parts;
      cut.push_back(y);
    }
    joins.push_back(j);
  }
  items.swap(cut);
}

struct AttnLists {
  bool few = false;       // forward tiles are of kAttnFewRows rows (its comment)
  int32_t row_tiles = 0;  // dq tiles of one key head
  int32_t parts = 0, kv_parts = 0;  // partial results of the forward pass, and of dk and dv
  std::vector<AttnItem> fwd, dq, dkv;
  std::vector<AttnJoin> joins, kv_joins;
};

// Sizes of a batch's lists before they are shared out (which only adds to short ones).
struct AttnCounts {
  bool few;               // AttnLists::few
  int64_t fwd, dq, dkv;   // items
};
inline AttnCounts count_items(const int64_t* qo, const int64_t* ko, int64_t nseq, int kv_heads,
                              int G) {
  int64_t most_rows = 0, most_keys = 0, rows128 = 0, rows32 = 0, keys = 0;
  for (int64_t s = 0; s < nseq; ++s) {
    const int64_t rows = (qo[s + 1] - qo[s]) * G;
    most_rows = std::max(most_rows, rows);
    most_keys = std::max(most_keys, ko[s + 1] - ko[s]);
    rows128 += (rows + kAttnRows - 1) / kAttnRows;
    rows32 += (rows + kAttnFewRows - 1) / kAttnFewRows;
    keys += (ko[s + 1] - ko[s] + kAttnKeys - 1) / kAttnKeys;
  }
  const bool few = most_rows <= kAttnFewRows && most_keys > kAttnFewKeys;
  return {few, (few ? rows32 : rows128) * kv_heads, rows128 * kv_heads, keys * kv_heads};
}

// Whether each list fits a launch; that of dK and dV has a work-group more for each head, for
// the bias's gradient.
inline bool lists_fit(const AttnCounts& n, int64_t heads) {
  return n.fwd <= kMaxItems && n.dq <= kMaxItems && n.dkv + heads <= kMaxItems;
}

// The items of a batch: qo and ko are nseq + 1 offsets each, G query heads to a key head.
// False where there are too many.
inline bool make_lists(const int64_t* qo, const int64_t* ko, int64_t nseq, int kv_heads, int G,
                       bool causal, AttnLists* out) {
  AttnLists& p = *out;
  const AttnCounts counts = count_items(qo, ko, nseq, kv_heads, G);
  if (!lists_fit(counts, (int64_t)kv_heads * G)) return false;
  p.few = counts.few;
  const int tile = p.few ? kAttnFewRows : kAttnRows;
  int32_t tile0 = 0;
  for (int64_t s = 0; s < nseq; ++s) {
    AttnItem x{};
    x.q0 = qo[s];
    x.k0 = ko[s];
    x.nq = (int32_t)(qo[s + 1] - qo[s]);
    x.nk = (int32_t)(ko[s + 1] - ko[s]);
    const int64_t rows = (int64_t)x.nq * G, shift = (int64_t)x.nk - x.nq;
    x.tile0 = tile0;
    x.ntiles = (int32_t)((rows + kAttnRows - 1) / kAttnRows);
    tile0 += x.ntiles;
    // keys that rows up to `last` see
    auto keys_of = [&](int64_t last) {
      return causal ? (int32_t)std::clamp<int64_t>(last / G + shift + 1, 0, x.nk) : x.nk;
    };
    for (x.kvh = 0; x.kvh < kv_heads; ++x.kvh) {
      x.lo = 0;
      x.part = -1;
      for (int64_t r = 0; r < rows; r += tile) {
        x.row = (int32_t)r;
        x.hi = keys_of(std::min<int64_t>(r + tile, rows) - 1);
        p.fwd.push_back(x);
      }
      for (int64_t r = 0; r < rows; r += kAttnRows) {
        x.row = (int32_t)r;
        x.hi = keys_of(std::min<int64_t>(r + kAttnRows, rows) - 1);
        x.part = x.tile0 + (int32_t)(r / kAttnRows);
        p.dq.push_back(x);
      }
      x.hi = (int32_t)rows;
      x.part = -1;
      for (int64_t k = 0; k < x.nk; k += kAttnKeys) {
        x.row = (int32_t)k;
        x.lo = causal ? (int32_t)std::clamp<int64_t>((k - shift) * G, 0, rows) : 0;
        p.dkv.push_back(x);
      }
    }
  }
  // too few items to fill the GPU: share the keys (the rows) of the long ones out
  share_out(p.fwd, p.joins, kWantItems, kMinKeys, p.parts,
            [](const AttnItem& x) { return AttnJoin{x.q0, x.nq, x.kvh, x.row, 0, 0, 0}; });
  share_out(p.dkv, p.kv_joins, kWantKvItems, kMinRows, p.kv_parts,
            [](const AttnItem& x) { return AttnJoin{x.k0, x.nk, x.kvh, x.row, 0, 0, 0}; });
  p.row_tiles = tile0;
  order_items(p.fwd);
  order_items(p.dq);
  order_items(p.dkv);
  return true;
}

}  // namespace sieve
