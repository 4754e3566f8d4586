// seq_plan.hpp -- in which order the window attention's workgroups take their work, and how
// its backward pass over keys is cut into workgroups.  Plain C++: the kernels and the host
// side use it, and it can be replayed without a GPU.
#pragma once

#include <algorithm>
#include <cstdint>

#include "../../include/qd_seq.h"

#ifdef __HIPCC__
#define SEQ_BOTH __host__ __device__ inline
#else
#define SEQ_BOTH inline
#endif

namespace seq {

constexpr int kFill = 512;             // workgroups that fill the card: two per compute unit
constexpr int kKeyRows = 128;          // keys of a block, which a workgroup has
constexpr int kUnitRows = 32;          // query rows of a unit of its work, of one head

SEQ_BOTH int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Workgroups that follow each other go round the card's eight XCDs, each with an L2
// cache of its own.  This puts the `per_list` items of a list, which read the same
// keys, on one XCD: lists are dealt to the XCDs in turn where their number allows
// (so that episodes of different lengths even out), else in contiguous pieces.
constexpr int kXcds = 8;
SEQ_BOTH int xcd_order(int id, int count, int per_list) {
  const int x = id % kXcds, y = id / kXcds;
  if (count / per_list % kXcds == 0) return (y / per_list * kXcds + x) * per_list + y % per_list;
  const int per = count / kXcds, rest = count % kXcds;
  return x * per + (x < rest ? x : rest) + y;
}

// The same with every list on every XCD: the items are dealt one of each list in turn,
// and one list further from item to item, so that a list's neighbours go round the XCDs.
SEQ_BOTH int spread_order(int id, int count, int per_list) {
  const uint32_t lists = (uint32_t)(count / per_list), y = (uint32_t)id / lists;
  return (int)(((uint32_t)id + y) % lists * (uint32_t)per_list + y);
}

SEQ_BOTH int item_order(bool spread, int id, int count, int per_list) {
  return spread ? spread_order(id, count, per_list) : xcd_order(id, count, per_list);
}

// A block of first tokens is seen by every later row, one of the band by about
// window + 128 rows of each head of the group: the former are cut into more pieces, so
// that no workgroup has far more to do than the others; both into more where there are
// few blocks.  Pieces of one block leave fp32 sums, which are added in their order; a
// block that is not cut has none.
struct KeyPlan {
  int32_t blocks, first;            // key blocks per key head; those that hold first tokens
  int32_t first_cut, band_cut;      // pieces of each kind
  int32_t items;                    // workgroups per key head
  int32_t sums;                     // those that leave sums
  bool ahead;                       // first blocks begin before all others
};

// Workgroup x of a key head.
struct KeyItem {
  int block, piece, cut;
  int sum;                          // its place among those that leave sums, where cut > 1
};
// Where the sums of a cut block begin.
SEQ_BOTH int key_sums(const KeyPlan& p, int block) {
  return block < p.first ? block * p.first_cut
                         : (p.first_cut > 1 ? p.first * p.first_cut : 0) + (block - p.first) * p.band_cut;
}
SEQ_BOTH KeyItem key_item(const KeyPlan& p, int x) {
  const bool is_first = x < p.first * p.first_cut;
  if (!is_first) x -= p.first * p.first_cut;
  const int cut = is_first ? p.first_cut : p.band_cut, block = (is_first ? 0 : p.first) + x / cut, piece = x % cut;
  return {block, piece, cut, key_sums(p, block) + piece};
}

// The list (one batch element's key head) of workgroup `id` of `count`, and its place there.
// Where a piece of a first block is longer than two blocks of the band, all lists' first blocks
// come first: what has the most to do must not be what begins last (64 x 4096 rows, 16 heads of
// 128, window 256, one first token, backward: 5.7 ms in the lists' order, 4.65 so).  Spread
// lists begin with them anyway.
struct KeyWork {
  int list, x;
};
SEQ_BOTH KeyWork key_work(const KeyPlan& p, bool spread, int id, int count) {
  const int ahead = p.ahead && !spread ? p.first * p.first_cut : 0, longs = count / p.items * ahead;
  const bool is_long = id < longs;
  const int per_list = is_long ? ahead : p.items - ahead, before = is_long ? 0 : longs;
  const int at = item_order(spread, id - before, is_long ? longs : count - longs, per_list);
  return {at / per_list, at % per_list + (is_long ? 0 : ahead)};
}

// The cut blocks of a key head are blocks from .. to - 1.
SEQ_BOTH int cut_from(const KeyPlan& p) { return p.first_cut > 1 ? 0 : p.first; }
SEQ_BOTH int cut_to(const KeyPlan& p) { return p.band_cut > 1 ? p.blocks : p.first; }

// The units of a piece: the rows that see its block, in tiles of 32 from the block's first
// row on, for each head of the group one after the other.  n: rows of the batch element.
struct KeyUnits {
  int per_head, begin, end;
};
SEQ_BOTH KeyUnits key_units(const KeyItem& item, int window, int sinks, int n, int group) {
  const int64_t j0 = (int64_t)item.block * kKeyRows;
  if (j0 >= n) return {1, 0, 0};
  const int64_t reach = j0 + kKeyRows - 1 + window - 1, last = j0 < sinks || reach > n - 1 ? n - 1 : reach;
  const int per_head = (int)((last - j0) / kUnitRows) + 1;
  const int64_t units = (int64_t)per_head * group;
  return {per_head, (int)(units * item.piece / item.cut), (int)(units * (item.piece + 1) / item.cut)};
}

inline KeyPlan key_plan(const qds_window_config* c) {
  KeyPlan p{};
  const int64_t group = c->heads / c->kv_heads, lists = (int64_t)c->batch * c->kv_heads;
  const int64_t sinks = c->sinks < c->length ? c->sinks : c->length;
  p.blocks = (int32_t)ceil_div(c->length, kKeyRows);
  p.first = (int32_t)ceil_div(sinks, kKeyRows);
  const int64_t all = ceil_div(c->length, kUnitRows);                                 // tiles that see a first block
  int64_t band = ceil_div((int64_t)c->window + kKeyRows, kUnitRows);                  // ... and one of the band
  if (band > all) band = all;
  // pieces of equal size that give about kFill workgroups, but of no less than 16 tiles
  // (the sequence's last blocks are seen by fewer tiles, 4 more from each to the one before;
  // counted as a whole band they left causal blocks whole, of which the first has twice the
  // mean: 16384 rows, 16 heads of 128 over 4, whole window, forward and backward 6.6 ms; 5.1 so)
  const int64_t bands = p.blocks - p.first, short_bands = std::min(bands, band / 4);
  const int64_t seen = (bands - short_bands) * band + 2 * short_bands * (short_bands + 1);
  const int64_t total = (p.first * all + seen) * group * lists;
  int64_t piece = ceil_div(total, kFill);
  if (piece < 16) piece = 16;
  // A first block in pieces as long as a block of the band, which then end with the others,
  // but of no less than a quarter of what a place on the card has to do: lists that fill the card
  // many times over even out by themselves, as first blocks then begin first.  All sums together then
  // belong to some 8 kFill pieces at most, whatever the number of lists.  Backward, us, in pieces of
  // the band's length | so: 64 x 4096 rows, 16 heads of 128, window 256, one first token: 5030 | 4650 (5.65 GB of
  // sums | none);  256 x 1000, 8 heads of 64, window 64, one: 1448 | 1107;  32 x 2048, 8 heads of 64, 128,
  // 300: 562 | 430;  64 x 4096, 8 heads of 64, 16, 4096: 16000 | 4670.
  const int64_t first_piece = std::min(piece, std::max(band * group, piece / 4));
  p.first_cut = p.first > 0 ? (int32_t)ceil_div(all * group, first_piece) : 1;
  p.band_cut = bands > 0 ? (int32_t)ceil_div(band * group, piece) : 1;
  p.ahead = p.first > 0 && first_piece > 2 * band * group;
  p.items = (int32_t)(p.first * p.first_cut + bands * p.band_cut);
  p.sums = (p.first_cut > 1 ? p.first * p.first_cut : 0) + (p.band_cut > 1 ? (int32_t)bands * p.band_cut : 0);
  return p;
}

// Bytes of a call's sums: dk and dv of 128 keys each.
inline uint64_t key_sums_bytes(const qds_window_config* c, const KeyPlan& p) {
  const uint64_t columns = c->dim <= 64 ? 64 : 128;
  return (uint64_t)c->batch * c->kv_heads * p.sums * 2 * kKeyRows * columns * sizeof(float);
}

}  // namespace seq
