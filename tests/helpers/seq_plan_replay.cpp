// Replays the work items of the window attention's backward pass over keys, from the
// header that the kernels use.  Arguments: batch length heads kv_heads dim window sinks, any
// number of times; prints "items sums first_cut band_cut" for each, and ends with 1 at the first that is wrong.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "../../paper_2202_01258_amd/csrc/seq_plan.hpp"

using namespace seq;

static int wrong(const char* what, int a, int b) {
  std::printf("%s: %d, %d\n", what, a, b);
  return 1;
}

static int check(const qds_window_config& c) {
  const KeyPlan p = key_plan(&c);
  const int group = c.heads / c.kv_heads;
  std::printf("%d %d %d %d\n", p.items, p.sums, p.first_cut, p.band_cut);
  if (p.blocks != (c.length + kKeyRows - 1) / kKeyRows) return wrong("blocks", p.blocks, c.length);
  if (p.first_cut < 1 || p.band_cut < 1) return wrong("cuts", p.first_cut, p.band_cut);
  // every piece of every block is one item's; every place of a sum is taken once, and read by the join
  std::vector<std::vector<KeyItem>> of(p.blocks);
  std::vector<int> taken(p.sums, 0);
  for (int x = 0; x < p.items; ++x) {
    const KeyItem it = key_item(p, x);
    if (it.block < 0 || it.block >= p.blocks) return wrong("block", x, it.block);
    if (it.piece != (int)of[it.block].size()) return wrong("piece", x, it.piece);
    of[it.block].push_back(it);
    if (it.cut > 1) {
      if (it.sum < 0 || it.sum >= p.sums || taken[it.sum]++) return wrong("sum", x, it.sum);
      if (it.sum != key_sums(p, it.block) + it.piece) return wrong("joined sum", x, it.sum);
    }
  }
  for (int s = 0; s < p.sums; ++s)
    if (!taken[s]) return wrong("unused sum", s, p.sums);
  for (int b = 0; b < p.blocks; ++b) {
    if ((int)of[b].size() != of[b][0].cut) return wrong("pieces", b, (int)of[b].size());
    if ((of[b][0].cut > 1) != (b >= cut_from(p) && b < cut_to(p))) return wrong("join", b, of[b][0].cut);
  }
  // every workgroup of the grid has an item of its own, in both orders
  const int lists = c.batch * c.kv_heads, grid = lists * p.items;
  for (int spread = 0; spread < 2 && grid <= 1 << 20; ++spread) {
    std::vector<char> seen(grid, 0);
    for (int id = 0; id < grid; ++id) {
      const KeyWork w = key_work(p, spread, id, grid);
      if (w.list < 0 || w.list >= lists || w.x < 0 || w.x >= p.items) return wrong("work", id, w.list);
      if (seen[w.list * p.items + w.x]++) return wrong("work taken twice", id, w.list);
    }
  }
  // the pieces of a block share out the rows that see it, for every length of an episode
  for (int n : {c.length, c.length - 1, c.length / 2, c.length / 3 + 1, 65, 1, 0}) {
    if (n < 0 || n > c.length) continue;
    for (int b = 0; b < p.blocks; ++b) {
      const int j0 = b * kKeyRows;
      int last = -1;                     // the last row that sees a key of the block
      for (int j = j0; j < j0 + kKeyRows && j < n; ++j) {
        const int i = j < c.sinks || c.window - 1 > n - 1 - j ? n - 1 : j + c.window - 1;
        if (i > last) last = i;
      }
      const int units = last < 0 ? 0 : ((last - j0) / kUnitRows + 1) * group;
      int at = 0;
      for (const KeyItem& it : of[b]) {
        const KeyUnits u = key_units(it, c.window, c.sinks, n, group);
        if (u.begin != at || u.end < u.begin) return wrong("units begin", b, u.begin);
        if (units && u.per_head * group != units) return wrong("units of a head", b, u.per_head);
        at = u.end;
      }
      if (at != units) return wrong("units", b, at);
    }
  }
  return 0;
}

int main(int argc, char** argv) {
  for (int i = 1; i + 7 <= argc; i += 7) {
    qds_window_config c{};
    c.abi_version = QDS_ABI_VERSION;
    c.batch = std::atoi(argv[i]), c.length = std::atoi(argv[i + 1]), c.heads = std::atoi(argv[i + 2]);
    c.kv_heads = std::atoi(argv[i + 3]), c.dim = std::atoi(argv[i + 4]);
    c.window = std::atoi(argv[i + 5]), c.sinks = std::atoi(argv[i + 6]);
    if (check(c)) {
      for (int k = 0; k < 7; ++k) std::printf("%s ", argv[i + k]);
      std::printf("\n");
      return 1;
    }
  }
  return 0;
}
