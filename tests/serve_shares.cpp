// How the kernels of the cache attention deal items to workgroups, with their own functions and costs: every unit goes to one workgroup, the
// parts of a divided item are those of neighbours in the order of the keys, and its first border, and no other, leaves word of how many
// there are.  Prints the first line of items that fails and returns 1.
#include <stdio.h>

#include <algorithm>
#include <random>
#include <vector>

#include "cache_shares.h"

using namespace sage;

struct Part {
  int w, j0, j1;
};

// Items of `units` and COST in front of each, the line of which `workgroups` share.
template <int COST>
int dealt_once(const std::vector<int>& units, int workgroups) {
  const int items = (int)units.size();
  std::vector<int> starts(1, 0);
  for (const int u : units) starts.push_back(starts.back() + u + COST);
  const AttendShares shares(starts.back(), workgroups);
  const auto bad = [&](const char* what, int w, int i) {
    printf("cost %d, %d items, total %d, %d workgroups: %s (workgroup %d, item %d)\n", COST, items, starts.back(), workgroups, what, w, i);
    return 1;
  };
  if (shares.n != std::min(workgroups, starts.back()) || shares.begin(0) != 0 || shares.begin(shares.n) != starts.back()) return bad("shares", 0, 0);
  std::vector<std::vector<Part>> parts(items);
  std::vector<int> word_from(items, -1), word(items, 0);
  for (int w = 0; w < shares.n; w++) {
    const int begin = shares.begin(w), end = shares.begin(w + 1);
    if (end <= begin) return bad("an empty share", w, 0);
    for (int x = begin; x < end; x++)
      if (shares.owner(x) != w) return bad("owner", w, 0);
    int i = (int)(std::upper_bound(starts.begin(), starts.end(), begin) - starts.begin()) - 1, j = cut_at<COST>(begin - starts[i]);
    if (cut_at<COST>(end - starts[i]) <= j) continue;          // (a share that ends inside an item's cost)
    if (shares.first_border<COST>(w, starts[i], j)) {
      if (word_from[i] >= 0) return bad("two first borders", w, i);
      word_from[i] = w;
      word[i] = shares.parts<COST>(w, starts[i], units[i]);
    }
    for (; i < items; i++, j = 0) {
      const int j1 = std::min(units[i], cut_at<COST>(end - starts[i]));
      if (j1 <= j) break;
      parts[i].push_back({w, j, j1});
      if (j1 < units[i]) break;
    }
  }
  for (int i = 0; i < items; i++) {
    int at = 0;
    for (size_t k = 0; k < parts[i].size(); k++) {
      if (parts[i][k].j0 != at || parts[i][k].w != parts[i][0].w + (int)k) return bad("a part out of order", parts[i][k].w, i);
      at = parts[i][k].j1;
    }
    if (at != units[i]) return bad("units left", 0, i);
    const bool divided = parts[i].size() > 1;
    if (divided != (word_from[i] >= 0)) return bad("word of the parts", word_from[i], i);
    if (divided && (word_from[i] != parts[i][1].w || word[i] != (int)parts[i].size())) return bad("number of parts", word_from[i], i);
    if (divided && (join_word(word[i], 256, 0, 0, 0).x & 0xFFFF) != word[i]) return bad("parts in a word", word_from[i], i);
  }
  return 0;
}

template <int COST>
int lines_of_every_kind() {
  std::mt19937 rng(COST);
  const auto below = [&](int n) { return (int)(rng() % (unsigned)n); };
  const int many[] = {1, 2, 3, 8, 255, 256, 512};
  for (int trial = 0; trial < 2000; trial++) {
    std::vector<int> units(1 + below(trial % 4 == 0 ? 400 : 40));
    const int most = 1 + below(trial % 3 == 0 ? 300 : 9), equal = below(3) == 0;
    for (int& u : units) u = equal ? most : 1 + below(most);
    if (dealt_once<COST>(units, many[below(7)])) return 1;
  }
  for (int u = 1; u <= 600; u++)          // one request alone
    for (const int n : {1, 256, 512})
      if (dealt_once<COST>({u}, n)) return 1;
  return 0;
}

int every_row_tile_has_a_place() {
  for (int tiles = 1; tiles <= 600; tiles++) {
    std::vector<char> taken(tiles, 0);
    for (int place = 0; place < tiles; place++) {
      const int t = chunk_tile_at(place, tiles);
      if (t < 0 || t >= tiles || taken[t]++) return printf("place %d of %d row tiles: tile %d\n", place, tiles, t), 1;
    }
  }
  return 0;
}

int main() {
  return lines_of_every_kind<kItemCost>() || lines_of_every_kind<kChunkCost>() || lines_of_every_kind<SpanShape<2>::COST>() ||
         lines_of_every_kind<SpanShape<4>::COST>() || every_row_tile_has_a_place();
}
