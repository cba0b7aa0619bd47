// How the attention over the 4-bit cache deals its items out to workgroups: what their kernels and the launches that join parts agree on.
#pragma once

#include "common.h"

namespace sage {

// What an item costs beside its units, in units: its queries, the joining of its waves, its stores.  (Without it a workgroup with many
// short items ends last: 64 ragged requests 62.7 us, with 1, 2, 3: 58.0, 56.6, 54.0; 32 equal ones of 4 drafted tokens, whose items
// came out whole by chance, 48.2 and 52.6, 49.4, 51.7.)
constexpr int kItemCost = 2;
// The same of the kernels for many rows,
constexpr int kChunkCost = 6;
// and what a workgroup of the one for up to 128 has: RG groups of 32 rows by KG tiles of 64 tokens.
template <int RG>
struct SpanShape {
  static constexpr int KG = 8 / RG, ROWS = 32 * RG, UNIT = 64 * KG, COST = KG == 4 ? 2 : 3;
};

// Items lie on a line, request after request, then head (and row tile), each with its units and COST in front of them; the line is dealt to the
// workgroups in order, total / n each and one more to the first total % n.  (The host bounds the total by 2^30.)  A border inside an item's
// COST (or before it) cuts nothing off.
template <int COST>
__host__ __device__ __forceinline__ int cut_at(int offset) { return max(0, offset - COST); }
struct AttendShares {
  int each, more, n;
  __host__ __device__ __forceinline__ AttendShares() {}
  __host__ __device__ __forceinline__ AttendShares(int total, int workgroups) {
    n = min(workgroups, total);
    each = n > 0 ? total / n : 0;
    more = total - each * n;
  }
  __host__ __device__ __forceinline__ int begin(int w) const { return each * w + min(w, more); }
  // the workgroup that has a unit
  __host__ __device__ __forceinline__ int owner(int unit) const {
    const int big = (each + 1) * more;
    return unit < big ? unit / (each + 1) : more + (unit - big) / each;
  }
  // Workgroup w begins j units into the item at x (its units behind their cost): whether that is the first border that divides the item,
  template <int COST>
  __host__ __device__ __forceinline__ bool first_border(int w, int x, int j) const { return j > 0 && cut_at<COST>(begin(w - 1) - x) == 0; }
  // and then how many parts the item has, that of workgroup w - 1 the first of them.
  template <int COST>
  __host__ __device__ __forceinline__ int parts(int w, int x, int units) const { return owner(x + units + COST - 1) - w + 2; }
};
// (at most 512 parts, and 256 rows)
__host__ __device__ __forceinline__ int4 join_word(int parts, int rows, int begin, int head, int row0) { return int4{parts | rows << 16, begin, head, row0}; }
// The row tile at a place of a head's line: the last ones see most, so light and heavy take turns and a share of average length cuts every
// second item instead of each.
__host__ __device__ __forceinline__ int chunk_tile_at(int place, int tiles) { return place & 1 ? tiles - 1 - (place >> 1) : place >> 1; }

}  // namespace sage
