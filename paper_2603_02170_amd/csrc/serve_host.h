// What the host files of the serving calls share: limits, checks of arguments, and how a call of the cache attention is laid out.
#pragma once

#include "sagebwd_serve.h"

#include <hip/hip_runtime.h>
#include <math.h>

#include "cache8_attend_kernel.h"
#include "cache_kernels.h"

namespace sage {

#define SERVE_LAUNCH_CHECK() do { if (hipGetLastError() != hipSuccess) return SAGEBWD_HIP_ERROR; } while (0)

constexpr int64_t kMostElements = (int64_t)1 << 40;
// A launch's threads are counted in 32 bits, its workgroups along y in 16.
constexpr int64_t kMostThreads = (int64_t)1 << 31;
constexpr int kMostInY = 65535;
// Rows of a plan: its kernels step over them in 32 bits, by as many as a launch has threads (rows rounded up).
constexpr int kMostRows = 1 << 30;
// Entries of a block table whose pages are counted: what the sums of plan and trim hold (they stop there).
constexpr int64_t kMostEntries = kFull;

inline bool aligned(const void* p, size_t to = 16) { return ((uintptr_t)p & (to - 1)) == 0; }
inline bool stride_ok(int64_t s) { return s >= 0 && s % 8 == 0 && s <= kMostElements; }

inline int page_shift_of(int page) {
  for (int s = 5; s <= 8; s++)
    if (page == 1 << s) return s;
  return -1;
}

inline int check_cache(const sagebwd_cache_params* p, bool pool) {
  if (p == nullptr || p->H < 1 || (pool && p->pages < 1)) return SAGEBWD_INVALID_ARG;
  if (p->block != 0 && ((p->block != 32 && p->block != 64) || p->group != 0)) return SAGEBWD_INVALID_ARG;
  if ((p->d != 64 && p->d != 128) || (p->block == 0 && p->group != 32 && p->group != 64) || page_shift_of(p->page) < 0 || p->page < p->block ||
      p->H > 1024)
    return SAGEBWD_UNSUPPORTED_SHAPE;
  return SAGEBWD_OK;
}
inline CacheGeometry geometry(const sagebwd_cache_params& p) { return CacheGeometry{p.H, p.d, page_shift_of(p.page), p.group, p.pages}; }

constexpr int kCus = 256;
// Query rows of a request and head that cache_attend_kernel takes (32 requests of 4096 tokens, 32 rows: 59 us, the kernel for many rows 135; 64 rows in
// four tiles a wave, which its registers do not hold at d = 128, 206).
constexpr int kFewRows = 32;
// Of a cache held in 8 bits: rows in several tiles of 32, each a pass over the keys, while the line that they are dealt out on holds them.
constexpr int kTiledRows = 128;
// Query rows of a request and head at most, and its keys.
inline int64_t most_rows(const sagebwd_cache_params& p, const sagebwd_cache_call& c) { return (int64_t)(c.max_new < c.T ? c.max_new : c.T) * (c.Hq / p.H); }
inline int most_length(const sagebwd_cache_params& p, const sagebwd_cache_call& c) {
  const int64_t all = (int64_t)c.columns * p.page;
  return (int)(c.max_length > 0 && c.max_length < all ? c.max_length : all);
}
// Where every request brings so many rows and a CU has much to do, tiles of 48 or 64 rows by one wave a SIMD, with all its registers, unpack less often
// than those of 32 by two; in short calls the latter end sooner.  (us, 32 -> 48 or 64 rows a tile, 8 heads of 128 in the cache: 32 requests of 4096
// tokens, 48 rows 90 -> 67, 64 rows 88 -> 81, 128 rows 166 -> 147; 24 ragged ones of up to 3000 of 4 heads, 48 rows 19.0 -> 20.4; heads of 64, 64 rows 48 -> 54.)
inline int tile_tiles_of(const sagebwd_cache_params& p, const sagebwd_cache_call& c, int64_t rows) {      // of 16 rows
  const int64_t units = (int64_t)c.R * p.H * ((most_length(p, c) + kUnit - 1) / kUnit);
  if (p.block == 0 || p.d != 128 || rows <= 32 || units < 16 * kCus || 5 * (int64_t)c.T < 3 * (int64_t)c.R * c.max_new) return rows <= 16 ? 1 : 2;
  return rows <= 48 || (rows > 64 && rows <= 96) ? 3 : 4;
}
inline int few_rows_of(const sagebwd_cache_params& p, const sagebwd_cache_call& c) {
  const int64_t line = (int64_t)c.R * p.H * (kTiledRows / 32) * ((most_length(p, c) + kUnit - 1) / kUnit + kItemCost);
  return p.block > 0 && line <= 1 << 29 ? kTiledRows : kFewRows;
}
// The rows of a workgroup of the kernel for many.  Of a cache held in 4 bits cache_span_kernel has 64 or 128 and unpacks 256 or 128 tokens at a time (tiles of
// 256 rows -> these, us: 32 requests of 4096 tokens, 64 rows 123 -> 87, 128 rows 126 -> 107; 64 of 40 rows, 1000 tokens, 60 -> 46; four requests of 64
// tokens 15 -> 19; 65 to 128 rows as two tiles of 64 188, 256 as two of 128, 3000 tokens, 79 -> 93).
inline int tile_rows_of(const sagebwd_cache_params& p, const sagebwd_cache_call& c) {
  const int64_t most = most_rows(p, c);
  return p.block > 0 || most > 128 || most_length(p, c) <= 256 ? kChunkRows : most > 64 ? 128 : 64;
}
// Row tiles of the kernel for many rows, over all heads, at most; 0 where no request goes to it.
inline int64_t chunk_tiles_of(const sagebwd_cache_params& p, const sagebwd_cache_call& c) {
  if (most_rows(p, c) <= few_rows_of(p, c)) return 0;
  return ((int64_t)c.T * (c.Hq / p.H) / tile_rows_of(p, c) + c.R) * p.H;
}

inline int check_call(const sagebwd_cache_params* p, const sagebwd_cache_call* c) {
  const int rc = check_cache(p, true);
  if (rc != SAGEBWD_OK) return rc;
  if (c == nullptr || c->R < 0 || c->T < 0 || c->Hq < 1 || c->columns < 1 || c->max_new < 1 || c->max_length < 0 ||
      (c->causal != 0 && c->causal != 1) || !(c->sm_scale >= 0.f) || !isfinite(c->sm_scale) || !stride_ok(c->q_token_stride) ||
      !stride_ok(c->q_head_stride))
    return SAGEBWD_INVALID_ARG;
  if (c->Hq % p->H != 0 || c->Hq / p->H > 64 || (int64_t)c->T * c->Hq * p->d >= kMostElements || c->R > 1 << 20 ||
      (int64_t)c->columns * p->page > INT32_MAX / 2 || (int64_t)c->R * p->H * (c->columns * (int64_t)p->page / kUnit + 1 + kItemCost) > 1 << 29 ||
      chunk_tiles_of(*p, *c) > kMostThreads / 512 || (int64_t)c->T * (c->Hq / p->H) > INT32_MAX / 2)
    return SAGEBWD_UNSUPPORTED_SHAPE;
  return SAGEBWD_OK;
}

// Keys of a request up to this many units are not divided (four requests of 500 tokens 11.0 -> 9.3 us, 256 of 650 56.4 -> 52.0: the joining
// launch is 4 to 5 us, a unit 0.6 where the machine is empty).
constexpr int kWholeUnits = 8;
// Held in 8 bits, where undivided items fill half of the machine, they may be this long (keys of 1500: 16 requests of 8 heads 16.7 -> 14.8
// us, 64 42.9 -> 39.0; 64 of 16 heads, d = 64, 46.5 -> 38.5; with fewer items division is the faster: one request 11.4 -> 14.0 undivided).
constexpr int kWholeUnits8 = 12;
// Held in 8 bits, items of so many keys have a wave each, whatever their number.
constexpr int kShortLength = 128;
// Keys and values are unpacked beforehand where a request's meet so many row tiles (us, unpacked by every tile -> beforehand: one request of 512 new
// tokens x 4 heads of the group against 32768, 8 tiles, 288 -> 277, at d = 64 229 -> 180; 2048 x 4 against 10000, 32 tiles, 335 -> 293, at
// d = 64 264 -> 193; two of 2048 against 8192, 8 tiles, 149 -> 148; 16 ragged ones of at most 600 x 4 140 -> 143; 4 of 256 x 4, 4 tiles,
// slower by a sixth), and the workspace for them is at most this.
constexpr int kWideTiles = 8;
constexpr int64_t kMostUnpacked = (int64_t)4 << 30;

// One of the two kernels' part of a call.
struct AttendLaunch {
  int rows_from, rows_to;      // of the requests that it has
  int nq;                      // cache_attend_kernel: tiles of 16 rows
  int workgroups, join_rows;
  bool join_wide;              // items have few parts: several rows a workgroup
  int direct;                  // workgroups of each request (short_items: waves), or 0: items are dealt out
  bool short_items;
  int tile_rows;               // of the kernels for many rows
  bool split;
  size_t joins, sums, stats;
  bool wide;                   // the keys and values are unpacked beforehand
  int unpack_workgroups, most_tiles;
  size_t unpacked, tiles, poison;
};
// How a call is laid out.
struct AttendPlan {
  int max_length;
  bool few, many;              // there may be requests for either kernel
  AttendLaunch f, m;
  size_t total;
};
inline size_t align_up(size_t x, size_t a = 256) { return (x + a - 1) / a * a; }

inline AttendPlan attend_plan(const sagebwd_cache_params& p, const sagebwd_cache_call& c) {
  AttendPlan w;
  const int G = c.Hq / p.H;
  w.max_length = most_length(p, c);
  const int64_t most = most_rows(p, c);
  const int64_t rows = most > 0 ? most : 1;
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t o = off; off += align_up(bytes); return o; };
  const auto lay_out = [&](AttendLaunch& l, int tile) {
    const size_t parts = l.split ? (size_t)l.workgroups * 2 * tile : 0;
    l.joins = take((size_t)l.workgroups * sizeof(int4));
    l.sums = take(parts * p.d * 4);
    l.stats = take(parts * 8);
  };
  // Few rows a request: all of them to the one kernel.  Else the requests of one new token (and what fits the same tiles) go to it, the others to
  // the kernel for many rows; where every request brings the same number there are none of the former.  (That is read from T = R max_new: a T
  // padded to it, with requests of one token among them, is served by the kernel for many: 32 of 4096 tokens, 4 heads a group, T = 512: 82 us, T = 511
  // 38.  And 17 to 32 rows beside a prompt go to it too: the same 32 with 8 tokens each 52 us, a prompt of 2048 129, together 356; with 4 tokens each
  // together 170.)
  const int few_rows = few_rows_of(p, c);
  w.many = rows > few_rows;
  w.few = !w.many || (G <= few_rows && (int64_t)c.T < (int64_t)c.R * c.max_new);
  // (Held in 8 bits and small, two launches more cost more than tiles half empty: eight ragged requests of 1380 tokens with up to 915 rows 45 -> 30 us.)
  if (w.many && p.block > 0 && (int64_t)c.R * p.H * ((w.max_length + kChunkUnit - 1) / kChunkUnit) <= 2 * kCus) w.few = false;
  if (w.few) {
    AttendLaunch& l = w.f;
    const int64_t here = !w.many ? rows : few_rows > kFewRows ? few_rows : G > 16 ? G : 16;
    l.nq = w.many ? (here <= 16 ? 1 : 2) : tile_tiles_of(p, c, here);
    const int64_t tiles = (here + 16 * l.nq - 1) / (16 * l.nq);
    l.rows_from = 0;
    l.rows_to = here > 32 ? few_rows : 16 * l.nq;
    l.join_rows = (int)(here < 16 * l.nq ? here : 16 * l.nq);
    const int most_units = (w.max_length + kUnit - 1) / kUnit;
    l.split = most_units > (p.block > 0 && (int64_t)c.R * p.H * tiles >= kCus / 2 ? kWholeUnits8 : kWholeUnits);
    const int64_t units = (int64_t)c.R * p.H * tiles * (l.split ? most_units + kItemCost : 1);
    // (Held in 8 bits the keys alone bound a call of one tile, and a workgroup a CU has enough of them under way: 32 requests of 4096 tokens, 16 rows
    // 59.4 -> 55.1 us, 32 rows 63.2 -> 57.0, one of 131000 57.4 -> 55.2.  Of several tiles two: heads of 64, up to 100 rows 19.6 -> 18.4.)
    const int64_t slots = (p.block > 0 && (tiles == 1 || l.nq > 2) ? 1 : 2) * kCus;
    l.workgroups = (int)(units < slots ? (units > 0 ? units : 1) : slots);
    // a wave an item where they are short, or many
    l.short_items = p.block > 0 && !l.split && l.nq <= 2 && (w.max_length <= kShortLength || units > 4 * kCus) && units < 1 << 22;
    l.direct = p.block > 0 && !l.split && (l.short_items || units <= 4 * kCus) ? (int)(p.H * tiles) : 0;
    if (l.direct) l.workgroups = (int)(units > 0 ? units : 1);
    l.join_wide = p.block > 0 && (int64_t)c.R * p.H * tiles >= 64;
    lay_out(l, 16 * l.nq);
  }
  if (w.many) {
    AttendLaunch& l = w.m;
    l.direct = 0;
    l.short_items = false;
    l.rows_from = w.few ? w.f.rows_to : 0;
    l.rows_to = INT32_MAX;
    const int64_t total = (int64_t)c.T * G;
    const int64_t with = w.few ? (total / (l.rows_from + 1) < c.R ? total / (l.rows_from + 1) : c.R) : c.R;      // requests that it may have
    l.tile_rows = tile_rows_of(p, c);
    const int unit = l.tile_rows == 64 ? SpanShape<2>::UNIT : l.tile_rows == 128 ? SpanShape<4>::UNIT : kChunkUnit;
    const int64_t tiles = total / l.tile_rows + with, units = tiles * p.H * ((w.max_length + unit - 1) / unit + kChunkCost);
    const int64_t key_tiles = with * p.H * ((w.max_length + kChunkUnit - 1) / kChunkUnit);
    const int64_t wide_rows = kWideTiles * kChunkRows;
    l.wide = most >= wide_rows && (w.few || total >= wide_rows * with) && key_tiles * p.d * 256 <= kMostUnpacked;
    l.split = total * p.H / l.tile_rows < 4 * kCus && units < 1 << 30;
    const int64_t slots = l.wide && p.d == 64 ? 2 * kCus : kCus;      // (workgroups that the machine takes at a time)
    l.workgroups = (int)(l.split ? (units < slots ? (units > 0 ? units : 1) : slots) : tiles * p.H);
    lay_out(l, l.tile_rows);
    if (l.wide) {
      l.unpack_workgroups = (int)(key_tiles < 4 * kCus ? key_tiles : 4 * kCus);
      l.most_tiles = (int)key_tiles;
      l.unpacked = take((size_t)key_tiles * p.d * 256);
      l.tiles = take((size_t)key_tiles * (p.block ? sizeof(ByteKnown) : sizeof(WideTile)) + (p.block ? 256 : 0));      // (the last one's copy reads 256 bytes)
      l.poison = take(p.block ? 0 : (size_t)key_tiles * (p.d / p.group) * 64);
    }
  }
  w.total = off;
  return w;
}

// The launches of a call, `Kernels` those of a format.
template <typename Kernels, int NQ>
int launch_few(const AttendArgs& a, const AttendLaunch& l, hipStream_t st) {
  if constexpr (Kernels::BYTES && NQ <= 2) {
    if (l.short_items) Kernels::template few_short<NQ>((l.workgroups + 3) / 4, a, st);
    else Kernels::template few<NQ>(l.workgroups, a, st);
  } else {
    Kernels::template few<NQ>(l.workgroups, a, st);
  }
  SERVE_LAUNCH_CHECK();
  if (l.split && l.workgroups > 1) {
    if (!Kernels::BYTES || !l.join_wide) Kernels::template join_few<16 * NQ>(dim3(l.workgroups - 1, l.join_rows), a, st);
    if constexpr (Kernels::BYTES)
      if (l.join_wide) Kernels::template join_many<16 * NQ>(dim3(l.workgroups - 1, (l.join_rows * (Kernels::D / 4) + 255) / 256), a, st);
    SERVE_LAUNCH_CHECK();
  }
  return SAGEBWD_OK;
}
template <typename Kernels>
int launch_attend(AttendArgs a, const AttendPlan& w, char* ws, hipStream_t st) {
  const auto with = [&](const AttendLaunch& l) {
    a.joins = (int4*)(ws + l.joins);
    a.sums = (float*)(ws + l.sums);
    a.stats = (float2*)(ws + l.stats);
    a.workgroups = l.workgroups;
    a.split = l.split;
    a.rows_from = l.rows_from;
    a.rows_to = l.rows_to;
    a.direct = l.direct;
  };
  if (w.many) {
    with(w.m);
    if (w.m.wide) {
      a.most_tiles = w.m.most_tiles;
      a.unpacked = ws + w.m.unpacked;
      a.tiles = (WideTile*)(ws + w.m.tiles);
      a.poison = (unsigned char*)(ws + w.m.poison);
      Kernels::unpack(w.m.unpack_workgroups, a, st);
      SERVE_LAUNCH_CHECK();
      Kernels::wide(w.m.workgroups, a, st);
    } else if (w.m.tile_rows == kChunkRows) {
      Kernels::chunk(w.m.workgroups, a, st);
    } else {
      if constexpr (!Kernels::BYTES) w.m.tile_rows == 64 ? Kernels::template span<2>(w.m.workgroups, a, st) : Kernels::template span<4>(w.m.workgroups, a, st);
    }
    SERVE_LAUNCH_CHECK();
    if (w.m.split && w.m.workgroups > 1) {
      const dim3 grid(w.m.workgroups - 1, w.m.tile_rows / (256 / (Kernels::D / 4)));
      if (w.m.tile_rows == kChunkRows) Kernels::template join_many<kChunkRows>(grid, a, st);
      if constexpr (!Kernels::BYTES) {
        if (w.m.tile_rows == 64) Kernels::template join_many<64>(grid, a, st);
        if (w.m.tile_rows == 128) Kernels::template join_many<128>(grid, a, st);
      }
      SERVE_LAUNCH_CHECK();
    }
  }
  if (w.few) {
    with(w.f);
    if constexpr (Kernels::MOST_TILES > 2) {
      if (w.f.nq == 3) return launch_few<Kernels, 3>(a, w.f, st);
      if (w.f.nq == 4) return launch_few<Kernels, 4>(a, w.f, st);
    }
    return w.f.nq == 1 ? launch_few<Kernels, 1>(a, w.f, st) : launch_few<Kernels, 2>(a, w.f, st);
  }
  return SAGEBWD_OK;
}

// The calls of a cache held in 8 bits (params.block > 0) behind their checks.
int cache8_append(const StoreArgs& a, const sagebwd_cache_params& p, hipStream_t st);
int cache8_read(const StoreArgs& a, const sagebwd_cache_params& p, hipStream_t st);
int cache8_attend(const AttendArgs& a, const sagebwd_cache_params& p, const AttendPlan& w, char* ws, hipStream_t st);

}  // namespace sage
