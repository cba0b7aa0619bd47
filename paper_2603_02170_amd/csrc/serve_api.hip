// C-ABI host side of the operators around the attention: argument checks, workspace layout, launches.
// See include/sagebwd_serve.h for the contract of every entry point.
#include "sagebwd_serve.h"

#include <hip/hip_runtime.h>
#include <math.h>

#include <type_traits>

#include "cache_attend_kernel.h"
#include "cache_chunk_kernel.h"
#include "cache_kernels.h"
#include "rotary_kernel.h"

namespace {

using namespace sage;

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

int page_shift_of(int page) {
  for (int s = 5; s <= 8; s++)
    if (page == 1 << s) return s;
  return -1;
}

int check_cache(const sagebwd_cache_params* p, bool pool) {
  if (p == nullptr || p->reserved != 0 || p->H < 1 || (pool && p->pages < 1)) return SAGEBWD_INVALID_ARG;
  if ((p->d != 64 && p->d != 128) || (p->group != 32 && p->group != 64) || page_shift_of(p->page) < 0 || p->H > 1024)
    return SAGEBWD_UNSUPPORTED_SHAPE;
  return SAGEBWD_OK;
}
CacheGeometry geometry(const sagebwd_cache_params& p) { return CacheGeometry{p.H, p.d, page_shift_of(p.page), p.group, p.pages}; }

constexpr int kCus = 256;
// Query rows of a request and head that cache_attend_kernel takes (32 requests of 4096 tokens, 32 rows: 59 us, the kernel for many rows 135; 64 rows in
// four tiles a wave, which its registers do not hold at d = 128, 206).
constexpr int kFewRows = 32;
// Query rows of a request and head at most, keys of a request at most, and the rows of a workgroup of the kernel for many.  cache_span_kernel has 64 or
// 128 and unpacks 256 or 128 tokens at a time (tiles of 256 rows -> these, us: 32 requests of 4096 tokens, 64 rows 123 -> 87, 128 rows 126 ->
// 107; 64 of 40 rows, 1000 tokens, 60 -> 46; four requests of 64 tokens 15 -> 19; 65 to 128 rows as two tiles of 64 188, 256 as two of 128, 3000
// tokens, 79 -> 93).
int64_t most_rows(const sagebwd_cache_params& p, const sagebwd_cache_call& c) { return (int64_t)(c.max_new < c.T ? c.max_new : c.T) * (c.Hq / p.H); }
int most_length(const sagebwd_cache_params& p, const sagebwd_cache_call& c) {
  const int64_t all = (int64_t)c.columns * p.page;
  return (int)(c.max_length > 0 && c.max_length < all ? c.max_length : all);
}
int tile_rows_of(const sagebwd_cache_params& p, const sagebwd_cache_call& c) {
  const int64_t most = most_rows(p, c);
  return most > 128 || most_length(p, c) <= 256 ? kChunkRows : most > 64 ? 128 : 64;
}
// Row tiles of the kernel for many rows, over all heads, at most; 0 where no request goes to it.
int64_t chunk_tiles_of(const sagebwd_cache_params& p, const sagebwd_cache_call& c) {
  if (most_rows(p, c) <= kFewRows) return 0;
  return ((int64_t)c.T * (c.Hq / p.H) / tile_rows_of(p, c) + c.R) * p.H;
}

int check_call(const sagebwd_cache_params* p, const sagebwd_cache_call* c) {
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

AttendPlan attend_plan(const sagebwd_cache_params& p, const sagebwd_cache_call& c) {
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
  w.many = rows > kFewRows;
  w.few = !w.many || (G <= kFewRows && (int64_t)c.T < (int64_t)c.R * c.max_new);
  if (w.few) {
    AttendLaunch& l = w.f;
    const int64_t here = w.many ? (G > 16 ? G : 16) : rows;
    l.nq = here <= 16 ? 1 : 2;
    l.rows_from = 0;
    l.rows_to = 16 * l.nq;
    l.join_rows = (int)(here < l.rows_to ? here : l.rows_to);
    const int most_units = (w.max_length + kUnit - 1) / kUnit;
    l.split = most_units > kWholeUnits;
    const int64_t units = (int64_t)c.R * p.H * (l.split ? most_units + kItemCost : 1);
    const int64_t slots = 2 * kCus;
    l.workgroups = (int)(units < slots ? (units > 0 ? units : 1) : slots);
    lay_out(l, 16 * l.nq);
  }
  if (w.many) {
    AttendLaunch& l = w.m;
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
      l.tiles = take((size_t)key_tiles * sizeof(WideTile));
      l.poison = take((size_t)key_tiles * (p.d / p.group) * 64);
    }
  }
  w.total = off;
  return w;
}

template <int D, int GROUP, int NQ>
int launch_few(const AttendArgs& a, const AttendLaunch& l, hipStream_t st) {
  cache_attend_kernel<D, GROUP, NQ><<<l.workgroups, 256, 0, st>>>(a);
  SERVE_LAUNCH_CHECK();
  if (l.split && l.workgroups > 1) {
    cache_join_kernel<D, 16 * NQ><<<dim3(l.workgroups - 1, l.join_rows), 256, 0, st>>>(a);
    SERVE_LAUNCH_CHECK();
  }
  return SAGEBWD_OK;
}
template <int D, int GROUP>
int launch_attend(AttendArgs a, const AttendPlan& w, char* ws, hipStream_t st) {
  const auto with = [&](const AttendLaunch& l) {
    a.joins = (int4*)(ws + l.joins);
    a.sums = (float*)(ws + l.sums);
    a.stats = (float2*)(ws + l.stats);
    a.workgroups = l.workgroups;
    a.split = l.split;
    a.rows_from = l.rows_from;
    a.rows_to = l.rows_to;
  };
  if (w.many) {
    with(w.m);
    if (w.m.wide) {
      a.most_tiles = w.m.most_tiles;
      a.unpacked = ws + w.m.unpacked;
      a.tiles = (WideTile*)(ws + w.m.tiles);
      a.poison = (unsigned char*)(ws + w.m.poison);
      cache_unpack_kernel<D, GROUP><<<w.m.unpack_workgroups, 512, 0, st>>>(a);
      SERVE_LAUNCH_CHECK();
      cache_wide_kernel<D, GROUP><<<w.m.workgroups, 512, 0, st>>>(a);
    } else if (w.m.tile_rows == 64) {
      cache_span_kernel<D, GROUP, 2><<<w.m.workgroups, 512, 0, st>>>(a);
    } else if (w.m.tile_rows == 128) {
      cache_span_kernel<D, GROUP, 4><<<w.m.workgroups, 512, 0, st>>>(a);
    } else {
      cache_chunk_kernel<D, GROUP><<<w.m.workgroups, 512, 0, st>>>(a);
    }
    SERVE_LAUNCH_CHECK();
    if (w.m.split && w.m.workgroups > 1) {
      const dim3 grid(w.m.workgroups - 1, w.m.tile_rows / (256 / (D / 4)));
      if (w.m.tile_rows == 64) cache_join_rows_kernel<D, 64><<<grid, 256, 0, st>>>(a);
      else if (w.m.tile_rows == 128) cache_join_rows_kernel<D, 128><<<grid, 256, 0, st>>>(a);
      else cache_join_rows_kernel<D, kChunkRows><<<grid, 256, 0, st>>>(a);
      SERVE_LAUNCH_CHECK();
    }
  }
  if (w.few) {
    with(w.f);
    return w.f.nq == 1 ? launch_few<D, GROUP, 1>(a, w.f, st) : launch_few<D, GROUP, 2>(a, w.f, st);
  }
  return SAGEBWD_OK;
}

template <typename F>
int with_format(const sagebwd_cache_params& p, F f) {
  if (p.d == 64) return p.group == 32 ? f(std::integral_constant<int, 64>(), std::integral_constant<int, 32>())
                                      : f(std::integral_constant<int, 64>(), std::integral_constant<int, 64>());
  return p.group == 32 ? f(std::integral_constant<int, 128>(), std::integral_constant<int, 32>())
                       : f(std::integral_constant<int, 128>(), std::integral_constant<int, 64>());
}

}  // namespace

extern "C" {

int sagebwd_cache_page_bytes(const sagebwd_cache_params* params, size_t* bytes) {
  const int rc = check_cache(params, false);
  if (rc != SAGEBWD_OK) return rc;
  if (bytes == nullptr) return SAGEBWD_INVALID_ARG;
  *bytes = geometry(*params).page_bytes();
  return SAGEBWD_OK;
}

int sagebwd_cache_plan(const int32_t* held, const int32_t* added, int32_t* block_table, const int32_t* free_pages, const int32_t* free_count,
                       int32_t R, int32_t columns, int32_t page, int32_t capacity, int32_t rows, int64_t* slots, int32_t* positions,
                       int32_t* cu_new, int32_t* lengths, int32_t* granted, int32_t* free_left, void* stream) {
  if (R < 0 || rows < 0 || columns < 1 || capacity < 0) return SAGEBWD_INVALID_ARG;
  if ((R > 0 && (held == nullptr || added == nullptr || block_table == nullptr || lengths == nullptr || granted == nullptr)) ||
      (capacity > 0 && free_pages == nullptr) || free_count == nullptr || cu_new == nullptr || free_left == nullptr ||
      (rows > 0 && (slots == nullptr || positions == nullptr)))
    return SAGEBWD_INVALID_ARG;
  if (page_shift_of(page) < 0 || (int64_t)columns * page > INT32_MAX / 2 || R > 1 << 20 || (int64_t)R * columns > kMostEntries || rows > kMostRows)
    return SAGEBWD_UNSUPPORTED_SHAPE;
  const PlanArgs a{held, added, free_pages, free_count, block_table, slots, positions, cu_new, lengths, granted, free_left,
                   R, columns, page_shift_of(page), capacity, rows};
  hipStream_t st = (hipStream_t)stream;
  // Several workgroups read what one of them writes where the lengths are updated in place; more requests than a workgroup has threads are summed
  // in several steps: many rows are then a launch of their own.
  const bool in_place = lengths == held || free_left == free_count;
  const bool several = R <= 1024 && !in_place;
  const int with_rows = several || rows <= 2048;
  if (R <= 64 && rows <= 256) cache_plan_kernel<1><<<1, 64, 0, st>>>(a, 1);
  else if (R <= 256 && rows <= 1024) cache_plan_kernel<4><<<1, 256, 0, st>>>(a, 1);
  else cache_plan_kernel<16><<<several && rows > 0 ? (rows + 1023) / 1024 : 1, 1024, 0, st>>>(a, with_rows);
  SERVE_LAUNCH_CHECK();
  if (with_rows) return SAGEBWD_OK;
  cache_plan_rows_kernel<<<(rows + 255) / 256, 256, 0, st>>>(a);
  SERVE_LAUNCH_CHECK();
  return SAGEBWD_OK;
}

int sagebwd_cache_trim(const int32_t* keep, int32_t* lengths, int32_t* block_table, int32_t* free_pages, int32_t* free_count, int32_t R,
                       int32_t columns, int32_t page, int32_t capacity, void* stream) {
  if (R < 0 || columns < 1 || capacity < 0 || free_count == nullptr || (capacity > 0 && free_pages == nullptr) ||
      (R > 0 && (keep == nullptr || lengths == nullptr || block_table == nullptr)))
    return SAGEBWD_INVALID_ARG;
  if (page_shift_of(page) < 0 || (int64_t)columns * page > INT32_MAX / 2 || R > 1 << 20 || (int64_t)R * columns > kMostEntries)
    return SAGEBWD_UNSUPPORTED_SHAPE;
  if (R == 0) return SAGEBWD_OK;
  cache_trim_kernel<<<1, 1024, 0, (hipStream_t)stream>>>(
      TrimArgs{keep, lengths, block_table, free_pages, free_count, R, columns, page_shift_of(page), capacity});
  SERVE_LAUNCH_CHECK();
  return SAGEBWD_OK;
}

int sagebwd_cache_append(const void* K, const void* V, int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride,
                         int64_t v_head_stride, const int64_t* slots, int32_t T, const float* k_mean, const float* v_mean,
                         const sagebwd_cache_params* params, void* pool, void* stream) {
  const int rc = check_cache(params, true);
  if (rc != SAGEBWD_OK) return rc;
  if (T < 0 || !stride_ok(k_token_stride) || !stride_ok(k_head_stride) || !stride_ok(v_token_stride) || !stride_ok(v_head_stride))
    return SAGEBWD_INVALID_ARG;
  if (T == 0) return SAGEBWD_OK;
  if (K == nullptr || V == nullptr || slots == nullptr || pool == nullptr || !aligned(K) || !aligned(V) || !aligned(pool)) return SAGEBWD_INVALID_ARG;
  const int64_t per = 256 / (params->d / 8), groups = (T + per - 1) / per;      // tokens of a workgroup, and workgroups of a head
  if (groups * params->H * 256 > kMostThreads) return SAGEBWD_UNSUPPORTED_SHAPE;
  const StoreArgs a{(const __bf16*)K, (const __bf16*)V, {k_token_stride, k_head_stride}, {v_token_stride, v_head_stride}, slots, k_mean, v_mean,
                    (unsigned char*)pool, nullptr, nullptr, T, geometry(*params)};
  return with_format(*params, [&](auto d, auto group) -> int {
    cache_append_kernel<decltype(d)::value, decltype(group)::value><<<dim3((unsigned)groups, params->H), 256, 0, (hipStream_t)stream>>>(a);
    SERVE_LAUNCH_CHECK();
    return SAGEBWD_OK;
  });
}

int sagebwd_cache_read(const int64_t* slots, int32_t T, const float* k_mean, const float* v_mean, const sagebwd_cache_params* params,
                       const void* pool, void* K, void* V, void* stream) {
  const int rc = check_cache(params, true);
  if (rc != SAGEBWD_OK) return rc;
  if (T < 0) return SAGEBWD_INVALID_ARG;
  if (T == 0) return SAGEBWD_OK;
  if (K == nullptr || V == nullptr || slots == nullptr || pool == nullptr || !aligned(K) || !aligned(V) || !aligned(pool)) return SAGEBWD_INVALID_ARG;
  const int64_t per = 256 / (params->d / 8), groups = (T + per - 1) / per;      // tokens of a workgroup, and workgroups of a head
  if (groups * params->H * 256 > kMostThreads) return SAGEBWD_UNSUPPORTED_SHAPE;
  const StoreArgs a{nullptr, nullptr, {0, 0}, {0, 0}, slots, k_mean, v_mean, (unsigned char*)pool, (__bf16*)K, (__bf16*)V, T, geometry(*params)};
  return with_format(*params, [&](auto d, auto group) -> int {
    cache_read_kernel<decltype(d)::value, decltype(group)::value><<<dim3((unsigned)groups, params->H), 256, 0, (hipStream_t)stream>>>(a);
    SERVE_LAUNCH_CHECK();
    return SAGEBWD_OK;
  });
}

int sagebwd_cache_workspace_bytes(const sagebwd_cache_params* params, const sagebwd_cache_call* call, size_t* bytes) {
  const int rc = check_call(params, call);
  if (rc != SAGEBWD_OK) return rc;
  if (bytes == nullptr) return SAGEBWD_INVALID_ARG;
  *bytes = attend_plan(*params, *call).total;
  return SAGEBWD_OK;
}

int sagebwd_cache_attention(const void* Q, const void* pool, const int32_t* block_table, const int32_t* lengths, const int32_t* cu,
                            const float* v_mean, const sagebwd_cache_params* params, const sagebwd_cache_call* call, void* O, float* LSE,
                            void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_call(params, call);
  if (rc != SAGEBWD_OK) return rc;
  if (call->R == 0 || call->T == 0) return SAGEBWD_OK;
  if (Q == nullptr || pool == nullptr || block_table == nullptr || lengths == nullptr || cu == nullptr || O == nullptr || !aligned(Q) ||
      !aligned(pool) || !aligned(O))
    return SAGEBWD_INVALID_ARG;
  const AttendPlan w = attend_plan(*params, *call);
  if (workspace_bytes < w.total) return SAGEBWD_WORKSPACE_TOO_SMALL;
  if (workspace == nullptr || !aligned(workspace, 256)) return SAGEBWD_INVALID_ARG;
  char* ws = (char*)workspace;
  AttendArgs a = {};
  a.Q = (const __bf16*)Q;
  a.pool = (const unsigned char*)pool;
  a.table = block_table;
  a.lengths = lengths;
  a.cu = cu;
  a.v_mean = v_mean;
  a.O = (__bf16*)O;
  a.LSE = LSE;
  a.g = geometry(*params);
  a.R = call->R;
  a.T = call->T;
  a.Hq = call->Hq;
  a.G = call->Hq / params->H;
  a.columns = call->columns;
  a.max_new = call->max_new;
  a.max_length = w.max_length;
  a.causal = call->causal;
  a.scale_log2 = (call->sm_scale > 0.f ? call->sm_scale : 1.f / sqrtf((float)params->d)) * 1.4426950408889634f;
  a.q_token = call->q_token_stride;
  a.q_head = call->q_head_stride;
  return with_format(*params, [&](auto d, auto group) { return launch_attend<decltype(d)::value, decltype(group)::value>(a, w, ws, (hipStream_t)stream); });
}

int sagebwd_rotary(const void* Q, const void* K, void* Qo, void* Ko, const void* positions, const float* inv_freq,
                   const sagebwd_rotary_params* p, void* stream) {
  if (p == nullptr || p->B < 0 || p->N < 0 || p->Hq < 1 || p->Hk < 0 || p->axes < 1 || p->axes > 4 || (p->adjacent != 0 && p->adjacent != 1) ||
      (p->inverse != 0 && p->inverse != 1) || (p->positions64 != 0 && p->positions64 != 1))
    return SAGEBWD_INVALID_ARG;
  if (p->d < 16 || p->d > 512 || p->d % 16 != 0 || p->rotary_dim < 16 || p->rotary_dim > p->d || p->rotary_dim % 16 != 0 ||
      (int64_t)p->B * p->N > INT32_MAX / 64 || (int64_t)p->Hq + p->Hk > kMostInY)
    return SAGEBWD_UNSUPPORTED_SHAPE;
  int64_t sum = 0;
  for (int k = 0; k < p->axes; k++) {
    if (p->sections[k] < 0) return SAGEBWD_INVALID_ARG;
    sum += p->sections[k];
  }
  if (sum != p->rotary_dim / 2) return SAGEBWD_INVALID_ARG;
  for (int k = 0; k < 3; k++)
    if (!stride_ok(p->q_strides[k]) || !stride_ok(p->qo_strides[k]) || (p->Hk > 0 && (!stride_ok(p->k_strides[k]) || !stride_ok(p->ko_strides[k]))))
      return SAGEBWD_INVALID_ARG;
  if (p->B == 0 || p->N == 0) return SAGEBWD_OK;
  if (Q == nullptr || Qo == nullptr || positions == nullptr || inv_freq == nullptr || !aligned(Q) || !aligned(Qo) ||
      (p->Hk > 0 && (K == nullptr || Ko == nullptr || !aligned(K) || !aligned(Ko))))
    return SAGEBWD_INVALID_ARG;
  RotaryArgs a;
  a.x[0] = (const __bf16*)Q;
  a.x[1] = (const __bf16*)K;
  a.y[0] = (__bf16*)Qo;
  a.y[1] = (__bf16*)Ko;
  for (int k = 0; k < 3; k++) {
    a.xs[0][k] = p->q_strides[k];
    a.xs[1][k] = p->k_strides[k];
    a.ys[0][k] = p->qo_strides[k];
    a.ys[1][k] = p->ko_strides[k];
  }
  a.positions = positions;
  a.inv_freq = inv_freq;
  a.N = p->N;
  a.tokens = p->B * p->N;
  a.d = p->d;
  a.half = p->rotary_dim / 2;
  a.heads[0] = p->Hq;
  a.heads[1] = p->Hk;
  a.axes = p->axes;
  int at = 0;
  for (int k = 0; k < 4; k++) {
    if (k < p->axes) at += p->sections[k];
    a.end[k] = at;
  }
  a.sign = p->inverse ? -1.f : 1.f;
  // Many tokens: eight frequencies a thread, for as many of up to eight heads as leave the machine 2^16 threads (of a training batch, 4109 tokens of 126
  // heads of 128, one head 74 us, eight 57; 2048 of 40 14.6 and, with two, 10.2; 8192 of 64 of 64 40 and 30; asked to leave 2^19, 16381
  // of 32 of 64 go from 122 to 134 forth and back); few: two, for one head.
  const int64_t many = (int64_t)a.tokens * (p->d / 16);
  const bool wide = many >= 4096;
  a.pieces = p->d / (wide ? 16 : 4);
  a.heads_per_thread = 1;
  for (int n = 8; n > 1 && a.heads_per_thread == 1; n /= 2)
    if (wide && many * ((p->Hq + n - 1) / n + (p->Hk + n - 1) / n) >= 1 << 16) a.heads_per_thread = n;
  for (int k = 0; k < 2; k++) a.head_groups[k] = (a.heads[k] + a.heads_per_thread - 1) / a.heads_per_thread;
  const dim3 grid((unsigned)(((int64_t)a.tokens * a.pieces + 255) / 256), a.head_groups[0] + a.head_groups[1]);
  hipStream_t st = (hipStream_t)stream;
  const auto launch = [&](auto adjacent, auto pos) {
    typedef decltype(pos) P;
    if (wide) rotary_kernel<8, decltype(adjacent)::value, P><<<grid, 256, 0, st>>>(a);
    else rotary_kernel<2, decltype(adjacent)::value, P><<<grid, 256, 0, st>>>(a);
  };
  if (p->adjacent) p->positions64 ? launch(std::true_type(), int64_t()) : launch(std::true_type(), int32_t());
  else p->positions64 ? launch(std::false_type(), int64_t()) : launch(std::false_type(), int32_t());
  SERVE_LAUNCH_CHECK();
  return SAGEBWD_OK;
}

}  // extern "C"
