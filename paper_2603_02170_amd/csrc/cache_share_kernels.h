// Pages that requests share: freeing, forking, owning, compacting (gfx950 only).  What the calls do is in sagebwd_serve.h.
//
// shares [3, pages]: the holders of a page beyond its first; a bit for each page that may have lost its last; nothing (own: who asks).  Holders are
// counted with integer atomics, whose order changes nothing; what depends on an order (the stack of free pages, who keeps a page) is decided
// by page numbers or request numbers afterwards.
//
// Steps: a workgroup has kColumns columns of a request's row of the table, a thread four of them, whose loads are under way together; one workgroup
// settles the stack.  Small calls are one launch of one workgroup.  (A wave a row, one trip to memory after the other: 25 requests of 530 pages 55 us
// for free, fork and own; so 24.)
#pragma once

#include "cache_kernels.h"

namespace sage {

struct PagesArgs {
  const int32_t* asked;            // keep, parents or added
  int32_t *lengths, *table, *free_pages, *free_count, *shares;
  int32_t *rows, *new_lengths;     // fork: the new rows of the table
  int32_t* granted;                // own: added, or 0
  int2* moves;                     // own, compact: page from, page to (own: -1 for none)
  int R, columns, page_shift, capacity, pages;
  __device__ __forceinline__ uint32_t* bits() const { return (uint32_t*)shares + pages; }
  __device__ __forceinline__ int pages_of(int length) const {
    return (int)min(((int64_t)length + (1 << page_shift) - 1) >> page_shift, (int64_t)columns);
  }
  __device__ __forceinline__ bool is_page(int entry) const { return (unsigned)entry < (unsigned)pages; }
};

// What another step of the same workgroup, or another workgroup's atomic, wrote.
__device__ __forceinline__ int now_in(const int32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// (Whoever takes the count below zero says so: of a page that ends there someone does, also where others count it up meanwhile.  With a bit from each of five holders
// of 530 pages free took 14.3 us, so 4.2.)
__device__ __forceinline__ void lose_page(const PagesArgs& a, int entry) {
  if (atomicSub(a.shares + entry, 1) <= 0) atomicOr(a.bits() + (entry >> 5), 1u << (entry & 31));
}

// Pages whose last holder went go on the stack, the lowest last.  One workgroup; 64 pages a thread at a time, from the highest: each wave finds the ones
// among 64, a lane a page, then their places are summed.
constexpr int kAtOnce = 4;      // loads of a lane under way
template <int WAVES>
struct SettleScratch {
  uint64_t freed[64 * WAVES];
  unsigned sums[WAVES][1], total;
};
template <int WAVES>
__device__ __forceinline__ void settle_pages(const PagesArgs& a, SettleScratch<WAVES>& s) {
  constexpr int THREADS = 64 * WAVES;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int groups = (a.pages + 63) >> 6, words = (a.pages + 31) >> 5;
  int64_t count = max(0, min(now_in(a.free_count), a.capacity));
  for (int end = groups; end > 0; end -= THREADS) {
    const int here = min(end, THREADS);
    for (int i0 = wave; i0 < here; i0 += WAVES * kAtOnce) {
      uint32_t word[kAtOnce];
      int holders[kAtOnce];
#pragma unroll
      for (int k = 0; k < kAtOnce; k++) {
        const int i = i0 + WAVES * k, group = end - 1 - i, at = 2 * group + (lane >> 5), page = 64 * group + lane;
        word[k] = i < here && at < words ? (uint32_t)now_in((const int32_t*)a.bits() + at) : 0;
        holders[k] = i < here && page < a.pages ? now_in(a.shares + page) : 0;
      }
#pragma unroll
      for (int k = 0; k < kAtOnce; k++) {
        const int i = i0 + WAVES * k, group = end - 1 - i;
        if (i >= here) break;
        if ((lane & 31) == 0 && word[k] != 0) a.bits()[2 * group + (lane >> 5)] = 0;
        const bool freed = (word[k] >> (lane & 31) & 1) && holders[k] < 0;
        if (freed) a.shares[64 * group + lane] = 0;
        const uint64_t mask = __ballot(freed);
        if (lane == 0) s.freed[i] = mask;
      }
    }
    __syncthreads();
    unsigned to[1] = {tid < here ? (unsigned)__popcll(s.freed[tid]) : 0};
    block_scan<WAVES>(to, s.sums);
    if (tid == THREADS - 1) s.total = to[0];
    if (tid < here) {
      uint64_t mask = s.freed[tid];
      int64_t at = count + to[0] - __popcll(mask);
      while (mask != 0) {
        const int bit = 63 - __builtin_clzll(mask);
        mask ^= 1ull << bit;
        if (at < a.capacity) a.free_pages[at] = 64 * (end - 1 - tid) + bit;
        at++;
      }
    }
    __syncthreads();
    count += s.total;
    __syncthreads();
  }
  if (tid == 0) a.free_count[0] = (int)min(count, (int64_t)a.capacity);
}

constexpr int kColumns = 1024;
template <typename F>
__device__ __forceinline__ void each_column(const PagesArgs& a, F f) {
  const int chunks = (a.columns + kColumns - 1) / kColumns, r = blockIdx.x / chunks;
  f(r, (int)(blockIdx.x - r * chunks) * kColumns + (int)threadIdx.x);
}
template <int THREADS, typename F>
__device__ __forceinline__ void each_entry(const PagesArgs& a, F f) {      // of a small call
  for (int i = threadIdx.x; i < a.R * a.columns; i += THREADS) f(i / a.columns, i % a.columns);
}

// ---- free ----------------------------------------------------------------------------------------------------------
__device__ __forceinline__ bool keeps(const PagesArgs& a, int r) { return a.asked[r] >= 0 && a.asked[r] <= a.lengths[r]; }
// What a request gives up of N columns, `step` apart.
template <int N>
__device__ __forceinline__ void free_columns(const PagesArgs& a, int r, int c0, int step) {
  const int length = a.lengths[r], keep = a.asked[r];
  if (keep < 0 || keep > length) return;
  const int first = a.pages_of(keep), end = a.pages_of(length);
  int32_t* row = a.table + (size_t)r * a.columns;
  int entry[N];
#pragma unroll
  for (int k = 0; k < N; k++) {
    const int c = c0 + k * step;
    entry[k] = c >= first && c < end ? row[c] : -1;
  }
#pragma unroll
  for (int k = 0; k < N; k++) {
    const int c = c0 + k * step;
    if (a.is_page(entry[k])) lose_page(a, entry[k]);
    if (c >= first && c < end) row[c] = -1;
  }
}
__global__ __launch_bounds__(256) void cache_free_rows_kernel(PagesArgs a) {
  each_column(a, [&](int r, int c) { free_columns<4>(a, r, c, 256); });
}
// the first workgroup settles, the others have the lengths
__global__ __launch_bounds__(1024) void cache_freed_kernel(PagesArgs a) {
  __shared__ SettleScratch<16> s;
  if (blockIdx.x == 0) {
    settle_pages(a, s);
    return;
  }
  const int r = (blockIdx.x - 1) * 1024 + threadIdx.x;
  if (r < a.R && keeps(a, r)) a.lengths[r] = a.asked[r];
}
template <int WAVES>
__global__ __launch_bounds__(64 * WAVES) void cache_free_kernel(PagesArgs a) {
  __shared__ SettleScratch<WAVES> s;
  each_entry<64 * WAVES>(a, [&](int r, int c) { free_columns<1>(a, r, c, 0); });
  __threadfence_block();
  __syncthreads();
  for (int r = threadIdx.x; r < a.R; r += 64 * WAVES)
    if (keeps(a, r)) a.lengths[r] = a.asked[r];
  settle_pages(a, s);
}

// ---- fork ----------------------------------------------------------------------------------------------------------
__device__ __forceinline__ bool forked(const PagesArgs& a, int r) {
  const int p = a.asked[r];
  return p >= 0 && p < a.R && p != r;
}
// N columns of the row that a request goes on with, to `rows`, as a row may be another one's parent; pages that stay where they are count for nothing.
template <int N>
__device__ __forceinline__ void fork_columns(const PagesArgs& a, int r, int c0, int step) {
  if (!forked(a, r)) return;
  const int p = a.asked[r], length = a.lengths[p], n = a.pages_of(length), had = a.pages_of(a.lengths[r]);
  const int32_t *from = a.table + (size_t)p * a.columns, *old = a.table + (size_t)r * a.columns;
  int entry[N], before[N];
#pragma unroll
  for (int k = 0; k < N; k++) {
    const int c = c0 + k * step;
    entry[k] = c < n ? from[c] : -1;
    before[k] = c < had ? old[c] : -1;
  }
#pragma unroll
  for (int k = 0; k < N; k++) {
    const int c = c0 + k * step;
    if (c < a.columns) a.rows[(size_t)r * a.columns + c] = entry[k];
    if (entry[k] == before[k]) continue;
    if (a.is_page(entry[k])) atomicAdd(a.shares + entry[k], 1);
    if (a.is_page(before[k])) lose_page(a, before[k]);
  }
  if (c0 == 0) a.new_lengths[r] = length;
}
template <int N>
__device__ __forceinline__ void forked_columns(const PagesArgs& a, int r, int c0, int step) {
  if (!forked(a, r)) return;
#pragma unroll
  for (int k = 0; k < N; k++) {
    const int c = c0 + k * step;
    if (c < a.columns) a.table[(size_t)r * a.columns + c] = a.rows[(size_t)r * a.columns + c];
  }
  if (c0 == 0) a.lengths[r] = a.new_lengths[r];
}
__global__ __launch_bounds__(256) void cache_fork_rows_kernel(PagesArgs a) {
  each_column(a, [&](int r, int c) { fork_columns<4>(a, r, c, 256); });
}
// the first workgroup settles, the others have kColumns of a row each
__global__ __launch_bounds__(1024) void cache_forked_kernel(PagesArgs a) {
  __shared__ SettleScratch<16> s;
  if (blockIdx.x == 0) {
    settle_pages(a, s);
    return;
  }
  const int chunks = (a.columns + kColumns - 1) / kColumns, i = blockIdx.x - 1, r = i / chunks;
  forked_columns<1>(a, r, (i - r * chunks) * kColumns + (int)threadIdx.x, 0);
}
template <int WAVES>
__global__ __launch_bounds__(64 * WAVES) void cache_fork_kernel(PagesArgs a) {
  __shared__ SettleScratch<WAVES> s;
  each_entry<64 * WAVES>(a, [&](int r, int c) { fork_columns<1>(a, r, c, 0); });
  __threadfence_block();
  __syncthreads();
  each_entry<64 * WAVES>(a, [&](int r, int c) { forked_columns<1>(a, r, c, 0); });
  settle_pages(a, s);
}

// ---- own -----------------------------------------------------------------------------------------------------------
// Who writes into a page that others hold gets a copy of it; if all its holders are about to write, the last of them keeps it.  One
// workgroup; the copies are a launch of their own.
template <int WAVES>
__global__ __launch_bounds__(64 * WAVES) void cache_own_kernel(PagesArgs a) {
  constexpr int THREADS = 64 * WAVES;
  __shared__ unsigned sums[WAVES][1], total;
  const int tid = threadIdx.x;
  int32_t *asks = a.shares + a.pages, *last = asks + a.pages;      // of a page: how many are about to write, and 1 + the last of them
  // the page that a request's next token goes into, if that has tokens
  const auto page_of = [&](int r) {
    const int length = a.lengths[r];
    if (a.asked[r] <= 0 || length <= 0 || (length & ((1 << a.page_shift) - 1)) == 0 || length >> a.page_shift >= a.columns) return -1;
    const int entry = a.table[(size_t)r * a.columns + (length >> a.page_shift)];
    return a.is_page(entry) ? entry : -1;
  };
  // (the thread's first request stays in registers from step to step)
  const auto holders_of = [&](int entry) { return entry >= 0 ? a.shares[entry] : 0; };
  const int entry0 = tid < a.R ? page_of(tid) : -1, holders0 = holders_of(entry0);
  for (int r = tid; r < a.R; r += THREADS) {
    const int entry = r == tid ? entry0 : page_of(r), holders = r == tid ? holders0 : holders_of(entry);
    if (holders <= 0) continue;
    atomicAdd(asks + entry, 1);
    atomicMax(last + entry, r + 1);
  }
  const unsigned count = (unsigned)max(0, min(a.free_count[0], a.capacity));
  __threadfence_block();
  __syncthreads();
  unsigned before = 0;
  int2 move0 = {-1, -1};
  for (int base = 0; base < a.R; base += THREADS) {
    const int r = base + tid;
    const int entry = base == 0 ? entry0 : r < a.R ? page_of(r) : -1, holders = base == 0 ? holders0 : holders_of(entry);
    const bool wants = holders > 0;
    const bool copies = wants && !(now_in(asks + entry) == holders + 1 && now_in(last + entry) == r + 1);
    unsigned need[1] = {copies ? 1u : 0u};
    block_scan<WAVES>(need, sums);
    if (tid == THREADS - 1) total = need[0];
    const unsigned needs = min(before + need[0], kFull);
    const bool granted = !wants || needs <= count;
    int2 move = {entry, -1};
    if (r < a.R) {
      a.granted[r] = granted ? a.asked[r] : 0;
      if (copies && granted) {
        const int to = a.free_pages[count - needs];
        a.table[(size_t)r * a.columns + (a.lengths[r] >> a.page_shift)] = to;
        move.y = a.is_page(to) ? to : -2;      // (a stack of something else: nothing is copied there)
      }
      a.moves[r] = move;
    }
    if (base == 0) move0 = move;
    __syncthreads();
    before = min(before + total, kFull);
    __syncthreads();
  }
  for (int r = tid; r < a.R; r += THREADS) {
    const int2 move = r == tid ? move0 : a.moves[r];
    if (move.x < 0) continue;
    asks[move.x] = 0;
    last[move.x] = 0;
    if (move.y != -1) atomicSub(a.shares + move.x, 1);
  }
  if (tid == 0) a.free_count[0] = (int)(count - min(before, count));
}

// Pages are copied in pieces of 16 KiB, four loads of a thread in flight.
constexpr int kCopyPiece = 16384;
__device__ __forceinline__ void copy_piece(unsigned char* pool, size_t page_bytes, const int2& move, int piece) {
  const unsigned char* from = pool + (size_t)move.x * page_bytes;
  unsigned char* to = pool + (size_t)move.y * page_bytes;
  const size_t at0 = (size_t)piece * kCopyPiece + threadIdx.x * 16;
  v4i x[4];
#pragma unroll
  for (int i = 0; i < 4; i++)
    if (at0 + i * 4096 < page_bytes) x[i] = *(const v4i*)(from + at0 + i * 4096);
#pragma unroll
  for (int i = 0; i < 4; i++)
    if (at0 + i * 4096 < page_bytes) *(v4i*)(to + at0 + i * 4096) = x[i];
}
__global__ __launch_bounds__(256) void cache_copy_pages_kernel(const int2* moves, unsigned char* pool, size_t page_bytes) {
  const int2 move = moves[blockIdx.x];
  if (move.y >= 0) copy_piece(pool, page_bytes, move, blockIdx.y);
}

// ---- compact -------------------------------------------------------------------------------------------------------
struct CompactArgs {
  PagesArgs p;               // its shares, free_pages and free_count are written; `moves` has room for half of the pages
  int32_t* table_out;
  int32_t* used;
  uint64_t* masks;           // of every 64 pages, which are in use,
  int32_t* before;           // and how many in front of them
  int32_t* sizes;            // pages in use, those of them that have to move
  unsigned char* pool;
  size_t page_bytes;
  int pieces;
};
// The holders of a request's pages, in the second row of shares.
template <int N>
__device__ __forceinline__ void count_columns(const PagesArgs& a, int r, int c0, int step) {
  const int n = a.pages_of(max(a.lengths[r], 0));
  int entry[N];
#pragma unroll
  for (int k = 0; k < N; k++) entry[k] = c0 + k * step < n ? a.table[(size_t)r * a.columns + c0 + k * step] : -1;
#pragma unroll
  for (int k = 0; k < N; k++)
    if (a.is_page(entry[k])) atomicAdd(a.shares + a.pages + entry[k], 1);
}
// 1024 threads: which pages are in use, and which of them go where.
struct CompactScratch {
  unsigned sums[16][1], total, below;
};
__device__ __forceinline__ void choose_moves(const CompactArgs& c, CompactScratch& s) {
  const PagesArgs& a = c.p;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int groups = (a.pages + 63) >> 6;
  for (int g0 = wave; g0 < groups; g0 += 16 * kAtOnce) {
    int holders[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; k++) {
      const int page = 64 * (g0 + 16 * k) + lane;
      holders[k] = page < a.pages ? now_in(a.shares + a.pages + page) : 0;
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; k++) {
      const uint64_t mask = __ballot(holders[k] > 0);
      if (lane == 0 && g0 + 16 * k < groups) c.masks[g0 + 16 * k] = mask;
    }
  }
  __threadfence_block();
  __syncthreads();
  unsigned n = 0;
  for (int base = 0; base < groups; base += 1024) {
    const int g = base + tid;
    const unsigned mine = g < groups ? (unsigned)__popcll(c.masks[g]) : 0;
    unsigned to[1] = {mine};
    block_scan<16>(to, s.sums);
    if (g < groups) c.before[g] = (int)(n + to[0] - mine);
    if (tid == 1023) s.total = to[0];
    __syncthreads();
    n += s.total;
    __syncthreads();
  }
  if (tid == 0) s.below = (int)n == a.pages ? n : (unsigned)c.before[n >> 6] + __popcll(c.masks[n >> 6] & ((1ull << (n & 63)) - 1));
  __syncthreads();
  const int below = (int)s.below;      // in use among the first n: the others of those are where the rest goes
  for (int g = wave; g < groups; g += 16) {
    const int page = 64 * g + lane;
    const uint64_t mask = c.masks[g];
    const bool in_use = mask >> lane & 1;
    const int upto = c.before[g] + __popcll(mask & ((1ull << lane) - 1));
    if (page < (int)n && !in_use) a.moves[page - upto].y = page;
    if (page >= (int)n && in_use) a.moves[upto - below].x = page;
  }
  if (tid == 0) {
    c.sizes[0] = (int)n;
    c.sizes[1] = (int)n - below;
    c.used[0] = (int)n;
    a.free_count[0] = a.pages - (int)n;
  }
}
__global__ __launch_bounds__(256) void cache_count_kernel(CompactArgs c) {
  each_column(c.p, [&](int r, int at) { count_columns<4>(c.p, r, at, 256); });
}
__global__ __launch_bounds__(1024) void cache_choose_kernel(CompactArgs c) {
  __shared__ CompactScratch s;
  choose_moves(c, s);
}
__global__ __launch_bounds__(1024) void cache_count_and_choose_kernel(CompactArgs c) {
  __shared__ CompactScratch s;
  each_entry<1024>(c.p, [&](int r, int at) { count_columns<1>(c.p, r, at, 0); });
  __threadfence_block();
  __syncthreads();
  choose_moves(c, s);
}
// The new table, stack and shares, and the copies: every workgroup has some of each.
__global__ __launch_bounds__(256) void cache_compact_kernel(CompactArgs c) {
  const PagesArgs& a = c.p;
  const int n = c.sizes[0], moves = c.sizes[1];
  const int64_t first = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
  const int below = n - moves;
  const auto place_of = [&](int page) {      // of a page in use
    if (page < n) return page;
    const int g = page >> 6;
    return a.moves[c.before[g] + __popcll(c.masks[g] & ((1ull << (page & 63)) - 1)) - below].y;
  };
  for (int64_t i = first; i < (int64_t)a.R * a.columns; i += step) {
    const int r = (int)(i / a.columns), at = (int)(i - (int64_t)r * a.columns);
    const int entry = at < a.pages_of(max(a.lengths[r], 0)) ? a.table[i] : -1;
    c.table_out[i] = a.is_page(entry) ? place_of(entry) : -1;
  }
  for (int64_t i = first; i < a.capacity; i += step) a.free_pages[i] = i < a.pages - n ? (int)(a.pages - 1 - i) : -1;
  for (int64_t i = first; i < a.pages; i += step) {
    const int holders = a.shares[a.pages + i];
    if (holders > 0) a.shares[place_of((int)i)] = holders - 1;
    if (i >= n) a.shares[i] = 0;
    a.shares[a.pages + i] = 0;
  }
  for (int64_t i = blockIdx.x; i < (int64_t)moves * c.pieces; i += gridDim.x) {
    const int k = (int)(i / c.pieces);
    copy_piece(c.pool, c.page_bytes, a.moves[k], (int)(i - (int64_t)k * c.pieces));
  }
}

}  // namespace sage
