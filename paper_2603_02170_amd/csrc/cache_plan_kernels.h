// Bookkeeping of a cache's pages: a step's new tokens, and requests that end (gfx950 only).  What the calls do is in sagebwd_serve.h.
#pragma once

#include "cache_kernels.h"

namespace sage {

struct PlanArgs {
  const int32_t *held, *added, *free_pages, *free_count;
  int32_t* table;
  int64_t* slots;
  int32_t *positions, *cu, *lengths, *granted, *free_left;
  int R, columns, page_shift, capacity, rows;
};

// Slot and position of row `row`; `cu` (the array or a copy of it), `lengths`, `granted` and the table are complete.
__device__ __forceinline__ void plan_row(const PlanArgs& a, const int32_t* cu, int row) {
  int64_t slot = -1;
  int position = 0;
  if (row < cu[a.R]) {
    int lo = 0, hi = a.R;            // the last request that begins at or before the row and has tokens
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (cu[mid] <= row) lo = mid;
      else hi = mid;
    }
    if (a.granted[lo]) {
      const int n = cu[lo + 1] - cu[lo];
      position = a.lengths[lo] - n + row - cu[lo];
      const int entry = a.table[(size_t)lo * a.columns + (position >> a.page_shift)];
      if (entry >= 0) slot = ((int64_t)entry << a.page_shift) + (position & ((1 << a.page_shift) - 1));
    }
  }
  a.slots[row] = slot;
  a.positions[row] = position;
}

// Everything but the rows, and those too where `with_rows`.  The sums over the requests are what everything waits for, and as many requests as a
// workgroup has threads are one step of them.  (32 requests take 1 wave 2.9 us, 4 waves 3.4; 16 waves, of which each knew its 64-bit
// sums only, 5.9.)  Where one step is all, the rows take what they need from LDS, and of many rows several workgroups each form the
// sums again, for rows of their own: the first writes the rest.  (300 requests, 4739 rows: with a launch of the rows 8.7 us, so 6.2, of which the host
// takes 5.5.)
template <int WAVES>
__global__ __launch_bounds__(64 * WAVES) void cache_plan_kernel(PlanArgs a, int with_rows) {
  constexpr int THREADS = 64 * WAVES;
  __shared__ unsigned sums2[WAVES][2], sums1[WAVES][1];
  __shared__ unsigned taken_to[THREADS];      // pages granted up to and with a request of this step
  __shared__ int first_page[THREADS];         // column of a request's first new page
  __shared__ int end_of[THREADS], held_of[THREADS];      // its rows' end, and tokens held (-1: not granted)
  __shared__ unsigned total[3];
  const int tid = threadIdx.x;
  const bool writes = blockIdx.x == 0;
  const int64_t page = 1 << a.page_shift;
  const unsigned count = (unsigned)max(0, min(a.free_count[0], a.capacity));
  unsigned tokens0 = 0, need0 = 0, taken0 = 0;      // sums of the steps before
  for (int base = 0; base < a.R; base += THREADS) {
    const int r = base + tid;
    int64_t held = 0, n = 0;
    unsigned need = 0;
    bool valid = false;
    if (r < a.R) {
      held = a.held[r];
      n = a.added[r];
      valid = held >= 0 && n >= 0 && held + n <= (int64_t)a.columns * page;
      if (!valid) n = 0;
      need = valid ? (unsigned)(((held + n + page - 1) >> a.page_shift) - ((held + page - 1) >> a.page_shift)) : 0;
    }
    unsigned both[2] = {(unsigned)n, need};
    block_scan<WAVES>(both, sums2);
    const unsigned tokens = min(tokens0 + both[0], kFull), needs = min(need0 + both[1], kFull);
    const bool granted = valid && tokens <= (unsigned)a.rows && (need == 0 || needs <= count);
    unsigned one[1] = {granted ? need : 0};
    block_scan<WAVES>(one, sums1);
    const unsigned taken = taken0 + one[0];           // (at most count)
    taken_to[tid] = taken;
    first_page[tid] = (int)((held + page - 1) >> a.page_shift);
    end_of[tid] = (int)min(tokens, (unsigned)a.rows);
    held_of[tid] = granted ? (int)held : -1;
    if (r < a.R && writes) {
      a.cu[r + 1] = end_of[tid];
      a.granted[r] = granted;
      a.lengths[r] = (int)(granted ? held + n : held);
    }
    if (tid == THREADS - 1) {
      total[0] = tokens;
      total[1] = needs;
      total[2] = taken;
    }
    __syncthreads();
    tokens0 = total[0];
    need0 = total[1];
    const unsigned end = total[2];
    for (unsigned k = taken0 + tid; writes && k < end; k += THREADS) {       // (k < end <= count <= capacity)
      int lo = 0, hi = THREADS - 1;         // the first request of this step with taken_to > k
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (taken_to[mid] > k) hi = mid;
        else lo = mid + 1;
      }
      const unsigned before = lo > 0 ? taken_to[lo - 1] : taken0;
      a.table[(size_t)(base + lo) * a.columns + first_page[lo] + (k - before)] = a.free_pages[count - 1 - k];
    }
    taken0 = end;
    if (base + THREADS < a.R) __syncthreads();
  }
  if (tid == 0 && writes) {
    a.cu[0] = 0;
    a.free_left[0] = (int)(count - taken0);
  }
  if (!with_rows) return;
  if (a.R <= THREADS) {
    const int end = (int)min(tokens0, (unsigned)a.rows);
    for (int row = blockIdx.x * THREADS + tid; row < a.rows; row += gridDim.x * THREADS) {
      int64_t slot = -1;
      int position = 0;
      if (row < end) {
        int lo = 0, hi = a.R - 1;        // the first request that ends behind the row
        while (lo < hi) {
          const int mid = (lo + hi) >> 1;
          if (end_of[mid] > row) hi = mid;
          else lo = mid + 1;
        }
        if (held_of[lo] >= 0) {
          position = held_of[lo] + row - (lo > 0 ? end_of[lo - 1] : 0);
          const int column = position >> a.page_shift, k = column - first_page[lo];      // (a new page: what goes into the table, from the stack)
          const int entry = k < 0 ? a.table[(size_t)lo * a.columns + column] : a.free_pages[count - 1 - ((lo > 0 ? taken_to[lo - 1] : 0) + k)];
          if (entry >= 0) slot = ((int64_t)entry << a.page_shift) + (position & ((1 << a.page_shift) - 1));
        }
      }
      a.slots[row] = slot;
      a.positions[row] = position;
    }
  } else {
    __threadfence_block();
    __syncthreads();
    for (int row = tid; row < a.rows; row += THREADS) plan_row(a, a.cu, row);
  }
}
// (the search of a row's request runs in LDS where cu fits: 300 requests, 4739 rows 5.0 -> 3.5 us)
__global__ __launch_bounds__(256) void cache_plan_rows_kernel(PlanArgs a) {
  constexpr int MOST = 4096;
  __shared__ int32_t cu[MOST];
  const int row = blockIdx.x * 256 + threadIdx.x;
  const bool fits = a.R < MOST;
  if (fits) {
    for (int i = threadIdx.x; i <= a.R; i += 256) cu[i] = a.cu[i];
    __syncthreads();
  }
  if (row >= a.rows) return;
  if (fits) plan_row(a, cu, row);
  else plan_row(a, a.cu, row);
}

struct TrimArgs {
  const int32_t* keep;
  int32_t *lengths, *table, *free_pages, *free_count;
  int R, columns, page_shift, capacity;
};
__global__ __launch_bounds__(1024) void cache_trim_kernel(TrimArgs a) {
  __shared__ unsigned sums[16][1];
  __shared__ unsigned freed_to[1024];
  __shared__ int first_page[1024];
  __shared__ unsigned total, in_step;
  const int tid = threadIdx.x;
  const int64_t page = 1 << a.page_shift;
  const unsigned count = (unsigned)max(0, min(a.free_count[0], a.capacity));
  // pages of a request from the first it loses to its last
  auto freed_of = [&](int r, int& first) -> unsigned {
    const int len = a.lengths[r], keep = a.keep[r];
    first = 0;
    if (keep < 0 || keep > len) return 0;
    first = (int)((keep + page - 1) >> a.page_shift);
    const int end = (int)min((len + page - 1) >> a.page_shift, (int64_t)a.columns);
    return (unsigned)max(0, end - first);
  };
  // Twice over what is freed, 1024 entries of the table at a time: how many of them are pages (entries that are not have none to give back),
  // then each to its place, the first page freed on top.
  unsigned all = 0;
  for (int pass = 0; pass < 2; pass++) {
    unsigned before_step = 0, freed = 0;       // entries, and pages among them, of the steps before
    for (int base = 0; base < a.R; base += 1024) {
      const int r = base + tid;
      int first = 0;
      unsigned n[1] = {r < a.R ? freed_of(r, first) : 0};
      block_scan<16>(n, sums);
      const unsigned to = min(before_step + n[0], kFull);
      freed_to[tid] = to;
      first_page[tid] = first;
      if (tid == 1023) total = to;
      __syncthreads();
      const unsigned end = total;
      for (unsigned k0 = before_step; k0 < end; k0 += 1024) {
        const unsigned k = k0 + tid;
        int32_t* entry = nullptr;
        if (k < end) {
          int lo = 0, hi = 1023;
          while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (freed_to[mid] > k) hi = mid;
            else lo = mid + 1;
          }
          const unsigned before = lo > 0 ? freed_to[lo - 1] : before_step;
          entry = a.table + (size_t)(base + lo) * a.columns + first_page[lo] + (k - before);
        }
        const bool has = entry != nullptr && *entry >= 0;
        unsigned rank[1] = {has ? 1u : 0u};
        block_scan<16>(rank, sums);
        if (pass == 1 && entry != nullptr) {
          const int64_t at = (int64_t)count + ((int64_t)all - freed - rank[0]);
          if (has && at < a.capacity) a.free_pages[at] = *entry;
          *entry = -1;
        }
        if (tid == 1023) in_step = rank[0];
        __syncthreads();
        freed += in_step;
      }
      if (pass == 1 && r < a.R) {
        const int len = a.lengths[r], keep = a.keep[r];
        if (keep >= 0 && keep <= len) a.lengths[r] = keep;
      }
      before_step = end;
      __syncthreads();
    }
    all = freed;
  }
  if (tid == 0) a.free_count[0] = (int)min((int64_t)count + all, (int64_t)a.capacity);
}

}  // namespace sage
