// The 4-bit cache beside its attention: bookkeeping of pages, storing and reading tokens (gfx950 only).
// The format of a page and the quantiser are in sagebwd_serve.h.
#pragma once

#include "common.h"

namespace sage {

// Where things stand in one head's part of a page.
struct CacheGeometry {
  int H, d, page_shift, group;
  int pages;
  __host__ __device__ int page() const { return 1 << page_shift; }
  __host__ __device__ int head_bytes() const { return page() * (d + 4 * d / group); }
  __host__ __device__ size_t page_bytes() const { return (size_t)H * head_bytes(); }
  __host__ __device__ int v_codes() const { return page() * d / 2; }
  __host__ __device__ int k_scales() const { return page() * d; }
  __host__ __device__ int v_scales() const { return page() * (d + 2 * d / group); }
};

// ---- bookkeeping -----------------------------------------------------------------------------------------------
// Inclusive sum over the 1024 threads of a workgroup.
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t* wave_sums) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int k = 1; k < 64; k <<= 1) {
    const int64_t u = __shfl_up(v, k);
    if (lane >= k) v += u;
  }
  __syncthreads();
  if (lane == 63) wave_sums[wave] = v;
  __syncthreads();
  int64_t before = 0;
  for (int k = 0; k < 16; k++)
    if (k < wave) before += wave_sums[k];
  return v + before;
}

struct PlanArgs {
  const int32_t *held, *added, *free_pages, *free_count;
  int32_t* table;
  int64_t* slots;
  int32_t *positions, *cu, *lengths, *granted, *free_left;
  int R, columns, page_shift, capacity, rows;
};

// Slot and position of row `row`; `cu`, `lengths`, `granted` and the table are complete.
__device__ __forceinline__ void plan_row(const PlanArgs& a, int row) {
  int64_t slot = -1;
  int position = 0;
  if (row < a.cu[a.R]) {
    int lo = 0, hi = a.R;            // the last request that begins at or before the row and has tokens
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (a.cu[mid] <= row) lo = mid;
      else hi = mid;
    }
    if (a.granted[lo]) {
      const int n = a.cu[lo + 1] - a.cu[lo];
      position = a.lengths[lo] - n + row - a.cu[lo];
      const int entry = a.table[(size_t)lo * a.columns + (position >> a.page_shift)];
      if (entry >= 0) slot = ((int64_t)entry << a.page_shift) + (position & ((1 << a.page_shift) - 1));
    }
  }
  a.slots[row] = slot;
  a.positions[row] = position;
}

// Everything but the rows (and those too where ROWS: few of them).  One workgroup: the sums over the requests are what everything waits
// for, and a thousand requests are one step of them.
template <bool ROWS>
__global__ __launch_bounds__(1024) void cache_plan_kernel(PlanArgs a) {
  __shared__ int64_t wave_sums[16];
  __shared__ int64_t taken_to[1024];      // pages granted up to and with a request of this step
  __shared__ int first_page[1024];        // column of a request's first new page
  __shared__ int64_t total[3];
  const int tid = threadIdx.x;
  const int64_t page = 1 << a.page_shift;
  const int count = max(0, min(a.free_count[0], a.capacity));
  int64_t tokens0 = 0, need0 = 0, taken0 = 0;      // sums of the steps before
  for (int base = 0; base < a.R; base += 1024) {
    const int r = base + tid;
    int64_t held = 0, n = 0, need = 0;
    bool valid = false;
    if (r < a.R) {
      held = a.held[r];
      n = a.added[r];
      valid = held >= 0 && n >= 0 && held + n <= (int64_t)a.columns * page;
      if (!valid) n = 0;
      need = valid ? ((held + n + page - 1) >> a.page_shift) - ((held + page - 1) >> a.page_shift) : 0;
    }
    const int64_t tokens = tokens0 + block_scan(n, wave_sums), needs = need0 + block_scan(need, wave_sums);
    const bool granted = valid && tokens <= a.rows && (need == 0 || needs <= count);
    const int64_t taken = taken0 + block_scan(granted ? need : 0, wave_sums);
    taken_to[tid] = taken;
    first_page[tid] = (int)((held + page - 1) >> a.page_shift);
    if (r < a.R) {
      a.cu[r + 1] = (int)min(tokens, (int64_t)a.rows);
      a.granted[r] = granted;
      a.lengths[r] = (int)(granted ? held + n : held);
    }
    if (tid == 1023) {
      total[0] = tokens;
      total[1] = needs;
      total[2] = taken;
    }
    __syncthreads();
    tokens0 = total[0];
    need0 = total[1];
    const int64_t end = total[2];
    for (int64_t k = taken0 + tid; k < end; k += 1024) {       // (k < end <= count <= capacity)
      int lo = 0, hi = 1023;         // the first request of this step with taken_to > k
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (taken_to[mid] > k) hi = mid;
        else lo = mid + 1;
      }
      const int64_t before = lo > 0 ? taken_to[lo - 1] : taken0;
      a.table[(size_t)(base + lo) * a.columns + first_page[lo] + (k - before)] = a.free_pages[count - 1 - k];
    }
    taken0 = end;
    __syncthreads();
  }
  if (tid == 0) {
    a.cu[0] = 0;
    a.free_left[0] = count - (int)taken0;
  }
  if (ROWS) {
    __threadfence_block();
    __syncthreads();
    for (int row = tid; row < a.rows; row += 1024) plan_row(a, row);
  }
}
__global__ __launch_bounds__(256) void cache_plan_rows_kernel(PlanArgs a) {
  const int row = blockIdx.x * 256 + threadIdx.x;
  if (row < a.rows) plan_row(a, row);
}

struct TrimArgs {
  const int32_t* keep;
  int32_t *lengths, *table, *free_pages, *free_count;
  int R, columns, page_shift, capacity;
};
__global__ __launch_bounds__(1024) void cache_trim_kernel(TrimArgs a) {
  __shared__ int64_t wave_sums[16];
  __shared__ int64_t freed_to[1024];
  __shared__ int first_page[1024];
  __shared__ int64_t total;
  const int tid = threadIdx.x;
  const int64_t page = 1 << a.page_shift;
  const int count = max(0, min(a.free_count[0], a.capacity));
  // pages of a request from the first it loses to its last
  auto freed_of = [&](int r, int& first) -> int {
    const int len = a.lengths[r], keep = a.keep[r];
    first = 0;
    if (keep < 0 || keep > len) return 0;
    first = (int)((keep + page - 1) >> a.page_shift);
    const int end = (int)min((len + page - 1) >> a.page_shift, (int64_t)a.columns);
    return max(0, end - first);
  };
  int64_t all = 0;
  {
    int64_t mine = 0;
    for (int r = tid; r < a.R; r += 1024) {
      int first;
      mine += freed_of(r, first);
    }
    const int64_t s = block_scan(mine, wave_sums);
    if (tid == 1023) total = s;
    __syncthreads();
    all = total;
    __syncthreads();
  }
  int64_t before_step = 0;
  for (int base = 0; base < a.R; base += 1024) {
    const int r = base + tid;
    int first = 0;
    const int n = r < a.R ? freed_of(r, first) : 0;
    const int64_t to = before_step + block_scan(n, wave_sums);
    freed_to[tid] = to;
    first_page[tid] = first;
    if (tid == 1023) total = to;
    __syncthreads();
    const int64_t end = total;
    for (int64_t k = before_step + tid; k < end; k += 1024) {
      int lo = 0, hi = 1023;
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (freed_to[mid] > k) hi = mid;
        else lo = mid + 1;
      }
      const int64_t before = lo > 0 ? freed_to[lo - 1] : before_step;
      int32_t* entry = a.table + (size_t)(base + lo) * a.columns + first_page[lo] + (k - before);
      const int64_t at = count + (all - 1 - k);      // the first page freed ends on top
      if (at < a.capacity) a.free_pages[at] = *entry;
      *entry = -1;
    }
    if (r < a.R) {
      const int len = a.lengths[r], keep = a.keep[r];
      if (keep >= 0 && keep <= len) a.lengths[r] = keep;
    }
    before_step = end;
    __syncthreads();
  }
  if (tid == 0) a.free_count[0] = (int)min(count + all, (int64_t)a.capacity);
}

// ---- storing and reading ---------------------------------------------------------------------------------------
// Largest of a group's |x|, as bits, so that an infinity and a NaN are the largest: over the lane's 8 channels and GROUP / 8 lanes.
template <int GROUP>
__device__ __forceinline__ unsigned group_max(const float* x) {
  unsigned m = 0;
#pragma unroll
  for (int i = 0; i < 8; i++) m = max(m, __float_as_uint(x[i]) & 0x7FFFFFFFu);
#pragma unroll
  for (int k = 1; k < GROUP / 8; k <<= 1) m = max(m, (unsigned)__shfl_xor((int)m, k));
  return m;
}
// Codes (-7 .. 7) of a lane's 8 channels; returns the scale's bf16 bits.
template <int GROUP>
__device__ __forceinline__ unsigned short quantise4(const float* x, int* q) {
  const unsigned top = group_max<GROUP>(x);
  if (top < 0x0D800000u || top >= 0x7F000000u) {     // below 2^-100: zeros; from 2^127 on, infinities and NaN: a scale that is NaN
#pragma unroll
    for (int i = 0; i < 8; i++) q[i] = 0;
    return top < 0x0D800000u ? 0 : 0x7FC0;
  }
  const unsigned bits = (__float_as_uint(__fdiv_rn(__uint_as_float(top), 7.0f)) + 0x7FFFFu) & 0xFFF80000u;
  const float s = __uint_as_float(bits), r = __fdiv_rn(1.0f, s);
#pragma unroll
  for (int i = 0; i < 8; i++) {
    // x / s rounded to nearest: the product with the rounded reciprocal and one step on its residual, which the scales' 5 bits need
    // (bf16 inputs meet them in exact ties)
    const float t = x[i] * r;
    q[i] = (int)rintf(__builtin_fmaf(__builtin_fmaf(-t, s, x[i]), r, t));
  }
  return (unsigned short)(bits >> 16);
}

struct StoreArgs {
  const __bf16 *K, *V;
  int64_t ks[2], vs[2];            // token and head strides in elements
  const int64_t* slots;
  const float *k_mean, *v_mean;
  unsigned char* pool;
  __bf16 *Ko, *Vo;                 // reading
  int T;
  CacheGeometry g;
};

// d / 8 lanes have a token of a head, 8 channels each.  A lane's channels of K are one word; of V they lie in eight half-words, whose
// other nibbles three lanes of the same half have (2, 4 and 6 away): those are joined and each lane stores two.
template <int D, int GROUP>
__global__ __launch_bounds__(256) void cache_append_kernel(StoreArgs a) {
  constexpr int LANES = D / 8, ROWS = 256 / LANES;
  const int l = threadIdx.x % LANES;
  const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES;
  const bool exists = row < (int64_t)a.T * a.g.H;
  const int t = exists ? (int)(row / a.g.H) : 0, h = exists ? (int)(row % a.g.H) : 0;
  const int64_t slot = a.slots[t];
  const bool stored = exists && slot >= 0 && slot < ((int64_t)a.g.pages << a.g.page_shift);
  const int c = 8 * l;
  float k[8], v[8];
  {
    const v8bf x = *(const v8bf*)(a.K + t * a.ks[0] + h * a.ks[1] + c), y = *(const v8bf*)(a.V + t * a.vs[0] + h * a.vs[1] + c);
#pragma unroll
    for (int i = 0; i < 8; i++) {
      k[i] = (float)x[i] - (a.k_mean != nullptr ? a.k_mean[h * D + c + i] : 0.f);
      v[i] = (float)y[i] - (a.v_mean != nullptr ? a.v_mean[h * D + c + i] : 0.f);
    }
  }
  int kq[8], vq[8];
  const unsigned short ksc = quantise4<GROUP>(k, kq), vsc = quantise4<GROUP>(v, vq);
  unsigned kw = 0;
#pragma unroll
  for (int i = 0; i < 8; i++) kw |= (unsigned)(kq[i] + 8) << (4 * (i / 2 + 4 * (i % 2)));
  // channel 64 h + 16 j + m: j = l / 2 % 4, m = 8 (l % 2) + i
  const int j = l / 2 % 4;
  unsigned w[4];
#pragma unroll
  for (int i = 0; i < 4; i++) {
    w[i] = ((unsigned)(vq[2 * i] + 8) | (unsigned)(vq[2 * i + 1] + 8) << 16) << (4 * j);
    w[i] |= (unsigned)__shfl_xor((int)w[i], 2);
    w[i] |= (unsigned)__shfl_xor((int)w[i], 4);
  }
  if (!stored) return;
  const int at = (int)(slot & (a.g.page() - 1)), octet = at >> 3, i = at & 7;
  unsigned char* p = a.pool + (size_t)(slot >> a.g.page_shift) * a.g.page_bytes() + (size_t)h * a.g.head_bytes();
  *(unsigned*)(p + at * (D / 2) + (l % 4) * (D / 8) + l / 4 * 4) = kw;
  const unsigned mine = j == 0 ? w[0] : j == 1 ? w[1] : j == 2 ? w[2] : w[3];
  unsigned char* pv = p + a.g.v_codes() + octet * (4 * D) + l / 8 * 256 + (8 * (l % 2) + 2 * j) * 16 + 2 * i;
  *(unsigned short*)pv = (unsigned short)mine;
  *(unsigned short*)(pv + 16) = (unsigned short)(mine >> 16);
  if (l % (GROUP / 8) == 0) {
    const int sc = (octet * (D / GROUP) + l / (GROUP / 8)) * 16 + 2 * i;
    *(unsigned short*)(p + a.g.k_scales() + sc) = ksc;
    *(unsigned short*)(p + a.g.v_scales() + sc) = vsc;
  }
}

template <int D, int GROUP>
__global__ __launch_bounds__(256) void cache_read_kernel(StoreArgs a) {
  constexpr int LANES = D / 8, ROWS = 256 / LANES;
  const int l = threadIdx.x % LANES;
  const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES;
  const bool exists = row < (int64_t)a.T * a.g.H;
  const int t = exists ? (int)(row / a.g.H) : 0, h = exists ? (int)(row % a.g.H) : 0;
  const int64_t slot = a.slots[t];
  const bool stored = slot >= 0 && slot < ((int64_t)a.g.pages << a.g.page_shift);
  const int c = 8 * l, j = l / 2 % 4;
  const int at = stored ? (int)(slot & (a.g.page() - 1)) : 0, octet = at >> 3, i = at & 7;
  const unsigned char* p = a.pool + (size_t)(stored ? slot >> a.g.page_shift : 0) * a.g.page_bytes() + (size_t)h * a.g.head_bytes();
  const unsigned kw = *(const unsigned*)(p + at * (D / 2) + (l % 4) * (D / 8) + l / 4 * 4);
  const unsigned char* pv = p + a.g.v_codes() + octet * (4 * D) + l / 8 * 256 + (8 * (l % 2) + 2 * j) * 16 + 2 * i;
  const unsigned mine = *(const unsigned short*)pv | (unsigned)*(const unsigned short*)(pv + 16) << 16;
  // half-words m = 2 j', 2 j' + 1 of the lane's eight are with the lane of nibble j'
  unsigned w[4];
#pragma unroll
  for (int k = 0; k < 4; k++) w[k] = (unsigned)__shfl((int)mine, (l & 9) | 2 * k, LANES) >> (4 * j);
  const int sc = (octet * (D / GROUP) + l / (GROUP / 8)) * 16 + 2 * i;
  const float ks = bf16_bits_to_float(*(const unsigned short*)(p + a.g.k_scales() + sc));
  const float vs = bf16_bits_to_float(*(const unsigned short*)(p + a.g.v_scales() + sc));
  if (!exists) return;
  v8bf k, v;
#pragma unroll
  for (int e = 0; e < 8; e++) {
    float x = (float)((int)(kw >> (4 * (e / 2 + 4 * (e % 2))) & 15) - 8) * ks;
    float y = (float)((int)(w[e / 2] >> (16 * (e % 2)) & 15) - 8) * vs;
    if (a.k_mean != nullptr) x += a.k_mean[h * D + c + e];
    if (a.v_mean != nullptr) y += a.v_mean[h * D + c + e];
    k[e] = (__bf16)(stored ? x : 0.f);
    v[e] = (__bf16)(stored ? y : 0.f);
  }
  *(v8bf*)(a.Ko + row * D + c) = k;
  *(v8bf*)(a.Vo + row * D + c) = v;
}

}  // namespace sage
