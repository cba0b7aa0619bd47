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
// Inclusive sums over the threads of a workgroup of WAVES waves, N of them at once, that stop at kFull (sizes that are not valid are taken out
// before, but many valid ones may sum to more than 32 bits hold; what they are compared with is less).
constexpr unsigned kFull = 0x7FFFFFFFu;
template <int WAVES, int N>
__device__ __forceinline__ void block_scan(unsigned (&v)[N], unsigned (*wave_sums)[N]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
#pragma unroll
    for (int i = 0; i < N; i++) {
      const unsigned u = __shfl_up(v[i], k);
      if (lane >= k) v[i] = min(v[i] + u, kFull);
    }
  }
  if (WAVES == 1) return;
  __syncthreads();
  if (lane == 63) {
#pragma unroll
    for (int i = 0; i < N; i++) wave_sums[wave][i] = v[i];
  }
  __syncthreads();
  for (int k = 0; k < wave; k++) {
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = min(v[i] + wave_sums[k][i], kFull);
  }
}

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

__device__ __forceinline__ void subtract_mean(float* x, const float* mean, int at) {
  typedef v4f v4f_dword __attribute__((aligned(4)));
  if (mean == nullptr) return;
  const v4f a = *(const v4f_dword*)(mean + at), b = *(const v4f_dword*)(mean + at + 4);
#pragma unroll
  for (int i = 0; i < 8; i++) x[i] -= i < 4 ? a[i & 3] : b[i & 3];
}

// d / 8 lanes have a token of a head, 8 channels each.  A lane's channels of K are one word; of V they lie in eight half-words, whose
// other nibbles three lanes of the same half have (2, 4 and 6 away): those are joined and each lane stores two.  Neighbouring rows are
// neighbouring tokens, whose bytes of V are neighbours: in the L2 they meet (8191 tokens of 8 heads of 128: 10.4 us, 4.1 TB/s, 12.4 where a row was found by a division; with the heads of
// a token as neighbours 15.6).
template <int D, int GROUP>
__global__ __launch_bounds__(256) void cache_append_kernel(StoreArgs a) {
  constexpr int LANES = D / 8, ROWS = 256 / LANES;
  const int l = threadIdx.x % LANES;
  const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES;
  const bool exists = row < a.T;
  const int h = blockIdx.y, t = exists ? (int)row : 0;
  const int64_t slot = a.slots[t];
  const bool stored = exists && slot >= 0 && slot < ((int64_t)a.g.pages << a.g.page_shift);
  const int c = 8 * l;
  float k[8], v[8];
  {
    const v8bf x = *(const v8bf*)(a.K + t * a.ks[0] + h * a.ks[1] + c), y = *(const v8bf*)(a.V + t * a.vs[0] + h * a.vs[1] + c);
#pragma unroll
    for (int i = 0; i < 8; i++) {
      k[i] = (float)x[i];
      v[i] = (float)y[i];
    }
    subtract_mean(k, a.k_mean, h * D + c);
    subtract_mean(v, a.v_mean, h * D + c);
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
  const bool exists = row < a.T;
  const int h = blockIdx.y, t = exists ? (int)row : 0;
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
  const size_t to = ((size_t)t * a.g.H + h) * D + c;
  *(v8bf*)(a.Ko + to) = k;
  *(v8bf*)(a.Vo + to) = v;
}

}  // namespace sage
