// The 4-bit cache beside its attention: where things stand in a page, storing and reading tokens (gfx950 only).
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
