// The cache held in 8 bits: storing and reading tokens (gfx950 only).  The format of a page and the quantiser are in sagebwd_serve.h.
#pragma once

#include "cache_kernels.h"

namespace sage {

// Where things stand in one head's part of a page: K's codes, V's, the magnitudes.  (CacheGeometry's own functions are those of the 4 bits.)
template <int D>
struct Bytes8 {
  static __host__ __device__ __forceinline__ int magnitudes(const CacheGeometry& g) { return 2 * g.page() * D; }
  static __host__ __device__ __forceinline__ int head_bytes(const CacheGeometry& g) { return 2 * g.page() * D + (g.page() > 64 ? g.page() / 4 : 16); }
  // of 8 tokens (from `octet` on) and channels c and c + 16 (c / 16 even), 16 bytes; of a token and 8 channels from c on, 8 bytes
  static __device__ __forceinline__ int v(const CacheGeometry& g, int octet, int c) {
    return g.page() * D + (octet >> 2) * (32 * D) + (c >> 5) * 1024 + (octet & 3) * 256 + (c & 15) * 16 + (c >> 4 & 1) * 8;
  }
  static __device__ __forceinline__ int k(int t, int c) {
    return (t >> 5) * (32 * D) + (c >> 6) * 2048 + (t >> 2 & 1) * 1024 + (c >> 4 & 3) * 256 + (t >> 3 & 3) * 64 + (t & 3) * 16 + (c & 15);
  }
};

// The largest magnitude of a block as it is stored, from its bits (of an infinity and a NaN the largest).
__device__ __forceinline__ float magnitude8(unsigned top) {
  return __uint_as_float(top < 0x0D800000u ? 0u : top >= 0x7F000000u ? 0x7FC00000u : top);
}
// What turns a block's numbers into codes, and codes held into codes of a larger magnitude.
__device__ __forceinline__ float to_codes8(float a) { return a > 0.f ? __fdiv_rn(127.f, a) : 0.f; }
__device__ __forceinline__ unsigned code8(float x, float r) { return (unsigned)(int)rintf(x * r) & 255u; }
__device__ __forceinline__ unsigned recode8(unsigned w, float f) {      // four of them
  unsigned y = 0;
#pragma unroll
  for (int i = 0; i < 4; i++) y |= ((unsigned)(int)rintf((float)(signed char)(w >> 8 * i) * f) & 255u) << 8 * i;
  return y;
}

// A run is what a call brings of one block: tokens one after the other with slots that rise by one.  Its first row finds it, and one workgroup
// has it for a head: the block's largest magnitude has to be known before the first code is written, and where it grows the codes held are
// written again.  A workgroup looks through `window` rows for first ones.
template <int D>
__global__ __launch_bounds__(256) void cache8_append_kernel(StoreArgs a, int block_shift, int window) {
  constexpr int PIECES = D / 8, MOST = 64 * PIECES / 256;      // 8 channels of a token each, and those of a thread
  __shared__ __attribute__((aligned(16))) unsigned char codes[64][D + 8];
  __shared__ unsigned tops[4][2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h = blockIdx.y;
  const int row0 = blockIdx.x * window;
  const int block = 1 << block_shift;
  const int64_t end = (int64_t)a.g.pages << a.g.page_shift;
  uint64_t firsts;
  {
    const int row = row0 + lane;
    const bool in = lane < window && row < a.T;
    const int64_t slot = in ? a.slots[row] : -1, before = in && row > 0 ? a.slots[row - 1] : -2;
    firsts = __ballot(slot >= 0 && slot < end && (slot - before != 1 || (slot & (block - 1)) == 0));
  }
  for (; firsts != 0; firsts &= firsts - 1) {
    const int first = row0 + __builtin_ctzll(firsts);
    const int64_t slot0 = a.slots[first];
    const int o = (int)(slot0 & (block - 1));
    int n;
    {
      const int64_t row = (int64_t)first + lane;
      const bool in = lane < block - o && row < a.T && a.slots[row] == slot0 + lane;
      const uint64_t others = ~__ballot(in);
      n = others == 0 ? 64 : __builtin_ctzll(others);
    }
    const int at = (int)(slot0 & (a.g.page() - 1)) - o;          // the block's first token in its page
    unsigned char* p = a.pool + ((size_t)(slot0 >> a.g.page_shift) * a.g.H + h) * Bytes8<D>::head_bytes(a.g);
    float* magnitudes = (float*)(p + Bytes8<D>::magnitudes(a.g) + at / 4);
    const float held[2] = {o > 0 ? magnitudes[0] : 0.f, o > 0 ? magnitudes[1] : 0.f};
    v8bf x[2][MOST];
    unsigned top[2] = {0, 0};
    const auto numbers = [&](float* f, int which, int i) {      // of the thread's i-th piece
      const int c = tid % PIECES * 8;
#pragma unroll
      for (int e = 0; e < 8; e++) f[e] = (float)x[which][i][e];
      subtract_mean(f, which == 0 ? a.k_mean : a.v_mean, h * D + c);
    };
#pragma unroll
    for (int i = 0; i < MOST; i++) {
      const int t = tid / PIECES + i * (256 / PIECES), c = tid % PIECES * 8;
      if (t >= n) continue;
      x[0][i] = *(const v8bf*)(a.K + (int64_t)(first + t) * a.ks[0] + h * a.ks[1] + c);
      x[1][i] = *(const v8bf*)(a.V + (int64_t)(first + t) * a.vs[0] + h * a.vs[1] + c);
    }
#pragma unroll
    for (int i = 0; i < MOST; i++) {
      const int t = tid / PIECES + i * (256 / PIECES);
      if (t >= n) continue;
#pragma unroll
      for (int which = 0; which < 2; which++) {
        float f[8];
        numbers(f, which, i);
#pragma unroll
        for (int e = 0; e < 8; e++) top[which] = max(top[which], __float_as_uint(f[e]) & 0x7FFFFFFFu);
      }
    }
#pragma unroll
    for (int which = 0; which < 2; which++) {
#pragma unroll
      for (int k = 1; k < 64; k <<= 1) top[which] = max(top[which], (unsigned)__shfl_xor((int)top[which], k));
      if (lane == 0) tops[wave][which] = top[which];
    }
    __syncthreads();
    float now[2], r[2], again[2];
    bool grown[2];
#pragma unroll
    for (int which = 0; which < 2; which++) {
      unsigned t = max(max(tops[0][which], tops[1][which]), max(tops[2][which], tops[3][which]));
      t = max(t, __float_as_uint(held[which]) & 0x7FFFFFFFu);
      now[which] = magnitude8(t);
      r[which] = to_codes8(now[which]);
      grown[which] = o > 0 && now[which] > held[which];
      again[which] = grown[which] ? __fdiv_rn(held[which], now[which]) : 1.f;
    }
    // new codes: K's to the page, V's to LDS, where 8 tokens of a channel meet
#pragma unroll
    for (int i = 0; i < MOST; i++) {
      const int t = tid / PIECES + i * (256 / PIECES), c = tid % PIECES * 8;
      if (t >= n) continue;
#pragma unroll
      for (int which = 0; which < 2; which++) {
        float f[8];
        numbers(f, which, i);
        uint2 w = {0, 0};
        if (r[which] > 0.f) {
#pragma unroll
          for (int e = 0; e < 4; e++) {
            w.x |= code8(f[e], r[which]) << 8 * e;
            w.y |= code8(f[4 + e], r[which]) << 8 * e;
          }
        }
        if (which == 0) *(uint2*)(p + Bytes8<D>::k(at + o + t, c)) = w;
        else *(uint2*)&codes[o + t][c] = w;
      }
    }
    if (grown[0]) {
      for (int i = tid; i < o * PIECES; i += 256) {
        uint2* q = (uint2*)(p + Bytes8<D>::k(at + i / PIECES, i % PIECES * 8));
        const uint2 w = *q;
        *q = uint2{recode8(w.x, again[0]), recode8(w.y, again[0])};
      }
    }
    __syncthreads();
    {
      const int octet0 = grown[1] ? 0 : o >> 3, octets = ((o + n + 7) >> 3) - octet0;
      for (int i = tid; i < octets * (D / 2); i += 256) {
        const int octet = octet0 + i / (D / 2), q = i % (D / 2), c = q / 16 * 32 + q % 16;
        uint4* to = (uint4*)(p + Bytes8<D>::v(a.g, at / 8 + octet, c));
        const int from = min(max(o - 8 * octet, 0), 8), upto = min(o + n - 8 * octet, 8);      // new tokens of the octet
        uint4 w = {0, 0, 0, 0};
        if (from > 0 || upto < 8) {
          w = *to;
          if (grown[1]) {
            const uint4 y = {recode8(w.x, again[1]), recode8(w.y, again[1]), recode8(w.z, again[1]), recode8(w.w, again[1])};
            // (tokens behind the new ones are not the call's)
            const uint64_t mask = from == 8 ? ~0ull : (1ull << 8 * from) - 1;
            const unsigned lo = (unsigned)mask, hi = (unsigned)(mask >> 32);
            w = uint4{(w.x & ~lo) | (y.x & lo), (w.y & ~hi) | (y.y & hi), (w.z & ~lo) | (y.z & lo), (w.w & ~hi) | (y.w & hi)};
          }
        }
#pragma unroll
        for (int t = 0; t < 8; t++) {
          if (t < from || t >= upto) continue;
          const unsigned mask = 255u << 8 * (t & 3), u = (unsigned)codes[8 * octet + t][c] << 8 * (t & 3),
                         v = (unsigned)codes[8 * octet + t][c + 16] << 8 * (t & 3);
          if (t < 4) {
            w.x = (w.x & ~mask) | u;
            w.z = (w.z & ~mask) | v;
          } else {
            w.y = (w.y & ~mask) | u;
            w.w = (w.w & ~mask) | v;
          }
        }
        *to = w;
      }
    }
    if (tid < block >> 5) *(float2*)(magnitudes + 2 * tid) = float2{now[0], now[1]};
    __syncthreads();
  }
}

// d / 8 lanes have a token of a head, 8 channels each.
template <int D>
__global__ __launch_bounds__(256) void cache8_read_kernel(StoreArgs a) {
  constexpr int LANES = D / 8, ROWS = 256 / LANES;
  const int l = threadIdx.x % LANES, c = 8 * l;
  const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES;
  if (row >= a.T) return;
  const int h = blockIdx.y, t = (int)row;
  const int64_t slot = a.slots[t];
  const bool stored = slot >= 0 && slot < ((int64_t)a.g.pages << a.g.page_shift);
  const int at = stored ? (int)(slot & (a.g.page() - 1)) : 0;
  const unsigned char* p = a.pool + ((size_t)(stored ? slot >> a.g.page_shift : 0) * a.g.H + h) * Bytes8<D>::head_bytes(a.g);
  const uint2 w = *(const uint2*)(p + Bytes8<D>::k(at, c));
  const float2 top = *(const float2*)(p + Bytes8<D>::magnitudes(a.g) + at / 32 * 8);
  const unsigned char* pv = p + Bytes8<D>::v(a.g, at / 8, c) + at % 8;
  const float ks = __fdiv_rn(top.x, 127.f), vs = __fdiv_rn(top.y, 127.f);
  v8bf k, v;
#pragma unroll
  for (int e = 0; e < 8; e++) {
    float x = (float)(signed char)((e < 4 ? w.x : w.y) >> 8 * (e % 4)) * ks;
    float y = (float)(signed char)pv[16 * e] * vs;
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
