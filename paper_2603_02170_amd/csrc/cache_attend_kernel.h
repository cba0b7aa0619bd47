// Attention over the 4-bit cache for few query rows a request: decoding, drafted tokens (gfx950 only).
//
//   S = q k^T,  k = s_k (n_k - 8);   O = sum_t p_t s_v,t (n_v,t - 8) / sum_t p_t
//
// A nibble n in the top four mantissa bits of a bf16 number of exponent 4 reads as 16 + n, so that an AND and an OR make two operands
// of a matrix instruction, and both products run on these exact numbers.  The 24 that is too much is taken off inside the chains: K's
// start from -24 sum(q), V's have a product with -24 beside each.  K's scales multiply the logits' parts of a group of channels in
// FP32; V's are multiplied into the probabilities, which are rounded to bf16 then (as any probabilities are that meet a matrix
// instruction).
//
// 16 x 16 x 32 products.  A wave has 32 tokens at a time: S^T = K Q^T in two of 16 tokens (rows) by 16 queries (columns), O^T = V^T P^T.
// Row 4 g + i of the two tiles is token 8 g + i and 8 g + 4 + i, so that a lane (column n, g) ends with the logits of the octet of tokens
// 8 g .. 8 g + 7, which is what it has to hold of P^T's operand; nothing moves between lanes but a maximum now and then.
#pragma once

#include "cache_kernels.h"

namespace sage {

struct AttendArgs {
  const __bf16* Q;
  const unsigned char* pool;
  const int32_t *table, *lengths, *cu;
  const float* v_mean;
  __bf16* O;
  float* LSE;
  int32_t* prefix;      // [row tiles, R + 1] units up to a request
  float* sums;          // [row tiles, 2 slots of every workgroup, rows, D]: parts of items that workgroups share
  float2* stats;        // their maximum (log2) and sum
  CacheGeometry g;
  int R, T, Hq, G, columns, max_new, max_length, causal;
  float scale_log2;     // sm_scale * log2(e)
  int64_t q_token, q_head;
  int workgroups;
};

constexpr int kUnit = 128;          // tokens that a workgroup of four waves takes at a time

struct AttendRequest {
  int begin, n, rows, len;          // first row, new tokens, query rows computed of each head, keys
  int first_sees;                   // keys that token 0 sees with the mask (may be negative), else len
};
__device__ __forceinline__ AttendRequest attend_request(const AttendArgs& a, int r) {
  AttendRequest q;
  q.begin = min(max(a.cu[r], 0), a.T);
  q.n = min(max(a.cu[r + 1], q.begin), a.T) - q.begin;
  q.rows = min(q.n, a.max_new) * a.G;
  q.len = min(max(a.lengths[r], 0), a.max_length);
  q.first_sees = a.causal ? q.len - q.n + 1 : q.len;
  return q;
}
// Keys that rows [row0, row0 + count) see at most.
__device__ __forceinline__ int attend_visible(const AttendArgs& a, const AttendRequest& q, int row0, int count) {
  if (!a.causal) return q.len;
  const int last = (min(q.rows, row0 + count) - 1) / a.G;
  return max(0, min(q.len, q.first_sees + last));
}
__device__ __forceinline__ int attend_units(const AttendArgs& a, int r, int row0, int count) {
  const AttendRequest q = attend_request(a, r);
  if (q.rows <= row0) return 0;
  return max(1, (attend_visible(a, q, row0, count) + kUnit - 1) / kUnit);     // (rows without a key are an item too: zeros)
}

// Items are (request, key/value head), request after request, of attend_units units each; workgroup w of n has units
// [w total / n, (w + 1) total / n).
__device__ __forceinline__ int64_t attend_share(int64_t total, int n, int w) { return total * w / n; }

// Two bf16 numbers 16 + n from nibble E of a word's half-words.
template <int E>
__device__ __forceinline__ int nibble_pair(int w) {
  const unsigned u = (unsigned)w;
  return (int)(((E == 0 ? u << 3 : u >> (4 * E - 3)) & 0x00780078u) | 0x41804180u);
}
__device__ __forceinline__ v8bf as_bf16(const v4i& x) {
  v8bf r;
  __builtin_memcpy(&r, &x, 16);
  return r;
}
__device__ __forceinline__ int pack_bf16(float a, float b) {
  typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
  const v2bf p = {(__bf16)a, (__bf16)b};
  int r;
  __builtin_memcpy(&r, &p, 4);
  return r;
}
__device__ __forceinline__ float low_bf16(int w) { return __uint_as_float((unsigned)w << 16); }
__device__ __forceinline__ float high_bf16(int w) { return __uint_as_float((unsigned)w & 0xFFFF0000u); }
// max, sum over the four lanes of a column
__device__ __forceinline__ float column_max(float v) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return half_swap_max_f32(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float column_sum(float v) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return half_swap_sum_f32(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// 32 tokens of a head as a lane (column m, g) takes them.
template <int D, int GROUP>
struct CacheTile {
  int k[2][D / 32];       // token 8 (m / 4) + m % 4 (+ 4), channels of quarter g
  v4i v[D / 64];          // octet g, channels m + 16 j of each half
  v4i ks[D / GROUP], vs[D / GROUP];   // octet g
  bool exists;

  __device__ __forceinline__ void load(const AttendArgs& a, const int32_t* table, int head, int t0) {
    const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const int entry = __builtin_amdgcn_readfirstlane(table[t0 >> a.g.page_shift]);
    exists = (unsigned)entry < (unsigned)a.g.pages;
    const unsigned char* p = a.pool + (size_t)(exists ? entry : 0) * a.g.page_bytes() + (size_t)head * a.g.head_bytes();
    const int at = t0 & (a.g.page() - 1), octet = (at >> 3) + g;
    const unsigned char* pk = p + (at + 8 * (m >> 2) + (m & 3)) * (D / 2) + g * (D / 8);
    if (D == 128) {
      const v4i x = *(const v4i*)pk, y = *(const v4i*)(pk + 4 * (D / 2));
#pragma unroll
      for (int j = 0; j < D / 32; j++) { k[0][j] = x[j]; k[1][j] = y[j]; }
    } else {
      const v2i x = *(const v2i*)pk, y = *(const v2i*)(pk + 4 * (D / 2));
#pragma unroll
      for (int j = 0; j < D / 32; j++) { k[0][j] = x[j]; k[1][j] = y[j]; }
    }
#pragma unroll
    for (int f = 0; f < D / 64; f++) v[f] = *(const v4i*)(p + a.g.v_codes() + octet * (4 * D) + f * 256 + m * 16);
#pragma unroll
    for (int s = 0; s < D / GROUP; s++) {
      ks[s] = *(const v4i*)(p + a.g.k_scales() + (octet * (D / GROUP) + s) * 16);
      vs[s] = *(const v4i*)(p + a.g.v_scales() + (octet * (D / GROUP) + s) * 16);
    }
  }
};

// One tile of 16 queries by what a wave has of an item's keys.
template <int D, int GROUP>
struct AttendRows {
  static constexpr int NG = D / GROUP, NJ = D / 32, NV = D / 16;
  v4i q[NJ];            // B operand: query n, channels 32 j + 8 g ..
  float start[NG];      // -24 sum(q) over a group
  v4f o[NV];            // channel 16 v + 4 g + i of query n
  float m, l;           // reference (log2), this lane's part of the sum
  int sees;             // keys that the query sees

  __device__ __forceinline__ void begin(const AttendArgs& a, const AttendRequest& rq, int head, int row0) {
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int row = row0 + n, i = row / a.G;
    const bool exists = row < rq.rows;
    const __bf16* p = a.Q + (int64_t)(rq.begin + (exists ? i : 0)) * a.q_token + (int64_t)(head * a.G + (exists ? row - i * a.G : 0)) * a.q_head + 8 * g;
#pragma unroll
    for (int s = 0; s < NG; s++) start[s] = 0.f;
#pragma unroll
    for (int j = 0; j < NJ; j++) {
      q[j] = exists ? *(const v4i*)(p + 32 * j) : v4i{0, 0, 0, 0};
      float t = 0.f;
#pragma unroll
      for (int e = 0; e < 4; e++) t += low_bf16(q[j][e]) + high_bf16(q[j][e]);
      start[32 * j / GROUP] += t;
    }
#pragma unroll
    for (int s = 0; s < NG; s++) start[s] = -24.f * column_sum(start[s]);
#pragma unroll
    for (int v = 0; v < NV; v++) o[v] = v4f{0.f, 0.f, 0.f, 0.f};
    m = -INFINITY;
    l = 0.f;
    sees = a.causal ? min(rq.len, rq.first_sees + i) : rq.len;
    if (!exists) sees = rq.len;
  }

  template <bool MASKED>
  __device__ __forceinline__ void add(const CacheTile<D, GROUP>& t, int t0, float scale_log2) {
    const int g = (threadIdx.x & 63) >> 4;
    float s[8];
#pragma unroll
    for (int b = 0; b < 2; b++) {
#pragma unroll
      for (int gr = 0; gr < NG; gr++) {
        v4f c = {start[gr], start[gr], start[gr], start[gr]};
#pragma unroll
        for (int j = gr * GROUP / 32; j < (gr + 1) * GROUP / 32; j++) {
          const int w = t.k[b][j];
          const v4i k = {nibble_pair<0>(w), nibble_pair<1>(w), nibble_pair<2>(w), nibble_pair<3>(w)};
          c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(k), as_bf16(q[j]), c, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 4; i++) {
          const int w = t.ks[gr][2 * b + i / 2];
          const float x = i % 2 == 0 ? low_bf16(w) : high_bf16(w);
          s[4 * b + i] = gr == 0 ? x * c[i] : __builtin_fmaf(x, c[i], s[4 * b + i]);
        }
      }
    }
    const int behind = sees - t0 - 8 * g;        // tokens of the octet that the query sees
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; i++) {
      if (MASKED) s[i] = i < behind ? s[i] : -INFINITY;
      top = fmaxf(top, s[i]);
    }
    // The reference only has to be near the maximum: it is raised where a logit is 2^8 above it (O / l and m + log l do not depend on it).
    if (__any(top * scale_log2 > m + 8.f)) {
      const float to = fmaxf(m, column_max(top) * scale_log2);
      const float f = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - to);
#pragma unroll
      for (int v = 0; v < NV; v++) o[v] *= f;
      l *= f;
      m = to;
    }
    const float ref = m == -INFINITY ? 0.f : m;
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
      p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], scale_log2, -ref));
      l += p[i];
    }
    const int minus24 = (int)0xC1C0C1C0;
    const v8bf less = as_bf16(v4i{minus24, minus24, minus24, minus24});
#pragma unroll
    for (int gr = 0; gr < NG; gr++) {
      v4i pb;
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const int w = t.vs[gr][i];
        float x = p[2 * i] * low_bf16(w), y = p[2 * i + 1] * high_bf16(w);
        if (MASKED) {              // (the scale of a token that is not seen may be anything)
          x = 2 * i < behind ? x : 0.f;
          y = 2 * i + 1 < behind ? y : 0.f;
        }
        pb[i] = pack_bf16(x, y);
      }
      const v8bf pt = as_bf16(pb);
#pragma unroll
      for (int v = gr * GROUP / 16; v < (gr + 1) * GROUP / 16; v++) {
        const v4i& w = t.v[v / 4];
        v4i x;
#pragma unroll
        for (int i = 0; i < 4; i++) x[i] = v % 4 == 0 ? nibble_pair<0>(w[i]) : v % 4 == 1 ? nibble_pair<1>(w[i]) : v % 4 == 2 ? nibble_pair<2>(w[i]) : nibble_pair<3>(w[i]);
        o[v] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(less, pt, o[v], 0, 0, 0);
        o[v] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(x), pt, o[v], 0, 0, 0);
      }
    }
  }
};

// Writes channels c .. c + N - 1 of a finished row.
template <int N>
__device__ __forceinline__ void attend_store(const AttendArgs& a, const AttendRequest& rq, int head, int row, int D, int c, float m, float l, const float* o) {
  const int i = row / a.G, hq = head * a.G + row - i * a.G;
  const int64_t token = rq.begin + i;
  const bool any = !(l == 0.f);
  const float r = any ? 1.f / l : 0.f;
  __bf16* p = a.O + (token * a.Hq + hq) * D + c;
  typedef __bf16 vec __attribute__((ext_vector_type(N)));
  vec x;
#pragma unroll
  for (int k = 0; k < N; k++) x[k] = (__bf16)(any ? o[k] * r + (a.v_mean != nullptr ? a.v_mean[head * D + c + k] : 0.f) : 0.f);
  *(vec*)p = x;
  if (c == 0 && a.LSE != nullptr) a.LSE[(int64_t)hq * a.T + token] = any ? (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : -INFINITY;
}

template <int D, int GROUP, int NQ>
__global__ __launch_bounds__(256, NQ == 4 ? 1 : 2) void cache_attend_kernel(AttendArgs a) {
  constexpr int ROWS = 16 * NQ, PITCH = D + 4, NC = D / 16;
  __shared__ float stage[4][16][PITCH];
  __shared__ float wave_m[4][ROWS], wave_l[4][ROWS];
  __shared__ int64_t wave_units[4];
  __shared__ int found_request;
  __shared__ int64_t found_prefix;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int H = a.g.H, row0 = blockIdx.y * ROWS;

  // units up to every thread's requests (R / 256 each)
  const int per = (a.R + 255) / 256, r0 = min(tid * per, a.R), r1 = min(r0 + per, a.R);
  int64_t mine = 0;
  for (int r = r0; r < r1; r++) mine += attend_units(a, r, row0, ROWS);
  int64_t upto = mine;
  for (int k = 1; k < 64; k <<= 1) {
    const int64_t u = __shfl_up(upto, k);
    if (lane >= k) upto += u;
  }
  if (lane == 63) wave_units[wave] = upto;
  __syncthreads();
  int64_t units = 0;
#pragma unroll
  for (int k = 0; k < 4; k++) {
    if (k < wave) upto += wave_units[k];
    units += wave_units[k];
  }
  const int64_t total = units * H;
  const int n = (int)min((int64_t)a.workgroups, total);
  if (blockIdx.x == 0) {           // for the launch that joins
    int32_t* prefix = a.prefix + (size_t)blockIdx.y * (a.R + 1);
    int64_t at = upto - mine;
    for (int r = r0; r < r1; r++) {
      prefix[r] = (int)at;
      at += attend_units(a, r, row0, ROWS);
    }
    if (tid == 0) prefix[a.R] = (int)units;
  }
  if ((int)blockIdx.x >= n) return;
  int64_t x = attend_share(total, n, blockIdx.x);
  const int64_t end = attend_share(total, n, blockIdx.x + 1);
  if ((upto - mine) * H <= x && x < upto * H) {
    int64_t at = upto - mine;
    for (int r = r0; r < r1; r++) {
      const int u = attend_units(a, r, row0, ROWS);
      if (x < (at + u) * H) {
        found_request = r;
        found_prefix = at;
        break;
      }
      at += u;
    }
  }
  __syncthreads();
  int r = __builtin_amdgcn_readfirstlane(found_request);
  int64_t prefix = found_prefix;

  while (x < end) {
    const int u = __builtin_amdgcn_readfirstlane(attend_units(a, r, row0, ROWS));
    const int64_t rel = x - prefix * H;
    if (rel >= (int64_t)u * H) {    // the next request
      prefix += u;
      r++;
      continue;
    }
    const AttendRequest rq = attend_request(a, r);
    const int head = __builtin_amdgcn_readfirstlane((int)(rel / u)), j0 = __builtin_amdgcn_readfirstlane((int)(rel % u));
    const int j1 = __builtin_amdgcn_readfirstlane((int)min((int64_t)u, j0 + (end - x)));
    x += j1 - j0;
    AttendRows<D, GROUP> rows[NQ];
#pragma unroll
    for (int q = 0; q < NQ; q++) rows[q].begin(a, rq, head, row0 + 16 * q);
    const int visible = attend_visible(a, rq, row0, ROWS);
    const int all_see = a.causal ? rq.first_sees + row0 / a.G : rq.len;       // keys that every row of the tile sees
    const int32_t* table = a.table + (size_t)r * a.columns;
    CacheTile<D, GROUP> tile;
    int t0 = j0 * kUnit + wave * 32;
    if (t0 < visible) tile.load(a, table, head, t0);
    for (int j = j0; j < j1 && t0 < visible; j++, t0 += kUnit) {
      CacheTile<D, GROUP> next;
      const bool more = j + 1 < j1 && t0 + kUnit < visible;
      if (more) next.load(a, table, head, t0 + kUnit);
      if (tile.exists) {
        if (t0 + 32 > all_see) {
#pragma unroll
          for (int q = 0; q < NQ; q++) rows[q].template add<true>(tile, t0, a.scale_log2);
        } else {
#pragma unroll
          for (int q = 0; q < NQ; q++) rows[q].template add<false>(tile, t0, a.scale_log2);
        }
      }
      if (more) tile = next;
    }
    // join the waves
    const bool whole = j0 == 0 && j1 == u;
    const int64_t slot = ((int64_t)blockIdx.y * a.workgroups + blockIdx.x) * 2 + (j0 == 0 ? 1 : 0);
#pragma unroll
    for (int q = 0; q < NQ; q++) {
      const float l = column_sum(rows[q].l);
      if (lane < 16) {
        wave_m[wave][16 * q + lane] = rows[q].m;
        wave_l[wave][16 * q + lane] = l;
      }
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < NQ; q++) {
      {
        const int k = 16 * q + (lane & 15);
        const float M = fmaxf(fmaxf(wave_m[0][k], wave_m[1][k]), fmaxf(wave_m[2][k], wave_m[3][k]));
        const float f = rows[q].m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(rows[q].m - M);
#pragma unroll
        for (int v = 0; v < D / 16; v++) *(v4f*)&stage[wave][lane & 15][16 * v + 4 * (lane >> 4)] = rows[q].o[v] * f;
      }
      __syncthreads();
      const int row = tid / 16, c = (tid % 16) * NC, k = 16 * q + row;
      const float M = fmaxf(fmaxf(wave_m[0][k], wave_m[1][k]), fmaxf(wave_m[2][k], wave_m[3][k]));
      float o[NC], l = 0.f;
#pragma unroll
      for (int i = 0; i < NC; i++) o[i] = (stage[0][row][c + i] + stage[1][row][c + i]) + (stage[2][row][c + i] + stage[3][row][c + i]);
#pragma unroll
      for (int w = 0; w < 4; w++) l += wave_m[w][k] == -INFINITY ? 0.f : wave_l[w][k] * __builtin_amdgcn_exp2f(wave_m[w][k] - M);
      if (row0 + k < rq.rows) {
        if (whole) {
          attend_store<NC>(a, rq, head, row0 + k, D, c, M, l, o);
        } else {
          float* p = a.sums + (slot * ROWS + k) * D + c;
#pragma unroll
          for (int i = 0; i < NC; i++) p[i] = o[i];
          if (c == 0) a.stats[slot * ROWS + k] = float2{M, l};
        }
      }
      __syncthreads();
    }
  }
}

// Items that several workgroups had parts of.  Workgroup (w, rows) looks at the border in front of workgroup w's share and joins the item
// that it divides, if it is the first border to do so: the parts in the order of the keys.  A wave has a row.
template <int D, int NQ>
__global__ __launch_bounds__(256) void cache_join_kernel(AttendArgs a) {
  constexpr int ROWS = 16 * NQ, NC = D / 64;
  const int32_t* prefix = a.prefix + (size_t)blockIdx.z * (a.R + 1);
  const int H = a.g.H;
  const int64_t total = (int64_t)prefix[a.R] * H;
  const int n = (int)min((int64_t)a.workgroups, total), w = blockIdx.x + 1;
  if (w >= n) return;
  const int64_t border = attend_share(total, n, w);
  int r = 0;
  for (int hi = a.R; hi - r > 1;) {
    const int mid = (r + hi) >> 1;
    if ((int64_t)prefix[mid] * H <= border) r = mid;
    else hi = mid;
  }
  const int u = prefix[r + 1] - prefix[r];
  const int64_t rel = border - (int64_t)prefix[r] * H;
  const int head = (int)(rel / u);
  const int64_t first = border - rel % u, last = first + u;
  if (first == border || attend_share(total, n, w - 1) > first) return;
  const AttendRequest rq = attend_request(a, r);
  const int lane = threadIdx.x & 63, k = blockIdx.y * 4 + (threadIdx.x >> 6), row = blockIdx.z * ROWS + k;
  if (row >= rq.rows) return;
  const int64_t slot0 = ((int64_t)blockIdx.z * a.workgroups + w) * 2;
  float M = a.stats[(slot0 - 1) * ROWS + k].x;
  int parts = 1;
  for (; attend_share(total, n, w + parts - 1) < last; parts++) M = fmaxf(M, a.stats[(slot0 + 2 * (parts - 1)) * ROWS + k].x);
  float o[NC], l = 0.f;
#pragma unroll
  for (int i = 0; i < NC; i++) o[i] = 0.f;
  for (int p = 0; p < parts; p++) {
    const int64_t at = (p == 0 ? slot0 - 1 : slot0 + 2 * (p - 1)) * ROWS + k;
    const float2 s = a.stats[at];
    const float f = s.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s.x - M);
    l += s.y * f;
#pragma unroll
    for (int i = 0; i < NC; i++) o[i] += a.sums[at * D + NC * lane + i] * f;
  }
  attend_store<NC>(a, rq, head, row, D, NC * lane, M, l, o);
}

}  // namespace sage
