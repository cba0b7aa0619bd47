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
#include "cache_shares.h"

namespace sage {

struct WideTile;
struct AttendArgs {
  const __bf16* Q;
  const unsigned char* pool;
  const int32_t *table, *lengths, *cu;
  const float* v_mean;
  __bf16* O;
  float* LSE;
  int4* joins;          // of every workgroup, of the item that its first unit divides: parts (or 0) and 2^16 rows, first row of Q, head, first query row
  float* sums;          // [2 slots of every workgroup, rows, D]: parts of items that workgroups share
  float2* stats;        // their maximum (log2) and sum
  char* unpacked;       // where keys and values are unpacked beforehand: fragments of 64 tokens of a head,
  WideTile* tiles;   // what is to be known of each,
  unsigned char* poison;    // and tokens that are not numbers
  int most_tiles;           // that there is room for
  CacheGeometry g;
  int R, T, Hq, G, columns, max_new, max_length, causal;
  float scale_log2;     // sm_scale * log2(e)
  int64_t q_token, q_head;
  int workgroups;
  int split;            // 1: an item's units may go to several workgroups
  int rows_from, rows_to;   // the launch has the requests of rows_from < rows (new tokens times G) <= rows_to
};

constexpr int kUnit = 128;          // tokens that a workgroup of four waves takes at a time
__device__ __forceinline__ int attend_cut(int offset) { return cut_at<kItemCost>(offset); }

struct AttendRequest {
  int begin, n, rows, len;          // first row, new tokens, query rows computed of each head, keys
  int first_sees;                   // keys that token 0 sees with the mask (may be negative), else len
};
__device__ __forceinline__ AttendRequest attend_request(const AttendArgs& a, int r) {
  AttendRequest q;
  q.begin = min(max(a.cu[r], 0), a.T);
  q.n = min(max(a.cu[r + 1], q.begin), a.T) - q.begin;
  q.rows = min(q.n, a.max_new) * a.G;
  if (q.rows <= a.rows_from || q.rows > a.rows_to) q.rows = 0;
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
__device__ __forceinline__ int attend_units(const AttendArgs& a, int r) {
  const AttendRequest q = attend_request(a, r);
  return q.rows == 0 ? 0 : max(1, (attend_visible(a, q, 0, q.rows) + kUnit - 1) / kUnit);     // (rows without a key are an item too: zeros)
}

__device__ __forceinline__ float wave_max_f32(float v) {
  for (int k = 1; k < 64; k <<= 1) v = fmaxf(v, __shfl_xor(v, k));
  return v;
}

// Two bf16 numbers 16 + n from nibble E of a word's half-words.  The AND and the OR are one instruction if the compiler does not see that
// their constants are constants (two literals fit none), hence a register of each kind that it knows nothing about.
struct Unpack {
  int mask, sixteens;
  __device__ __forceinline__ Unpack() : mask(0x00780078), sixteens(0x41804180) {
    asm("" : "+s"(mask));
    asm("" : "+v"(sixteens));
  }
  template <int E>
  __device__ __forceinline__ int pair(int w) const {
    const unsigned u = (unsigned)w;
    return (int)((E == 0 ? u << 3 : u >> (4 * E - 3)) & (unsigned)mask) | sixteens;
  }
};
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
// copy_16 and copy_4 of a ring whose reads are counted by hand.  Behind the builtin the compiler lets every read of LDS wait for every copy in
// flight, as it cannot tell a ring's slots apart, so that a ring is one tile deep; of this it sees no access, only that memory changes: what
// is read has to have been waited for (vmcnt_only), and its own waits for loads come out early at worst.  (The copies have no register for a
// result; m0 is reserved to the compiler, which does not honour a clobber of it: nothing else of a kernel with these may use it, and the tests look.  Wait
// states: of m0, and of a base that a vector instruction wrote.)
template <int BYTES>
__device__ __forceinline__ void ring_copy(gbytes_t base, unsigned lane_offset, const void* lds_base) {
  const unsigned to = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(lptr_t)lds_base);
  if (BYTES == 16) asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(lane_offset), "s"(base), "s"(to) : "memory");
  else asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tglobal_load_lds_dword %0, %1" ::"v"(lane_offset), "s"(base), "s"(to) : "memory");
}
// Waits here for a load, once, and not wherever its result is used: a use that some path reaches with the load under way waits for everything in
// flight on every path, copies to LDS that were meant to stay there included.
template <typename T>
__device__ __forceinline__ void arrived(T& x) { asm volatile("" : "+v"(x)); }
// max, sum over the four lanes of a column
__device__ __forceinline__ float column_max(float v) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return half_swap_max_f32(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float column_sum(float v) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return half_swap_sum_f32(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// 32 tokens of a head.  They come past the registers into a ring of the wave's own in LDS (K's codes, V's, the scales, as they lie in
// the page), two tiles ahead; a lane (column m, g) then takes its operands.  (In registers one tile ahead was all that fitted, and
// the 16 lanes of a group each fetched the same scales: the launch of 64 requests took 61 us, then 53.)
template <int D, int GROUP>
struct CacheTile {
  static constexpr int NG = D / GROUP, CODES = 16 * D, SCALES = 64 * NG, SLOT = 2 * CODES + (2 * SCALES > 256 ? 2 * SCALES : 256);
  static constexpr int COPIES = 2 * CODES / 1024 + (NG == 4 ? 2 : 1);

  v4i v[D / 64];          // octet g, channels m + 16 j of each half
  int k[2][D / 32];       // token 8 (m / 4) + m % 4 (+ 4), channels of quarter g
  v4i ks[NG], vs[NG];     // octet g

  // Starts the copies of the 32 tokens from `at` of a page; `p` is the head's part of it.
  static __device__ __forceinline__ void fetch(const CacheGeometry& geo, const unsigned char* p, int at, char* slot) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int c = 0; c < CODES / 1024; c++) {
      ring_copy<16>(uniform(p + at * (D / 2) + c * 1024), lane * 16, slot + c * 1024);
      ring_copy<16>(uniform(p + geo.v_codes() + at * (D / 2) + c * 1024), lane * 16, slot + CODES + c * 1024);
    }
    const gbytes_t ps = uniform(p + geo.k_scales() + at * (2 * NG));
    const int apart = geo.v_scales() - geo.k_scales();
    if (NG == 4) {
      ring_copy<4>(ps, lane * 4, slot + 2 * CODES);
      ring_copy<4>(ps, apart + lane * 4, slot + 2 * CODES + SCALES);
    } else {
      const int l = lane % (32 * NG);        // (with one group the upper half of the lanes copies the same to where nothing is read)
      ring_copy<4>(ps, l < 16 * NG ? 4 * l : apart + 4 * l - SCALES, slot + 2 * CODES);
    }
  }
  __device__ __forceinline__ void take(const char* slot) {
    const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const char* pk = slot + (8 * (m >> 2) + (m & 3)) * (D / 2) + g * (D / 8);
#pragma unroll
    for (int b = 0; b < 2; b++) {
      if (D == 128) {
        const v4i x = *(const v4i*)(pk + b * 4 * (D / 2));
#pragma unroll
        for (int j = 0; j < D / 32; j++) k[b][j] = x[j];
      } else {
        const v2i x = *(const v2i*)(pk + b * 4 * (D / 2));
#pragma unroll
        for (int j = 0; j < D / 32; j++) k[b][j] = x[j];
      }
    }
#pragma unroll
    for (int f = 0; f < D / 64; f++) v[f] = *(const v4i*)(slot + CODES + g * (4 * D) + f * 256 + m * 16);
#pragma unroll
    for (int s = 0; s < NG; s++) {
      ks[s] = *(const v4i*)(slot + 2 * CODES + (g * NG + s) * 16);
      vs[s] = *(const v4i*)(slot + 2 * CODES + SCALES + (g * NG + s) * 16);
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

  int row, token, head_of;   // the lane's query row: new token, head of the group

  __device__ __forceinline__ void place(const AttendArgs& a, int row0) {
    row = row0 + (threadIdx.x & 15);
    token = row / a.G;
    head_of = row - token * a.G;
  }
  template <typename Piece>
  __device__ __forceinline__ void fetch(const AttendArgs& a, const Piece& p) {
    const int g = (threadIdx.x & 63) >> 4;
    const bool exists = row < p.n_rows;
    const __bf16* x = a.Q + (int64_t)(p.begin + (exists ? token : 0)) * a.q_token + (int64_t)(p.head * a.G + (exists ? head_of : 0)) * a.q_head + 8 * g;
#pragma unroll
    for (int j = 0; j < NJ; j++) q[j] = exists ? *(const v4i*)(x + 32 * j) : v4i{0, 0, 0, 0};
    sees = exists && a.causal ? min(p.len, p.first_sees + token) : p.len;
  }
  __device__ __forceinline__ void begin() {
#pragma unroll
    for (int s = 0; s < NG; s++) start[s] = 0.f;
#pragma unroll
    for (int j = 0; j < NJ; j++) {
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
  }
};

// 32 tokens into NQ tiles of queries.  `masked`: some row does not see all of them.
template <int D, int GROUP, int NQ>
__device__ __forceinline__ void attend_tile(AttendRows<D, GROUP> (&rows)[NQ], CacheTile<D, GROUP>& t, int t0, bool masked, float scale_log2, const Unpack& un) {
  constexpr int NG = D / GROUP;
  const int g = (threadIdx.x & 63) >> 4;
  float s[NQ][8];
#pragma unroll
  for (int b = 0; b < 2; b++) {
#pragma unroll
    for (int gr = 0; gr < NG; gr++) {
      v4f c[NQ];
#pragma unroll
      for (int q = 0; q < NQ; q++) c[q] = v4f{rows[q].start[gr], rows[q].start[gr], rows[q].start[gr], rows[q].start[gr]};
#pragma unroll
      for (int j = gr * GROUP / 32; j < (gr + 1) * GROUP / 32; j++) {
        const int w = t.k[b][j];
        const v8bf k = as_bf16(v4i{un.pair<0>(w), un.pair<1>(w), un.pair<2>(w), un.pair<3>(w)});
#pragma unroll
        for (int q = 0; q < NQ; q++) c[q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, as_bf16(rows[q].q[j]), c[q], 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const int w = t.ks[gr][2 * b + i / 2];
        const float x = i % 2 == 0 ? low_bf16(w) : high_bf16(w);
#pragma unroll
        for (int q = 0; q < NQ; q++) s[q][4 * b + i] = gr == 0 ? x * c[q][i] : __builtin_fmaf(x, c[q][i], s[q][4 * b + i]);
      }
    }
  }
  __builtin_amdgcn_sched_barrier(0);           // (left to itself the compiler unpacks everything first, which the registers do not hold)
  int seen[NQ][4];
#pragma unroll
  for (int q = 0; q < NQ; q++) {
    AttendRows<D, GROUP>& R = rows[q];
    // of the octet's scales of V: one that is not seen may be anything
#pragma unroll
    for (int i = 0; i < 4; i++) seen[q][i] = -1;
    if (masked) {
      asm volatile("");                          // (stays a branch: as selects it is a tenth of the tile's instructions)
      const int behind = R.sees - t0 - 8 * g;    // tokens of the octet that the query sees
#pragma unroll
      for (int i = 0; i < 8; i++) s[q][i] = i < behind ? s[q][i] : -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; i++) seen[q][i] = (2 * i < behind ? 0xFFFF : 0) | (2 * i + 1 < behind ? (int)0xFFFF0000 : 0);
    }
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; i++) top = fmaxf(top, s[q][i]);
    // The reference only has to be near the maximum: it is raised where a logit is 2^8 above it (O / l and m + log l do not depend on it).
    if (__any(top * scale_log2 > R.m + 8.f)) {
      const float to = fmaxf(R.m, column_max(top) * scale_log2);
      const float f = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(R.m - to);
#pragma unroll
      for (int v = 0; v < D / 16; v++) R.o[v] *= f;
      R.l *= f;
      R.m = to;
    }
    const float ref = R.m == -INFINITY ? 0.f : R.m;
#pragma unroll
    for (int i = 0; i < 8; i++) {
      s[q][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[q][i], scale_log2, -ref));
      R.l += s[q][i];
    }
  }
  const int minus24 = (int)0xC1C0C1C0;
  const v8bf less = as_bf16(v4i{minus24, minus24, minus24, minus24});
#pragma unroll
  for (int gr = 0; gr < NG; gr++) {
    __builtin_amdgcn_sched_barrier(0);
    v8bf pt[NQ];
#pragma unroll
    for (int q = 0; q < NQ; q++) {
      v4i pb;
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const int w = t.vs[gr][i] & seen[q][i];
        pb[i] = pack_bf16(s[q][2 * i] * low_bf16(w), s[q][2 * i + 1] * high_bf16(w));
      }
      pt[q] = as_bf16(pb);
    }
#pragma unroll
    for (int v = gr * GROUP / 16; v < (gr + 1) * GROUP / 16; v++) {
      const v4i& w = t.v[v / 4];
      v4i x;
#pragma unroll
      for (int i = 0; i < 4; i++)
        x[i] = v % 4 == 0 ? un.pair<0>(w[i]) : v % 4 == 1 ? un.pair<1>(w[i]) : v % 4 == 2 ? un.pair<2>(w[i]) : un.pair<3>(w[i]);
#pragma unroll
      for (int q = 0; q < NQ; q++) {
        rows[q].o[v] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(less, pt[q], rows[q].o[v], 0, 0, 0);
        rows[q].o[v] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(x), pt[q], rows[q].o[v], 0, 0, 0);
      }
    }
  }
  __builtin_amdgcn_sched_barrier(0);
}

// V's means of N channels from `at` on, which a finished row gets back.
template <int N>
__device__ __forceinline__ auto value_means(const AttendArgs& a, int at) {
  typedef float vec __attribute__((ext_vector_type(N)));
  typedef vec vec_dword __attribute__((aligned(4)));
  vec mean = {};
  if (a.v_mean != nullptr) mean = *(const vec_dword*)(a.v_mean + at);
  return mean;
}
// Writes channels c .. c + N - 1 of a finished row.
template <int N, typename Mean>
__device__ __forceinline__ void attend_store(const AttendArgs& a, int begin, int head, int row, int D, int c, float m, float l, const float* o, const Mean& mean) {
  const int i = row / a.G, hq = head * a.G + row - i * a.G;
  const int64_t token = begin + i;
  const bool any = !(l == 0.f);
  const float r = any ? 1.f / l : 0.f;
  __bf16* p = a.O + (token * a.Hq + hq) * D + c;
  typedef __bf16 vec __attribute__((ext_vector_type(N)));
  vec x;
#pragma unroll
  for (int k = 0; k < N; k++) x[k] = (__bf16)(any ? o[k] * r + mean[k] : 0.f);
  *(vec*)p = x;
  if (c == 0 && a.LSE != nullptr) a.LSE[(int64_t)hq * a.T + token] = any ? (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : -INFINITY;
}

constexpr int kStages = 3;          // tiles of a wave's ring

// What a workgroup does with one item: units j0 .. j1 - 1 of the u of (request, head).  All of it is the same in every lane.
struct AttendPiece {
  int r, head, j0, j1, u;
  int begin, n_rows, len, first_sees, visible;
};

constexpr int kKnown = 256;
// 64 requests at a time, one a lane: where one ends the next one's sizes are at hand.
struct AttendCursor {
  int base;                                                // request of lane 0
  int begin, n_rows, len, first_sees, visible, units;      // of request base + lane
  int r, head, j;                                          // the next piece begins here: request, head, unit
  int (*known)[kKnown];                                    // the same of all requests in LDS, if they are few
  int x, end;                                              // where its item begins in what is dealt out, and where the share ends
  __device__ __forceinline__ bool more(const AttendArgs& a) const { return a.split ? attend_cut(end - x) > j : x < end; }

  __device__ __forceinline__ void take(const AttendArgs& a, const AttendRequest& q) {
    begin = q.begin;
    n_rows = q.rows;
    len = q.len;
    first_sees = q.first_sees;
    visible = q.rows > 0 ? attend_visible(a, q, 0, q.rows) : 0;
    units = q.rows > 0 ? max(1, (visible + kUnit - 1) / kUnit) : 0;
  }
  __device__ __forceinline__ void look(const AttendArgs& a, int from) {
    base = from;
    const int i = min(from + (int)(threadIdx.x & 63), a.R - 1);
    if (a.R <= kKnown) {
      begin = known[0][i];
      n_rows = known[1][i];
      len = known[2][i];
      first_sees = known[3][i];
      visible = known[4][i];
      units = known[5][i];
    } else {
      take(a, attend_request(a, i));
    }
  }
  // (more)
  __device__ __forceinline__ AttendPiece next(const AttendArgs& a) {
    AttendPiece p;
    int at;
    do {
      if (r >= base + 64) look(a, r);
      at = r - base;
      p.u = __builtin_amdgcn_readlane(units, at);
      if (p.u == 0) r++;
    } while (p.u == 0);
    p.r = r;
    p.head = head;
    p.begin = __builtin_amdgcn_readlane(begin, at);
    p.n_rows = __builtin_amdgcn_readlane(n_rows, at);
    p.len = __builtin_amdgcn_readlane(len, at);
    p.first_sees = __builtin_amdgcn_readlane(first_sees, at);
    p.visible = __builtin_amdgcn_readlane(visible, at);
    p.j0 = j;
    p.j1 = a.split ? min(p.u, attend_cut(end - x)) : p.u;
    j = p.j1;
    if (j == p.u) {
      x += a.split ? p.u + kItemCost : 1;
      j = 0;
      if (++head == a.g.H) {
        head = 0;
        r++;
      }
    }
    return p;
  }
};

template <int D, int GROUP, int NQ>
__global__ __launch_bounds__(256, 2) void cache_attend_kernel(AttendArgs a) {
  typedef CacheTile<D, GROUP> Tile;
  constexpr int ROWS = 16 * NQ, PITCH = 64 + 4, RING = kStages * Tile::SLOT;
  __shared__ __attribute__((aligned(16))) char lds[4 * RING];          // the ring of every wave
  __shared__ __attribute__((aligned(16))) float stage[4][16][PITCH];   // their sums for 16 rows and 64 channels
  __shared__ float wave_m[4][ROWS], wave_l[4][ROWS];
  __shared__ int wave_units[4], found[2], known[6][kKnown];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int H = a.g.H;
  char* ring = lds + wave * RING;
  const Unpack un;
  const auto shared_units = [&](int u) { return u == 0 ? 0 : a.split ? u + kItemCost : 1; };      // what is dealt out of an item

  // units up to every thread's requests (R / 256 each; where that is one it is kept)
  const int per = (a.R + 255) / 256, r0 = min(tid * per, a.R), r1 = min(r0 + per, a.R);
  AttendCursor cursor;
  cursor.known = known;
  int mine = 0;
  if (a.R <= kKnown) {
    if (tid < a.R) {
      cursor.take(a, attend_request(a, tid));
      const int x[6] = {cursor.begin, cursor.n_rows, cursor.len, cursor.first_sees, cursor.visible, cursor.units};
#pragma unroll
      for (int i = 0; i < 6; i++) known[i][tid] = x[i];
      mine = shared_units(cursor.units);
    }
  } else {
    for (int r = r0; r < r1; r++) mine += shared_units(attend_units(a, r));
  }
  int upto = mine;
  for (int k = 1; k < 64; k <<= 1) {
    const int u = __shfl_up(upto, k);
    if (lane >= k) upto += u;
  }
  if (lane == 63) wave_units[wave] = upto;
  __syncthreads();
  int units = 0;
#pragma unroll
  for (int k = 0; k < 4; k++) {
    if (k < wave) upto += wave_units[k];
    units += wave_units[k];
  }
  const AttendShares shares(__builtin_amdgcn_readfirstlane(units) * H, a.workgroups);
  const int w = blockIdx.x;
  if (a.split && tid == 0) a.joins[w] = int4{0, 0, 0, 0};
  if (w >= shares.n) return;
  const int begin = shares.begin(w);
  if ((upto - mine) * H <= begin && begin < upto * H) {
    int at = upto - mine;
    for (int r = r0; r < r1; r++) {
      const int u = shared_units(a.R <= kKnown ? known[5][r] : attend_units(a, r));
      if (begin < (at + u) * H) {
        found[0] = r;
        found[1] = begin - at * H;
        break;
      }
      at += u;
    }
  }
  __syncthreads();
  cursor.r = __builtin_amdgcn_readfirstlane(found[0]);
  cursor.look(a, cursor.r);
  {
    const int rel = __builtin_amdgcn_readfirstlane(found[1]), u = a.split ? __builtin_amdgcn_readlane(cursor.units, 0) + kItemCost : 1;
    cursor.head = rel / u;
    cursor.j = attend_cut(rel - cursor.head * u);
    cursor.x = begin - (rel - cursor.head * u);
    cursor.end = shares.begin(w + 1);
  }
  if (!cursor.more(a)) return;
  if (tid == 0 && shares.first_border<kItemCost>(w, cursor.x, cursor.j))
    a.joins[w] = join_word(shares.parts<kItemCost>(w, cursor.x, __builtin_amdgcn_readlane(cursor.units, 0)),
                           __builtin_amdgcn_readlane(cursor.n_rows, 0), __builtin_amdgcn_readlane(cursor.begin, 0), cursor.head, 0);

  AttendRows<D, GROUP> rows[NQ];
#pragma unroll
  for (int q = 0; q < NQ; q++) rows[q].place(a, 16 * q);
  AttendPiece piece = cursor.next(a);
  // The wave's tiles: `count`, every 128 tokens from `first`.  Those of pages that do not exist are passed over where tiles are chosen.  (A branch
  // round a tile's arithmetic has the sums in other registers behind it, 48.4 us for 64 ragged requests in place of 47.5; their arithmetic
  // under a mask takes as long as that of any other: 64 requests of 8192 tokens of which an eighth is left 94, so 21.)
  int first, count;
  int pages, window;          // a lane has the page of one of 64 tiles, from `window` on: a tile's address then waits for no load
  uint64_t left;              // those of them that exist and are not on their way yet
  int on_way, to, t0[kStages] = {};      // tiles on their way into the ring, where the next one goes, their first tokens
  const auto pages_from = [&](int k) {
    return a.table[(size_t)piece.r * a.columns + (min(first + (k + lane) * kUnit, max(piece.visible - 1, 0)) >> a.g.page_shift)];
  };
  const auto take_pages = [&] {
    arrived(pages);
    left = __ballot(window + lane < count && (unsigned)pages < (unsigned)a.g.pages);
  };
  const auto look = [&] {      // loads what the piece's copies wait for, and its queries
    first = piece.j0 * kUnit + wave * 32;
    count = max(0, min(piece.j1 - piece.j0, (piece.visible - first + kUnit - 1) / kUnit));
    window = 0;
    pages = pages_from(0);
#pragma unroll
    for (int q = 0; q < NQ; q++) rows[q].fetch(a, piece);
  };
  const auto fetch = [&] {      // the next tile's copies, if there is one
    while (left == 0) {
      window += 64;
      if (window >= count) return;
      pages = pages_from(window);
      take_pages();
    }
    const int i = __builtin_ctzll(left), k = window + i, entry = __builtin_amdgcn_readlane(pages, i);
    left &= left - 1;
    const unsigned char* p = a.pool + (size_t)entry * a.g.page_bytes() + (size_t)(piece.head * a.g.head_bytes());
    Tile::fetch(a.g, p, (first + k * kUnit) & (a.g.page() - 1), ring + to * Tile::SLOT);
    to = to == kStages - 1 ? 0 : to + 1;
#pragma unroll
    for (int q = 0; q < kStages; q++) t0[q] = q == on_way ? first + k * kUnit : t0[q];
    on_way++;
  };
  const auto start = [&] {
    take_pages();
#pragma unroll
    for (int q = 0; q < NQ; q++)
#pragma unroll
      for (int j = 0; j < D / 32; j++) arrived(rows[q].q[j]);
    on_way = to = 0;
#pragma unroll 1
    for (int k = 0; k < kStages - 1; k++) fetch();       // (one copy of the code: of 4 short requests it is 3 % of the call)
  };
  look();
  start();

  for (;;) {
    const int all_see = a.causal ? piece.first_sees : piece.len;       // keys that every row sees
#pragma unroll
    for (int q = 0; q < NQ; q++) rows[q].begin();
    for (int slot = 0; on_way > 0; slot = slot == kStages - 1 ? 0 : slot + 1) {
      compiler_fence();
      fetch();
      compiler_fence();
      if (on_way >= 3) __builtin_amdgcn_s_waitcnt(vmcnt_only(2 * Tile::COPIES));
      else if (on_way == 2) __builtin_amdgcn_s_waitcnt(vmcnt_only(Tile::COPIES));
      else __builtin_amdgcn_s_waitcnt(vmcnt_only(0));
      compiler_fence();
      Tile tile;
      tile.take(ring + slot * Tile::SLOT);
      attend_tile<D, GROUP, NQ>(rows, tile, t0[0], t0[0] + 32 > all_see, a.scale_log2, un);
      on_way--;
#pragma unroll
      for (int q = 1; q < kStages; q++) t0[q - 1] = t0[q];
    }
    // Join the waves; the next piece's loads and first copies are on their way meanwhile.
    const AttendPiece done = piece;
    v4f mean[D / 64];             // (asked for in front of the next piece's copies, which a load behind them would wait for)
#pragma unroll
    for (int h = 0; h < D / 64; h++) mean[h] = value_means<4>(a, done.head * D + 64 * h + tid % 16 * 4);
    const bool more = cursor.more(a);
    if (more) {
      piece = cursor.next(a);
      look();
    } else {
      count = 0;
    }
    const bool whole = done.j0 == 0 && done.j1 == done.u;
    const size_t part = (size_t)w * 2 + (done.j0 == 0 ? 1 : 0);
    barrier_lds_only();           // (the sums of the piece before are read)
#pragma unroll
    for (int q = 0; q < NQ; q++) {
      const float l = column_sum(rows[q].l);
      if (lane < 16) {
        wave_m[wave][16 * q + lane] = rows[q].m;
        wave_l[wave][16 * q + lane] = l;
      }
    }
#pragma unroll
    for (int q = 0; q < NQ; q++) {
      const int row = tid / 16, c = tid % 16 * 4, k = 16 * q + row;
      float M = 0.f, f[4], l = 0.f;
#pragma unroll
      for (int half = 0; half < D / 64; half++) {
        if (q + half > 0) barrier_lds_only();
#pragma unroll
        for (int v = 0; v < 4; v++) *(v4f*)&stage[wave][lane & 15][16 * v + 4 * (lane >> 4)] = rows[q].o[4 * half + v];
        if (q + half == 0) {
#pragma unroll
          for (int h = 0; h < D / 64; h++) arrived(mean[h]);
          start();
        }
        barrier_lds_only();
        if (half == 0) {
          M = fmaxf(fmaxf(wave_m[0][k], wave_m[1][k]), fmaxf(wave_m[2][k], wave_m[3][k]));
#pragma unroll
          for (int w = 0; w < 4; w++) {
            f[w] = wave_m[w][k] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(wave_m[w][k] - M);
            l += wave_l[w][k] * f[w];
          }
        }
        v4f o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; w++) o += *(const v4f*)&stage[w][row][c] * f[w];
        if (k < done.n_rows) {
          const int channel = 64 * half + c;
          if (whole) {
            attend_store<4>(a, done.begin, done.head, k, D, channel, M, l, (const float*)&o, mean[half]);
          } else {
            *(v4f*)(a.sums + (part * ROWS + k) * D + channel) = o;
            if (channel == 0) a.stats[part * ROWS + k] = float2{M, l};
          }
        }
      }
    }
    if (!more) break;
  }
}

// Joins the parts of an item that several workgroups had, in the order of the keys: the workgroup at the first border inside it has left word
// (AttendArgs::joins).  Of few rows, with many parts: a workgroup has a row, every lane weighs a part, then each wave takes every fourth part,
// several loads in flight, and they meet in LDS (one wave and one part after the other took 97 us for the 128 parts of a request alone, now 7).
template <int D, int ROWS>
__global__ __launch_bounds__(256) void cache_join_kernel(AttendArgs a) {
  constexpr int NC = D / 64, MOST = 256;
  const int w = blockIdx.x + 1, k = blockIdx.y;
  const int4 join = a.joins[w];
  const int parts = join.x & 0xFFFF;
  if (k >= join.x >> 16) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const auto mean = value_means<NC>(a, join.z * D + NC * lane);
  const size_t slot0 = (size_t)w * 2;
  const auto at = [&](int p) { return (p == 0 ? slot0 - 1 : slot0 + 2 * (p - 1)) * ROWS + k; };
  float M = -INFINITY;
  for (int p = lane; p < parts; p += 64) M = fmaxf(M, a.stats[at(p)].x);
  M = wave_max_f32(M);
  float o[NC], l = 0.f;
#pragma unroll
  for (int i = 0; i < NC; i++) o[i] = 0.f;
  __shared__ float weight[MOST], meet[4][D + 2];
  for (int p0 = 0; p0 < parts; p0 += MOST) {
    const int here = min(parts - p0, MOST);
    __syncthreads();
    if (tid < here) {
      const float2 s = a.stats[at(p0 + tid)];
      const float f = s.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s.x - M);
      weight[tid] = f;
      l += s.y * f;
    }
    __syncthreads();
#pragma unroll 4
    for (int p = wave; p < here; p += 4) {
      const float f = weight[p];
      const float* x = a.sums + at(p0 + p) * D + NC * lane;
#pragma unroll
      for (int i = 0; i < NC; i++) o[i] += x[i] * f;
    }
  }
#pragma unroll
  for (int i = 0; i < NC; i++) meet[wave][NC * lane + i] = o[i];
  for (int x = 1; x < 64; x <<= 1) l += __shfl_xor(l, x);
  if (lane == 0) meet[wave][D] = l;
  __syncthreads();
  if (wave != 0) return;
  l = (meet[0][D] + meet[1][D]) + (meet[2][D] + meet[3][D]);
#pragma unroll
  for (int i = 0; i < NC; i++) o[i] = (meet[0][NC * lane + i] + meet[1][NC * lane + i]) + (meet[2][NC * lane + i] + meet[3][NC * lane + i]);
  attend_store<NC>(a, join.y, join.z, join.w + k, D, NC * lane, M, l, o, mean);
}

// The same of many rows, with few parts each: D / 4 lanes have a row and take four parts at a time, one trip to memory for up to four.  (A wave a row,
// two channels a lane, the maxima asked for first: vector instructions were 83 % of its cycles; 255 divided tiles of 256 rows of 128
// channels 20 us, the call 327 -> 319; 511 borders of a mixed batch, 64 channels, 72.5 -> 67.5.)
template <int D, int ROWS>
__global__ __launch_bounds__(256) void cache_join_rows_kernel(AttendArgs a) {
  constexpr int LANES = D / 4, HERE = 256 / LANES, BATCH = 4;
  const int w = blockIdx.x + 1, k = blockIdx.y * HERE + threadIdx.x / LANES;
  const int4 join = a.joins[w];
  const int parts = join.x & 0xFFFF;
  if (k >= join.x >> 16) return;
  const int c = threadIdx.x % LANES * 4;
  const auto mean = value_means<4>(a, join.z * D + c);
  const size_t slot0 = (size_t)w * 2;
  float m = -INFINITY, l = 0.f;
  v4f o = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = 0; p0 < parts; p0 += BATCH) {
    float2 s[BATCH];
    v4f x[BATCH];
#pragma unroll
    for (int i = 0; i < BATCH; i++) {
      const int p = min(p0 + i, parts - 1);
      const size_t at = (p == 0 ? slot0 - 1 : slot0 + 2 * (p - 1)) * ROWS + k;
      s[i] = a.stats[at];
      x[i] = *(const v4f*)(a.sums + at * D + c);
    }
    float to = m;
#pragma unroll
    for (int i = 0; i < BATCH; i++) to = fmaxf(to, s[i].x);
    const float ref = to == -INFINITY ? 0.f : to, f = __builtin_amdgcn_exp2f(m - ref);
    l *= f;
    o *= f;
#pragma unroll
    for (int i = 0; i < BATCH; i++) {
      const float g = p0 + i < parts ? __builtin_amdgcn_exp2f(s[i].x - ref) : 0.f;
      l = p0 + i < parts ? l + s[i].y * g : l;
      o = p0 + i < parts ? o + x[i] * g : o;
    }
    m = to;
  }
  attend_store<4>(a, join.y, join.z, join.w + k, D, c, m, l, (const float*)&o, mean);
}

}  // namespace sage
