// Attention over the cache held in 8 bits (gfx950 only): what is its own beside cache_attend_kernel.h and cache_chunk_kernel.h.
//
//   S = q k^T,  k = a_k / 127 n_k;   O = sum_t p_t a_v,t / 127 n_v,t / sum_t p_t,   a: one number for a block of 32 or 64 tokens and head
//
// A code -127 .. 127 is a bf16 number, so the matrix instructions multiply the codes themselves and nothing is rounded but the probabilities: K's
// scale goes with sm_scale into the exponents, V's into the probabilities before they become bf16.  A code takes one and a half vector
// instructions (a byte to FP32, two of them to a word).
//
// Few rows: the codes lie in the page in the order of the operands of 16 x 16 x 32 products (tokens and tiles as in cache_attend_kernel.h),
// 16 bytes a lane, so that a tile of 32 tokens comes straight to registers, the next one under it.
#pragma once

#include "cache8_kernels.h"
#include "cache_chunk_kernel.h"

namespace sage {

// Eight codes to an operand.
__device__ __forceinline__ v8bf codes_to_bf16(int w0, int w1) {
  const auto f = [](int w, int i) { return (float)(signed char)(w >> 8 * i); };
  return as_bf16(v4i{pack_bf16(f(w0, 0), f(w0, 1)), pack_bf16(f(w0, 2), f(w0, 3)), pack_bf16(f(w1, 0), f(w1, 1)), pack_bf16(f(w1, 2), f(w1, 3))});
}

// 32 tokens of a head.
template <int D>
struct ByteTile {
  static constexpr int SLOT = 0;      // of a ring
  v4i k[2][D / 64];       // token 8 (m / 4) + m % 4 (+ 4), channels 64 j + 16 g ..
  v4i v[D / 32];          // octet g, channels 32 j + m and 16 more
  float ka, va;           // largest magnitudes

  // `p`: the head's part of a page, `at`: a token of it; not `any`: loads from where it is.
  __device__ __forceinline__ void load(const CacheGeometry& geo, const unsigned char* p, int at, bool any) {
    const int lane = any ? (threadIdx.x & 63) * 16 : 0;
    const unsigned char *pk = p + at * D, *pv = pk + geo.page() * D;
#pragma unroll
    for (int j = 0; j < D / 64; j++)
#pragma unroll
      for (int b = 0; b < 2; b++) k[b][j] = *(const v4i*)(pk + (2 * j + b) * 1024 + lane);
#pragma unroll
    for (int j = 0; j < D / 32; j++) v[j] = *(const v4i*)(pv + j * 1024 + lane);
    const float* a = (const float*)(p + Bytes8<D>::magnitudes(geo) + at / 4);
    ka = a[0];
    va = a[1];
  }
};

template <int D>
struct ByteRows : AttendRows<D, D> {
  typedef AttendRows<D, D> Base;
  // q[2 j + h]: channels 64 j + 16 g + 8 h ..
  template <typename Piece>
  __device__ __forceinline__ void fetch(const AttendArgs& a, const Piece& p) {
    const int g = (threadIdx.x & 63) >> 4;
    const bool exists = Base::row < p.n_rows;
    const __bf16* x =
        a.Q + (int64_t)(p.begin + (exists ? Base::token : 0)) * a.q_token + (int64_t)(p.head * a.G + (exists ? Base::head_of : 0)) * a.q_head + 16 * g;
#pragma unroll
    for (int j = 0; j < Base::NJ; j++) Base::q[j] = exists ? *(const v4i*)(x + 64 * (j / 2) + 8 * (j % 2)) : v4i{0, 0, 0, 0};
    Base::sees = exists && a.causal ? min(p.len, p.first_sees + Base::token) : p.len;
  }
  __device__ __forceinline__ void begin() {
#pragma unroll
    for (int v = 0; v < Base::NV; v++) Base::o[v] = v4f{0.f, 0.f, 0.f, 0.f};
    Base::m = -INFINITY;
    Base::l = 0.f;
  }
};

constexpr float kBy127 = 1.f / 127.f;

template <int D_>
struct ByteForm {
  static constexpr int D = D_;
  typedef ByteTile<D> Tile;
  typedef ByteRows<D> Rows;
  struct Unpacking {};
  static constexpr bool RING = false, TILED = true;
  static __device__ __forceinline__ const unsigned char* part(const AttendArgs& a, int entry, int head) {
    return a.pool + ((size_t)entry * a.g.H + head) * Bytes8<D>::head_bytes(a.g);
  }

  // 32 tokens into NQ tiles of queries.  `masked`: some row does not see all of them.
  template <int NQ>
  static __device__ __forceinline__ void attend(Rows (&rows)[NQ], Tile& t, int t0, bool masked, float scale_log2, const Unpacking&) {
    const int g = (threadIdx.x & 63) >> 4;
    v4f s[NQ][2];
#pragma unroll
    for (int q = 0; q < NQ; q++) s[q][0] = s[q][1] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int b = 0; b < 2; b++)
#pragma unroll
      for (int j = 0; j < D / 32; j++) {
        const v8bf k = codes_to_bf16(t.k[b][j / 2][2 * (j % 2)], t.k[b][j / 2][2 * (j % 2) + 1]);
#pragma unroll
        for (int q = 0; q < NQ; q++) s[q][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, as_bf16(rows[q].q[j]), s[q][b], 0, 0, 0);
      }
    const float k_scale = t.ka * kBy127 * scale_log2, v_scale = t.va * kBy127;
    // The probabilities times V's scale in bf16, and what that rounding left in a second product, which where the keys bound the call costs nothing: O's error
    // is then that of its own rounding, 0.0017, else 0.0024.  (Not in tiles of more rows, where products count: 128 rows, 32 requests of 4096 tokens, 147 -> 175 us.)
    constexpr bool REST = NQ <= 2;
    v8bf pt[NQ], rest[NQ];
#pragma unroll
    for (int q = 0; q < NQ; q++) {
      Rows& R = rows[q];
      const int behind = R.sees - t0 - 8 * g;      // tokens of the octet that the query sees
      float x[8], c = k_scale;
#pragma unroll
      for (int i = 0; i < 8; i++) x[i] = s[q][i / 4][i % 4];
      if (masked) {
        asm volatile("");                          // (stays a branch)
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = i < behind ? x[i] * c : -INFINITY;      // (c may be 0)
        c = 1.f;
      }
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 8; i++) top = fmaxf(top, x[i]);
      top *= c;
      // (the reference need only be near the maximum)
      if (__any(top > R.m + 8.f)) {
        const float to = fmaxf(R.m, column_max(top));
        const float f = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(R.m - to);
#pragma unroll
        for (int v = 0; v < D / 16; v++) R.o[v] *= f;
        R.l *= f;
        R.m = to;
      }
      const float ref = R.m == -INFINITY ? 0.f : R.m;
#pragma unroll
      for (int i = 0; i < 8; i++) {
        x[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], c, -ref));
        R.l += x[i];
        x[i] *= v_scale;
      }
      if (masked) {
        asm volatile("");
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = i < behind ? x[i] : 0.f;                // (V's scale may be NaN)
      }
      v4i hi, lo;
#pragma unroll
      for (int i = 0; i < 4; i++) {
        hi[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
        if (REST) lo[i] = pack_bf16(x[2 * i] - low_bf16(hi[i]), x[2 * i + 1] - high_bf16(hi[i]));
      }
      pt[q] = as_bf16(hi);
      if (REST) rest[q] = as_bf16(lo);
    }
#pragma unroll
    for (int v = 0; v < D / 16; v++) {
      const v8bf w = codes_to_bf16(t.v[v / 2][2 * (v % 2)], t.v[v / 2][2 * (v % 2) + 1]);
#pragma unroll
      for (int q = 0; q < NQ; q++) {
        rows[q].o[v] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, pt[q], rows[q].o[v], 0, 0, 0);
        if (REST) rows[q].o[v] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, rest[q], rows[q].o[v], 0, 0, 0);
      }
    }
  }
};

template <int D, int NQ>
__global__ __launch_bounds__(256, NQ > 2 ? 1 : 2) void cache8_attend_kernel(AttendArgs a) {
  attend_items<ByteForm<D>, NQ>(a);
}

// Short requests, a wave each of their items: no sum over the requests, nothing to join, no LDS.  (Four waves an item, dealt out to a workgroup a CU: 405
// requests of 3 tokens, 14 heads, 73 us; so 23, 17 MB in and out each.)
template <int D, int NQ>
__global__ __launch_bounds__(256, 2) void cache8_short_kernel(AttendArgs a) {
  typedef ByteForm<D> Form;
  const int lane = threadIdx.x & 63, g = lane >> 4;
  const int item = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)), r = item / a.direct;
  if (r >= a.R) return;
  const AttendRequest rq = attend_request(a, r);
  const int tiles = (rq.rows + 16 * NQ - 1) / (16 * NQ), index = item - r * a.direct;
  if (index >= a.g.H * tiles) return;
  struct {
    int begin, n_rows, head, len, first_sees;
  } piece;
  piece.begin = rq.begin;
  piece.n_rows = rq.rows;
  piece.head = index / tiles;
  piece.len = rq.len;
  piece.first_sees = rq.first_sees;
  const int row0 = (index - piece.head * tiles) * 16 * NQ, visible = attend_visible(a, rq, row0, 16 * NQ);
  const int all_see = a.causal ? rq.first_sees + row0 / a.G : rq.len, last = max(visible - 1, 0);
  const int32_t* table = a.table + (size_t)r * a.columns;
  ByteRows<D> rows[NQ];
#pragma unroll
  for (int q = 0; q < NQ; q++) {
    rows[q].place(a, row0 + 16 * q);
    rows[q].fetch(a, piece);
    rows[q].begin();
  }
  const typename Form::Unpacking un;
  ByteTile<D> t[2];
  bool there[2];
  const auto load = [&](int x, int t0) {      // (as in attend_items: loads every time)
    const int entry = __builtin_amdgcn_readfirstlane(table[min(t0, last) >> a.g.page_shift]);
    there[x] = t0 < visible && (unsigned)entry < (unsigned)a.g.pages;
    t[x].load(a.g, Form::part(a, there[x] ? entry : 0, piece.head), t0 & (a.g.page() - 1), there[x]);
  };
  load(0, 0);
  for (int t0 = 0; t0 < visible; t0 += 64) {
#pragma unroll
    for (int x = 0; x < 2; x++) {
      const int at = t0 + 32 * x;
      load(1 - x, at + 32);
      if (there[x]) Form::template attend<NQ>(rows, t[x], at, at + 32 > all_see, a.scale_log2, un);
    }
  }
  // A tile's rows, turned in the wave's part of LDS so that 16 lanes write a row.
  __shared__ __attribute__((aligned(16))) char turned[4][16][2 * D + 16];
  char(*out)[2 * D + 16] = turned[threadIdx.x >> 6];
#pragma unroll
  for (int q = 0; q < NQ; q++) {
    const ByteRows<D>& R = rows[q];
    const float l = column_sum(R.l);
    const bool any = !(l == 0.f);
    const float f = any ? 1.f / l : 0.f;
#pragma unroll
    for (int v = 0; v < D / 16; v++) {
      const auto mean = value_means<4>(a, piece.head * D + 16 * v + 4 * g);
      float y[4];
#pragma unroll
      for (int i = 0; i < 4; i++) y[i] = any ? R.o[v][i] * f + mean[i] : 0.f;
      *(v2i*)(out[lane & 15] + 32 * v + 8 * g) = v2i{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
    }
    if (g == 0 && R.row < rq.rows && a.LSE != nullptr)
      a.LSE[(int64_t)(piece.head * a.G + R.head_of) * a.T + rq.begin + R.token] = any ? (R.m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : -INFINITY;
    __builtin_amdgcn_wave_barrier();
    constexpr int LANES = D / 8, AT_ONCE = 64 / LANES;      // of a row, rows
#pragma unroll
    for (int k = 0; k < 16 / AT_ONCE; k++) {
      const int i = k * AT_ONCE + lane / LANES, row = row0 + 16 * q + i;
      const v4i x = *(const v4i*)(out[i] + lane % LANES * 16);
      if (row >= rq.rows) continue;
      const int token = row / a.G, hq = piece.head * a.G + row - token * a.G;
      *(v4i*)(a.O + ((int64_t)(rq.begin + token) * a.Hq + hq) * D + lane % LANES * 8) = x;
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// ---- many rows ---------------------------------------------------------------------------------------------------------
// V's scale of a half goes into its exponents (log2 of it), so that they give the probabilities times it, and out of their sum.  (Of a scale of zero, whose
// codes are zeros, any other will do, and for one that is no number poison() stands in.)  It saves 32 products of a lane and tile: 2048 new tokens of
// 4 heads of a group against 10000 313 -> 304 us.  Only of a magnitude that the quantiser may have stored, zero or 2^-100 and more: where nothing was stored any
// bits may be, and the logarithm of a number so small that its scale flushes to zero would make the sum of a half of which no row sees a token 0 times infinity.
// What is folded in is at most 2^64 either way: exp2 flushes what is below 2^-126, so that the sum loses weights of less than 2^-62 of the reference (2^30 keys
// of them are 2^-32; of a magnitude of 2^-100 it would lose those of 2^-19, and LSE depend on V).  The few magnitudes beyond leave a power of two to be
// multiplied into the probabilities behind the sum, in the branch of blocks that are not numbers.  (In the softmax that took 12 to 17 registers more and 308 -> 319
// us; into V's fragments where they are stored, four of 5000 tokens with 300 new ones 136 -> 142; so 134 -> 132.)
struct ByteKnown {
  int flags[2];           // bit 0: the half's page exists; bit 1: and its values are not numbers; bit 2: and its keys; from bit 8 on, signed: the power of two
  float k[2], log_v[2];
  __device__ __forceinline__ void set(int half, bool is_page, float ka, float va) {
    const auto number = [](float x) { return x >= 0.f && x < INFINITY; };      // (where nothing was stored any bits may be)
    const bool stored = is_page && number(va) && va >= kLeast8;
    const int e = (int)(__float_as_uint(va) >> 23) - 127, left = stored && (e < -57 || e > 70) ? e - 7 : 0;
    flags[half] = (is_page ? 1 | (number(va) ? 0 : 2) | (number(ka) ? 0 : 4) : 0) | left * 256;
    k[half] = number(ka) ? ka * kBy127 : 0.f;
    log_v[half] = stored ? __builtin_amdgcn_logf(__builtin_ldexpf(va * kBy127, -left)) : 0.f;
  }
  // Of all lanes the same: to scalar registers.
  __device__ __forceinline__ ByteKnown uniform(int lane) const {
    ByteKnown w;
#pragma unroll
    for (int b = 0; b < 2; b++) {
      w.flags[b] = __builtin_amdgcn_readlane(flags[b], lane);
      w.k[b] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(k[b]), lane));
      w.log_v[b] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(log_v[b]), lane));
    }
    return w;
  }
};

// 64 tokens on their way from the pages to bf16 fragments of codes: waves 0 to 3 have K's, the others V's, 16 bytes at a time as they lie
// in the page (one of which is two lanes' octets of channels, or of tokens).
template <int D_>
struct ByteChunk {
  static constexpr int D = D_, FRAG = D / 16 * 1024, N = D / 64, NG = 0;
  typedef ByteKnown Known;
  v4i code[N];
  float k, v;             // of the half with the same number as (u & 127) / 64
  int valid;

  __device__ __forceinline__ void load(const AttendArgs& a, int head, int from, int page0, int page1, int visible) {
    const int tid = threadIdx.x, u = tid & 255;
    const auto of = [&](int b) {
      const int entry = __builtin_amdgcn_readfirstlane(b ? page1 : page0);
      return a.pool + ((size_t)((unsigned)entry < (unsigned)a.g.pages ? entry : 0) * a.g.H + head) * Bytes8<D>::head_bytes(a.g);
    };
#pragma unroll
    for (int i = 0; i < N; i++) {
      const int b = N == 2 ? i : u >> 7, at = (from + 32 * b) & (a.g.page() - 1);
      const int q = N == 2 ? u : u & 127;
      code[i] = *(const v4i*)(of(b) + (tid < 256 ? 0 : a.g.page() * D) + at * D + q * 16);
    }
    const int b = u >> 6 & 1, at = (from + 32 * b) & (a.g.page() - 1);
    const float* s = (const float*)(of(b) + Bytes8<D>::magnitudes(a.g) + at / 4);
    k = s[0];
    v = s[1];
    valid = (unsigned)(b ? page1 : page0) < (unsigned)a.g.pages;
  }
  __device__ __forceinline__ void store(char* K, char* V, Known& known, unsigned char*, int*, int) const {
    const int tid = threadIdx.x, u = tid & 255;
    if (tid < 128 && (tid & 63) == 0) {
      known.set(tid >> 6, valid, k, v);
    }
#pragma unroll
    for (int i = 0; i < N; i++) {
      const int b = N == 2 ? i : u >> 7, q = N == 2 ? u : u & 127;
      const v8bf x = codes_to_bf16(code[i][0], code[i][1]), y = codes_to_bf16(code[i][2], code[i][3]);
      if (tid < 256) {      // j = q / 128, s = q / 64 % 2, g = q / 16 % 4, m = q % 16: token 8 (m / 4) + 4 s + m % 4, channels 64 j + 16 g ..
        const int m = q & 15, rho = 16 * (m >> 3) + 8 * (q >> 6 & 1) + 4 * (m >> 2 & 1) + (m & 3);
        char* to = K + b * FRAG + ((4 * (q >> 7) + (q >> 4 & 3)) * 64 + rho) * 16;
        *(v8bf*)to = x;
        *(v8bf*)(to + 512) = y;
      } else {              // j = q / 64, octet q / 16 % 4, channels 32 j + q % 16 and 16 more
        const int o = 4 * b + (q >> 4 & 3);
        char* to = V + ((q >> 6) * 4 + (o >> 1)) * 1024 + ((o & 1) * 32 + (q & 15)) * 16;
        *(v8bf*)to = x;
        *(v8bf*)(to + 256) = y;
      }
    }
  }
};

// The probabilities are rounded to bf16, once: the matrix pipe bounds these calls, and a product of what that leaves, as tiles of few rows have, takes a
// third and more (2048 new tokens against 10000 307 -> 415 us, heads of 64 210 -> 317; four of 5000 with 300 130 -> 163) for an error of O of 0.0017 in
// place of 0.0024.
template <int D>
struct ByteChunkRows : ChunkRows<D> {
  typedef ChunkRows<D> Base;
  __device__ __forceinline__ void softmax(v16f (&s)[2], v8bf (&p)[4], int t0, const ByteKnown& of_tile, float scale_log2) {
    const ByteKnown known = of_tile.uniform(0);
    // (above zero, as a hidden logit is -infinity times it; a scale of zero has codes of zeros)
    const auto scalar = [](float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); };
    const float c[2] = {scalar(fmaxf(known.k[0] * scale_log2, 1e-37f)), scalar(fmaxf(known.k[1] * scale_log2, 1e-37f))};
    if (t0 + kChunkUnit > Base::all_see || !known.flags[0] || !known.flags[1]) {
      const int h = threadIdx.x >> 5 & 1;
#pragma unroll
      for (int b = 0; b < 2; b++) {
        const int behind = known.flags[b] ? Base::sees - t0 - 32 * b - 8 * h : 0;
#pragma unroll
        for (int i = 0; i < 16; i++) s[b][i] = 16 * (i / 8) + i % 8 < behind ? s[b][i] : -INFINITY;
      }
    }
    float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int b = 0; b < 2; b++) {
#pragma unroll
      for (int i = 0; i < 16; i++) top[b] = fmaxf(top[b], s[b][i]);
      top[b] *= c[b];
    }
    if (__any(fmaxf(top[0], top[1]) > Base::m + 8.f)) {
      const float to = fmaxf(Base::m, half_swap_max_f32(fmaxf(top[0], top[1])));
      const float f = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(Base::m - to);
#pragma unroll
      for (int i = 0; i < Base::NC; i++) Base::o[i] *= f;
      Base::l *= f;
      Base::m = to;
    }
    const float ref = Base::m == -INFINITY ? 0.f : Base::m;
#pragma unroll
    for (int b = 0; b < 2; b++) {
      const float off = known.log_v[b] - ref;
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 16; i++) {
        s[b][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], c[b], off));
        sum += s[b][i];
      }
      Base::l = __builtin_fmaf(sum, __builtin_amdgcn_exp2f(-known.log_v[b]), Base::l);
#pragma unroll
      for (int k = 0; k < 2; k++)
        p[2 * b + k] = as_bf16(v4i{pack_bf16(s[b][8 * k], s[b][8 * k + 1]), pack_bf16(s[b][8 * k + 2], s[b][8 * k + 3]),
                                   pack_bf16(s[b][8 * k + 4], s[b][8 * k + 5]), pack_bf16(s[b][8 * k + 6], s[b][8 * k + 7])});
    }
  }
  // What the probabilities are still to be multiplied by.
  static __device__ __forceinline__ void scale(v8bf (&p)[4], const ByteKnown& known) {
#pragma unroll
    for (int b = 0; b < 2; b++) {
      const float by = __builtin_ldexpf(1.f, known.flags[b] >> 8);
#pragma unroll
      for (int k = 0; k < 2; k++)
#pragma unroll
        for (int i = 0; i < 8; i++) p[2 * b + k][i] = (__bf16)((float)p[2 * b + k][i] * by);
    }
  }
  // A block whose keys or values are not numbers, to the rows that see some of it.
  __device__ __forceinline__ void poison(const ByteKnown& known, int t0) {
#pragma unroll
    for (int b = 0; b < 2; b++)
      if ((known.flags[b] & 6) != 0 && Base::sees > t0 + 32 * b) {
#pragma unroll
        for (int c = 0; c < Base::NC; c++) Base::o[c] += __builtin_nanf("");
        if (known.flags[b] & 4) Base::l = __builtin_nanf("");
      }
  }
};

template <int D_>
struct ByteChunks {
  static constexpr int D = D_;
  typedef ByteChunk<D> Tile;
  typedef ByteChunkRows<D> Rows;
  typedef ByteKnown Known;
  static __device__ __forceinline__ void before_values(Rows& rows, v8bf (&p)[4], const Known& known, int t0) {
    if (__builtin_expect(__builtin_amdgcn_readfirstlane(known.flags[0] | known.flags[1]) & ~1, 0)) {
      Rows::scale(p, known);
      rows.poison(known, t0);
    }
  }
  static __device__ __forceinline__ void poison(Rows&, bool, const unsigned char*, const Known&, int) {}      // (before_values has)
  static constexpr bool WORDS_IN_RING = true;      // (six registers of them are more than the kernel for heads of 64 has)
  typedef ByteKnown Word;
  static __device__ __forceinline__ Word word(const Known& known, bool) { return known; }
  struct Words {};
  static __device__ __forceinline__ const Known& known(const Word& w) { return w; }
  static __device__ __forceinline__ bool any_bad(const Word&) { return false; }
};

template <int D>
__global__ __launch_bounds__(512, 2) void cache8_chunk_kernel(AttendArgs a) {
  chunk_items<ByteChunks<D>>(a);
}
template <int D>
__global__ __launch_bounds__(512) void cache8_unpack_kernel(AttendArgs a) {
  unpack_items<ByteChunks<D>>(a);
}
template <int D>
__global__ __launch_bounds__(512, D == 64 ? 4 : 2) void cache8_wide_kernel(AttendArgs a) {
  wide_items<ByteChunks<D>>(a);
}

}  // namespace sage
