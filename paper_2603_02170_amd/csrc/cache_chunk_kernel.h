// Attention over the 4-bit cache for many query rows a request: prompts, chunks of them (gfx950 only).
//
// The matrix pipe bounds it: 4 d operations a (row, key), of which a workgroup of eight waves does 256 rows (query x head of the group) by 64
// keys at a time.  What the cache holds are bf16 numbers, so the waves of a workgroup turn 64 tokens into bf16 fragments in LDS once for
// all (three instructions a value, a 512th of them a thread) and each wave runs 32 x 32 x 16 products of its own 32 rows on them:
// S^T = K Q^T, in which a lane has one query, and O^T = V^T P^T, of which P^T is the accumulator as it stands: row 8 a + 4 h + b of a
// 32 x 32 accumulator (register 4 a + b, lane half h) is given token 16 (a / 2) + 8 h + 4 (a % 2) + b, so that a lane's eight registers 8 k .. 8 k + 7 are the octet of
// tokens 16 k + 8 h .. that it has to hold of the operand.  The next 64 tokens are unpacked into the other half of the LDS under this.
#pragma once

#include "cache_attend_kernel.h"

namespace sage {

constexpr int kChunkRows = 256, kChunkUnit = 64;

// What the rows have to know of 64 tokens that lie in LDS or in the workspace: whether the pages of its halves exist.
struct ChunkKnown {
  int exists[2];
};

// 64 tokens on their way from the pages to bf16 fragments: waves 0 to 3 have K's, the others V's.
template <int D_, int GROUP_>
struct ChunkTile {
  static constexpr int D = D_, GROUP = GROUP_, NG = D / GROUP, FRAG = D / 16 * 1024;     // bytes of 32 tokens of K, of 32 tokens' worth of V
  typedef ChunkKnown Known;
  v4i code, s0, s1;
  int valid;               // tokens of the thread's own that exist, counted from its first

  // `from`: the tile's first token; `pages`: the table's entries of its two halves
  __device__ __forceinline__ void load(const AttendArgs& a, int head, int from, int page0, int page1, int visible) {
    const int tid = threadIdx.x, u = tid & 255;
    const bool keys = tid < 256;
    const int o = D == 128 ? u >> 5 : (u >> 4) & 7;          // V: octet of the tile
    const int b = keys ? u >> 7 : o >> 2;                    // half of the tile
    const int entry = __builtin_amdgcn_readfirstlane(b ? page1 : page0);
    const bool exists = (unsigned)entry < (unsigned)a.g.pages;
    const unsigned char* p = a.pool + (size_t)(exists ? entry : 0) * a.g.page_bytes() + (size_t)head * a.g.head_bytes();
    const int t0 = from + 32 * b, at = t0 & (a.g.page() - 1);
    if (keys) {
      const int rho = u & 31, q = (u >> 5) & 3;
      const int t = at + 16 * (rho >> 4) + 8 * (rho >> 2 & 1) + 4 * (rho >> 3 & 1) + (rho & 3);
      const unsigned char* pk = p + t * (D / 2) + q * (D / 8);
      if (D == 128) {
        code = *(const v4i*)pk;
      } else {
        const v2i x = *(const v2i*)pk;
        code = v4i{x[0], x[1], 0, 0};
      }
      const unsigned short* ps = (const unsigned short*)(p + a.g.k_scales() + (t >> 3) * NG * 16) + (t & 7);
#pragma unroll
      for (int s = 0; s < NG; s++) s0[s] = ps[8 * s];
      valid = exists;
    } else {
      const int octet = (at >> 3) + (o & 3), f = D == 128 ? u >> 4 & 1 : 0, m = u & 15;
      code = *(const v4i*)(p + a.g.v_codes() + octet * (4 * D) + f * 256 + m * 16);
      const unsigned char* ps = p + a.g.v_scales() + (octet * NG + f * (64 / GROUP)) * 16;
      s0 = *(const v4i*)ps;
      if (GROUP == 32) s1 = *(const v4i*)(ps + 16);
      valid = exists ? visible - (from + 8 * o) : 0;
    }
  }

  // Writes the fragments.  `poison`: tokens whose scale of V is not a number (bit s: of the group s), which the product may not meet
  // (0 times NaN in the rows that do not see the token); `poisoned` says that there is one.
  __device__ __forceinline__ void store(char* K, char* V, Known& known, unsigned char* poison, int* poisoned, int tag) const {
    const int tid = threadIdx.x, u = tid & 255;
    if (tid < 256) {
      const int rho = u & 31, q = (u >> 5) & 3, b = u >> 7;
      if ((u & 127) == 0) known.exists[b] = valid;
#pragma unroll
      for (int j = 0; j < D / 32; j++) {
        const float s = bf16_bits_to_float((unsigned short)s0[32 * j / GROUP]), s8 = -8.f * s;
        const unsigned lo = (unsigned)code[j] & 0x0F0F0F0Fu, hi = (unsigned)code[j] >> 4 & 0x0F0F0F0Fu;
        const auto value = [&](unsigned w, int byte) { return __builtin_fmaf((float)(w >> 8 * byte & 255), s, s8); };
        const v4i x = {pack_bf16(value(lo, 0), value(lo, 2)), pack_bf16(value(hi, 0), value(hi, 2)), pack_bf16(value(lo, 1), value(lo, 3)),
                       pack_bf16(value(hi, 1), value(hi, 3))};
        *(v4i*)(K + b * FRAG + ((2 * j + (q >> 1)) * 64 + (q & 1) * 32 + rho) * 16) = x;
      }
      return;
    }
    if (D == 64 && u >= 128) return;
    const int o = D == 128 ? u >> 5 : u >> 4, f = D == 128 ? u >> 4 & 1 : 0, m = u & 15;
    constexpr int NS = GROUP == 32 ? 2 : 1;      // scales of a token over the thread's channels m + 16 j
    v4i sc[NS];
    sc[0] = s0;
    if (NS == 2) sc[NS - 1] = s1;
    unsigned top = 0;                            // (an exponent of ones carries into the sign's place)
#pragma unroll
    for (int k = 0; k < NS; k++)
#pragma unroll
      for (int i = 0; i < 4; i++) top |= ((unsigned)sc[k][i] & 0x7F807F80u) + 0x00800080u;
    unsigned bad[NS] = {};
    if (__any(valid < 8 || (top & 0x80008000u) != 0)) {
      asm volatile("");                          // (stays a branch)
#pragma unroll
      for (int k = 0; k < NS; k++) {
#pragma unroll
        for (int i = 0; i < 8; i++) {
          const int half = i % 2 == 0 ? 0xFFFF : (int)0xFFFF0000;
          const bool number = (sc[k][i / 2] & half & 0x7F807F80) != (half & 0x7F807F80);
          if (!number && i < valid) bad[k] |= 1u << i;
          sc[k][i / 2] = number && i < valid ? sc[k][i / 2] : sc[k][i / 2] & ~half;
        }
        if (__any(bad[k] != 0)) *poisoned = tag;
      }
    }
    if (m == 0) {
#pragma unroll
      for (int k = 0; k < NS; k++)               // a byte a token
        *(uint2*)(poison + (f * (64 / GROUP) + k) * 64 + 8 * o) = uint2{(bad[k] & 15) * 0x00204081u & 0x01010101u, (bad[k] >> 4) * 0x00204081u & 0x01010101u};
    }
    v4i x[4];                                    // channel m + 16 j
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const unsigned lo = (unsigned)code[i] & 0x0F0F0F0Fu, hi = (unsigned)code[i] >> 4 & 0x0F0F0F0Fu;
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const int w = sc[NS == 2 ? j / 2 : 0][i];
        const float s = low_bf16(w), t = high_bf16(w);
        const unsigned bytes = (j % 2 ? hi : lo) >> 8 * (j / 2);
        x[j][i] = pack_bf16(__builtin_fmaf((float)(bytes & 255), s, -8.f * s), __builtin_fmaf((float)(bytes >> 16 & 255), t, -8.f * t));
      }
    }
#pragma unroll
    for (int j = 0; j < 4; j++) *(v4i*)(V + ((2 * f + j / 2) * 4 + (o >> 1)) * 1024 + ((o & 1) * 32 + 16 * (j % 2) + m) * 16) = x[j];
  }
};

// Line of what is dealt out: request, then head, then row tile of 256, each its units + a cost of its own; or (not split) one each,
// request, then row tile from the last, which sees most, then head.

// Tiles of 64 tokens that a head of the request has for the rows to see.
__device__ __forceinline__ int chunk_key_tiles(const AttendRequest& q) { return q.rows == 0 ? 0 : max(1, (q.len + kChunkUnit - 1) / kChunkUnit); }

struct ChunkScratch {
  unsigned sums[8][2];
  int total, found[4];
};
// A workgroup's way along the line: (request, head, row tile of ROWS) from unit j0 (of UNIT tokens) on.
template <int ROWS, int UNIT, int COST>
struct ChunkWalk {
  static __device__ __forceinline__ int chunk_tiles(int rows) { return (rows + ROWS - 1) / ROWS; }
  static __device__ __forceinline__ int chunk_units(const AttendArgs& a, const AttendRequest& q, int tile) {
    return max(1, (attend_visible(a, q, tile * ROWS, ROWS) + UNIT - 1) / UNIT);
  }
  static __device__ __forceinline__ int chunk_cut(int offset) { return cut_at<COST>(offset); }
  // of a request and head
  static __device__ __forceinline__ int chunk_weight(const AttendArgs& a, const AttendRequest& q) {
    const int tiles = chunk_tiles(q.rows);
    if (!a.split) return tiles;
    int w = 0;
    for (int t = 0; t < tiles; t++) w += chunk_units(a, q, t) + COST;
    return w;
  }

  int w, x, end, j0;       // its number; where its item begins in the line; where its share ends
  int r, head, place, tile;
  int before;              // tiles of 64 tokens of the requests in front (of one head)
  AttendRequest rq;
  AttendShares shares;

  // All 512 threads; false: the workgroup has nothing.  Leaves no word for the joining launch.
  __device__ __forceinline__ bool start(const AttendArgs& a, ChunkScratch& s) {
    const int tid = threadIdx.x, H = a.g.H;
    const int per = (a.R + 511) / 512, r0 = min(tid * per, a.R), r1 = min(r0 + per, a.R);
    unsigned mine = 0, tiles = 0;
    for (int i = r0; i < r1; i++) {
      const AttendRequest q = attend_request(a, i);
      mine = min(mine + (unsigned)chunk_weight(a, q), kFull);
      tiles += chunk_key_tiles(q);
    }
    unsigned to[2] = {mine, tiles};
    block_scan<8>(to, s.sums);
    if (tid == 511) s.total = (int)to[0];
    __syncthreads();
    const int units = s.total;
    // (the host has bounded this for a `cu` that rises; another one gets nothing)
    if ((int64_t)units * H > 1 << 30) {
      if (tid == 0) a.joins[blockIdx.x] = int4{0, 0, 0, 0};
      return false;
    }
    const int upto = (int)to[0], tiles_to = (int)to[1];
    shares = AttendShares(__builtin_amdgcn_readfirstlane(units) * H, a.workgroups);
    // (neighbours in the line to one XCD, whose L2 then holds a head's keys for all its row tiles)
    w = a.split && shares.n == a.workgroups && shares.n % 8 == 0 ? (blockIdx.x & 7) * (shares.n / 8) + (blockIdx.x >> 3) : blockIdx.x;
    if (tid == 0) a.joins[w] = int4{0, 0, 0, 0};
    if (w >= shares.n) return false;
    const int begin = shares.begin(w);
    end = shares.begin(w + 1);
    if ((upto - (int)mine) * H <= begin && begin < upto * H) {
      int at = upto - (int)mine, t = tiles_to - (int)tiles;
      for (int i = r0; i < r1; i++) {
        const AttendRequest q = attend_request(a, i);
        const int u = chunk_weight(a, q);
        if (begin < (at + u) * H) {
          s.found[0] = i;
          s.found[1] = at * H;
          s.found[2] = u;
          s.found[3] = t;
          break;
        }
        at += u;
        t += chunk_key_tiles(q);
      }
    }
    __syncthreads();
    r = __builtin_amdgcn_readfirstlane(s.found[0]);
    x = __builtin_amdgcn_readfirstlane(s.found[1]);
    before = __builtin_amdgcn_readfirstlane(s.found[3]);
    const int weight = __builtin_amdgcn_readfirstlane(s.found[2]);
    rq = attend_request(a, r);
    j0 = 0;
    if (a.split) {
      head = (begin - x) / weight;
      x += head * weight;
      place = 0;
      for (int u; x + (u = chunk_units(a, rq, chunk_tile_at(place, chunk_tiles(rq.rows))) + COST) <= begin; place++) x += u;
      place = __builtin_amdgcn_readfirstlane(place);
      tile = chunk_tile_at(place, chunk_tiles(rq.rows));
      j0 = chunk_cut(begin - x);
    } else {
      const int i = begin - x;
      tile = weight - 1 - i / H;
      head = i - i / H * H;
      x = begin;
    }
    head = __builtin_amdgcn_readfirstlane(head);
    tile = __builtin_amdgcn_readfirstlane(tile);
    x = __builtin_amdgcn_readfirstlane(x);
    j0 = __builtin_amdgcn_readfirstlane(j0);
    return a.split ? chunk_cut(end - x) > j0 : true;
  }
  // Units j0 .. of the item that are this workgroup's; leaves word for the joining launch at the first border inside it.
  __device__ __forceinline__ int last_unit(const AttendArgs& a, int units) const {
    if (shares.template first_border<COST>(w, x, j0) && threadIdx.x == 0)
      a.joins[w] = join_word(shares.template parts<COST>(w, x, units), min(rq.rows - tile * ROWS, ROWS), rq.begin, head,
                             tile * ROWS);
    return a.split ? min(units, chunk_cut(end - x)) : units;
  }
  // Behind an item of so many units of which all up to j1 are done: false at the share's end.
  __device__ __forceinline__ bool next(const AttendArgs& a, int units, int j1) {
    if (j1 < units || !a.split) return false;        // (not split, a workgroup has one)
    x += units + COST;
    if (chunk_cut(end - x) <= 0) return false;
    j0 = 0;
    if (++place == chunk_tiles(rq.rows)) {
      place = 0;
      if (++head == a.g.H) {
        head = 0;
        before += chunk_key_tiles(rq);
        do rq = attend_request(a, ++r); while (rq.rows == 0);     // (there is one: the share goes on)
      }
    }
    tile = chunk_tile_at(place, chunk_tiles(rq.rows));
    return true;
  }
};

// The rows of a wave: 32 queries, a lane (n, h) has half of the channels of one.
template <int D>
struct ChunkRows {
  static constexpr int NK = D / 16, NC = D / 32;
  v4i q[NK];
  v16f o[NC];
  float m, l;
  int token, head_of, sees, all_see, wave_sees;
  bool real;

  __device__ __forceinline__ void begin(const AttendArgs& a, const AttendRequest& rq, int head, int wave_row0) {
    const int n = threadIdx.x & 31, h = threadIdx.x >> 5 & 1, row = wave_row0 + n;
    token = row / a.G;
    head_of = row - token * a.G;
    real = row < rq.rows;
    const __bf16* p = a.Q + (int64_t)(rq.begin + (real ? token : 0)) * a.q_token + (int64_t)(head * a.G + (real ? head_of : 0)) * a.q_head + 8 * h;
#pragma unroll
    for (int s = 0; s < NK; s++) q[s] = real ? *(const v4i*)(p + 16 * s) : v4i{0, 0, 0, 0};
    sees = real && a.causal ? min(rq.len, rq.first_sees + token) : rq.len;
    all_see = __builtin_amdgcn_readfirstlane(a.causal ? rq.first_sees + wave_row0 / a.G : rq.len);
    wave_sees = __builtin_amdgcn_readfirstlane(wave_row0 < rq.rows ? attend_visible(a, rq, wave_row0, 32) : 0);
#pragma unroll
    for (int c = 0; c < NC; c++) o[c] = v16f{};
    m = -INFINITY;
    l = 0.f;
  }
  // The queries are there.
  __device__ __forceinline__ void wait() {
#pragma unroll
    for (int s = 0; s < NK; s++) arrived(q[s]);
  }
  // N products whose operand comes from LDS, kAhead reads ahead of each, in this order.  (The compiler by itself reads, waits and multiplies,
  // one after the other, and looks past groups of instructions that it is asked for.)
  static constexpr int kAhead = 4;
  template <int N, typename Read, typename Product>
  static __device__ __forceinline__ void products(Read read, Product product) {
    v4i f[kAhead];
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < kAhead; i++) f[i] = read(i);
#pragma unroll
    for (int i = 0; i < N; i++) {
      __builtin_amdgcn_sched_barrier(0);
      product(i, as_bf16(f[i % kAhead]));
      if (i + kAhead < N) f[i % kAhead] = read(i + kAhead);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  __device__ __forceinline__ void logits(const char* K, v16f (&s)[2]) const {
    K += (threadIdx.x & 63) * 16;
    s[0] = v16f{};
    s[1] = v16f{};
    products<2 * NK>([&](int i) { return *(const v4i*)(K + ((i & 1) * NK + (i >> 1)) * 1024); },
                     [&](int i, const v8bf& f) { s[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, as_bf16(q[i >> 1]), s[i & 1], 0, 0, 0); });
  }
  // Logits of the tokens t0 .. t0 + 63 to probabilities.
  __device__ __forceinline__ void softmax(v16f (&s)[2], v8bf (&p)[4], int t0, const ChunkKnown& known, float scale_log2) {
    const int e0 = known.exists[0], e1 = known.exists[1];
    if (t0 + kChunkUnit > all_see || e0 + e1 != 2) {
      const int h = threadIdx.x >> 5 & 1;
#pragma unroll
      for (int b = 0; b < 2; b++) {
        const int behind = (b ? e1 : e0) ? sees - t0 - 32 * b - 8 * h : 0;
#pragma unroll
        for (int i = 0; i < 16; i++) s[b][i] = 16 * (i / 8) + i % 8 < behind ? s[b][i] : -INFINITY;
      }
    }
    float top = -INFINITY;
#pragma unroll
    for (int b = 0; b < 2; b++)
#pragma unroll
      for (int i = 0; i < 16; i++) top = fmaxf(top, s[b][i]);
    if (__any(top * scale_log2 > m + 8.f)) {
      const float to = fmaxf(m, half_swap_max_f32(top) * scale_log2);
      const float f = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - to);
#pragma unroll
      for (int c = 0; c < NC; c++) o[c] *= f;
      l *= f;
      m = to;
    }
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int b = 0; b < 2; b++) {
#pragma unroll
      for (int i = 0; i < 16; i++) {
        s[b][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], scale_log2, -ref));
        l += s[b][i];
      }
#pragma unroll
      for (int k = 0; k < 2; k++)
        p[2 * b + k] = as_bf16(v4i{pack_bf16(s[b][8 * k], s[b][8 * k + 1]), pack_bf16(s[b][8 * k + 2], s[b][8 * k + 3]),
                                   pack_bf16(s[b][8 * k + 4], s[b][8 * k + 5]), pack_bf16(s[b][8 * k + 6], s[b][8 * k + 7])});
    }
  }
  __device__ __forceinline__ void values(const char* V, const v8bf (&p)[4]) {
    V += (threadIdx.x & 63) * 16;
    products<4 * NC>([&](int i) { return *(const v4i*)(V + (i % NC * 4 + i / NC) * 1024); },
                     [&](int i, const v8bf& f) { o[i % NC] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, p[i / NC], o[i % NC], 0, 0, 0); });
  }
  // Tokens whose values are not numbers, to the rows that see them.
  __device__ __forceinline__ void poison(const unsigned char* bad, int group, int t0, const ChunkKnown& known) {
    const int e0 = known.exists[0], e1 = known.exists[1];
    for (int t = 0; t < kChunkUnit; t++)
#pragma unroll
      for (int c = 0; c < NC; c++)
        if (bad[32 * c / group * 64 + t] && (t < 32 ? e0 : e1) && t < sees - t0) o[c] += __builtin_nanf("");
  }
  // A finished row, or (part) what a workgroup has of it.
  __device__ __forceinline__ void end(const AttendArgs& a, const AttendRequest& rq, int head, bool whole, size_t part) {
    const int h = threadIdx.x >> 5 & 1;
    l = half_swap_sum_f32(l);
    if (!real) return;
    if (whole) {
      const bool any = !(l == 0.f);
      const float f = any ? 1.f / l : 0.f;
      const int hq = head * a.G + head_of;
      __bf16* p = a.O + ((int64_t)(rq.begin + token) * a.Hq + hq) * D;
#pragma unroll
      for (int c = 0; c < NC; c++)
#pragma unroll
        for (int i = 0; i < 4; i++) {
          float y[4];
#pragma unroll
          for (int e = 0; e < 4; e++) {
            const float mean = a.v_mean != nullptr ? a.v_mean[head * D + 32 * c + 8 * i + 4 * h + e] : 0.f;
            y[e] = any ? o[c][4 * i + e] * f + mean : 0.f;
          }
          *(v2i*)(p + 32 * c + 8 * i + 4 * h) = v2i{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
        }
      if (h == 0 && a.LSE != nullptr) a.LSE[(int64_t)hq * a.T + rq.begin + token] = any ? (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : -INFINITY;
    } else {
#pragma unroll
      for (int c = 0; c < NC; c++)
#pragma unroll
        for (int i = 0; i < 4; i++)
          *(v4f*)(a.sums + part * D + 32 * c + 8 * i + 4 * h) = v4f{o[c][4 * i], o[c][4 * i + 1], o[c][4 * i + 2], o[c][4 * i + 3]};
      if (h == 0) a.stats[part] = float2{m, l};
    }
  }
};

struct WideTile {
  int flags;        // bit 0, 1: the pages of its halves exist; bit 2: some value is not a number
};

// What the kernels need of a cache's format.
template <int D_, int GROUP>
struct NibbleChunks {
  static constexpr int D = D_;
  typedef ChunkTile<D, GROUP> Tile;
  typedef ChunkRows<D> Rows;
  typedef ChunkKnown Known;
  // What is to be done in front of the product of 64 tokens' probabilities and values.
  static __device__ __forceinline__ void before_values(Rows&, v8bf (&)[4], const Known&, int) {}
  // Of 64 tokens: `bad` has those that are not numbers, if there are any.
  static __device__ __forceinline__ void poison(Rows& rows, bool any, const unsigned char* bad, const Known& known, int t0) {
    if (any) rows.poison(bad, GROUP, t0, known);
  }
  // What is known of tiles unpacked beforehand, of 64 of them, one a lane.
  static constexpr bool WORDS_IN_RING = false;      // (else it comes with each tile)
  typedef WideTile Word;
  static __device__ __forceinline__ Word word(const Known& known, bool any) { return Word{(known.exists[0] != 0) | (known.exists[1] != 0) << 1 | any << 2}; }
  struct Words {
    int flags;
    __device__ __forceinline__ void take(const AttendArgs& a, size_t tile) { flags = a.tiles[tile].flags; }
    __device__ __forceinline__ void wait() { arrived(flags); }
    __device__ __forceinline__ Word of(int lane) const { return Word{__builtin_amdgcn_readlane(flags, lane)}; }
  };
  static __device__ __forceinline__ Known known(const Word& w) { return Known{{w.flags & 1, w.flags >> 1 & 1}}; }
  static __device__ __forceinline__ bool any_bad(const Word& w) { return w.flags & 4; }
};

template <typename Form>
__device__ __forceinline__ void chunk_items(AttendArgs a) {
  typedef typename Form::Tile Tile;
  constexpr int HALF = 2 * Tile::FRAG;
  __shared__ __attribute__((aligned(16))) char Ks[2][HALF], Vs[3][HALF];
  __shared__ __attribute__((aligned(8))) unsigned char poison[4][Tile::NG * 64];
  __shared__ typename Form::Known known[4];
  __shared__ int poisoned[4];
  __shared__ ChunkScratch scratch;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (tid < 4) poisoned[tid] = -1;
  const bool late = wave >= 4;
  ChunkWalk<kChunkRows, kChunkUnit, kChunkCost> walk;
  if (!walk.start(a, scratch)) return;
  int tag = 0;      // of a tile, over all items
  for (bool more = true; more;) {
    const AttendRequest& rq = walk.rq;
    const int visible = __builtin_amdgcn_readfirstlane(attend_visible(a, rq, walk.tile * kChunkRows, kChunkRows));
    const int u = max(1, (visible + kChunkUnit - 1) / kChunkUnit), j0 = walk.j0, j1 = walk.last_unit(a, u);
    typename Form::Rows rows;
    rows.begin(a, rq, walk.head, walk.tile * kChunkRows + 32 * wave);
    // a lane has the page of one of the next 64 blocks of 32 tokens
    const int32_t* table = a.table + (size_t)walk.r * a.columns;
    const auto pages_from = [&](int j) { return table[min(j * kChunkUnit + 32 * lane, max(visible - 1, 0)) >> a.g.page_shift]; };
    int pages = pages_from(j0);
    arrived(pages);
    rows.wait();
    const auto load = [&](Tile& t, int j) {
      const int k = 2 * (j - j0) & 63;
      if (k == 0 && j != j0) pages = pages_from(j);
      t.load(a, walk.head, j * kChunkUnit, __builtin_amdgcn_readlane(pages, k), __builtin_amdgcn_readlane(pages, k + 1), visible);
    };
    Tile next;
    const int count = visible > 0 ? j1 - j0 : 0;
    int v_at = 0;      // (k + 1) % 3 of the tile that is stored next
    const auto store = [&](int k) {
      next.store(Ks[k & 1], Vs[v_at], known[k & 3], poison[k & 3], &poisoned[k & 3], tag + k);
      v_at = v_at == 2 ? 0 : v_at + 1;
    };
    if (count > 0) {
      load(next, j0);
      store(0);
      if (count > 1) load(next, j0 + 1);
    }
    __syncthreads();
    // In interval k every wave has the values of tile k - 1 and the logits of tile k on the matrix pipe; half of the waves form tile k's
    // probabilities after that, the other half tile k - 1's before it, so that of the two waves of a SIMD one multiplies under the
    // softmax and the unpacking of the other.
    v16f s[2];
    v8bf p[4];
    const auto probabilities = [&](int k) {
      const int t0 = (j0 + k) * kChunkUnit;
      if (t0 < rows.wave_sees) rows.softmax(s, p, t0, known[k & 3], a.scale_log2);
    };
    for (int k = 0, v = 2; k <= count; k++, v = v == 2 ? 0 : v + 1) {      // v = (k + 2) % 3
      if (late && k > 0) probabilities(k - 1);
      if (k > 0 && (j0 + k - 1) * kChunkUnit < rows.wave_sees) {
        Form::before_values(rows, p, known[k - 1 & 3], (j0 + k - 1) * kChunkUnit);
        rows.values(Vs[v], p);
        Form::poison(rows, poisoned[k - 1 & 3] == tag + k - 1, poison[k - 1 & 3], known[k - 1 & 3], (j0 + k - 1) * kChunkUnit);
      }
      if (k < count && (j0 + k) * kChunkUnit < rows.wave_sees) rows.logits(Ks[k & 1], s);
      if (!late && k < count) probabilities(k);
      if (k + 1 < count) {
        store(k + 1);
        if (k + 2 < count) load(next, j0 + k + 2);
      }
      __syncthreads();
    }
    tag += count;
    rows.end(a, rq, walk.head, j0 == 0 && j1 == u, ((size_t)walk.w * 2 + (j0 == 0 ? 1 : 0)) * kChunkRows + 32 * wave + (lane & 31));
    more = walk.next(a, u, j1);
  }
}
template <int D, int GROUP>
__global__ __launch_bounds__(512, 2) void cache_chunk_kernel(AttendArgs a) {
  chunk_items<NibbleChunks<D, GROUP>>(a);
}

// ---- up to 128 query rows a request ---------------------------------------------------------------------------------
// Of the 256 rows of cache_chunk_kernel's tile most do not exist then, and their waves wait.  Here a workgroup's eight waves are RG groups
// of 32 rows by KG = 8 / RG tiles of 64 tokens: all of them unpack KG tiles, then every wave has its rows by one of the tiles, and at an
// item's end the KG sums of a row meet in LDS.  The next tiles' codes are on their way to registers meanwhile; where LDS holds two sets they
// are unpacked while slower waves still multiply.  Unpacking is what bounds it: about 1300 vector instructions for 64 tokens of 128 channels.
// (32 requests of 4096 tokens, 8 heads, 64 rows: 123 -> 87 us, 128 rows 126 -> 107; at d = 64 102 -> 73, 119 -> 91.  With a branch round each tile
// behind the last token, which a request's last unit may have, the tiles are unpacked one after the other: 108.)
template <typename Form, int RG>
__device__ __forceinline__ void span_items(AttendArgs a) {
  typedef typename Form::Tile Tile;
  typedef SpanShape<RG> Shape;
  constexpr int D = Form::D;
  constexpr int KG = Shape::KG, ROWS = Shape::ROWS, UNIT = Shape::UNIT, HALF = 2 * Tile::FRAG, SETS = KG * 4 * HALF <= 131072 ? 2 : 1;
  __shared__ __attribute__((aligned(16))) char lds[SETS][KG][2 * HALF];
  __shared__ __attribute__((aligned(8))) unsigned char poison[SETS][KG][Tile::NG * 64];
  __shared__ typename Form::Known known[SETS][KG];
  __shared__ int poisoned[SETS][KG];
  __shared__ ChunkScratch scratch;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), rg = wave % RG, kg = wave / RG;
  if (tid < SETS * KG) (&poisoned[0][0])[tid] = -1;
  ChunkWalk<ROWS, UNIT, Shape::COST> walk;
  if (!walk.start(a, scratch)) return;
  int tag = 0;      // of a unit, over all items
  for (bool more = true; more;) {
    const AttendRequest& rq = walk.rq;
    const int visible = __builtin_amdgcn_readfirstlane(attend_visible(a, rq, walk.tile * ROWS, ROWS));
    const int u = max(1, (visible + UNIT - 1) / UNIT), j0 = walk.j0, j1 = walk.last_unit(a, u);
    const int count = visible > 0 ? j1 - j0 : 0;
    typename Form::Rows rows;
    rows.begin(a, rq, walk.head, walk.tile * ROWS + 32 * rg);
    // a lane has the page of one of the next 64 blocks of 32 tokens
    const int32_t* table = a.table + (size_t)walk.r * a.columns;
    const auto pages_from = [&](int j) { return table[min(j * UNIT + 32 * lane, max(visible - 1, 0)) >> a.g.page_shift]; };
    int pages = pages_from(j0);
    arrived(pages);
    rows.wait();
    Tile next[KG];
    const auto load = [&](int k) {
      const int at = 2 * KG * k & 63;
      if (at == 0 && k != 0) pages = pages_from(j0 + k);
#pragma unroll
      for (int i = 0; i < KG; i++)
        next[i].load(a, walk.head, (j0 + k) * UNIT + 64 * i, __builtin_amdgcn_readlane(pages, at + 2 * i), __builtin_amdgcn_readlane(pages, at + 2 * i + 1),
                     visible);
    };
    const auto store = [&](int k) {
      const int set = SETS == 2 ? k & 1 : 0;
#pragma unroll
      for (int i = 0; i < KG; i++)
        next[i].store(lds[set][i], lds[set][i] + HALF, known[set][i], poison[set][i], &poisoned[set][i], tag + k);
    };
    const auto attend = [&](int k) {
      const int set = SETS == 2 ? k & 1 : 0, t0 = (j0 + k) * UNIT + 64 * kg;
      if (t0 >= rows.wave_sees) return;
      const typename Form::Known of = known[set][kg];
      v16f s[2];
      v8bf p[4];
      rows.logits(lds[set][kg], s);
      rows.softmax(s, p, t0, of, a.scale_log2);
      Form::before_values(rows, p, of, t0);
      rows.values(lds[set][kg] + HALF, p);
      Form::poison(rows, poisoned[set][kg] == tag + k, poison[set][kg], of, t0);
    };
    if (count > 0) load(0);
    if (SETS == 2) {
      for (int k = -1; k < count; k++) {
        if (k >= 0) attend(k);
        if (k + 1 < count) {
          store(k + 1);
          if (k + 2 < count) load(k + 2);
        }
        __syncthreads();
      }
    } else {
      for (int k = 0; k < count; k++) {
        store(k);
        if (k + 1 < count) load(k + 1);
        __syncthreads();
        attend(k);
        __syncthreads();
      }
    }
    tag += count;
    // the sums of the KG waves of a row (of those that had a tile), two at a time
    const int tiles = count > 1 ? KG : (visible - j0 * UNIT + 63) / 64;
    float* slots = (float*)&lds[0][0][0];
    constexpr int SLOT = D * 32 + 128;
#pragma unroll
    for (int half = KG / 2; half > 0; half /= 2) {
      if (half >= tiles) continue;
      float* slot = slots + ((kg < half ? kg : kg - half) * RG + rg) * SLOT;
      if (kg >= half && kg < 2 * half) {
#pragma unroll
        for (int c = 0; c < ChunkRows<D>::NC; c++)
#pragma unroll
          for (int i = 0; i < 4; i++)
            *(v4f*)(slot + ((4 * c + i) * 64 + lane) * 4) = v4f{rows.o[c][4 * i], rows.o[c][4 * i + 1], rows.o[c][4 * i + 2], rows.o[c][4 * i + 3]};
        slot[D * 32 + lane] = rows.m;
        slot[D * 32 + 64 + lane] = rows.l;
      }
      __syncthreads();
      if (kg < half) {
        const float m = slot[D * 32 + lane], l = slot[D * 32 + 64 + lane], to = fmaxf(rows.m, m), ref = to == -INFINITY ? 0.f : to;
        const float f = __builtin_amdgcn_exp2f(rows.m - ref), g = __builtin_amdgcn_exp2f(m - ref);
#pragma unroll
        for (int c = 0; c < ChunkRows<D>::NC; c++)
#pragma unroll
          for (int i = 0; i < 4; i++) {
            const v4f x = *(const v4f*)(slot + ((4 * c + i) * 64 + lane) * 4);
#pragma unroll
            for (int e = 0; e < 4; e++) rows.o[c][4 * i + e] = rows.o[c][4 * i + e] * f + x[e] * g;
          }
        rows.l = rows.l * f + l * g;
        rows.m = to;
      }
      __syncthreads();
    }
    if (kg == 0) rows.end(a, rq, walk.head, j0 == 0 && j1 == u, ((size_t)walk.w * 2 + (j0 == 0 ? 1 : 0)) * ROWS + 32 * rg + (lane & 31));
    more = walk.next(a, u, j1);
  }
}
template <int D, int GROUP, int RG>
__global__ __launch_bounds__(512, 2) void cache_span_kernel(AttendArgs a) {
  span_items<NibbleChunks<D, GROUP>, RG>(a);
}

// ---- the same with the keys and values unpacked beforehand ------------------------------------------------------------
// Where a request's keys meet several row tiles, unpacking them in each costs more vector instructions than the softmax: a launch writes the
// fragments to the workspace once (as they lie in LDS, 256 d bytes for 64 tokens of a head, request after request, head, tile), and the
// attention copies them into a ring past the registers.
template <typename Form>
__device__ __forceinline__ void unpack_items(AttendArgs a) {
  typedef typename Form::Tile Tile;
  constexpr int D = Form::D;
  __shared__ ChunkScratch s;
  __shared__ typename Form::Known known;
  __shared__ int poisoned;
  const int tid = threadIdx.x, H = a.g.H;
  const int per = (a.R + 511) / 512, r0 = min(tid * per, a.R), r1 = min(r0 + per, a.R);
  unsigned tiles = 0;
  for (int i = r0; i < r1; i++) tiles += chunk_key_tiles(attend_request(a, i));
  unsigned to[2] = {tiles, 0};
  block_scan<8>(to, s.sums);
  if (tid == 0) poisoned = -1;
  if (tid == 511) s.total = (int)to[0];
  __syncthreads();
  const int upto = (int)to[0];
  const AttendShares shares(__builtin_amdgcn_readfirstlane(s.total) * H, gridDim.x);
  if ((int)blockIdx.x >= shares.n) return;
  // (the workspace has room for every request that `cu` can hold, if it rises: what does not fit is left)
  const int begin = shares.begin(blockIdx.x), end = min(shares.begin(blockIdx.x + 1), a.most_tiles);
  if ((upto - (int)tiles) * H <= begin && begin < upto * H) {
    int at = upto - (int)tiles;
    for (int i = r0; i < r1; i++) {
      const int u = chunk_key_tiles(attend_request(a, i));
      if (begin < (at + u) * H) {
        s.found[0] = i;
        s.found[1] = at * H;
        break;
      }
      at += u;
    }
  }
  __syncthreads();
  int r = __builtin_amdgcn_readfirstlane(s.found[0]), x = __builtin_amdgcn_readfirstlane(s.found[1]);
  AttendRequest rq = attend_request(a, r);
  for (int y = begin; y < end; y++) {
    while (y >= x + chunk_key_tiles(rq) * H) {
      x += chunk_key_tiles(rq) * H;
      rq = attend_request(a, ++r);
    }
    const int n = chunk_key_tiles(rq), head = (y - x) / n, j = y - x - head * n;
    const int32_t* table = a.table + (size_t)r * a.columns;
    const int last = max(rq.len - 1, 0), t0 = j * kChunkUnit;
    Tile t;
    t.load(a, head, t0, table[min(t0, last) >> a.g.page_shift], table[min(t0 + 32, last) >> a.g.page_shift], rq.len);
    char* to = a.unpacked + (size_t)y * (256 * D);
    t.store(to, to + 128 * D, known, a.poison + (size_t)y * (Tile::NG * 64), &poisoned, y);
    __syncthreads();
    if (tid == 0) ((typename Form::Word*)a.tiles)[y] = Form::word(known, poisoned == y);
    __syncthreads();
  }
}
template <int D, int GROUP>
__global__ __launch_bounds__(512) void cache_unpack_kernel(AttendArgs a) {
  unpack_items<NibbleChunks<D, GROUP>>(a);
}

constexpr int kWideStages = 4;

template <typename Form>
__device__ __forceinline__ void wide_items(AttendArgs a) {
  constexpr int D = Form::D;
  constexpr int TILE = 256 * D, COPIES = TILE / 8 / 1024, LOADS = COPIES + (Form::WORDS_IN_RING ? 1 : 0);
  __shared__ __attribute__((aligned(16))) char ring[kWideStages][TILE];
  __shared__ __attribute__((aligned(16))) char word_ring[kWideStages][Form::WORDS_IN_RING ? 256 : 0];      // (all waves copy them, to the same place)
  __shared__ ChunkScratch scratch;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  ChunkWalk<kChunkRows, kChunkUnit, kChunkCost> walk;
  if (!walk.start(a, scratch)) return;
  const bool late = wave >= 4;
  for (bool more = true; more;) {
    const AttendRequest& rq = walk.rq;
    const int visible = __builtin_amdgcn_readfirstlane(attend_visible(a, rq, walk.tile * kChunkRows, kChunkRows));
    const int u = max(1, (visible + kChunkUnit - 1) / kChunkUnit), j0 = walk.j0, j1 = walk.last_unit(a, u);
    int count = visible > 0 ? j1 - j0 : 0;
    size_t tile0 = (size_t)walk.before * a.g.H + (size_t)walk.head * chunk_key_tiles(rq) + j0;      // of the unpacked ones
    if (tile0 + max(count, 1) > (size_t)a.most_tiles) tile0 = count = 0;
    typename Form::Rows rows;
    rows.begin(a, rq, walk.head, walk.tile * kChunkRows + 32 * wave);
    typename Form::Words words;        // of the next 64 tiles, one a lane
    if constexpr (!Form::WORDS_IN_RING) words.take(a, tile0 + min(lane, max(count - 1, 0)));
    const auto fetch = [&](int k) {
      const gbytes_t from = uniform(a.unpacked + (tile0 + k) * TILE + wave * (COPIES * 1024));
#pragma unroll
      for (int c = 0; c < COPIES; c++) ring_copy<16>(from, c * 1024 + lane * 16, ring[k % kWideStages] + wave * (COPIES * 1024) + c * 1024);
      if constexpr (Form::WORDS_IN_RING) ring_copy<4>(uniform((const typename Form::Word*)a.tiles + tile0 + k), lane * 4, word_ring[k % kWideStages]);
    };
    // (intervals as in cache_chunk_kernel)
    v16f s[2];
    v8bf p[4];
    typename Form::Word word = {}, word_before = {};
    const auto probabilities = [&](int k, const typename Form::Word& word) {
      const int t0 = (j0 + k) * kChunkUnit;
      if (t0 < rows.wave_sees) rows.softmax(s, p, t0, Form::known(word), a.scale_log2);
    };
    if constexpr (!Form::WORDS_IN_RING) words.wait();
    rows.wait();
    compiler_fence();
    fetch(0);
    if (count > 1) fetch(1);
    for (int k = 0; k <= count; k++) {
      compiler_fence();
      if (k + 1 < count) __builtin_amdgcn_s_waitcnt(vmcnt_only(LOADS));
      else __builtin_amdgcn_s_waitcnt(vmcnt_only(0));
      barrier_lds_only();                  // the tile has landed, and every wave is through with the one two before it
      compiler_fence();
      if (k + 2 < count) fetch(k + 2);
      compiler_fence();
      if constexpr (!Form::WORDS_IN_RING) {
        if (k % 64 == 0 && k != 0) {
          words.take(a, tile0 + min(k + lane, count - 1));
          words.wait();
        }
      }
      word_before = word;
      if constexpr (Form::WORDS_IN_RING) word = ((const typename Form::Word*)word_ring[k % kWideStages])->uniform(0);
      else word = words.of(k % 64);
      if (late && k > 0) probabilities(k - 1, word_before);
      if (k > 0 && (j0 + k - 1) * kChunkUnit < rows.wave_sees) {
        Form::before_values(rows, p, Form::known(word_before), (j0 + k - 1) * kChunkUnit);
        rows.values(ring[(k - 1) % kWideStages] + TILE / 2, p);
        Form::poison(rows, Form::any_bad(word_before), a.poison + (tile0 + k - 1) * (Form::Tile::NG * 64), Form::known(word_before), (j0 + k - 1) * kChunkUnit);
      }
      if (k < count) {
        if ((j0 + k) * kChunkUnit < rows.wave_sees) rows.logits(ring[k % kWideStages], s);
        if (!late) probabilities(k, word);
      }
    }
    rows.end(a, rq, walk.head, j0 == 0 && j1 == u, ((size_t)walk.w * 2 + (j0 == 0 ? 1 : 0)) * kChunkRows + 32 * wave + (lane & 31));
    more = walk.next(a, u, j1);
    barrier_all_memory();                  // (the ring is the next item's)
  }
}
template <int D, int GROUP>
__global__ __launch_bounds__(512, D == 64 ? 4 : 2) void cache_wide_kernel(AttendArgs a) {
  wide_items<NibbleChunks<D, GROUP>>(a);
}

}  // namespace sage
