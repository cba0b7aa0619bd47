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

// 64 tokens on their way from the pages to bf16 fragments: waves 0 to 3 have K's, the others V's.
template <int D, int GROUP>
struct ChunkTile {
  static constexpr int NG = D / GROUP, FRAG = D / 16 * 1024;     // bytes of 32 tokens of K, of 32 tokens' worth of V
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
  __device__ __forceinline__ void store(char* K, char* V, int* exists, unsigned char* poison, int* poisoned, int tag) const {
    const int tid = threadIdx.x, u = tid & 255;
    if (tid < 256) {
      const int rho = u & 31, q = (u >> 5) & 3, b = u >> 7;
      if ((u & 127) == 0) exists[b] = valid;
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
#pragma unroll
    for (int pair = 0; pair < 2; pair++) {      // channels m + 16 j, j = 2 pair and 2 pair + 1
      const v4i& sc = GROUP == 32 && pair == 1 ? s1 : s0;
      float s[8], s8[8];
      unsigned bad = 0;
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const float x = i % 2 == 0 ? low_bf16(sc[i / 2]) : high_bf16(sc[i / 2]);
        const bool number = fabsf(x) < INFINITY;
        if (!number && i < valid) bad |= 1u << i;
        s[i] = i < valid && number ? x : 0.f;
        s8[i] = -8.f * s[i];
      }
      if (__any(bad != 0)) *poisoned = tag;
      if (m == 0 && (GROUP == 32 || pair == 0)) {
        const int group = f * (64 / GROUP) + pair;
#pragma unroll
        for (int i = 0; i < 8; i++) poison[group * 64 + 8 * o + i] = bad >> i & 1;
      }
#pragma unroll
      for (int k = 0; k < 2; k++) {
        const int j = 2 * pair + k;
        v4i x;
#pragma unroll
        for (int i = 0; i < 4; i++) {
          const unsigned w = (unsigned)code[i] >> 4 * j;
          x[i] = pack_bf16(__builtin_fmaf((float)(w & 15), s[2 * i], s8[2 * i]), __builtin_fmaf((float)(w >> 16 & 15), s[2 * i + 1], s8[2 * i + 1]));
        }
        *(v4i*)(V + ((2 * f + pair) * 4 + (o >> 1)) * 1024 + ((o & 1) * 32 + 16 * k + m) * 16) = x;
      }
    }
  }
};

// Line of what is dealt out: request, then head, then row tile of 256, each attend_units(tile) + kChunkCost; or (not split) one each,
// request, then row tile from the last, which sees most, then head.
constexpr int kChunkCost = 6;
__device__ __forceinline__ int chunk_tiles(int rows) { return (rows + kChunkRows - 1) / kChunkRows; }
__device__ __forceinline__ int chunk_units(const AttendArgs& a, const AttendRequest& q, int tile) {
  return max(1, (attend_visible(a, q, tile * kChunkRows, kChunkRows) + kChunkUnit - 1) / kChunkUnit);
}
// of a request and head
__device__ __forceinline__ int chunk_weight(const AttendArgs& a, const AttendRequest& q) {
  const int tiles = chunk_tiles(q.rows);
  if (!a.split) return tiles;
  int w = 0;
  for (int t = 0; t < tiles; t++) w += chunk_units(a, q, t) + kChunkCost;
  return w;
}
__device__ __forceinline__ int chunk_cut(int offset) { return max(0, offset - kChunkCost); }

template <int D, int GROUP>
__global__ __launch_bounds__(512, 2) void cache_chunk_kernel(AttendArgs a) {
  typedef ChunkTile<D, GROUP> Tile;
  constexpr int NK = D / 16, NC = D / 32, HALF = 2 * Tile::FRAG;
  __shared__ __attribute__((aligned(16))) char Ks[2][HALF], Vs[2][HALF];
  __shared__ unsigned char poison[2][Tile::NG * 64];
  __shared__ int exists[2][2], poisoned[2];
  __shared__ int wave_units[8], found[3];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, h = lane >> 5;
  const int H = a.g.H;

  const int per = (a.R + 511) / 512, r0 = min(tid * per, a.R), r1 = min(r0 + per, a.R);
  int mine = 0;
  for (int r = r0; r < r1; r++) mine += chunk_weight(a, attend_request(a, r));
  int upto = mine;
  for (int k = 1; k < 64; k <<= 1) {
    const int u = __shfl_up(upto, k);
    if (lane >= k) upto += u;
  }
  if (lane == 63) wave_units[wave] = upto;
  if (tid < 2) poisoned[tid] = -1;
  __syncthreads();
  int units = 0;
#pragma unroll
  for (int k = 0; k < 8; k++) {
    if (k < wave) upto += wave_units[k];
    units += wave_units[k];
  }
  const AttendShares shares(__builtin_amdgcn_readfirstlane(units) * H, a.workgroups);
  // (neighbours in the line to one XCD, whose L2 then holds a head's keys for all its row tiles)
  const int w = a.split && shares.n == a.workgroups && shares.n % 8 == 0 ? (blockIdx.x & 7) * (shares.n / 8) + (blockIdx.x >> 3) : blockIdx.x;
  if (tid == 0) a.joins[w] = int4{0, 0, 0, 0};
  if (w >= shares.n) return;
  const int begin = shares.begin(w), end = shares.begin(w + 1);
  if ((upto - mine) * H <= begin && begin < upto * H) {
    int at = upto - mine;
    for (int r = r0; r < r1; r++) {
      const int u = chunk_weight(a, attend_request(a, r));
      if (begin < (at + u) * H) {
        found[0] = r;
        found[1] = at * H;
        found[2] = u;
        break;
      }
      at += u;
    }
  }
  __syncthreads();
  int r = __builtin_amdgcn_readfirstlane(found[0]), weight = __builtin_amdgcn_readfirstlane(found[2]);
  int x = __builtin_amdgcn_readfirstlane(found[1]);      // where (r, head, tile) begins in the line
  int head, tile;
  AttendRequest rq = attend_request(a, r);
  if (a.split) {
    head = (begin - x) / weight;
    x += head * weight;
    tile = 0;
    for (int u; x + (u = chunk_units(a, rq, tile) + kChunkCost) <= begin; tile++) x += u;
  } else {
    const int i = begin - x;
    tile = weight - 1 - i / H;
    head = i - i / H * H;
    x = begin;
  }
  head = __builtin_amdgcn_readfirstlane(head);
  tile = __builtin_amdgcn_readfirstlane(tile);
  x = __builtin_amdgcn_readfirstlane(x);
  int j0 = a.split ? chunk_cut(begin - x) : 0;

  int tag = 0;      // of a tile, over all items
  while (a.split ? chunk_cut(end - x) > j0 : x < end) {
    const int row0 = tile * kChunkRows;
    const int visible = __builtin_amdgcn_readfirstlane(attend_visible(a, rq, row0, kChunkRows));
    const int u = max(1, (visible + kChunkUnit - 1) / kChunkUnit), j1 = a.split ? min(u, chunk_cut(end - x)) : u;
    if (j0 > 0 && chunk_cut(shares.begin(w - 1) - x) == 0 && tid == 0)      // the first border in this item
      a.joins[w] = int4{shares.owner(x + u + kChunkCost - 1) - w + 2, r, head, row0};
    // the wave's queries
    const int row = row0 + 32 * wave + n, token = row / a.G;
    const bool real = row < rq.rows;
    v4i q[NK];
    {
      const __bf16* p = a.Q + (int64_t)(rq.begin + (real ? token : 0)) * a.q_token + (int64_t)(head * a.G + (real ? row - token * a.G : 0)) * a.q_head + 8 * h;
#pragma unroll
      for (int s = 0; s < NK; s++) q[s] = real ? *(const v4i*)(p + 16 * s) : v4i{0, 0, 0, 0};
    }
    const int sees = real && a.causal ? min(rq.len, rq.first_sees + token) : rq.len;
    const int wave_row0 = row0 + 32 * wave;
    const int all_see = __builtin_amdgcn_readfirstlane(a.causal ? rq.first_sees + wave_row0 / a.G : rq.len);
    const int wave_sees = __builtin_amdgcn_readfirstlane(wave_row0 < rq.rows ? attend_visible(a, rq, wave_row0, 32) : 0);
    v16f o[NC];
#pragma unroll
    for (int c = 0; c < NC; c++) o[c] = v16f{};
    float m = -INFINITY, l = 0.f;

    // a lane has the page of one of the next 64 blocks of 32 tokens
    const int32_t* table = a.table + (size_t)r * a.columns;
    const auto pages_from = [&](int j) { return table[min(j * kChunkUnit + 32 * lane, max(visible - 1, 0)) >> a.g.page_shift]; };
    int pages = pages_from(j0);
    const auto load = [&](Tile& t, int j) {
      const int k = 2 * (j - j0) & 63;
      if (k == 0 && j != j0) pages = pages_from(j);
      t.load(a, head, j * kChunkUnit, __builtin_amdgcn_readlane(pages, k), __builtin_amdgcn_readlane(pages, k + 1), visible);
    };
    Tile next;
    const int count = visible > 0 ? j1 - j0 : 0;
    if (count > 0) {
      load(next, j0);
      next.store(Ks[0], Vs[0], exists[0], poison[0], &poisoned[0], tag);
      if (count > 1) load(next, j0 + 1);
    }
    __syncthreads();
    for (int k = 0; k < count; k++) {
      const int t0 = (j0 + k) * kChunkUnit, at = k & 1;
      const bool busy = t0 < wave_sees;
      v16f s[2];
      if (busy) {
#pragma unroll
        for (int b = 0; b < 2; b++) {
          s[b] = v16f{};
#pragma unroll
          for (int c = 0; c < NK; c++) {
            const v4i f = *(const v4i*)(Ks[at] + b * Tile::FRAG + c * 1024 + lane * 16);
            s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16(f), as_bf16(q[c]), s[b], 0, 0, 0);
          }
        }
      }
      if (k + 1 < count) {
        next.store(Ks[at ^ 1], Vs[at ^ 1], exists[at ^ 1], poison[at ^ 1], &poisoned[at ^ 1], tag + 1);
        if (k + 2 < count) load(next, j0 + k + 2);
      }
      if (busy) {
        if (t0 + kChunkUnit > all_see || exists[at][0] + exists[at][1] != 2) {
#pragma unroll
          for (int b = 0; b < 2; b++) {
            const int behind = exists[at][b] ? sees - t0 - 32 * b - 8 * h : 0;
#pragma unroll
            for (int i = 0; i < 16; i++) s[b][i] = 16 * (i / 8) + i % 8 < behind ? s[b][i] : -INFINITY;
          }
        }
        float top = -INFINITY;
#pragma unroll
        for (int b = 0; b < 2; b++)
#pragma unroll
          for (int i = 0; i < 16; i++) top = fmaxf(top, s[b][i]);
        if (__any(top * a.scale_log2 > m + 8.f)) {
          const float to = fmaxf(m, half_swap_max_f32(top) * a.scale_log2);
          const float f = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - to);
#pragma unroll
          for (int c = 0; c < NC; c++) o[c] *= f;
          l *= f;
          m = to;
        }
        const float ref = m == -INFINITY ? 0.f : m;
        v8bf p[4];
#pragma unroll
        for (int b = 0; b < 2; b++) {
#pragma unroll
          for (int i = 0; i < 16; i++) {
            s[b][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], a.scale_log2, -ref));
            l += s[b][i];
          }
#pragma unroll
          for (int kk = 0; kk < 2; kk++)
            p[2 * b + kk] = as_bf16(v4i{pack_bf16(s[b][8 * kk], s[b][8 * kk + 1]), pack_bf16(s[b][8 * kk + 2], s[b][8 * kk + 3]),
                                        pack_bf16(s[b][8 * kk + 4], s[b][8 * kk + 5]), pack_bf16(s[b][8 * kk + 6], s[b][8 * kk + 7])});
        }
#pragma unroll
        for (int c = 0; c < NC; c++)
#pragma unroll
          for (int kk = 0; kk < 4; kk++) {
            const v4i f = *(const v4i*)(Vs[at] + (c * 4 + kk) * 1024 + lane * 16);
            o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16(f), p[kk], o[c], 0, 0, 0);
          }
        if (poisoned[at] == tag) {
          for (int t = 0; t < kChunkUnit; t++)
#pragma unroll
            for (int c = 0; c < NC; c++)
              if (poison[at][32 * c / GROUP * 64 + t] && exists[at][t / 32] && t < sees - t0) o[c] += __builtin_nanf("");
        }
      }
      tag++;
      __syncthreads();
    }
    l = half_swap_sum_f32(l);
    if (real) {
      if (j0 == 0 && j1 == u) {
        const bool any = !(l == 0.f);
        const float f = any ? 1.f / l : 0.f;
        const int hq = head * a.G + row - token * a.G;
        __bf16* p = a.O + ((int64_t)(rq.begin + token) * a.Hq + hq) * D;
#pragma unroll
        for (int c = 0; c < NC; c++) {
          int d[4][2];
#pragma unroll
          for (int i = 0; i < 4; i++) {
            float y[4];
#pragma unroll
            for (int e = 0; e < 4; e++) {
              const float mean = a.v_mean != nullptr ? a.v_mean[head * D + 32 * c + 8 * i + 4 * h + e] : 0.f;
              y[e] = any ? o[c][4 * i + e] * f + mean : 0.f;
            }
            d[i][0] = pack_bf16(y[0], y[1]);
            d[i][1] = pack_bf16(y[2], y[3]);
            *(v2i*)(p + 32 * c + 8 * i + 4 * h) = v2i{d[i][0], d[i][1]};
          }
        }
        if (h == 0 && a.LSE != nullptr) a.LSE[(int64_t)hq * a.T + rq.begin + token] = any ? (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : -INFINITY;
      } else {
        const size_t at = ((size_t)w * 2 + (j0 == 0 ? 1 : 0)) * kChunkRows + 32 * wave + n;
#pragma unroll
        for (int c = 0; c < NC; c++)
#pragma unroll
          for (int i = 0; i < 4; i++)
            *(v4f*)(a.sums + at * D + 32 * c + 8 * i + 4 * h) = v4f{o[c][4 * i], o[c][4 * i + 1], o[c][4 * i + 2], o[c][4 * i + 3]};
        if (h == 0) a.stats[at] = float2{m, l};
      }
    }
    // the next item
    if (j1 < u || !a.split) break;        // (not split, a workgroup has one)
    x += u + kChunkCost;
    j0 = 0;
    if (++tile == chunk_tiles(rq.rows)) {
      tile = 0;
      if (++head == H) {
        head = 0;
        do r++; while (r < a.R && (rq = attend_request(a, r)).rows == 0);
        if (r == a.R) break;
        r = __builtin_amdgcn_readfirstlane(r);
      }
    }
  }
}

}  // namespace sage
