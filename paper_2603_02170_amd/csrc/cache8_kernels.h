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

constexpr float kLeast8 = 0x1p-100f;      // of magnitudes stored, but for zero
// The largest magnitude of a block as it is stored, from its bits (of an infinity and a NaN the largest).
__device__ __forceinline__ float magnitude8(unsigned top) {
  return __uint_as_float(top < 0x0D800000u ? 0u : top >= 0x7F000000u ? 0x7FC00000u : top);
}
// What turns a block's numbers into codes, and codes held into codes of a larger magnitude.
__device__ __forceinline__ float to_codes8(float a) { return a > 0.f ? __fdiv_rn(127.f, a) : 0.f; }
// Four numbers times r, rounded to nearest: the sum with 1.5 * 2^23 has the integer in its low bits.  (The product is rounded first, as the header has it:
// half of the magnitude is a tie in it, not in an fma.)
__device__ __forceinline__ unsigned codes8(const float* x, float r) {
#pragma clang fp contract(off)
  unsigned u[4];
#pragma unroll
  for (int i = 0; i < 4; i++) u[i] = __float_as_uint(x[i] * r + 12582912.f);
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(u[3], u[2], 0x0C0C0400u), __builtin_amdgcn_perm(u[1], u[0], 0x0C0C0400u), 0x05040100u);
}
__device__ __forceinline__ unsigned recode8(unsigned w, float f) {      // four codes of another scale
  float x[4];
#pragma unroll
  for (int i = 0; i < 4; i++) x[i] = (float)(signed char)(w >> 8 * i);
  return codes8(x, f);
}

// 8 tokens (an octet) of a head are the work of D / 2 lanes, and a wave has EACH at a time.  K: a lane has 16 channels of a token, as they lie in
// the page.  V: lane (j, q, i) has 16 bytes of channels c = 32 j + 4 q + i and c + 16, which turned are channels 32 j + 4 q .. and 16 more of tokens i
// and 4 + i.  (A byte at a time, of V in LDS or in the page, storing 7700 tokens of 8 heads of 128 took 19.1 us and
// reading them 22.8, now 14.5 and 13.9.)
template <int D>
struct Octet8 {
  static constexpr int LANES = D / 2, EACH = 64 / LANES;
  int k_token, k_channel;                 // of the octet
  int v_token, v_channel, v_byte;         // (and 4 more; and 16 more); of the bytes, from the octet's first
  __device__ __forceinline__ Octet8() {
    const int l = threadIdx.x % LANES;
    k_token = l / (D / 16);
    k_channel = l % (D / 16) * 16;
    v_token = l & 3;
    v_channel = (l >> 4) * 32 + (l >> 2 & 3) * 4;
    v_byte = (l >> 4) * 1024 + (l & 15) * 16;
  }
  // of the octet's first token
  static __device__ __forceinline__ int v_at(const CacheGeometry& g, int token) { return g.page() * D + (token >> 5) * (32 * D) + (token >> 3 & 3) * 256; }
};

// 4 x 4 bytes over the four lanes of a quad: byte k of lane i to byte i of lane k.
struct Turn8 {
  unsigned one, two;
  __device__ __forceinline__ Turn8() : one(threadIdx.x & 1 ? 0x03070105u : 0x06020400u), two(threadIdx.x & 2 ? 0x03020706u : 0x05040100u) {}
  __device__ __forceinline__ unsigned operator()(unsigned w) const {
    w = __builtin_amdgcn_perm((unsigned)__builtin_amdgcn_mov_dpp((int)w, 0xB1, 0xF, 0xF, true), w, one);      // (lanes 1, 0, 3, 2)
    return __builtin_amdgcn_perm((unsigned)__builtin_amdgcn_mov_dpp((int)w, 0x4E, 0xF, 0xF, true), w, two);   // (lanes 2, 3, 0, 1)
  }
};

typedef __bf16 v4bf __attribute__((ext_vector_type(4)));

// Rows of a call whose slots rise by one inside a unit of tokens (a block, an octet) are a run, which its first row finds.  A wave looks at
// 64 rows and the 64 behind them with one trip to memory: the runs that begin in the first `window` of them.
struct Runs8 {
  int64_t slot;                     // of the lane's row
  uint64_t firsts, on, on_behind;   // rows that begin a run; that go on with the one before
  __device__ __forceinline__ Runs8(const StoreArgs& a, int row0, int window, int unit, bool all) {
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)row0 + lane, end = (int64_t)a.g.pages << a.g.page_shift;
    const auto at = [&](int64_t r) { return r >= 0 && r < a.T ? a.slots[r] : -1; };
    const int64_t before = at(row - 1), before_behind = at(row + 63), behind = at(row + 64);
    slot = at(row);
    const auto valid = [&](int64_t x) { return x >= 0 && x < end; };
    const auto goes_on = [&](int64_t x, int64_t y) { return valid(x) && y >= 0 && x - 1 == y && (x & (unit - 1)) != 0; };
    on = __ballot(goes_on(slot, before));
    on_behind = __ballot(goes_on(behind, before_behind));
    firsts = __ballot(lane < window && row < a.T && (all || valid(slot))) & ~on;      // (all: rows without a slot, each by itself)
  }
  __device__ __forceinline__ int length(int i) const {      // of the run that begins at row i
    const uint64_t rest = i == 63 ? on_behind : on >> (i + 1) | on_behind << (63 - i);
    return rest == ~0ull ? 64 : 1 + __builtin_ctzll(~rest);
  }
};

// One workgroup has a run of a block's keys or values (blockIdx.z), for a head: the block's largest magnitude has to be known before the first code is written,
// and where it grows the codes held are written again.  A thread has 16 numbers at a time.  (With 16 of K and 16 of V registers halve the waves of a CU:
// 7700 tokens of 8 heads
// 15.8 us, so 14.5; a thread having two such in turn, and the slots asked for once more for each run, 20.0.)
template <int D, int BLOCK, int WAVES, bool VALUES>
__device__ __forceinline__ void store_runs(const StoreArgs& a, int window, unsigned (*tops)[WAVES]) {
  typedef Octet8<D> Octet;
  constexpr int THREADS = 64 * WAVES, AT_ONCE = WAVES * Octet::EACH;      // octets
  constexpr bool ONCE = AT_ONCE >= BLOCK / 8;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h = blockIdx.y;
  const Octet me;
  const Turn8 turn;
  const float* mean = VALUES ? a.v_mean : a.k_mean;
  const __bf16* from_head = VALUES ? a.V + h * a.vs[1] + me.v_channel : a.K + h * a.ks[1] + me.k_channel;
  const int64_t stride = VALUES ? a.vs[0] : a.ks[0];
  const int row0 = blockIdx.x * window;
  const Runs8 runs(a, row0, window, BLOCK, false);
  int side = 0;
  for (uint64_t firsts = runs.firsts; firsts != 0; firsts &= firsts - 1, side ^= 1) {
    const int index = __builtin_ctzll(firsts), first = row0 + index, n = runs.length(index);
    const int64_t slot0 = (int64_t)((uint64_t)(unsigned)__builtin_amdgcn_readlane((int)(runs.slot >> 32), index) << 32 |
                                    (unsigned)__builtin_amdgcn_readlane((int)runs.slot, index));
    const int o = (int)(slot0 & (BLOCK - 1));
    const int at = (int)(slot0 & (a.g.page() - 1)) - o;          // the block's first token in its page
    unsigned char* p = a.pool + ((size_t)(slot0 >> a.g.page_shift) * a.g.H + h) * Bytes8<D>::head_bytes(a.g);
    float* magnitude = (float*)(p + Bytes8<D>::magnitudes(a.g) + at / 4) + (VALUES ? 1 : 0);
    const float held = o > 0 ? *magnitude : 0.f;
    const int octets = ((o + n + 7) >> 3) - (o >> 3), rounds = ONCE ? 1 : (octets + AT_ONCE - 1) / AT_ONCE;      // with new tokens
    // The thread's octet of the block: all of them at once, so that the codes held are on their way with the new numbers; or, in rounds, those with new tokens.
    int t0 = 8 * ((ONCE ? 0 : o >> 3) + tid / Octet::LANES);
    const auto bytes_of = [&](int t0) { return (uint4*)(p + (VALUES ? Octet::v_at(a.g, at + t0) + me.v_byte : Bytes8<D>::k(at + t0 + me.k_token, me.k_channel))); };
    uint4 codes = {0, 0, 0, 0};      // held
    if (ONCE && (VALUES ? t0 < o || (t0 < o + n && o + n < t0 + 8) : t0 + me.k_token < o)) codes = *bytes_of(t0);
    const auto is_new = [&](int t) { return t >= o && t < o + n; };
    v4bf x[4];      // K: 16 channels of a token; V: [2 * (token i or 4 + i) + (channels c or c + 16)]
    const auto fetch = [&] {
#pragma unroll
      for (int i = 0; i < 4; i++) x[i] = v4bf{};
      if (VALUES) {
#pragma unroll
        for (int half = 0; half < 2; half++) {
          const int t = t0 + me.v_token + 4 * half;
          if (!is_new(t)) continue;
          const __bf16* y = from_head + (int64_t)(first + t - o) * stride;
          x[2 * half] = *(const v4bf*)y;
          x[2 * half + 1] = *(const v4bf*)(y + 16);
        }
      } else if (is_new(t0 + me.k_token)) {
        const __bf16* y = from_head + (int64_t)(first + t0 + me.k_token - o) * stride;
        const v8bf lo = *(const v8bf*)y, hi = *(const v8bf*)(y + 8);
#pragma unroll
        for (int e = 0; e < 4; e++) {
          x[0][e] = lo[e];
          x[1][e] = lo[4 + e];
          x[2][e] = hi[e];
          x[3][e] = hi[4 + e];
        }
      }
    };
    const auto numbers = [&](int i, float* f) {
      typedef v4f v4f_dword __attribute__((aligned(4)));
#pragma unroll
      for (int e = 0; e < 4; e++) f[e] = (float)x[i][e];
      if (mean == nullptr) return;
      const v4f m = *(const v4f_dword*)(mean + h * D + (VALUES ? me.v_channel + 16 * (i & 1) : me.k_channel + 4 * i));
#pragma unroll
      for (int e = 0; e < 4; e++) f[e] -= m[e];
    };
    unsigned top = 0;
    float f[4];
#pragma unroll 1
    for (int round = 0; round < rounds; round++, t0 += 8 * AT_ONCE) {
      fetch();
#pragma unroll
      for (int i = 0; i < 4; i++) {
        if (!is_new(t0 + (VALUES ? me.v_token + 4 * (i >> 1) : me.k_token))) continue;
        numbers(i, f);
#pragma unroll
        for (int e = 0; e < 4; e++) top = max(top, __float_as_uint(f[e]) & 0x7FFFFFFFu);
      }
    }
    t0 -= 8 * AT_ONCE * rounds;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) top = max(top, (unsigned)__shfl_xor((int)top, k));
    if (lane == 0) tops[side][wave] = top;
    __syncthreads();               // (the next run has the other side of them)
    top = __float_as_uint(held) & 0x7FFFFFFFu;
#pragma unroll
    for (int w = 0; w < WAVES; w++) top = max(top, tops[side][w]);
    const float now = magnitude8(top), r = to_codes8(now);
    const bool grown = o > 0 && now > held;
    const float again = grown ? __fdiv_rn(held, now) : 1.f;
    const auto recode = [&](const uint4& w) { return uint4{recode8(w.x, again), recode8(w.y, again), recode8(w.z, again), recode8(w.w, again)}; };
#pragma unroll 1
    for (int round = 0; round < rounds; round++, t0 += 8 * AT_ONCE) {
      if (!ONCE && rounds > 1) fetch();      // (once more)
      unsigned w[4];
#pragma unroll
      for (int i = 0; i < 4; i++) {
        numbers(i, f);
        w[i] = codes8(f, r);
      }
      if (!VALUES) {
        if (is_new(t0 + me.k_token)) *bytes_of(t0) = uint4{w[0], w[1], w[2], w[3]};
        else if (ONCE && grown && t0 + me.k_token < o) *bytes_of(t0) = recode(codes);
        continue;
      }
      const int from = min(max(o - t0, 0), 8), upto = min(max(o + n - t0, 0), 8);      // new tokens of the octet
      uint4 z = {turn(w[0]), turn(w[2]), turn(w[1]), turn(w[3])};                      // channel c, tokens 0 .. 3 and 4 .. 7; channel c + 16
      if (upto > from || (ONCE && grown && from > 0)) {
        if (from > 0 || upto < 8) {
          const uint4 old = ONCE ? codes : *bytes_of(t0), y = grown ? recode(old) : old;
          const auto bytes = [](int n) { return n == 8 ? ~0ull : (1ull << 8 * n) - 1; };
          const uint64_t below = bytes(from), fresh = bytes(upto) & ~below, behind = ~(below | fresh);      // (behind the new tokens nothing is the call's)
          const auto merge = [&](unsigned z, unsigned y, unsigned old, int half) {
            return (z & (unsigned)(fresh >> half)) | (y & (unsigned)(below >> half)) | (old & (unsigned)(behind >> half));
          };
          z = uint4{merge(z.x, y.x, old.x, 0), merge(z.y, y.y, old.y, 32), merge(z.z, y.z, old.z, 0), merge(z.w, y.w, old.w, 32)};
        }
        *bytes_of(t0) = z;
      }
    }
    if (!ONCE && grown) {      // octets of tokens held (of K up to the last of them)
      constexpr int EACH = VALUES ? Octet::LANES : D / 16;
#pragma unroll 1
      for (int i = tid; i < (VALUES ? o >> 3 : o) * EACH; i += THREADS) {
        uint4* q = (uint4*)(p + (VALUES ? Octet::v_at(a.g, at + i / EACH * 8) + (i % EACH >> 4) * 1024 + (i & 15) * 16 : Bytes8<D>::k(at + i / EACH, i % EACH * 16)));
        *q = recode(*q);
      }
    }
    if (tid < BLOCK / 32) magnitude[2 * tid] = now;
  }
}
template <int D, int BLOCK, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void cache8_append_kernel(StoreArgs a, int window) {
  __shared__ unsigned tops[2][WAVES];
  if (blockIdx.z == 0) store_runs<D, BLOCK, WAVES, false>(a, window, tops);
  else store_runs<D, BLOCK, WAVES, true>(a, window, tops);
}

// The tokens of an octet that stand one after the other are read together; a wave has some of those that begin in the workgroup's `window` rows.
template <int D>
__global__ __launch_bounds__(256) void cache8_read_kernel(StoreArgs a, int window) {
  typedef Octet8<D> Octet;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h = blockIdx.y;
  const Octet me;
  const Turn8 turn;
  const int row0 = blockIdx.x * window;
  const int64_t end = (int64_t)a.g.pages << a.g.page_shift;
  const Runs8 runs(a, row0, window, 8, true);
  uint64_t firsts = runs.firsts;
  for (int skip = wave * Octet::EACH; skip > 0; skip--) firsts &= firsts - 1;
  while (firsts != 0) {
    uint64_t mine = firsts;
    if (lane >= Octet::LANES && (mine & (mine - 1)) != 0) mine &= mine - 1;      // (of two octets the second; where there is none both are the first)
    for (int skip = 4 * Octet::EACH; skip > 0; skip--) firsts &= firsts - 1;
    const int index = __builtin_ctzll(mine), first = row0 + index, n = runs.length(index);
    const int64_t slot0 = __shfl(runs.slot, index);
    const bool stored = slot0 >= 0 && slot0 < end;
    const int at = stored ? (int)(slot0 & (a.g.page() - 1)) : 0, t0 = at & ~7, o = at & 7;
    const unsigned char* p = a.pool + ((size_t)(stored ? slot0 >> a.g.page_shift : 0) * a.g.H + h) * Bytes8<D>::head_bytes(a.g);
    const uint4 kw = *(const uint4*)(p + Bytes8<D>::k(t0 + me.k_token, me.k_channel));
    const uint4 vw = *(const uint4*)(p + Octet::v_at(a.g, t0) + me.v_byte);
    const float2 top = *(const float2*)(p + Bytes8<D>::magnitudes(a.g) + t0 / 32 * 8);
    const float ks = stored ? __fdiv_rn(top.x, 127.f) : 0.f, vs = stored ? __fdiv_rn(top.y, 127.f) : 0.f;
    const auto row_of = [&](int t) { return t >= o && t < o + n ? first + t - o : -1; };      // of the octet's token t, if the call asks for it here
    const auto numbers = [&](unsigned w, float s, const float* mean, int c, __bf16* to) {      // four of them
#pragma clang fp contract(off)
      typedef v4f v4f_dword __attribute__((aligned(4)));
      v4f m = {0.f, 0.f, 0.f, 0.f};
      if (mean != nullptr && stored) m = *(const v4f_dword*)(mean + h * D + c);
#pragma unroll
      for (int e = 0; e < 4; e++) to[e] = (__bf16)(stored ? (float)(signed char)(w >> 8 * e) * s + m[e] : 0.f);
    };
    const int row = row_of(me.k_token);
    if (row >= 0) {
      v8bf x[2];
      const unsigned w[4] = {kw.x, kw.y, kw.z, kw.w};
#pragma unroll
      for (int i = 0; i < 4; i++) {
        __bf16 f[4];
        numbers(w[i], ks, a.k_mean, me.k_channel + 4 * i, f);
#pragma unroll
        for (int e = 0; e < 4; e++) x[i / 2][4 * (i % 2) + e] = f[e];
      }
      __bf16* to = a.Ko + ((size_t)row * a.g.H + h) * D + me.k_channel;
      *(v8bf*)to = x[0];
      *(v8bf*)(to + 8) = x[1];
    }
    const unsigned w[2][2] = {{turn(vw.x), turn(vw.y)}, {turn(vw.z), turn(vw.w)}};
#pragma unroll
    for (int half = 0; half < 2; half++) {
      const int row = row_of(me.v_token + 4 * half);
      if (row < 0) continue;
#pragma unroll
      for (int more = 0; more < 2; more++) {
        __bf16 f[4];
        numbers(w[more][half], vs, a.v_mean, me.v_channel + 16 * more, f);
        *(v4bf*)(a.Vo + ((size_t)row * a.g.H + h) * D + me.v_channel + 16 * more) = v4bf{f[0], f[1], f[2], f[3]};
      }
    }
  }
}

}  // namespace sage
