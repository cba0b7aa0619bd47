// Rotary positions of Q and K in one launch (gfx950 only).
#pragma once

#include "common.h"

namespace sage {

struct RotaryArgs {
  const __bf16* x[2];       // Q, K
  __bf16* y[2];
  int64_t xs[2][3], ys[2][3];   // batch, row, head strides in elements
  const void* positions;
  const float* inv_freq;
  int N, tokens, d, half;   // half = rotary_dim / 2 frequencies
  int heads[2];
  int axes, end[4];         // end[a]: first frequency behind axis a
  int pieces;               // threads a token and group of heads takes: d / (2 F)
  int heads_per_thread, head_groups[2];
  float sign;
};

// cos and sin of 2 pi t, |t| <= 1/2, as floats.
__device__ __forceinline__ void turn_of(double turns, float sign, float& c, float& s) {
  // (a position of up to 53 bits is exact in float64; its product with a frequency and that with 1 / 2 pi are rounded, with the constant's own error up to
  // 3 x 2^-53 of the turns: 3.5e-10 at 2^20 turns, of which only the fraction counts, which float32 holds to 3e-8)
  const float t = (float)(turns - __builtin_rint(turns));
  float sv, cv;
  sv = sinpif(2.f * t);
  cv = cospif(2.f * t);
  c = cv;
  s = sign * sv;
}

// A thread has F frequencies of a token (2 F channels; or 2 F channels that are copied) and up to heads_per_thread heads, for which it forms sine
// and cosine once: y1 = x1 cos - x2 sin, y2 = x2 cos + x1 sin.  The bytes of x and y are what bounds it; the angles cost about 50
// instructions a frequency, which eight heads share (16381 tokens of 32 heads of 64: 56 us, 4.8 TB/s).  A few tokens are bound by a thread's own
// chain: they take two frequencies a thread (32 tokens of 40 heads of 128: 4.5 -> 3.2 us).
template <int F, bool ADJACENT, typename POS>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a) {
  typedef __bf16 vec __attribute__((ext_vector_type(F)));
  const unsigned id = blockIdx.x * 256u + threadIdx.x;
  const unsigned token = id / (unsigned)a.pieces, piece = id % (unsigned)a.pieces;
  if (token >= (unsigned)a.tokens) return;
  int group = blockIdx.y;
  const int which = group >= a.head_groups[0];
  if (which) group -= a.head_groups[0];
  const int h0 = group * a.heads_per_thread;
  const int h1 = min(h0 + a.heads_per_thread, a.heads[which]);
  const unsigned b = token / (unsigned)a.N, n = token % (unsigned)a.N;
  const __bf16* x = a.x[which] + b * a.xs[which][0] + n * a.xs[which][1];
  __bf16* y = a.y[which] + b * a.ys[which][0] + n * a.ys[which][1];
  const int64_t xh = a.xs[which][2], yh = a.ys[which][2];

  // halves: F channels from f0 and F from half + f0; adjacent, or channels that pass through: 2 F channels from 2 f0
  const int f0 = piece * F;
  const bool passes = f0 >= a.half, split = !ADJACENT && !passes;
  const int c0 = split ? f0 : 2 * f0, c1 = split ? a.half + f0 : 2 * f0 + F;
  vec u = *(const vec*)(x + h0 * xh + c0), w = *(const vec*)(x + h0 * xh + c1);      // (the angles are formed under the loads)
  float cs[F], sn[F];
  if (!passes) {
    const POS* pos = (const POS*)a.positions + token;
    double p[4];
#pragma unroll
    for (int k = 0; k < 4; k++) p[k] = k < a.axes ? (double)pos[(size_t)k * a.tokens] : 0.0;
#pragma unroll
    for (int i = 0; i < F; i++) {
      const int f = f0 + i;
      const double at = f < a.end[0] ? p[0] : f < a.end[1] ? p[1] : f < a.end[2] ? p[2] : p[3];
      turn_of(at * (double)a.inv_freq[f] * 0.15915494309189533577, a.sign, cs[i], sn[i]);
    }
  }
  for (int h = h0; h < h1; h++) {
    if (h > h0) {
      u = *(const vec*)(x + h * xh + c0);
      w = *(const vec*)(x + h * xh + c1);
    }
    vec r = u, t = w;
    if (!passes) {
#pragma unroll
      for (int i = 0; i < F; i++) {
        // pair i: (u[i], w[i]), or channels 2 i, 2 i + 1 of the two pieces
        const int j = 2 * i % F;
        const float x1 = ADJACENT ? (float)(2 * i < F ? u[j] : w[j]) : (float)u[i];
        const float x2 = ADJACENT ? (float)(2 * i < F ? u[j + 1] : w[j + 1]) : (float)w[i];
        const __bf16 y1 = (__bf16)(x1 * cs[i] - x2 * sn[i]), y2 = (__bf16)(x2 * cs[i] + x1 * sn[i]);
        if (!ADJACENT) {
          r[i] = y1;
          t[i] = y2;
        } else if (2 * i < F) {
          r[j] = y1;
          r[j + 1] = y2;
        } else {
          t[j] = y1;
          t[j + 1] = y2;
        }
      }
    }
    *(vec*)(y + h * yh + c0) = r;
    *(vec*)(y + h * yh + c1) = t;
  }
}

}  // namespace sage
