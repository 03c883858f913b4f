// Rotary positions: cos and sin of a pair's turn, shared by rope.hip and kv_append.hip.
#pragma once

#include "dqt_device.h"

namespace dqt {

// cos and sin of 2 pi t 2^-64 in double.  t is cut into the nearest quarter turn and a
// rest of an eighth at most, whose sine and cosine are Taylor sums: the terms left out
// are below 2^-54, less than the sums' own roundings, so the rounding to fp32 is the one of
// the exact value unless that lies within 2^-49 of the middle of two.  (Double runs at
// the rate of fp32 here.)
__device__ __forceinline__ void turn(uint64_t t, double& c, double& s) {
  const uint32_t quarter = (uint32_t)((t + (1ull << 61)) >> 62);
  const int64_t r = (int64_t)(t - ((uint64_t)quarter << 62));
  const double hi = (double)(int32_t)(r >> 32), lo = (double)(uint32_t)r;
  const double x = __builtin_fma(hi, 4294967296.0, lo) * (6.283185307179586 / 18446744073709551616.0);
  const double y = x * x;
  double p = -7.647163731819816e-13;                                                 // 1 / 15!
  p = __builtin_fma(p, y, 1.6059043836821613e-10);                                   // 1 / 13!
  p = __builtin_fma(p, y, -2.505210838544172e-08);
  p = __builtin_fma(p, y, 2.7557319223985893e-06);
  p = __builtin_fma(p, y, -1.984126984126984e-04);
  p = __builtin_fma(p, y, 8.333333333333333e-03);
  p = __builtin_fma(p, y, -1.6666666666666666e-01);
  p = __builtin_fma(p * y, x, x);
  double q = 4.779477332387385e-14;                                                  // 1 / 16!
  q = __builtin_fma(q, y, -1.1470745597729725e-11);
  q = __builtin_fma(q, y, 2.08767569878681e-09);
  q = __builtin_fma(q, y, -2.755731922398589e-07);
  q = __builtin_fma(q, y, 2.48015873015873e-05);
  q = __builtin_fma(q, y, -1.388888888888889e-03);
  q = __builtin_fma(q, y, 4.1666666666666664e-02);
  q = __builtin_fma(q, y, -0.5);
  q = __builtin_fma(q, y, 1.0);
  const double a = (quarter & 1) ? p : q, b = (quarter & 1) ? q : p;
  c = ((quarter + 1) & 2) ? -a : a;
  s = (quarter & 2) ? -b : b;
}

// Cosines and sines of a token's rot / 2 = half pairs, times amp and in fp32, lie in a
// row of LDS.  Pairs 8 j, 8 j + 1 of all j lie side by side, then 8 j + 2, 8 j + 3 and so
// on: lanes of consecutive j read consecutive 16-byte words.
__device__ __forceinline__ int turn_place(int p, int half) { return ((p & 7) >> 1) * (half / 4) + 2 * (p >> 3) + (p & 1); }

// those of pairs 8 j .. 8 j + 7
struct Turns {
  float c[8], s[8];
  __device__ __forceinline__ void read(const float2* row, int j, int half) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(row + i * (half / 4) + 2 * j);
      c[2 * i] = v[0];
      s[2 * i] = v[1];
      c[2 * i + 1] = v[2];
      s[2 * i + 1] = v[3];
    }
  }
  // u, v: the two runs of 8 values; pairs are neighbours, or (u[i], v[i])
  __device__ __forceinline__ void apply(bool neighbours, float (&u)[8], float (&v)[8]) const {
    if (neighbours) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p = u[2 * i], q = u[2 * i + 1], r = v[2 * i], w = v[2 * i + 1];
        u[2 * i] = p * c[i] - q * s[i];
        u[2 * i + 1] = p * s[i] + q * c[i];
        v[2 * i] = r * c[4 + i] - w * s[4 + i];
        v[2 * i + 1] = r * s[4 + i] + w * c[4 + i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float p = u[i], q = v[i];
        u[i] = p * c[i] - q * s[i];
        v[i] = p * s[i] + q * c[i];
      }
    }
  }
};

}  // namespace dqt
