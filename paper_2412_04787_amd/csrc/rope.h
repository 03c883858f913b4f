// Rotary positions: cos and sin of a pair's turn, shared by rope.hip and kv_append.hip.
#pragma once

#include "dqt_device.h"

namespace dqt {

// cos and sin (times amp) of 2 pi t 2^-64.  t is cut into the nearest quarter turn
// and a rest of an eighth at most, whose sine and cosine are Taylor sums: the terms
// left out are below 2^-45, so the rounding to fp32 is the one of the exact value in
// all but one case in 2^20.  In double, which runs at the rate of fp32 here.
__device__ __forceinline__ void turn(uint64_t t, double amp, float& c, float& s) {
  const uint32_t quarter = (uint32_t)((t + (1ull << 61)) >> 62);
  const int64_t r = (int64_t)(t - ((uint64_t)quarter << 62));
  const double hi = (double)(int32_t)(r >> 32), lo = (double)(uint32_t)r;
  const double x = __builtin_fma(hi, 4294967296.0, lo) * (6.283185307179586 / 18446744073709551616.0);
  const double y = x * x;
  double p = 1.6059043836821613e-10;                                                 // 1 / 13!
  p = __builtin_fma(p, y, -2.505210838544172e-08);                                   // 1 / 11!
  p = __builtin_fma(p, y, 2.7557319223985893e-06);
  p = __builtin_fma(p, y, -1.984126984126984e-04);
  p = __builtin_fma(p, y, 8.333333333333333e-03);
  p = __builtin_fma(p, y, -1.6666666666666666e-01);
  p = __builtin_fma(p * y, x, x);
  double q = -1.1470745597729725e-11;                                                // 1 / 14!
  q = __builtin_fma(q, y, 2.08767569878681e-09);
  q = __builtin_fma(q, y, -2.755731922398589e-07);
  q = __builtin_fma(q, y, 2.48015873015873e-05);
  q = __builtin_fma(q, y, -1.388888888888889e-03);
  q = __builtin_fma(q, y, 4.1666666666666664e-02);
  q = __builtin_fma(q, y, -0.5);
  q = __builtin_fma(q, y, 1.0);
  const double a = (quarter & 1) ? p : q, b = (quarter & 1) ? q : p;
  c = (float)(((quarter + 1) & 2) ? -amp * a : amp * a);
  s = (float)((quarter & 2) ? -amp * b : amp * b);
}

}  // namespace dqt
