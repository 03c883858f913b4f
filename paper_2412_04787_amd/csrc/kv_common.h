// What the kernels of the 8-bit cache share: the sequence a block works for, and
// the pages' scales.
#pragma once

#include "dqt_launch.h"

namespace dqt {

constexpr int kMinExp = -64, kMaxExp = 112;          // of the scales

__device__ __forceinline__ int clamp_to(int x, int n) { return x < 0 ? 0 : x > n ? n : x; }

// A sequence's new tokens (queries) and length.  Nothing that stands in the arrays
// leads out of bounds: starts are clamped to the tensors, lengths to max_len.  An end
// beyond the following end is cut there, so that a single wrong start makes no two
// sequences write the same rows, in an order that no one knows.
struct KvSeq {
  int s, q0, lq, lk;
};
__device__ __forceinline__ KvSeq kv_seq(const KvArgs& a, int s) {
  KvSeq q;
  q.s = s;
  q.q0 = a.q_start == nullptr ? s : clamp_to(a.q_start[s], a.tq);
  const int end = a.q_start == nullptr ? s + 1 : clamp_to(min(a.q_start[s + 1], a.q_start[min(s + 2, a.n_seq)]), a.tq);
  q.lq = end > q.q0 ? end - q.q0 : 0;
  q.lk = clamp_to(a.kv_len[s], a.max_len);
  return q;
}

// Item p of all sequences' (tiles, pages) -> its sequence and number there.
// Sequence s's items begin at start(s) = q_start[s] mul / size + extra s (rounded
// down), which leaves room for lq mul / size + extra of each.  The wave looks at 64
// sequences at a time.
__device__ __forceinline__ KvSeq kv_find(const KvArgs& a, int p, int mul, int size, int extra, int& item) {
  if (a.q_start == nullptr && mul <= size && extra == 1) {       // an item for each sequence
    item = 0;
    return kv_seq(a, p);
  }
  const int lane = threadIdx.x & (kWave - 1);
  auto start = [&](int s) {
    return (int64_t)(a.q_start == nullptr ? s : clamp_to(a.q_start[s], a.tq)) * mul / size + (int64_t)extra * s;
  };
  int lo = 0, hi = a.n_seq;            // the last sequence whose items begin at or before p
  while (hi - lo > 1) {
    const int step = (hi - lo + kWave - 1) / kWave, s = lo + lane * step;
    const unsigned long long before = __ballot(s < hi && start(min(s, hi - 1)) <= p);
    lo += (before ? 63 - __builtin_clzll(before) : 0) * step;
    hi = min(hi, lo + step);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  item = __builtin_amdgcn_readfirstlane((int)(p - start(lo)));
  return kv_seq(a, lo);
}

// The smallest e in kMinExp .. kMaxExp with amax <= top 2^e (amax finite, >= 0):
// top is 1.75 2^8 (e4m3) or 1.984375 2^6 (int8).
template <bool E4M3>
__device__ __forceinline__ int scale_exp(float amax) {
  const uint32_t b = __float_as_uint(amax);
  const int e = (int)(b >> 23) - 127 - (E4M3 ? 8 : 6) + ((b & 0x7FFFFFu) > (E4M3 ? 0x600000u : 0x7E0000u) ? 1 : 0);
  return min(max(e, kMinExp), kMaxExp);
}
__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 .. 127
__device__ __forceinline__ int exp_of(float scale) {
  return min(max((int)((__float_as_uint(scale) >> 23) & 0xFFu) - 127, kMinExp), kMaxExp);
}

}  // namespace dqt
