// What the kernels of the 8-bit cache share: the sequence a block works for, and
// the pages' scales.
#pragma once

#include "cache_launch.h"

namespace dqt {

constexpr int kMinExp = -64, kMaxExp = 112;          // of the scales

__device__ __forceinline__ int clamp_to(int x, int n) { return x < 0 ? 0 : x > n ? n : x; }

// A sequence's new tokens (queries) and length.  Nothing that stands in the arrays
// leads out of bounds: starts are clamped to the tensors, lengths to max_len; and no two
// sequences have the same row (whose writers' order no one would know) where starts do not
// ascend.
struct KvSeq {
  int s, q0, lq, lk;
};
__device__ __forceinline__ KvSeq kv_span(const KvArgs& a, int s, int start, int end, int len) {
  KvSeq q;
  q.s = s;
  q.q0 = clamp_to(start, a.tq);
  q.lq = max(clamp_to(end, a.tq) - q.q0, 0);
  q.lk = clamp_to(len, a.max_len);
  return q;
}
// One new token for each sequence (no starts).
__device__ __forceinline__ KvSeq kv_seq(const KvArgs& a, int s) { return kv_span(a, s, s, s + 1, a.kv_len[s]); }

// Up to 64 sequences at once, lane s that of sequence s: a row is the last one's that starts at
// or before it.
__device__ __forceinline__ KvSeq kv_seq_of_lane(const KvArgs& a) {
  const int s = threadIdx.x & (kWave - 1);
  const bool there = s < a.n_seq;
  const int len = there ? a.kv_len[s] : 0;
  if (a.q_start == nullptr) return kv_span(a, s, s, there ? s + 1 : s, len);
  const int start = a.q_start[min(s, a.n_seq)];
  int end = a.q_start[min(s + 1, a.n_seq)];
  if (__ballot(there && start > end)) {
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) end = min(end, __shfl_down(end, off, kWave));      // (the last lanes' own)
  }
  return kv_span(a, s, start, there ? end : start, len);
}

// Item p of all sequences' (tiles, pages) -> its sequence and number there.
// Sequence s's items begin at start(s) = q_start[s] mul / size + extra s (rounded
// down), which leaves room for lq mul / size + extra of each.  The wave looks at 64
// sequences at a time, and takes the last whose items begin at or before p.
//
// A sequence has the rows that a search of this kind for a row, by the starts themselves, ends
// at it for: those from the starts that the looks went past, and before the others that they
// saw behind it.  Where starts ascend, that is all up to the start after it.  (3000 sequences:
// attention 45.6 us and appending 77; 45.2 and 74 by the next start alone, which leaves rows to
// two where starts descend; 72 and 152 by the least of all later starts.)
__device__ __forceinline__ KvSeq kv_find(const KvArgs& a, int p, int mul, int size, int extra, int& item) {
  if (a.q_start == nullptr && mul <= size && extra == 1) {       // an item for each sequence
    item = 0;
    return kv_seq(a, p);
  }
  const int lane = threadIdx.x & (kWave - 1);
  auto start = [&](int s, int x) { return (int64_t)(a.q_start == nullptr ? s : clamp_to(x, a.tq)) * mul / size + (int64_t)extra * s; };
  int lo = 0, hi = a.n_seq, passed = 0, later = a.tq;
  while (hi - lo > 1) {
    const int step = (hi - lo + kWave - 1) / kWave, s = lo + lane * step;
    const int x = a.q_start == nullptr ? 0 : a.q_start[min(s, hi - 1)];
    const unsigned long long before = __ballot(s < hi && start(min(s, hi - 1), x) <= p);
    const int at = before ? 63 - __builtin_clzll(before) : 0;
    if (s < hi && lane > at) later = min(later, x);
    if (at > 0) passed = max(passed, __builtin_amdgcn_readlane(x, at));
    lo += at * step;
    hi = min(hi, lo + step);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  if (a.q_start == nullptr) {
    item = __builtin_amdgcn_readfirstlane((int)(p - start(lo, 0)));
    return kv_seq(a, lo);
  }
  const int first = a.q_start[lo];
  item = __builtin_amdgcn_readfirstlane((int)(p - start(lo, first)));
  int end = min(a.q_start[lo + 1], a.q_start[a.n_seq]);
  if (__ballot(later < end)) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) later = min(later, __shfl_xor(later, off, kWave));
    end = min(end, __builtin_amdgcn_readfirstlane(later));
  }
  return kv_span(a, lo, max(first, passed), end, a.kv_len[lo]);
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
