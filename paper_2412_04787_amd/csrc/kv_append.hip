// New tokens into the 8-bit cache: their keys rotated by their positions and
// written with the values as codes on the page's scale, their queries rotated.
//
//   amax = largest finite |x| of the page's new tokens (key head, keys or values)
//   s = max(smallest power of two with amax <= top s, the scale that stands), or
//   without the latter when the page's row 0 is among them;  code = round(x / s)
// and, where s grows over codes that stand, code' = round(code s_old / s).  All
// divisions are by powers of two, so a code is rounded once from the fp32 value.
//
// The keys of a page and key head are one block's work, its values another's, and the
// queries of the heads that share the key head, half a page at a time, that of two more:
// with all of it in one block, 1104 long blocks on 256 units (five prompts of 301 to 3001
// tokens, 32 heads on 8) ended in a round that was nearly empty, 56 us.  A thread holds
// 16 values of each of two tokens' keys, or 8 channels of 4 tokens' values, between the
// page's maximum and its codes.  Rotations come from a table of cosines and sines in
// LDS.  Values go through LDS to lie as the cache has them (a channel's tokens
// together).  Bound by HBM for prompts (those five 44 us, 4.2 TB/s; the turns are 2 of
// it; the maximum as an integer and clamps in one operation took 1.6 off), by the chain
// of dependent loads (length, page, scale) for single tokens (32 sequences 4.7 us).
#include "kv_common.h"
#include "rope.h"

namespace dqt {

namespace {

// 8 bf16 values as fp32
__device__ __forceinline__ void widen8(i32x4 x, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float((uint32_t)x[i] << 16);
    v[2 * i + 1] = __uint_as_float((uint32_t)x[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void load16(const uint8_t* p, float (&v)[8]) { widen8(*reinterpret_cast<const i32x4*>(p), v); }

// values on their scale (not NaN) -> four codes
template <bool E4M3>
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  if constexpr (E4M3) {
    auto q = [](float v) { return __builtin_amdgcn_fmed3f(v, -448.0f, 448.0f); };
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(q(a), q(b), 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(q(c), q(d), w, true);
    return (uint32_t)w;
  }
  // (1.5 2^23 + v ends in v, rounded to nearest even)
  auto q = [](float v) { return __float_as_uint(__builtin_amdgcn_fmed3f(v, -127.0f, 127.0f) + 12582912.0f); };
  return __builtin_amdgcn_perm(q(b), q(a), 0x0C0C0400u) | (__builtin_amdgcn_perm(q(d), q(c), 0x0C0C0400u) << 16);
}
// four codes that stand for x -> those of x / 2^n
template <bool E4M3>
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float f) {
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    v[i] = (E4M3 ? e4m3_to_f32((w >> (8 * i)) & 0xFFu) : (float)(int8_t)(w >> (8 * i))) * f;
  return codes4<E4M3>(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }
constexpr uint32_t kInfBits = 0x7F800000u;
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, off, kWave));
  return v;
}

// A token's run of 16 values: rotated pairs 8 item .. + 7, or 16 values as they are.
struct Run {
  int i0, i1;            // first of its two runs of 8 values, second
  bool turns;
  __device__ __forceinline__ Run(const KvAppendArgs& a, int item) {
    turns = a.freq != nullptr && 16 * item < a.rot;
    i0 = turns && !a.pairs ? 8 * item : 16 * item;
    i1 = turns && !a.pairs ? a.rot / 2 + 8 * item : i0 + 8;
  }
};

// 4 tokens' codes of 4 channels (byte = channel) -> 4 channels' codes of 4 tokens
__device__ __forceinline__ void transpose4(const uint32_t (&a)[4], uint32_t (&b)[4]) {
  const uint32_t t0 = __builtin_amdgcn_perm(a[1], a[0], 0x05010400u), t1 = __builtin_amdgcn_perm(a[1], a[0], 0x07030602u);
  const uint32_t t2 = __builtin_amdgcn_perm(a[3], a[2], 0x05010400u), t3 = __builtin_amdgcn_perm(a[3], a[2], 0x07030602u);
  b[0] = __builtin_amdgcn_perm(t2, t0, 0x05040100u);
  b[1] = __builtin_amdgcn_perm(t2, t0, 0x07060302u);
  b[2] = __builtin_amdgcn_perm(t3, t1, 0x05040100u);
  b[3] = __builtin_amdgcn_perm(t3, t1, 0x07060302u);
}

constexpr int kTurnTokens = kPage / 2;               // of the table in LDS

// Cosines and sines of n tokens from position pos on.  A thread takes one pair through
// a run of tokens: the first one's turn, then products with that of one position (each
// adds what the two factors are off by and its own roundings, 2^-51, to what is rounded to
// fp32; seven at most).
template <int ROW>
__device__ __forceinline__ void turn_table(const KvAppendArgs& a, float2* cs, int pos, int n) {
  const int half = a.rot / 2, runs = 256 / half, p = threadIdx.x % half, len = (n + runs - 1) / runs, t0 = threadIdx.x / half * len;
  if (threadIdx.x >= runs * half || t0 >= n) return;
  const uint64_t f = a.freq[p];
  double c, s, c1 = 1.0, s1 = 0.0;
  turn((uint64_t)(pos + t0) * f, c, s);
  if (len > 1) turn(f, c1, s1);
  const int place = turn_place(p, half), end = min(t0 + len, n);
  for (int t = t0; t < end; ++t) {
    cs[t * ROW + place] = float2{(float)(a.amp * c), (float)(a.amp * s)};
    const double d = __builtin_fma(c, c1, -(s * s1));
    s = __builtin_fma(s, c1, c * s1);
    c = d;
  }
}

// The queries of the G heads that share a key head: n tokens from row0 on.
template <int D, int CROW>
__device__ __forceinline__ void turn_queries(const KvAppendArgs& a, const float2* cs, int64_t row0, int kvh, int n) {
  constexpr int ITEMS = D / 16, QSTEPS = 2;
  const int tid = threadIdx.x;
  const uint32_t G = (uint32_t)a.c.group, all = n * G * ITEMS;
  const uint8_t* q = a.q + row0 * a.q_tok + (int64_t)kvh * G * a.q_head;
  uint8_t* qr = a.qr + row0 * a.qr_tok + (int64_t)kvh * G * a.qr_head;
  for (uint32_t i0 = tid; i0 < all; i0 += 256 * QSTEPS) {
    i32x4 ru[QSTEPS], rv[QSTEPS];
    int t[QSTEPS], g[QSTEPS];
#pragma unroll
    for (int e = 0; e < QSTEPS; ++e) {
      const uint32_t i = i0 + 256 * e, tg = i / ITEMS;
      t[e] = (int)(tg / G);
      g[e] = (int)(tg - t[e] * G);
      if (i >= all) continue;
      const Run r(a, i % ITEMS);
      const uint8_t* p = q + t[e] * a.q_tok + g[e] * a.q_head;
      ru[e] = *reinterpret_cast<const i32x4*>(p + 2 * r.i0);
      rv[e] = *reinterpret_cast<const i32x4*>(p + 2 * r.i1);
    }
#pragma unroll
    for (int e = 0; e < QSTEPS; ++e) {
      const uint32_t i = i0 + 256 * e;
      if (i >= all) continue;
      const int item = i % ITEMS;
      const Run r(a, item);
      float u[8], v[8];
      widen8(ru[e], u);
      widen8(rv[e], v);
      if (r.turns) {
        Turns w;
        w.read(cs + t[e] * CROW, item, a.rot / 2);
        w.apply(a.pairs, u, v);
      }
      uint8_t* o = qr + t[e] * a.qr_tok + g[e] * a.qr_head;
      *reinterpret_cast<i32x4*>(o + 2 * r.i0) = i32x4{(int)pack_bf16x2(u[0], u[1]), (int)pack_bf16x2(u[2], u[3]),
                                                     (int)pack_bf16x2(u[4], u[5]), (int)pack_bf16x2(u[6], u[7])};
      *reinterpret_cast<i32x4*>(o + 2 * r.i1) = i32x4{(int)pack_bf16x2(v[0], v[1]), (int)pack_bf16x2(v[2], v[3]),
                                                     (int)pack_bf16x2(v[4], v[5]), (int)pack_bf16x2(v[6], v[7])};
    }
  }
}

template <int D, bool E4M3>
__global__ __launch_bounds__(256) void kv_append_kernel(KvAppendArgs a) {
  constexpr int ITEMS = D / 16, STEPS = kPage * ITEMS / 256;
  constexpr int CROW = D / 2 + 16;                   // (two tokens' rows fall on different halves of the banks)
  constexpr int VROW = kPage + 4;
  __shared__ __attribute__((aligned(16))) float2 cs[kTurnTokens * CROW];
  __shared__ uint32_t vt[D * VROW / 4];              // the values' codes, [channel][token]
  __shared__ uint32_t red[4];
  __shared__ int stood;
  // blocks of keys, of values, of the queries of each half of the page
  const int tid = threadIdx.x, part = (int)blockIdx.y / a.c.kv_heads, kvh = (int)blockIdx.y - part * a.c.kv_heads;
  int at;
  const KvSeq sq = kv_find(a.c, blockIdx.x, 1, kPage, a.c.q_start == nullptr ? 1 : 2, at);
  if (at < 0 || sq.lq == 0) return;
  const int pos0 = sq.lk - sq.lq;                    // of the first new token (below 0: it is left out)
  const int64_t page_at = (int64_t)max(pos0, 0) / kPage + at;
  if (page_at * kPage >= sq.lk) return;
  const int base = (int)page_at * kPage;             // the page's first position
  int lo = max(pos0 - base, 0), hi = min(sq.lk - base, kPage);
  if (part > 1) {
    lo = max(lo, (part - 2) * kTurnTokens);
    hi = min(hi, (part - 1) * kTurnTokens);
    if (lo >= hi) return;
  }
  const int n = hi - lo;
  const int64_t row0 = (int64_t)sq.q0 + (base + lo - pos0);        // the first of these tokens in the batch
  if (part > 1) {
    turn_table<CROW>(a, cs, base + lo, n);
    __syncthreads();
    turn_queries<D, CROW>(a, cs, row0, kvh, n);
    return;
  }
  const int64_t page = a.c.table[(int64_t)sq.s * a.c.table_stride + page_at];
  if (page < 0 || page >= a.c.pages) return;
  const bool keys = part == 0;
  float* sc = a.c.scales + 2 * (page * a.c.kv_heads + kvh) + part;

  float x[4][8];
#pragma unroll
  for (int st = 0; st < 4; ++st)
#pragma unroll
    for (int e = 0; e < 8; ++e) x[st][e] = 0.0f;
  const int unit = tid % (D / 8), grp = tid / (D / 8);        // values: 8 channels of 4 tokens
  if (keys) {
    const uint8_t* src = a.k + row0 * a.k_tok + (int64_t)kvh * a.k_head;
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
      const int i = tid + 256 * st, t = i / ITEMS;
      const Run r(a, i % ITEMS);
      if (t < n) {
        load16(src + t * a.k_tok + 2 * r.i0, x[2 * st]);
        load16(src + t * a.k_tok + 2 * r.i1, x[2 * st + 1]);
      }
    }
  } else {
    const uint8_t* src = a.v + row0 * a.v_tok + (int64_t)kvh * a.v_head;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int t = 4 * grp + b;                     // (of the page)
      if (t >= lo && t < hi) load16(src + (t - lo) * a.v_tok + 16 * unit, x[b]);
    }
  }
  // (read by the thread that will write it, before the others know the new one)
  if (tid == 0) stood = lo > 0 ? exp_of(*sc) : kMinExp;
  if (keys && a.freq != nullptr) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int t0 = half * kTurnTokens;
      if (t0 >= n) break;
      if (half > 0) __syncthreads();
      turn_table<CROW>(a, cs, base + lo + t0, min(n - t0, kTurnTokens));
      __syncthreads();
#pragma unroll
      for (int st = 0; st < STEPS; ++st) {
        const int i = tid + 256 * st, t = i / ITEMS, item = i % ITEMS;
        if (t >= t0 && t < min(n, t0 + kTurnTokens) && 16 * item < a.rot) {
          Turns w;
          w.read(cs + (t - t0) * CROW, item, a.rot / 2);
          w.apply(a.pairs, x[2 * st], x[2 * st + 1]);
        }
      }
    }
  }
  // the block's largest |x|, as bits
  auto largest = [&] {
    uint32_t m = 0;
#pragma unroll
    for (int st = 0; st < 4; ++st)
#pragma unroll
      for (int e = 0; e < 8; ++e) m = max(m, abs_bits(x[st][e]));
    m = wave_max_u32(m);
    if ((tid & 63) == 0) red[tid >> 6] = m;
    __syncthreads();
    return max(max(red[0], red[1]), max(red[2], red[3]));
  };
  uint32_t most = largest();
  if (most >= kInfBits) {
    // (rare: what is not finite does not count; then it is held as the largest code, NaN as 0)
    float keep[4][8];
#pragma unroll
    for (int st = 0; st < 4; ++st)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float v = x[st][e];
        keep[st][e] = v != v ? 0.0f : __builtin_amdgcn_fmed3f(v, -3.402823466e38f, 3.402823466e38f);
        if (abs_bits(v) >= kInfBits) x[st][e] = 0.0f;
      }
    __syncthreads();
    most = largest();
#pragma unroll
    for (int st = 0; st < 4; ++st)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[st][e] = keep[st][e];
  }
  const int was = stood, e = max(scale_exp<E4M3>(__uint_as_float(most)), was);
  const bool grows = lo > 0 && e > was;
  const float inv = exp2_int(-e), f = exp2_int(max(was - e, -126));
  if (tid == 0) *sc = exp2_int(e);
  uint8_t* dst = (keys ? a.c.K : a.c.V) + (page * a.c.kv_heads + kvh) * (int64_t)(kPage * D);
  auto codes = [&](const float (&y)[8], int from) {
    return codes4<E4M3>(y[from] * inv, y[from + 1] * inv, y[from + 2] * inv, y[from + 3] * inv);
  };
  if (keys) {
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
      const int i = tid + 256 * st, t = i / ITEMS;
      if (t >= n) continue;
      const Run r(a, i % ITEMS);
      uint8_t* p = dst + (lo + t) * D;
      *reinterpret_cast<uint2*>(p + r.i0) = uint2{codes(x[2 * st], 0), codes(x[2 * st], 4)};
      *reinterpret_cast<uint2*>(p + r.i1) = uint2{codes(x[2 * st + 1], 0), codes(x[2 * st + 1], 4)};
    }
    if (grows)           // rows 0 .. lo - 1 on the new scale
      for (int i = tid; i < lo * ITEMS; i += 256) {
        i32x4* p = reinterpret_cast<i32x4*>(dst) + i;
        i32x4 v = *p;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = (int)rescale4<E4M3>((uint32_t)v[j], f);
        *p = v;
      }
    return;
  }
  if (4 * grp + 3 >= lo && 4 * grp < hi) {
    uint32_t* p = vt + 8 * unit * (VROW / 4) + grp;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t w[4] = {codes(x[0], 4 * h), codes(x[1], 4 * h), codes(x[2], 4 * h), codes(x[3], 4 * h)};
      uint32_t y[4];
      transpose4(w, y);
#pragma unroll
      for (int j = 0; j < 4; ++j) p[(4 * h + j) * (VROW / 4)] = y[j];
    }
  }
  __syncthreads();
  if (n == 1 && !grows) {
    // one token: single bytes, without waiting for those beside them
    if (tid < D) dst[tid * kPage + lo] = reinterpret_cast<const uint8_t*>(vt)[tid * VROW + lo];
    return;
  }
  for (int i = tid; i < D * 4; i += 256) {
    const int row = i >> 2, t0 = 16 * (i & 3);
    if (t0 >= hi || (t0 + 16 <= lo && !grows)) continue;
    i32x4* p = reinterpret_cast<i32x4*>(dst + row * kPage + t0);
    i32x4 v;
    const bool whole = t0 >= lo && t0 + 16 <= hi;
    if (!whole) v = *p;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int t = t0 + 4 * j;                           // bytes t .. t + 3: old, new, or behind the end
      const uint32_t fresh = vt[row * (VROW / 4) + t / 4];
      if (whole) {
        v[j] = (int)fresh;
      } else {
        const uint32_t had = (uint32_t)v[j], moved = grows ? rescale4<E4M3>(had, f) : had;
        uint32_t w = 0;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const uint32_t from = t + b < lo ? moved : t + b < hi ? fresh : had;
          w |= from & (0xFFu << (8 * b));
        }
        v[j] = (int)w;
      }
    }
    *p = v;
  }
}

}  // namespace

hipError_t launch_kv_append(bool e4m3, const KvAppendArgs& a, hipStream_t s) {
  // pages of all sequences at most (see kv_find)
  const int64_t blocks = a.c.q_start == nullptr ? a.c.n_seq : a.c.tq / kPage + 2 * (int64_t)a.c.n_seq;
  const int parts = a.q == nullptr ? 2 : 2 + kPage / kTurnTokens;
  const dim3 grid((uint32_t)blocks, (uint32_t)(a.c.kv_heads * parts));
  auto go = [&](auto k) { return launch_kernel(k, grid, dim3(256), s, a); };
  if (a.c.d == 128) return e4m3 ? go(kv_append_kernel<128, true>) : go(kv_append_kernel<128, false>);
  return e4m3 ? go(kv_append_kernel<64, true>) : go(kv_append_kernel<64, false>);
}

}  // namespace dqt
