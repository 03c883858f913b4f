// New tokens into the 8-bit cache: their keys rotated by their positions and
// written with the values as codes on the page's scale, their queries rotated.
//
//   amax = largest finite |x| of the page's new tokens (key head, keys or values)
//   s = max(smallest power of two with amax <= top s, the scale that stands), or
//   without the latter when the page's row 0 is among them;  code = round(x / s)
// and, where s grows over codes that stand, code' = round(code s_old / s).  All
// divisions are by powers of two, so a code is rounded once from the fp32 value.
//
// A block takes the new tokens of one page and key head, and the queries of the heads
// that share it: waves 0 and 1 the keys, 2 and 3 the values, 16 values per thread
// and step, held in registers between the page's maximum and its codes.  Rotations
// come from a table of the page's cosines and sines in LDS, which keys and queries
// share.  Values go through LDS to lie as the cache has them (a channel's tokens
// together).  Bound by HBM for prompts, by the chain of dependent loads (length,
// page, scale) for single tokens.
#include "kv_common.h"
#include "rope.h"

namespace dqt {

namespace {

__device__ __forceinline__ void load16(const uint8_t* p, float (&v)[8]) {
  const i32x4 x = *reinterpret_cast<const i32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = bf16_bits_to_f32((uint32_t)x[i] & 0xFFFFu);
    v[2 * i + 1] = __uint_as_float((uint32_t)x[i] & 0xFFFF0000u);
  }
}

// values on their scale (not NaN) -> four codes
template <bool E4M3>
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  if constexpr (E4M3) return f32x4_to_e4m3x4(a, b, c, d);
  auto lim = [](float x) { return fminf(fmaxf(x, -127.0f), 127.0f); };
  return f32x4_to_i8x4(lim(a), lim(b), lim(c), lim(d));
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
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a <= 3.402823466e38f ? a : 0.0f;
}

// A token's run of 16 values: rotated pairs 8 item .. + 7, or 16 values as they are.
struct Run {
  int i0, i1, cs;        // first of its two runs of 8 values, second; its cosines (-1: none)
  __device__ __forceinline__ Run(const KvAppendArgs& a, int item) {
    const bool turns = a.freq != nullptr && item < a.rot / 16;
    cs = turns ? 8 * item : -1;
    i0 = turns && !a.pairs ? 8 * item : 16 * item;
    i1 = turns && !a.pairs ? a.rot / 2 + 8 * item : i0 + 8;
  }
  // cs_row: the token's cosines and sines
  __device__ __forceinline__ void rotate(const KvAppendArgs& a, const float2* cs_row, float (&u)[8], float (&v)[8]) const {
    if (cs < 0) return;
    if (a.pairs) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 f = cs_row[cs + i], g = cs_row[cs + 4 + i];
        const float p = u[2 * i], q = u[2 * i + 1], r = v[2 * i], w = v[2 * i + 1];
        u[2 * i] = p * f.x - q * f.y;
        u[2 * i + 1] = p * f.y + q * f.x;
        v[2 * i] = r * g.x - w * g.y;
        v[2 * i + 1] = r * g.y + w * g.x;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 f = cs_row[cs + i];
        const float p = u[i], q = v[i];
        u[i] = p * f.x - q * f.y;
        v[i] = p * f.y + q * f.x;
      }
    }
  }
};

template <int D, bool E4M3>
__global__ __launch_bounds__(256) void kv_append_kernel(KvAppendArgs a) {
  constexpr int ITEMS = D / 16, STEPS = kPage * ITEMS / 128, VROW = kPage + 4;
  __shared__ float2 cs[kPage][D / 2];
  __shared__ uint32_t vt[D * VROW / 4];              // the values' codes, [channel][token]
  __shared__ float red[4];
  __shared__ int stood[2];
  const int tid = threadIdx.x, kvh = blockIdx.y;
  int at;
  const KvSeq sq = kv_find(a.c, blockIdx.x, 1, kPage, a.c.q_start == nullptr ? 1 : 2, at);
  if (at < 0 || sq.lq == 0) return;
  const int pos0 = sq.lk - sq.lq;                    // of the first new token (below 0: it is left out)
  const int64_t page_at = (int64_t)max(pos0, 0) / kPage + at;
  if (page_at * kPage >= sq.lk) return;
  const int base = (int)page_at * kPage;             // the page's first position
  const int lo = max(pos0 - base, 0), hi = min(sq.lk - base, kPage), n = hi - lo;
  const int64_t row0 = (int64_t)sq.q0 + (base + lo - pos0);        // the first of these tokens in the batch
  const int64_t page = a.c.table[(int64_t)sq.s * a.c.table_stride + page_at];
  const bool there = page >= 0 && page < a.c.pages;

  // 16 values per item: waves 0, 1 of the keys, waves 2, 3 of the values
  const bool keys = tid < 128;
  const int first = tid & 127;
  const uint8_t* src = keys ? a.k + row0 * a.k_tok + (int64_t)kvh * a.k_head : a.v + row0 * a.v_tok + (int64_t)kvh * a.v_head;
  const int64_t tok = keys ? a.k_tok : a.v_tok;
  float x[STEPS][2][8];
#pragma unroll
  for (int st = 0; st < STEPS; ++st) {
    const int i = first + 128 * st, t = i / ITEMS, item = i % ITEMS;
    if (there && t < n) {
      int i0 = 16 * item, i1 = i0 + 8;
      if (keys) {
        const Run r(a, item);
        i0 = r.i0;
        i1 = r.i1;
      }
      load16(src + t * tok + 2 * i0, x[st][0]);
      load16(src + t * tok + 2 * i1, x[st][1]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[st][0][e] = x[st][1][e] = 0.0f;
    }
  }
  float* sc = a.c.scales + 2 * (page * a.c.kv_heads + kvh);
  // (read by the thread that will write it, before the others know the new one)
  if (there && first == 0) stood[keys ? 0 : 1] = lo > 0 ? exp_of(sc[keys ? 0 : 1]) : kMinExp;
  if (a.freq != nullptr) {
    const int half = a.rot / 2;
    for (int i = tid; i < n * half; i += 256) {
      const int t = i / half, f = i - t * half;
      float2 w;
      turn((uint64_t)(base + lo + t) * a.freq[f], a.amp, w.x, w.y);
      cs[t][f] = w;
    }
    __syncthreads();
  }
  if (there) {
    float most = 0.0f;
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
      const int i = first + 128 * st, t = i / ITEMS, item = i % ITEMS;
      if (keys && t < n) Run(a, item).rotate(a, cs[t], x[st][0], x[st][1]);
#pragma unroll
      for (int e = 0; e < 8; ++e) most = fmaxf(most, fmaxf(finite_abs(x[st][0][e]), finite_abs(x[st][1][e])));
    }
    most = wave_max(most);
    if ((tid & 63) == 0) red[tid >> 6] = most;
    __syncthreads();
    most = keys ? fmaxf(red[0], red[1]) : fmaxf(red[2], red[3]);
    const int was = stood[keys ? 0 : 1], e = max(scale_exp<E4M3>(most), was);
    const bool grows = lo > 0 && e > was;
    const float inv = exp2_int(-e), f = exp2_int(max(was - e, -126));
    if (first == 0) sc[keys ? 0 : 1] = exp2_int(e);
    uint8_t* dst = (keys ? a.c.K : a.c.V) + (page * a.c.kv_heads + kvh) * (int64_t)(kPage * D);
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
      const int i = first + 128 * st, t = i / ITEMS, item = i % ITEMS;
      if (t >= n) continue;
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float y[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const float z = x[st][j / 2][4 * (j & 1) + b];
          y[b] = z == z ? z * inv : 0.0f;
        }
        w[j] = codes4<E4M3>(y[0], y[1], y[2], y[3]);
      }
      if (keys) {
        const Run r(a, item);
        uint8_t* p = dst + (lo + t) * D;
        *reinterpret_cast<uint2*>(p + r.i0) = uint2{w[0], w[1]};
        *reinterpret_cast<uint2*>(p + r.i1) = uint2{w[2], w[3]};
      } else {
        uint8_t* p = reinterpret_cast<uint8_t*>(vt) + (16 * item) * VROW + lo + t;
#pragma unroll
        for (int j = 0; j < 16; ++j) p[j * VROW] = (uint8_t)(w[j / 4] >> (8 * (j & 3)));
      }
    }
    __syncthreads();
    if (keys) {
      if (grows)         // rows 0 .. lo - 1 on the new scale
        for (int i = first; i < lo * ITEMS; i += 128) {
          i32x4* p = reinterpret_cast<i32x4*>(dst) + i;
          i32x4 v = *p;
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] = (int)rescale4<E4M3>((uint32_t)v[j], f);
          *p = v;
        }
    } else if (n == 1 && !grows) {
      // one token: single bytes, without waiting for those beside them
      if (first < D) dst[first * kPage + lo] = reinterpret_cast<const uint8_t*>(vt)[first * VROW + lo];
    } else {
      for (int i = first; i < D * 4; i += 128) {
        const int row = i >> 2, t0 = 16 * (i & 3);
        if (t0 >= hi || (t0 + 16 <= lo && !grows)) continue;
        i32x4* p = reinterpret_cast<i32x4*>(dst + row * kPage + t0);
        i32x4 v;
        const bool whole = t0 >= lo && t0 + 16 <= hi;
        if (!whole) v = *p;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int t = t0 + 4 * j;                       // bytes t .. t + 3: old, new, or behind the end
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
  }
  // the queries of the heads that share this key head
  if (a.q != nullptr) {
    const int G = a.c.group;
    for (int i = tid; i < n * G * ITEMS; i += 256) {
      const int item = i % ITEMS, tg = i / ITEMS, t = tg / G, g = tg - t * G;
      const Run r(a, item);
      const int64_t head = (int64_t)kvh * G + g;
      float u[8], v[8];
      const uint8_t* p = a.q + (row0 + t) * a.q_tok + head * a.q_head;
      load16(p + 2 * r.i0, u);
      load16(p + 2 * r.i1, v);
      r.rotate(a, cs[t], u, v);
      uint8_t* o = a.qr + (row0 + t) * a.qr_tok + head * a.qr_head;
      *reinterpret_cast<i32x4*>(o + 2 * r.i0) = i32x4{(int)pack_bf16x2(u[0], u[1]), (int)pack_bf16x2(u[2], u[3]),
                                                     (int)pack_bf16x2(u[4], u[5]), (int)pack_bf16x2(u[6], u[7])};
      *reinterpret_cast<i32x4*>(o + 2 * r.i1) = i32x4{(int)pack_bf16x2(v[0], v[1]), (int)pack_bf16x2(v[2], v[3]),
                                                     (int)pack_bf16x2(v[4], v[5]), (int)pack_bf16x2(v[6], v[7])};
    }
  }
}

}  // namespace

hipError_t launch_kv_append(bool e4m3, const KvAppendArgs& a, hipStream_t s) {
  // pages of all sequences at most (see kv_find)
  const int64_t blocks = a.c.q_start == nullptr ? a.c.n_seq : a.c.tq / kPage + 2 * (int64_t)a.c.n_seq;
  const dim3 grid((uint32_t)blocks, (uint32_t)a.c.kv_heads);
  auto go = [&](auto k) { return launch_kernel(k, grid, dim3(256), s, a); };
  if (a.c.d == 128) return e4m3 ? go(kv_append_kernel<128, true>) : go(kv_append_kernel<128, false>);
  return e4m3 ? go(kv_append_kernel<64, true>) : go(kv_append_kernel<64, false>);
}

}  // namespace dqt
