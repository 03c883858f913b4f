// Rotary positions, forward and backward (the formulas and the fixed-point angles
// are in the header): pair (a, b) of a head at position p turns by t = p f,
//   a' = a cos t - b sin t,  b' = a sin t + b cos t,  backward by -t.
//
// Bound by HBM: every value is read and written once.  A thread takes 8 pairs of a
// token (16 values, or 16 of those that are copied) through several heads, so that
// the angles' sines and cosines (8 sums in double, about 300 instructions) are formed
// once for them; a token's threads lie side by side and read whole lines.
#include "dqt_launch.h"
#include "rope.h"

namespace dqt {

namespace {

// 8 consecutive values of X as fp32, and back
template <class T>
__device__ __forceinline__ void load8(const uint8_t* p, float (&v)[8]) {
  if constexpr (sizeof(T) == 2) {
    const i32x4 x = *reinterpret_cast<const i32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = bf16_bits_to_f32((uint32_t)x[i] & 0xFFFFu);
      v[2 * i + 1] = __uint_as_float((uint32_t)x[i] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const f32x4 x = reinterpret_cast<const f32x4*>(p)[i];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * i + e] = x[e];
    }
  }
}
template <class T>
__device__ __forceinline__ void store8(uint8_t* p, const float (&v)[8]) {
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<i32x4*>(p) = i32x4{(int)pack_bf16x2(v[0], v[1]), (int)pack_bf16x2(v[2], v[3]),
                                         (int)pack_bf16x2(v[4], v[5]), (int)pack_bf16x2(v[6], v[7])};
  } else {
    reinterpret_cast<f32x4*>(p)[0] = f32x4{v[0], v[1], v[2], v[3]};
    reinterpret_cast<f32x4*>(p)[1] = f32x4{v[4], v[5], v[6], v[7]};
  }
}

template <class T, bool PAIRS>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t tok = at / a.items;
  if (tok >= a.tokens) return;
  const int item = (int)(at - tok * a.items), turned = a.rot / 16;
  // first of the item's two runs of 8 values, and the second
  const bool turns = item < turned;
  const int i0 = PAIRS || !turns ? 16 * item : 8 * item, i1 = PAIRS || !turns ? i0 + 8 : a.rot / 2 + 8 * item;
  float c[8], s[8];
  if (turns) {
    const int64_t p = a.pos == nullptr ? tok : a.pos[tok];
    const uint64_t dir = a.back ? 0 - (uint64_t)p : (uint64_t)p;
#pragma unroll
    for (int i = 0; i < 8; ++i) turn(dir * a.freq[8 * item + i], a.amp, c[i], s[i]);
  }
  const int first = (int)((int64_t)a.all_heads * blockIdx.y / gridDim.y);
  const int last = (int)((int64_t)a.all_heads * (blockIdx.y + 1) / gridDim.y);
  int h0 = 0;                                       // the tensor's first head among all
  for (int t = 0; t < a.n; ++t) {
    const RopeIO& io = a.io[t];
    const int from = max(first, h0) - h0, to = min(last, h0 + io.heads) - h0;
    h0 += io.heads;
    if (!turns && io.X == io.Y) continue;           // (in place: what is copied is there)
    const uint8_t* x = io.X + tok * io.x_tok + (int64_t)from * io.x_head;
    uint8_t* y = io.Y + tok * io.y_tok + (int64_t)from * io.y_head;
#pragma unroll 2
    for (int h = from; h < to; ++h, x += io.x_head, y += io.y_head) {
      float u[8], v[8];
      load8<T>(x + i0 * sizeof(T), u);
      load8<T>(x + i1 * sizeof(T), v);
      if (turns) {
        if constexpr (PAIRS) {
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
      store8<T>(y + i0 * sizeof(T), u);
      store8<T>(y + i1 * sizeof(T), v);
    }
  }
}

}  // namespace

hipError_t launch_rope(bool bf16, const RopeArgs& in, hipStream_t s) {
  RopeArgs a = in;
  a.items = a.d / 16;
  const int64_t blocks = (a.tokens * a.items + 255) / 256;
  // few tokens: the heads are spread over blocks as well, up to about four a unit
  const int64_t split = (1024 + blocks - 1) / blocks;
  const dim3 grid((uint32_t)blocks, (uint32_t)(split < a.all_heads ? split : a.all_heads));
  auto go = [&](auto k) { return launch_kernel(k, grid, dim3(256), s, a); };
  if (bf16) return a.pairs ? go(rope_kernel<uint16_t, true>) : go(rope_kernel<uint16_t, false>);
  return a.pairs ? go(rope_kernel<float, true>) : go(rope_kernel<float, false>);
}

}  // namespace dqt
