// Rotary positions, forward and backward (the formulas and the fixed-point angles
// are in the header): pair (a, b) of a head at position p turns by t = p f,
//   a' = a cos t - b sin t,  b' = a sin t + b cos t,  backward by -t.
//
// Bound by HBM: every value is read and written once.  A block takes a few tokens and
// a range of the heads of all tensors: it forms the tokens' cosines and sines in LDS
// (once for all heads), then walks the values in the order of memory, 16 of a head per
// thread and step (8 pairs, or 16 values that are copied), two steps in flight: 16384
// tokens, 16 + 16 heads of 128, bf16, 52 us (5.2 TB/s; 73 us with a thread for 8 pairs of
// a token through all heads, whose waves asked the same channels at once).  Few tokens:
// a launch, 4.4 us for 32 tokens of 40 heads.
#include "cache_launch.h"
#include "rope.h"

namespace dqt {

namespace {

// 8 consecutive values as they lie in memory, as fp32, and back
template <class T>
struct Raw8 {
  i32x4 w[sizeof(T) / 2];
  __device__ __forceinline__ void load(const uint8_t* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = reinterpret_cast<const i32x4*>(p)[i];
  }
  __device__ __forceinline__ void widen(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (sizeof(T) == 4) v[i] = __uint_as_float((uint32_t)w[i / 4][i & 3]);
      else v[i] = __uint_as_float(i & 1 ? (uint32_t)w[0][i / 2] & 0xFFFF0000u : (uint32_t)w[0][i / 2] << 16);
    }
  }
};
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

constexpr int kRopeTokens = 8;       // of a block at most
constexpr int kRopeSteps = 2;

template <class T, bool PAIRS>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  extern __shared__ __attribute__((aligned(16))) float2 cs[];        // [block_tokens][rot / 2]
  const int tid = threadIdx.x, half = a.rot / 2;
  const int64_t t0 = (int64_t)blockIdx.x * a.block_tokens;
  const int nt = (int)min((int64_t)a.block_tokens, a.tokens - t0);
  for (int i = tid; i < nt * half; i += 256) {
    const int t = i / half, p = i - t * half;
    const int64_t pos = a.pos == nullptr ? t0 + t : a.pos[t0 + t];
    double c, s;
    turn((a.back ? 0 - (uint64_t)pos : (uint64_t)pos) * a.freq[p], c, s);
    cs[t * half + turn_place(p, half)] = float2{(float)(a.amp * c), (float)(a.amp * s)};
  }
  __syncthreads();
  const int first = (int)((int64_t)a.all_heads * blockIdx.y / gridDim.y);
  const int last = (int)((int64_t)a.all_heads * (blockIdx.y + 1) / gridDim.y);
  int h0 = 0;                                       // the tensor's first head among all
  for (int k = 0; k < a.n; ++k) {
    const RopeIO& io = a.io[k];
    const int from = max(first, h0) - h0, heads = min(last, h0 + io.heads) - h0 - from;
    h0 += io.heads;
    if (heads <= 0) continue;
    const bool copies = io.X != io.Y;               // (in place: what is copied is there)
    const uint32_t per = (uint32_t)heads * a.items, all = nt * per;
    for (uint32_t at = tid; at < all; at += 256 * kRopeSteps) {
      Raw8<T> ru[kRopeSteps], rv[kRopeSteps];
      uint8_t* y[kRopeSteps];
      int tok[kRopeSteps], item[kRopeSteps];
#pragma unroll
      for (int e = 0; e < kRopeSteps; ++e) {
        const uint32_t i = at + 256 * e;
        y[e] = nullptr;
        if (i >= all) continue;
        tok[e] = (int)(i / per);
        const uint32_t r = i - tok[e] * per, h = r / a.items;
        item[e] = (int)(r - h * a.items);
        const bool turns = 16 * item[e] < a.rot;
        if (!turns && !copies) continue;
        const int i0 = PAIRS || !turns ? 16 * item[e] : 8 * item[e], i1 = PAIRS || !turns ? i0 + 8 : half + i0;
        const uint8_t* x = io.X + (t0 + tok[e]) * io.x_tok + (int64_t)(from + h) * io.x_head;
        ru[e].load(x + i0 * sizeof(T));
        rv[e].load(x + i1 * sizeof(T));
        y[e] = io.Y + (t0 + tok[e]) * io.y_tok + (int64_t)(from + h) * io.y_head;
      }
#pragma unroll
      for (int e = 0; e < kRopeSteps; ++e) {
        if (y[e] == nullptr) continue;
        const bool turns = 16 * item[e] < a.rot;
        const int i0 = PAIRS || !turns ? 16 * item[e] : 8 * item[e], i1 = PAIRS || !turns ? i0 + 8 : half + i0;
        float u[8], v[8];
        ru[e].widen(u);
        rv[e].widen(v);
        if (turns) {
          Turns w;
          w.read(cs + tok[e] * half, item[e], half);
          w.apply(PAIRS, u, v);
        }
        store8<T>(y[e] + i0 * sizeof(T), u);
        store8<T>(y[e] + i1 * sizeof(T), v);
      }
    }
  }
}

}  // namespace

hipError_t launch_rope(bool bf16, const RopeArgs& in, hipStream_t s) {
  RopeArgs a = in;
  a.items = a.d / 16;
  // as many tokens to a block as leave two blocks to each compute unit; few tokens: the
  // heads are spread over blocks too, no fewer than 256 runs of 16 values to each
  a.block_tokens = 1;
  while (a.block_tokens < kRopeTokens && a.tokens >= 1024 * a.block_tokens) a.block_tokens *= 2;
  const int64_t blocks = (a.tokens + a.block_tokens - 1) / a.block_tokens;
  int64_t split = (1024 + blocks - 1) / blocks, most = ((int64_t)a.all_heads * a.items * a.block_tokens + 255) / 256;
  if (split > most) split = most;
  if (split > a.all_heads) split = a.all_heads;
  const dim3 grid((uint32_t)blocks, (uint32_t)split);
  const size_t lds = (size_t)a.block_tokens * (a.rot / 2) * sizeof(float2);
  auto go = [&](auto k) { return launch_kernel_lds(k, grid, dim3(256), lds, s, a); };
  if (bf16) return a.pairs ? go(rope_kernel<uint16_t, true>) : go(rope_kernel<uint16_t, false>);
  return a.pairs ? go(rope_kernel<float, true>) : go(rope_kernel<float, false>);
}

}  // namespace dqt
