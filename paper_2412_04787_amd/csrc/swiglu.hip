// The SwiGLU product of a LLaMA block and its 8-bit quantisation, in one
// launch, and its backward from 8-bit checkpoints of its inputs:
//   h = (g / (1 + exp(-g))) u,  m_row = max(max_k |h|, 1e-5)
//   Xq = quantise(h fl(Q / m_row)), xdq = fl(m_row / Q)      (Q = 127 or 448)
//   checkpoint of g and of u: groups of 128 consecutive elements of a row,
//     a = max(max |x|, 1e-5), code = clamp(rint(x fl(127 / a))), scale = fl(a / 127)
//   backward, with s = 1 / (1 + exp(-g)):
//     dU = dH (g s),  dG = dH u s (1 + g (1 - s))
// The forward's operations are correctly rounded fp32 (the exponential the
// device library's), so codes and scales do not depend on how rows are spread
// over threads.
//
// Forward: a block per row; h stays in registers between the row's maximum
// and the codes (rows of up to 4 chunks of 8 elements per thread; longer ones
// form h twice, from cache).  A checkpoint group is 16 neighbouring lanes.
// HBM traffic per element (bf16): 4 bytes read, 1 written, 2 more with the
// checkpoint: 16384 x 5632 in 150 us (4.3 TB/s; without it 8192 x 5632 in 43 us,
// 5.4 TB/s), bound by the vector units, which are never idle (an exponential, a
// division and three conversions an element).
// Backward: 8 elements per thread, 8 bytes of traffic per element (bf16 dH,
// dG and dU, checkpoint) and bound by it: the same size in 119 us, 6.2 TB/s, some
// of it from the last-level cache; from gate and up in bf16, 10 bytes, 161 us,
// 5.7 TB/s.
#include "dqt_launch.h"

namespace dqt {

namespace {

template <typename TX>
__device__ __forceinline__ void load8(const TX* p, float (&v)[8]) {
  if constexpr (sizeof(TX) == 2) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = bf16_bits_to_f32(w[i] & 0xFFFFu);
      v[2 * i + 1] = bf16_bits_to_f32(w[i] >> 16);
    }
  } else {
    const float4 a = *reinterpret_cast<const float4*>(p);
    const float4 b = *reinterpret_cast<const float4*>(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
}
template <typename TX>
__device__ __forceinline__ void store8(TX* p, const float (&v)[8]) {
  if constexpr (sizeof(TX) == 2) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                                              pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
  } else {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
  }
}
// The vector units are as busy as HBM here, so the divisions are shortened where
// that gives the same bits (with the conversions' clamps left out: forward and
// backward of 16384 x 5632 320 -> 300 us, 8192 x 5632 forward 46.7 -> 42.9): a / b
// as a rcp(b) and one correction of its remainder.
// For every fp32 g >= -69 and b = 1 + exp(-g) the result is that of the correctly
// rounded division (-0 gives +0, restored where a code has a sign), and so it is
// for 127 / b from 1e-5 to 2^100 and a / 127 from 1e-5 on: the tests compare all
// gates, and for the other two every significand and 2^18 values over all
// exponents.  Beyond (a denormal reciprocal) the division itself.
__device__ __forceinline__ float div_short(float a, float b) {
  const float r = __builtin_amdgcn_rcpf(b), q = a * r;
  return __builtin_fmaf(__builtin_fmaf(-b, q, a), r, q);
}
__device__ __forceinline__ float div127(float a) {
  constexpr float r = 1.0f / 127.0f;
  const float q = a * r;
  return __builtin_fmaf(__builtin_fmaf(-127.0f, q, a), r, q);
}
// h of 8 elements
template <bool SIGN>
__device__ __forceinline__ void silu_mul8(const float (&g)[8], const float (&u)[8], float (&h)[8]) {
  float lo = g[0];
#pragma unroll
  for (int j = 1; j < 8; ++j) lo = fminf(lo, g[j]);
  if (__any(lo < -69.0f)) {
#pragma unroll
    for (int j = 0; j < 8; ++j) h[j] = __fdiv_rn(g[j], 1.0f + expf(-g[j])) * u[j];
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float s = div_short(g[j], 1.0f + expf(-g[j]));
    h[j] = (SIGN ? copysignf(s, g[j]) : s) * u[j];
  }
}
// f32x4_to_i8x4 of values whose magnitude rounds to 127 at most
__device__ __forceinline__ uint32_t bounded_to_i8x4(float a, float b, float c, float d) {
  auto q = [](float v) { return __float_as_uint(v + 12582912.0f); };
  return (q(a) & 0xFFu) | ((q(b) & 0xFFu) << 8) | ((q(c) & 0xFFu) << 16) | (q(d) << 24);
}

// maximum with the value N lanes further on in the row of 16
template <int N>
__device__ __forceinline__ float max_of_16(float x) {
  return fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 | N, 0xF, 0xF, false)));
}

// The 8-bit checkpoint of 8 elements of a group held by 16 neighbouring lanes.
__device__ __forceinline__ void ckpt8(const float (&v)[8], bool in, int8_t* q, float* scale) {
  float a = 0.0f;
#pragma unroll
  for (int j = 0; j < 8; ++j) a = fmaxf(a, fabsf(v[j]));
  a = max_of_16<8>(max_of_16<4>(max_of_16<2>(max_of_16<1>(in ? a : 0.0f))));
  a = fmaxf(a, 1e-5f);
  const float inv = __any(!(a < 0x1p100f)) ? __fdiv_rn(127.0f, a) : div_short(127.0f, a);
  if (!in) return;
  *reinterpret_cast<uint2*>(q) = make_uint2(bounded_to_i8x4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv),
                                            bounded_to_i8x4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv));
  if ((threadIdx.x & 15) == 0) *scale = div127(a);
}

// NCH chunks of 8 elements per thread in registers; NCH = 0: any row length.
template <typename TX, bool E4M3, bool CKPT, int T, int NCH>
__global__ __launch_bounds__(T) void swiglu_quant_kernel(const TX* __restrict__ G, const TX* __restrict__ U, int64_t M,
                                                         int K, uint8_t* __restrict__ Xq, float* __restrict__ xdq,
                                                         Ckpt ck) {
  __shared__ float wmax[2][T / kWave];
  const int nchunk = K / 8, ngroup = (K + kCkptGroup - 1) / kCkptGroup;
  constexpr float qmax = E4M3 ? 448.0f : 127.0f;
  int flip = 0;
  for (int64_t row = blockIdx.x; row < M; row += gridDim.x, flip ^= 1) {
    const TX* gr = G + row * (int64_t)K;
    const TX* ur = U + row * (int64_t)K;
    float hv[NCH > 0 ? NCH : 1][8];
    float amax = 0.0f;
    auto chunk = [&](int c, float (&hh)[8]) {
      // (lanes without a chunk load the last one and do not use it)
      const bool in = c < nchunk;
      const int cc = in ? c : nchunk - 1;
      float g[8], u[8];
      load8(gr + 8 * cc, g);
      load8(ur + 8 * cc, u);
      silu_mul8<E4M3>(g, u, hh);
      float m = 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(hh[j]));
      amax = in ? fmaxf(amax, m) : amax;
      if constexpr (CKPT) {
        const int64_t sg = row * ngroup + cc / 16;
        ckpt8(g, in, ck.Gq + row * (int64_t)K + 8 * cc, ck.gs + sg);
        ckpt8(u, in, ck.Uq + row * (int64_t)K + 8 * cc, ck.us + sg);
      }
    };
    auto codes = [&](int c, const float (&hh)[8], float inv) {
      if (c >= nchunk) return;
      uint32_t w0, w1;
      if constexpr (E4M3) {
        w0 = f32x4_to_e4m3x4(hh[0] * inv, hh[1] * inv, hh[2] * inv, hh[3] * inv);
        w1 = f32x4_to_e4m3x4(hh[4] * inv, hh[5] * inv, hh[6] * inv, hh[7] * inv);
      } else {
        w0 = bounded_to_i8x4(hh[0] * inv, hh[1] * inv, hh[2] * inv, hh[3] * inv);
        w1 = bounded_to_i8x4(hh[4] * inv, hh[5] * inv, hh[6] * inv, hh[7] * inv);
      }
      *reinterpret_cast<uint2*>(Xq + row * (int64_t)K + 8 * c) = make_uint2(w0, w1);
    };
    if constexpr (NCH > 0) {
#pragma unroll
      for (int i = 0; i < NCH; ++i) chunk(i * T + threadIdx.x, hv[i]);
    } else {
      for (int b = 0; b < nchunk; b += T) chunk(b + threadIdx.x, hv[0]);
    }
    amax = wave_max(amax);
    if ((threadIdx.x & (kWave - 1)) == 0) wmax[flip][threadIdx.x / kWave] = amax;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < T / kWave; ++w) amax = fmaxf(amax, wmax[flip][w]);
    amax = fmaxf(amax, 1e-5f);
    const float inv = __fdiv_rn(qmax, amax);
    if (threadIdx.x == 0) xdq[row] = __fdiv_rn(amax, qmax);
    if constexpr (NCH > 0) {
#pragma unroll
      for (int i = 0; i < NCH; ++i) codes(i * T + threadIdx.x, hv[i], inv);
    } else {
      for (int c = threadIdx.x; c < nchunk; c += T) {
        float g[8], u[8];
        load8(gr + 8 * c, g);
        load8(ur + 8 * c, u);
        silu_mul8<E4M3>(g, u, hv[0]);
        codes(c, hv[0], inv);
      }
    }
  }
}

// Threads by the row's length, so that a thread holds up to 3 chunks (4 in rows of
// more than 12288) and few lanes idle.  8192 rows of bf16, this rule / 512 threads
// that form h twice / 256 threads with all chunks in registers / 512 or 1024 with
// one or two: K = 2048 20.0 / 44.1 / 19.8 / 31.5 us, 5632 44.6 / 86.9 / 45.5 /
// 57.3, 8192 69.4 / 104 / 73.8 / 69.5, 11008 98 to 108 / 148 / 98 / 152, 16384
// 140 / 200 / 138 / 164; few rows are faster with more threads.
template <typename TX, bool E4M3, bool CKPT>
hipError_t launch_fwd(const TX* g, const TX* u, int64_t M, int K, uint8_t* q, float* xdq, const Ckpt& ck, hipStream_t s) {
  const int nchunk = K / 8;
  const dim3 grid((unsigned)(M < 65536 ? M : 65536));
  auto go = [&](auto kernel, int t) { return launch_kernel(kernel, grid, dim3(t), s, g, u, M, K, q, xdq, ck); };
  if (nchunk <= 256) return go(swiglu_quant_kernel<TX, E4M3, CKPT, 256, 1>, 256);
  if (nchunk <= 512) return go(swiglu_quant_kernel<TX, E4M3, CKPT, 256, 2>, 256);
  if (nchunk <= 768) return go(swiglu_quant_kernel<TX, E4M3, CKPT, 256, 3>, 256);
  if (nchunk <= 1024) return go(swiglu_quant_kernel<TX, E4M3, CKPT, 512, 2>, 512);
  if (nchunk <= 1536) return go(swiglu_quant_kernel<TX, E4M3, CKPT, 512, 3>, 512);
  if (nchunk <= 2048) return go(swiglu_quant_kernel<TX, E4M3, CKPT, 512, 4>, 512);
  return go(swiglu_quant_kernel<TX, E4M3, CKPT, 512, 0>, 512);
}

// (dG or dU may be dH: no __restrict__ on them)
template <typename TH, bool CKPT>
__global__ __launch_bounds__(256) void swiglu_bwd_kernel(const TH* dH, const TH* __restrict__ G, const TH* __restrict__ U,
                                                         Ckpt ck, uint32_t n, uint32_t nchunk, TH* dG, TH* dU) {
  const uint32_t ngroup = (nchunk + 15) / 16;
  for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (uint64_t)gridDim.x * 256) {
    float d[8], g[8], u[8], og[8], ou[8];
    load8(dH + 8 * i, d);
    if constexpr (CKPT) {
      const uint32_t row = (uint32_t)i / nchunk, c = (uint32_t)i - row * nchunk;
      const uint64_t sg = (uint64_t)row * ngroup + c / 16;
      const float a = ck.gs[sg], b = ck.us[sg];
      const uint2 x = *reinterpret_cast<const uint2*>(ck.Gq + 8 * i), y = *reinterpret_cast<const uint2*>(ck.Uq + 8 * i);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        g[j] = (float)(int8_t)((j < 4 ? x.x : x.y) >> (8 * (j & 3))) * a;
        u[j] = (float)(int8_t)((j < 4 ? y.x : y.y) >> (8 * (j & 3))) * b;
      }
    } else {
      load8(G + 8 * i, g);
      load8(U + 8 * i, u);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float s = __builtin_amdgcn_rcpf(1.0f + expf(-g[j]));    // (within one unit in the last place)
      ou[j] = d[j] * (g[j] * s);
      og[j] = d[j] * u[j] * (s * (1.0f + g[j] * (1.0f - s)));
    }
    store8(dG + 8 * i, og);
    store8(dU + 8 * i, ou);
  }
}

}  // namespace

hipError_t launch_swiglu_act_quant(const void* G, const void* U, bool x_bf16, int64_t M, int K, bool e4m3, void* Xq,
                                   float* xdq, const Ckpt& ck, hipStream_t s) {
  uint8_t* q = static_cast<uint8_t*>(Xq);
  const bool c = ck.Gq != nullptr;
  auto go = [&](auto t) {
    using TX = decltype(t);
    const TX* g = static_cast<const TX*>(G);
    const TX* u = static_cast<const TX*>(U);
    if (e4m3) return c ? launch_fwd<TX, true, true>(g, u, M, K, q, xdq, ck, s) : launch_fwd<TX, true, false>(g, u, M, K, q, xdq, ck, s);
    return c ? launch_fwd<TX, false, true>(g, u, M, K, q, xdq, ck, s) : launch_fwd<TX, false, false>(g, u, M, K, q, xdq, ck, s);
  };
  return x_bf16 ? go(uint16_t{}) : go(float{});
}

hipError_t launch_swiglu_backward(const void* dH, bool h_bf16, const void* G, const void* U, const Ckpt& ck, int64_t M,
                                  int K, void* dG, void* dU, hipStream_t s) {
  const uint32_t nchunk = K / 8, n = (uint32_t)(M * nchunk);
  const uint32_t blocks = n / 256 + (n % 256 != 0);
  const dim3 grid(blocks < (1u << 20) ? blocks : 1u << 20), block(256);
  auto go = [&](auto t) {
    using TH = decltype(t);
    auto* k = ck.Gq != nullptr ? swiglu_bwd_kernel<TH, true> : swiglu_bwd_kernel<TH, false>;
    return launch_kernel(k, grid, block, s, static_cast<const TH*>(dH), static_cast<const TH*>(G),
                         static_cast<const TH*>(U), ck, n, nchunk, static_cast<TH*>(dG), static_cast<TH*>(dU));
  };
  return h_bf16 ? go(uint16_t{}) : go(float{});
}

}  // namespace dqt
