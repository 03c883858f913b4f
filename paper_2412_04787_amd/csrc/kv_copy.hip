// Copies of pages within caches: page src[i] to page dst[i], in each layer's cache.
// The lists come with the launch (the host checks them: no page is read and
// written).  A block copies 16 KB, 64 bytes in flight per thread.
#include "dqt_launch.h"

namespace dqt {

namespace {

constexpr int kChunk = 16384;

__global__ __launch_bounds__(256) void kv_copy_kernel(KvCopyArgs a) {
  const int pair = blockIdx.y, cache = blockIdx.z, tid = threadIdx.x;
  const int64_t src = a.p[pair].src, dst = a.p[pair].dst;
  const int parts = (int)((a.page_bytes + kChunk - 1) / kChunk);
  const bool values = (int)blockIdx.x >= parts;
  const int64_t at = (int64_t)((int)blockIdx.x - (values ? parts : 0)) * kChunk;
  uint8_t* base = values ? a.c[cache].V : a.c[cache].K;
  const uint8_t* from = base + src * a.page_bytes + at;
  uint8_t* to = base + dst * a.page_bytes + at;
  const int n = (int)min((int64_t)kChunk, a.page_bytes - at);       // a multiple of 4096
  i32x4 v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (4096 * i < n) v[i] = reinterpret_cast<const i32x4*>(from + 4096 * i)[tid];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (4096 * i < n) reinterpret_cast<i32x4*>(to + 4096 * i)[tid] = v[i];
  if (blockIdx.x == 0) {
    float* sc = a.c[cache].scales;
    for (int i = tid; i < 2 * a.kv_heads; i += 256) sc[dst * 2 * a.kv_heads + i] = sc[src * 2 * a.kv_heads + i];
  }
}

}  // namespace

hipError_t launch_kv_copy(const KvCopyArgs& a, int caches, int pages, hipStream_t s) {
  const uint32_t parts = (uint32_t)((a.page_bytes + kChunk - 1) / kChunk);
  return launch_kernel(kv_copy_kernel, dim3(2 * parts, (uint32_t)pages, (uint32_t)caches), dim3(256), s, a);
}

}  // namespace dqt
