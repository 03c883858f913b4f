// Copies of pages within caches: page src[i] to page dst[i], in each layer's cache.
// The lists come with the launch (the host checks them: no page is read and
// written).  Bound by HBM.  A block copies 4 KB, 16 bytes per thread, and its stores go
// past the caches: 16 pages in 24 layers of 16 heads of 128 (100 MB each way) 31 us, 6.4
// TB/s, 700 pages in 4 layers of 8 heads 136 us, 5.4 TB/s; 16 KB to a block 43 and 161
// us, with such stores 36.7 and 152.
#include "cache_launch.h"

namespace dqt {

namespace {

constexpr int kChunk = 4096;         // of which a page's codes are a multiple

__global__ __launch_bounds__(256) void kv_copy_kernel(KvCopyArgs a) {
  const int pair = blockIdx.y, cache = blockIdx.z, tid = threadIdx.x;
  const int64_t src = a.p[pair].src, dst = a.p[pair].dst;
  const uint32_t parts = gridDim.x / 2;
  const bool values = blockIdx.x >= parts;
  const int64_t at = (int64_t)(blockIdx.x - (values ? parts : 0)) * kChunk + 16 * tid;
  uint8_t* base = (values ? a.c[cache].V : a.c[cache].K) + at;
  __builtin_nontemporal_store(*reinterpret_cast<const i32x4*>(base + src * a.page_bytes),
                              reinterpret_cast<i32x4*>(base + dst * a.page_bytes));
  if (blockIdx.x == 0) {
    float* sc = a.c[cache].scales;
    for (int i = tid; i < 2 * a.kv_heads; i += 256) sc[dst * 2 * a.kv_heads + i] = sc[src * 2 * a.kv_heads + i];
  }
}

}  // namespace

hipError_t launch_kv_copy(const KvCopyArgs& a, int caches, int pages, hipStream_t s) {
  const uint32_t parts = (uint32_t)(a.page_bytes / kChunk);
  return launch_kernel(kv_copy_kernel, dim3(2 * parts, (uint32_t)pages, (uint32_t)caches), dim3(256), s, a);
}

}  // namespace dqt
