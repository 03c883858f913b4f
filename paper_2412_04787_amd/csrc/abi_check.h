// Argument checks that the C ABI's files share.
#pragma once

#include "../../include/dqt.h"
#include "dqt_launch.h"

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned8(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 7u) == 0; }
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

bool is_float_type(int32_t t) { return t == DQT_F32 || t == DQT_BF16; }

dqt_status from_hip(hipError_t e) { return e == hipSuccess ? DQT_OK : DQT_ERR_HIP; }

constexpr int64_t kMaxBlocks = int64_t(1) << 24;      // of 256 threads: the runtime's grids end at 2^32 threads

// r / g = (umulhi(r, mul) + (r & one)) >> shift for r < 2^31: mul = ceil(2^(31 + b) / g), b = ceil(log2 g)
void group_division(int64_t g, uint32_t* mul, uint32_t* one, int* shift) {
  *mul = 0;
  *one = g == 1 ? ~0u : 0u;
  *shift = 0;
  if (g == 1) return;
  int b = 1;
  while ((int64_t(1) << b) < g) ++b;
  *mul = (uint32_t)(((uint64_t(1) << (31 + b)) + g - 1) / g);
  *shift = b - 1;
}

// A strided tensor [tokens, heads, d] of bf16: non-negative strides that keep
// 16-byte alignment; an output's rows must not overlap.
dqt_status check_rows(const dqt_rows* t, int64_t tokens, int32_t heads, int32_t d, bool output) {
  if (t == nullptr) return DQT_ERR_NULL;
  if (tokens > 0 && t->p == nullptr) return DQT_ERR_NULL;
  if (!aligned16(t->p) || (t->token & 7) != 0 || (t->head & 7) != 0) return DQT_ERR_ALIGN;
  // (the kernels take a tile's rows, up to 128 tokens, at 32-bit offsets)
  if (t->token < 0 || t->head < 0 || t->token > (int64_t(1) << 23) || t->head > (int64_t(1) << 40)) return DQT_ERR_SHAPE;
  if (output && tokens > 0) {
    const bool by_token = (heads == 1 || t->head >= d) && (tokens == 1 || t->token >= (heads - 1) * t->head + d);
    const bool by_head = (tokens == 1 || t->token >= d) && (heads == 1 || t->head >= (tokens - 1) * t->token + d);
    if (!by_token && !by_head) return DQT_ERR_SHAPE;
  }
  return DQT_OK;
}

}  // namespace
