// Launch arguments of rotary positions and of the 8-bit cache of keys and values, for
// abi_cache.hip and their kernels.
#pragma once

#include "dqt_launch.h"

namespace dqt {

// Rotary positions (rope.hip); strides in bytes.
constexpr int kMaxRope = 4;
struct RopeIO {
  const uint8_t* X;
  uint8_t* Y;
  int64_t x_tok, x_head, y_tok, y_head;
  int heads;
};
struct RopeArgs {
  const uint64_t* freq;
  const int32_t* pos;          // [tokens], nullable
  RopeIO io[kMaxRope];
  int64_t tokens;
  double amp;
  int n, d, rot, pairs, back;
  int all_heads;               // of all tensors
  int items;                   // of a head: runs of 16 values
  int block_tokens;            // tokens of a block
};
hipError_t launch_rope(bool bf16, const RopeArgs& a, hipStream_t stream);

// The 8-bit cache of keys and values (kv_append.hip, kv_attn.hip, kv_copy.hip).
constexpr int kPage = 64;            // tokens
struct KvArgs {
  uint8_t *K, *V;                    // [pages, kv_heads, 64, d], [pages, kv_heads, d, 64]
  float* scales;                     // [pages, kv_heads, 2]
  int64_t pages;
  const int32_t *table, *kv_len, *q_start;
  int tq, n_seq, table_stride, max_len, heads, kv_heads, group;
  int d;
};
struct KvAppendArgs {
  KvArgs c;
  const uint8_t *k, *v, *q;          // new tokens (q nullable); strides in bytes
  uint8_t* qr;
  int64_t k_tok, k_head, v_tok, v_head, q_tok, q_head, qr_tok, qr_head;
  const uint64_t* freq;              // null: nothing is rotated
  double amp;
  int rot, pairs;
};
hipError_t launch_kv_append(bool e4m3, const KvAppendArgs& a, hipStream_t stream);

struct KvAttnArgs {
  KvArgs c;
  const uint8_t* Q;
  uint8_t* O;
  int64_t q_tok, q_head, o_tok, o_head;
  float* lse;                        // [heads, tq], nullable
  float scale;
  int causal;
  // r / group = (umulhi(r, gmul) + (r & gone)) >> gshift for r < 2^31
  uint32_t gmul, gone;
  int gshift;
  int tile_rows, tiles;              // rows per tile, tiles of all sequences at most
  int chunk, splits;                 // pages per split, splits
  float *part, *part_lse;            // [splits, tq, heads, d], [splits, tq, heads]
};
// fills tile_rows .. splits from the sizes
void kv_attn_plan(bool e4m3, KvAttnArgs* a);
hipError_t launch_kv_attn(bool e4m3, const KvAttnArgs& a, hipStream_t stream);

constexpr int kCopyCaches = 32, kCopyPages = 256;    // of one launch
struct KvCopyArgs {
  struct { uint8_t *K, *V; float* scales; } c[kCopyCaches];
  struct { int32_t src, dst; } p[kCopyPages];
  int64_t page_bytes;                // of K, as many of V
  int kv_heads;
};
hipError_t launch_kv_copy(const KvCopyArgs& a, int caches, int pages, hipStream_t stream);

}  // namespace dqt
