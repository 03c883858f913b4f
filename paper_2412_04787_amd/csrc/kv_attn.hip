// Attention of new tokens over the 8-bit cache.
//
// Query row r of a sequence and key head (token r / G, head r % G of the G query heads
// that share it) sees keys j <= token + lk - lq (causal).  With codes k_j, v_j of page
// scales a_j, b_j = 2^ev (powers of two) and c = scale log2 e:
//   u_j = c a_j q.k_j + ev,  M = max u_j so far,  w_j = 2^(u_j - M + 8),
//   o = sum w_j v_j / l,  l = sum w_j 2^-ev,  lse = ln 2 (M - 8 + log2 l)
// so that the values' scale rides in the exponent and o is summed from codes.  l is 0
// for a row that sees nothing and no other: where scores are NaN, which no maximum keeps,
// M may be -inf too, and l is NaN.
//
// Both products run on the matrix cores in 16-bit floating point (fp16), which holds
// every code exactly; the row of Q is brought to 2^14 .. 2^15 by a power of two (bf16
// values fit, those below 2^-31 of the row's largest or 2^-57 lose bits), and w, at most
// 2^14, is off by 2^-11 of itself (below 2^-14, which is 2^-22 of the largest, by 2^-25).
// In bf16 it would be off by 2^-8, as much as the result's own rounding.
#include "kv_common.h"

namespace dqt {

namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
using lds_f32 = __attribute__((address_space(3))) float;
using lds_i32x4 = __attribute__((address_space(3))) i32x4;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLift = 8.0f;        // w = 2^(u - M + kLift)
constexpr float kSlack = 6.0f;       // M moves when u passes it by more: w <= 2^14

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ int row_token(const KvAttnArgs& a, int r) {
  return (int)((__umulhi((uint32_t)r, a.gmul) + ((uint32_t)r & a.gone)) >> a.gshift);
}

// 4 codes -> 4 fp16 values, exactly
template <bool E4M3>
__device__ __forceinline__ uint2 widen4(uint32_t w) {
  if constexpr (E4M3) {
    return uint2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true))};
  } else {
    // x + 128 in the low byte of 1024.0 is 1024 + x + 128
    const uint32_t u = w ^ 0x80808080u;
    const f16x2 off = {(_Float16)1152, (_Float16)1152};
    const f16x2 lo = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) - off;
    const f16x2 hi = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) - off;
    return uint2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
  }
}
template <bool E4M3>
__device__ __forceinline__ f16x8 widen8(int w0, int w1) {
  const uint2 a = widen4<E4M3>((uint32_t)w0), b = widen4<E4M3>((uint32_t)w1);
  return __builtin_bit_cast(f16x8, i32x4{(int)a.x, (int)a.y, (int)b.x, (int)b.y});
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  const f32x2_t v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
}
// the power of two k with 2^14 <= most 2^-k < 2^15 (no less than -40: times the smallest
// scales of a call and of a page, 2^-20 and 2^-64, 2^k is still a normal number, which c
// has to be where scores are -inf)
__device__ __forceinline__ int row_shift(float most) {
  return max((int)(__float_as_uint(most) >> 23) - 127 - 14, -40);
}
__device__ __forceinline__ float finite_abs(uint32_t bits) {
  const float a = fabsf(__uint_as_float(bits));
  return a <= 3.402823466e38f ? a : 0.0f;
}
// 8 bf16 values times f -> fp16
__device__ __forceinline__ f16x8 scaled_row(i32x4 x, float f) {
  i32x4 y;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    y[i] = (int)pack_f16x2(__uint_as_float((uint32_t)x[i] << 16) * f, __uint_as_float((uint32_t)x[i] & 0xFFFF0000u) * f);
  return __builtin_bit_cast(f16x8, y);
}
__device__ __forceinline__ float row_most(i32x4 x) {
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    m = fmaxf(m, fmaxf(finite_abs((uint32_t)x[i] << 16), finite_abs((uint32_t)x[i] & 0xFFFF0000u)));
  return m;
}
__device__ __forceinline__ f32x16 splat(float x) {
  f32x16 v;
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = x;
  return v;
}
// bytes 4 i .. 4 i + 3 of 16, of which the first n count: a mask
__device__ __forceinline__ uint32_t keep_bytes(int n, int i) {
  const int k = n - 4 * i;
  return k >= 4 ? ~0u : k <= 0 ? 0u : (1u << (8 * k)) - 1;
}

// One tile of rows of one sequence and key head.
struct Tile {
  KvSeq q;
  int r0, rows;          // its first row, the sequence's rows
  int nblk;              // pages that its last row sees
};
__device__ __forceinline__ Tile tile_at(const KvAttnArgs& a, const KvSeq& q, int item) {
  Tile t{q, item * a.tile_rows, q.lq * a.c.group, 0};
  if (item >= 0 && t.r0 < t.rows) {
    const int last = a.causal ? row_token(a, min(t.r0 + a.tile_rows, t.rows) - 1) + q.lk - q.lq : q.lk - 1;
    t.nblk = last < 0 ? 0 : last / kPage + 1;
  }
  return t;
}

// ------------------------------------------------------------------ few rows
// 16 NT rows of a sequence and key head over a range of pages, which the block's four
// waves take in turn and join at the end.  Codes go from memory to registers and into
// the matrix cores, 16 consecutive bytes per lane and load, without LDS: a wave holds
// a whole page (64 tokens) of keys and one of values, and the next page's keys are
// loaded while this one's are worked on.  Bound by HBM for single tokens: 32 over 1 to
// 8192 tokens, 32 heads on 8, 50 us for 0.27 GB (5.4 TB/s) and the join of the parts 4.7;
// two sequences of 30000 and 65000, 3 to 5 tokens each, 16 heads, int8: 74.5 us for 0.39
// GB (5.3 TB/s), 4.6.  Three waves per SIMD (two for 32 rows).
//
// v_mfma_f32_16x16x32_f16: A lane l holds row l % 16, 8 values of the reduction from
// 8 (l / 16); B the same of columns; result register i is row 4 (l / 16) + i of column
// l % 16.  Scores are formed transposed, 16 tokens x 16 rows.  A lane's 16 bytes of a
// key row serve two steps of the reduction over d (Q is read in the same order), and
// token 16 (m / 4) + 4 t + m % 4 of a page is row m of token tile t, so that a lane's
// results of four tiles are tokens 16 (l / 16) + 0..15: those of the 16 bytes that
// it loads of a value channel, and, as they are, the second product's B operand.
template <bool ONCE>
__device__ __forceinline__ i32x4 load_codes(const uint8_t* p) {
  if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const i32x4*>(p));
  return *reinterpret_cast<const i32x4*>(p);
}

template <int D, bool E4M3, int NT, bool ONCE>
__global__ __launch_bounds__(256, NT == 1 ? 3 : 2) void kv_attn_kernel(KvAttnArgs a) {
  constexpr int KJ = D / 64, ND = D / 16, ROWS = 16 * NT, OROW = D + 4;
  __shared__ float part_o[4][ROWS][OROW];
  __shared__ float part_m[4][ROWS], part_l[4][ROWS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, g = lane >> 4;
  int id = blockIdx.x, item;
  const int kvh = id % a.c.kv_heads;
  id /= a.c.kv_heads;
  const int split = id / a.tiles, first = split * a.chunk;
  // a tile for each sequence and a cache that fits the last-level one: the table is asked
  // beside the length, not after it (16 x 4096 tokens, 32 heads on 8: 29.4 -> 27.8 us; with
  // larger ones the many blocks behind the ends of short sequences wait for it as well,
  // 32 over 1 to 8192: 55.6 -> 57.4)
  const bool one = !ONCE && a.tiles == a.c.n_seq;
  int early = -1;
  if (one && first + wave + 4 * lane < min(first + a.chunk, (a.c.max_len + kPage - 1) / kPage))
    early = a.c.table[(int64_t)(id - split * a.tiles) * a.c.table_stride + first + wave + 4 * lane];
  const Tile t = tile_at(a, kv_find(a.c, id - split * a.tiles, a.c.group, ROWS, 1, item), item);
  if (item < 0 || t.r0 >= t.rows) return;
  const int end = min(first + a.chunk, t.nblk);
  if (split > 0 && first >= t.nblk) return;
  const bool whole = t.nblk <= a.chunk;             // no other block works on these rows

  // the rows
  i32x4 qraw[NT][2 * KJ];
  int lim[NT], tok[NT], head[NT];
  f16x8 qf[NT][2 * KJ];
  float qc[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = min(t.r0 + 16 * nt + n, t.rows - 1);
    tok[nt] = row_token(a, r);
    head[nt] = kvh * a.c.group + (r - tok[nt] * a.c.group);
    lim[nt] = a.causal ? tok[nt] + t.q.lk - t.q.lq : t.q.lk - 1;
    const uint8_t* p = a.Q + (int64_t)(t.q.q0 + tok[nt]) * a.q_tok + head[nt] * a.q_head;
#pragma unroll
    for (int j = 0; j < KJ; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) qraw[nt][2 * j + e] = *reinterpret_cast<const i32x4*>(p + 2 * (64 * j + 16 * g + 8 * e));
  }
  const int lim_lo = __builtin_amdgcn_readfirstlane(lim[0]);

  // this wave's pages of up to 256 of the block's, one per lane
  int page;
  float ks, vs;
  auto find_pages = [&](int from) {
    const int blk = from + wave + 4 * lane;
    page = -1;
    ks = vs = 1.0f;
    if (blk < end) page = one && from == first ? early : a.c.table[(int64_t)t.q.s * a.c.table_stride + blk];
    if (page < 0 || page >= a.c.pages) page = -1;
    if (page >= 0) {
      const float2 s = *reinterpret_cast<const float2*>(a.c.scales + 2 * ((int64_t)page * a.c.kv_heads + kvh));
      ks = s.x;
      vs = s.y;
    }
  };

  // page i of this wave -> its codes
  const uint32_t koff = (16 * (n >> 2) + (n & 3)) * D + 16 * g, voff = n * kPage + 16 * g;
  auto block_at = [&](int i) {
    const int p = __builtin_amdgcn_readlane(page, i);
    return ((int64_t)p * a.c.kv_heads + kvh) * (int64_t)(kPage * D);
  };
  i32x4 kraw[4][KJ], vraw[ND];
  auto load_k = [&](int i) {
    const uint8_t* p = a.c.K + block_at(i);
#pragma unroll
    for (int mt = 0; mt < 4; ++mt)
#pragma unroll
      for (int j = 0; j < KJ; ++j) kraw[mt][j] = load_codes<ONCE>(p + koff + 4 * D * mt + 64 * j);
  };
  auto load_v = [&](int i) {
    const uint8_t* p = a.c.V + block_at(i);
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) vraw[dt] = load_codes<ONCE>(p + voff + 16 * kPage * dt);
  };

  unsigned long long todo;
  int i;
  auto begin = [&](int from) {
    find_pages(from);
    todo = __ballot(page >= 0);
    i = todo ? __builtin_ctzll(todo) : 0;
    if (todo) {
      load_k(i);
      load_v(i);
    }
  };
  begin(first);

#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float most = 0.0f;
#pragma unroll
    for (int j = 0; j < 2 * KJ; ++j) most = fmaxf(most, row_most(qraw[nt][j]));
    most = fmaxf(most, __shfl_xor(most, 16, kWave));
    most = fmaxf(most, __shfl_xor(most, 32, kWave));
    const int k = row_shift(most);
    const float f = exp2_int(-k);
    qc[nt] = a.scale * kLog2e * exp2_int(k);
#pragma unroll
    for (int j = 0; j < 2 * KJ; ++j) qf[nt][j] = scaled_row(qraw[nt][j], f);
  }

  f32x4 o[NT][ND];
  float m[NT], l[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    m[nt] = -__builtin_inff();
    l[nt] = 0.0f;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) o[nt][dt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }

  for (int from = first;;) {
    while (todo) {
      todo &= todo - 1;
      const int next = todo ? __builtin_ctzll(todo) : -1;
      const int at = (from + wave + 4 * i) * kPage;           // the page's first token
      const float kscale = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ks), i));
      const int ev = exp_of(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vs), i)));

      f32x4 s[NT][4];
#pragma unroll
      for (int mt = 0; mt < 4; ++mt) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s[nt][mt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < KJ; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const f16x8 k8 = widen8<E4M3>(kraw[mt][j][2 * e], kraw[mt][j][2 * e + 1]);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
              s[nt][mt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k8, qf[nt][2 * j + e], s[nt][mt], 0, 0, 0);
          }
      }
      if (next >= 0) load_k(next);

      f16x8 w[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        if (at + kPage - 1 > lim_lo) {
#pragma unroll
          for (int mt = 0; mt < 4; ++mt)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (at + 16 * g + 4 * mt + e > lim[nt]) s[nt][mt][e] = -__builtin_inff();
        }
        float mx = -__builtin_inff();
#pragma unroll
        for (int mt = 0; mt < 4; ++mt)
#pragma unroll
          for (int e = 0; e < 4; e += 2) mx = fmaxf(mx, fmaxf(s[nt][mt][e], s[nt][mt][e + 1]));
        mx = fmaxf(mx, __shfl_xor(mx, 16, kWave));
        mx = fmaxf(mx, __shfl_xor(mx, 32, kWave));
        const float c = kscale * qc[nt], u = mx * c + (float)ev;
        if (__ballot(u > m[nt] + kSlack)) {
          const float to = fmaxf(m[nt], u), f = to == m[nt] ? 1.0f : exp2_fast(m[nt] - to);
          m[nt] = to;
          l[nt] *= f;
#pragma unroll
          for (int dt = 0; dt < ND; ++dt) o[nt][dt] *= f;
        }
        const float b = (float)ev + kLift - (m[nt] == -__builtin_inff() ? 0.0f : m[nt]);
        float sum = 0.0f;
#pragma unroll
        for (int mt = 0; mt < 4; ++mt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s[nt][mt][e] = exp2_fast(__builtin_fmaf(s[nt][mt][e], c, b));
            sum += s[nt][mt][e];
          }
        l[nt] += sum * exp2_int(-ev);
#pragma unroll
        for (int h = 0; h < 2; ++h)
          w[nt][h] = __builtin_bit_cast(f16x8, i32x4{(int)pack_f16x2(s[nt][2 * h][0], s[nt][2 * h][1]),
                                                     (int)pack_f16x2(s[nt][2 * h][2], s[nt][2 * h][3]),
                                                     (int)pack_f16x2(s[nt][2 * h + 1][0], s[nt][2 * h + 1][1]),
                                                     (int)pack_f16x2(s[nt][2 * h + 1][2], s[nt][2 * h + 1][3])});
      }
      if (at + kPage > t.q.lk) {                               // what lies behind the last token is not read
        const int have = t.q.lk - at - 16 * g;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
          for (int e = 0; e < 4; ++e) vraw[dt][e] &= (int)keep_bytes(have, e);
      }
#pragma unroll
      for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const f16x8 v8 = widen8<E4M3>(vraw[dt][2 * h], vraw[dt][2 * h + 1]);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) o[nt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v8, w[nt][h], o[nt][dt], 0, 0, 0);
        }
      if (next >= 0) load_v(next);
      i = next;
    }
    from += 4 * kWave;
    if (from >= end) break;
    begin(from);
  }

  // the four waves' sums on a common M
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    l[nt] += __shfl_xor(l[nt], 16, kWave);
    l[nt] += __shfl_xor(l[nt], 32, kWave);
    if (g == 0) {
      part_m[wave][16 * nt + n] = m[nt];
      part_l[wave][16 * nt + n] = l[nt];
    }
  }
  __syncthreads();
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = 16 * nt + n;
    const float all = fmaxf(fmaxf(part_m[0][r], part_m[1][r]), fmaxf(part_m[2][r], part_m[3][r]));
    const float f = m[nt] == all ? 1.0f : exp2_fast(m[nt] - all);
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) *reinterpret_cast<f32x4*>(&part_o[wave][r][16 * dt + 4 * g]) = o[nt][dt] * f;
  }
  __syncthreads();
  for (int x = threadIdx.x; x < ROWS * (D / 4); x += 256) {
    const int r = x / (D / 4), d = 4 * (x % (D / 4));
    if (t.r0 + r >= t.rows) break;
    float all = part_m[0][r], sum = 0.0f;
#pragma unroll
    for (int v = 1; v < 4; ++v) all = fmaxf(all, part_m[v][r]);
#pragma unroll
    for (int v = 0; v < 4; ++v) sum += part_m[v][r] == all ? part_l[v][r] : part_l[v][r] * exp2_fast(part_m[v][r] - all);
    f32x4 y = *reinterpret_cast<const f32x4*>(&part_o[0][r][d]);
#pragma unroll
    for (int v = 1; v < 4; ++v) y += *reinterpret_cast<const f32x4*>(&part_o[v][r][d]);
    y *= sum == 0.0f ? 0.0f : 1.0f / sum;
    const float lse = sum == 0.0f ? -__builtin_inff() : all - kLift + log2f(sum);
    const int tk = row_token(a, t.r0 + r), hd = kvh * a.c.group + (t.r0 + r - tk * a.c.group);
    const int64_t row = t.q.q0 + tk;
    if (whole) {
      *reinterpret_cast<uint2*>(a.O + row * a.o_tok + hd * a.o_head + 2 * d) = uint2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
      if (d == 0 && a.lse != nullptr) a.lse[(int64_t)hd * a.c.tq + row] = lse * kLn2;
    } else {
      const int64_t at = ((int64_t)split * a.c.tq + row) * a.c.heads + hd;
      *reinterpret_cast<f32x4*>(a.part + at * D + d) = y;
      if (d == 0) a.part_lse[at] = lse;
    }
  }
}

// ------------------------------------------------------------------ many rows
// 128 rows of a sequence and key head, 32 per wave, by two groups of four waves, which
// take every second page each and join at the end (a block is done in half the time,
// which counts where contexts differ: the longest block ends the kernel).  A group
// loads a page's codes to registers while the page before is worked on, widens them
// once for its 128 rows and passes them through LDS as fp16, two stages.
//
// Bound by what a wave issues between its products: of 197 us (8 chunks of 130 to 512
// tokens over 460 to 7870, 32 heads on 8: 163 GFLOP, 825 TFLOP/s; 240 us for the first
// launches after a pause, 195 from some 40 ms of them on) the staging takes
// about 45, the reads of LDS 30, the exponentials 12.  The scheduling groups keep reads
// ahead of the products and vector work beside them (without: 209 us); three waves per
// SIMD do not fit their registers, groups half a round apart, raw codes two pages
// ahead and sums watched instead of maxima gave nothing; 256 rows, eight waves on one
// page, gain 6 % in rate but end later, their blocks being twice as long (236 us).
//
// v_mfma_f32_32x32x16_f16: A lane l holds row l % 32, 8 values of the reduction from
// 8 (l / 32); B the same of columns; result register i is row 8 (i / 4) + 4 (l / 32) +
// i % 4 of column l % 32.  Scores are formed transposed (A = keys); key 8 h + 4 x + y of
// 16 is row 8 x + 4 h + y of the tile, so that registers 8 k .. 8 k + 7 are keys
// 16 k + 8 (l / 32) + 0..7: the second product's B operand as they are, beside 16 bytes
// of a value channel, whose tokens the cache keeps together.
constexpr int kTileRows = 128, kMaxSplits = 32;

// The tile of rank p, those of the longest sequences first: a block's time goes by the
// pages that its sequence has, and the long ones that began last ended the kernel (8
// chunks over 460 to 7870 tokens: 19 % of it).  Up to 64 sequences, one per lane; more:
// in their order.
__device__ __forceinline__ KvSeq find_longest(const KvAttnArgs& a, int p, int& item) {
  if (a.c.n_seq > kWave) return kv_find(a.c, p, a.c.group, kTileRows, 1, item);
  const int lane = threadIdx.x & (kWave - 1);
  const KvSeq q = kv_seq_of_lane(a.c);
  const int n = (int)(((int64_t)q.lq * a.c.group + kTileRows - 1) / kTileRows);
  int before = 0;
  for (int s = 0; s < a.c.n_seq; ++s) {
    const int lk = __builtin_amdgcn_readlane(q.lk, s), tiles = __builtin_amdgcn_readlane(n, s);
    before += lk > q.lk || (lk == q.lk && s < lane) ? tiles : 0;
  }
  const unsigned long long here = __ballot(before <= p && p < before + n);
  if (here == 0) {
    item = -1;
    return KvSeq{0, 0, 0, 0};
  }
  const int s = __builtin_ctzll(here);
  item = p - __builtin_amdgcn_readlane(before, s);
  return KvSeq{s, __builtin_amdgcn_readlane(q.q0, s), __builtin_amdgcn_readlane(q.lq, s), __builtin_amdgcn_readlane(q.lk, s)};
}

template <int D, bool E4M3>
__global__ __launch_bounds__(512, D == 64 ? 4 : 2) void kv_tile_kernel(KvAttnArgs a) {
  // rows of a staged tile end in 16 bytes that nothing uses: the 16 rows that as many
  // lanes read at one place then fall on all banks, at offsets that are constants
  constexpr int NK = D / 16, ND = D / 32, CH = kPage * D / 16 / 256, GR = 2;
  constexpr int kAhead = D == 64 ? 2 : 6;          // reads ahead of the scores' products
  constexpr int KROW = 2 * D + 16, VROW = 2 * kPage + 16, KB = kPage * KROW, VB = D * VROW, GB = 2 * (KB + VB);
  __shared__ __attribute__((aligned(1024))) uint8_t smem[GR * GB];         // of each group: keys, values; two stages
  __shared__ float row_m[GR][kTileRows], row_l[GR][kTileRows];
  const int lane = threadIdx.x & 63, h = lane >> 5, n = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w = wave & 3, grp = wave >> 2;
  const int tid = threadIdx.x & 255;
  int id = blockIdx.x, item;
  const int kvh = id % a.c.kv_heads;
  id /= a.c.kv_heads;
  const int split = id / a.tiles;
  const Tile t = tile_at(a, find_longest(a, id - split * a.tiles, item), item);
  if (item < 0 || t.r0 >= t.rows) return;
  const int first = split * a.chunk, end = min(first + a.chunk, t.nblk);
  if (split > 0 && first >= t.nblk) return;
  const bool whole = t.nblk <= a.chunk;             // no other block works on these rows

  // this lane's row
  const int r = min(t.r0 + 32 * w + n, t.rows - 1);
  const int tok = row_token(a, r), head = kvh * a.c.group + (r - tok * a.c.group);
  const int lim = a.causal ? tok + t.q.lk - t.q.lq : t.q.lk - 1;
  const int lim_lo = __builtin_amdgcn_readlane(lim, 0);
  const int lim_hi = t.r0 + 32 * w < t.rows ? __builtin_amdgcn_readlane(lim, 31) : -1;
  i32x4 qraw[NK];
  const uint8_t* qp = a.Q + (int64_t)(t.q.q0 + tok) * a.q_tok + head * a.q_head;
#pragma unroll
  for (int ks = 0; ks < NK; ++ks) qraw[ks] = *reinterpret_cast<const i32x4*>(qp + 32 * ks + 16 * h);

  // pages of this group (up to 128 of the block's at a time), one per lane
  int page;
  float ks_, vs_;
  auto find_pages = [&](int from) {
    const int blk = from + grp + GR * lane;
    page = -1;
    ks_ = vs_ = 1.0f;
    if (blk < end) page = a.c.table[(int64_t)t.q.s * a.c.table_stride + blk];
    if (page < 0 || page >= a.c.pages) page = -1;
    if (page >= 0) {
      const float2 s = *reinterpret_cast<const float2*>(a.c.scales + 2 * ((int64_t)page * a.c.kv_heads + kvh));
      ks_ = s.x;
      vs_ = s.y;
    }
  };
  auto kscale = [&](int i) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ks_), i)); };
  auto vexp = [&](int i) { return exp_of(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vs_), i))); };
  // codes of page i (zeros of one that is not there, or behind the last)
  i32x4 kraw[CH], vraw[CH];
  // (of a page's keys a thread takes every 256th run of 16 bytes; of its values those of
  // one row for 16 lanes of a quarter each, whose stores fall on all banks)
  const int vrow = 16 * w + (lane & 15), vat = 4 * vrow + (lane >> 4);
  auto load = [&](const uint8_t* base, int first, int i, i32x4 (&raw)[CH]) {
    const int p = i < kWave ? __builtin_amdgcn_readlane(page, i) : -1;
    if (p < 0) {
#pragma unroll
      for (int c = 0; c < CH; ++c) raw[c] = i32x4{0, 0, 0, 0};
    } else {
      const i32x4* x = reinterpret_cast<const i32x4*>(base + ((int64_t)p * a.c.kv_heads + kvh) * (int64_t)(kPage * D));
#pragma unroll
      for (int c = 0; c < CH; ++c) raw[c] = x[first + 256 * c];
    }
  };
  auto load_k = [&](int i) { load(a.c.K, tid, i, kraw); };
  auto load_v = [&](int i) { load(a.c.V, vat, i, vraw); };
  lds_u8* lds = (lds_u8*)&smem[0] + grp * GB;
  // codes -> fp16 in stage st; of the values, tokens behind the sequence's end as 0
  auto stage_k = [&](int st) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int p = tid + 256 * c, row = p / (D / 16), col = 2 * (p % (D / 16));
#pragma unroll
      for (int e = 0; e < 2; ++e)
        *(lds_i32x4*)(lds + st * KB + row * KROW + 16 * (col + e)) = __builtin_bit_cast(i32x4, widen8<E4M3>(kraw[c][2 * e], kraw[c][2 * e + 1]));
    }
  };
  auto cut_v = [&](int at) {
    if (at + kPage > t.q.lk) {
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) vraw[c][e] &= (int)keep_bytes(t.q.lk - at - 16 * (lane >> 4), e);
    }
  };
  auto stage_v = [&](int st) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int row = vrow + 64 * c, col = 2 * (lane >> 4);
#pragma unroll
      for (int e = 0; e < 2; ++e)
        *(lds_i32x4*)(lds + 2 * KB + st * VB + row * VROW + 16 * (col + e)) = __builtin_bit_cast(i32x4, widen8<E4M3>(vraw[c][2 * e], vraw[c][2 * e + 1]));
    }
  };

  f16x8 qf[NK];
  float qc;
  {
    float most = 0.0f;
#pragma unroll
    for (int ks = 0; ks < NK; ++ks) most = fmaxf(most, row_most(qraw[ks]));
    most = fmaxf(most, __shfl_xor(most, 32, kWave));
    const int k = row_shift(most);
    const float f = exp2_int(-k);
    qc = a.scale * kLog2e * exp2_int(k);
#pragma unroll
    for (int ks = 0; ks < NK; ++ks) qf[ks] = scaled_row(qraw[ks], f);
  }
  // row n of a key tile's 32 is this key
  const int key = (n & 16) + ((n & 4) << 1) + ((n & 8) >> 1) + (n & 3);
  const lds_u8 *kread = lds + key * KROW + 16 * h, *vread = lds + 2 * KB + n * VROW + 16 * h;

  f32x16 o[ND];
#pragma unroll
  for (int db = 0; db < ND; ++db) o[db] = splat(0.0f);
  float m = -__builtin_inff(), l = 0.0f;

  // groups of up to 128 pages; both groups of waves go round as often, for the barriers
  for (int from = first; from < end; from += GR * kWave) {
    find_pages(from);
    const int rounds = (min(end - from, GR * kWave) + GR - 1) / GR;
    auto at_of = [&](int i) { return (from + grp + GR * i) * kPage; };       // page i's first token
    f32x16 s[2];
    load_k(0);
    load_v(0);
    stage_k(0);
    cut_v(at_of(0));
    stage_v(0);
    load_k(1);
    load_v(1);
    __syncthreads();
    auto round = [&](int i, auto stage) {
      constexpr int S = decltype(stage)::value;
      const int at = at_of(i);
      const bool there = __builtin_amdgcn_readlane(page, i) >= 0 && at <= lim_hi;
      // the scores, beside them the staging of what comes (behind the last page: zeros)
      cut_v(at + GR * kPage);
#pragma unroll
      for (int nb = 0; nb < 2; ++nb) s[nb] = splat(0.0f);
#pragma unroll
      for (int ks = 0; ks < NK; ++ks)
#pragma unroll
        for (int nb = 0; nb < 2; ++nb)
          s[nb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
              __builtin_bit_cast(f16x8, *(const lds_i32x4*)(kread + S * KB + nb * 32 * KROW + 32 * ks)), qf[ks], s[nb], 0, 0, 0);
      stage_k(1 - S);
      stage_v(1 - S);
      // (reads run six ahead of the products: one behind each was waited for)
      __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
      for (int e = 0; e < 2 * NK; ++e) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if (e < 2 * NK - kAhead) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, E4M3 ? 2 : 5, 0);
        if (e >= 2 * NK - kAhead) __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);
      }
      load_k(i + 2);
      load_v(i + 2);
      if (there) {
        if (at + kPage - 1 > lim_lo) {
          const int left = lim - at - 8 * h;       // the last key seen, from this lane's first
#pragma unroll
          for (int nb = 0; nb < 2; ++nb)
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (32 * nb + 16 * (e / 8) + e % 8 > left) s[nb][e] = -__builtin_inff();
        }
        float mx = s[0][0];
#pragma unroll
        for (int e = 1; e < 32; ++e) mx = fmaxf(mx, s[e / 16][e % 16]);
        mx = fmaxf(mx, __shfl_xor(mx, 32, kWave));
        const int ev = vexp(i);
        const float c = kscale(i) * qc, u = mx * c + (float)ev;
        if (__ballot(u > m + kSlack)) {
          const float to = fmaxf(m, u), f = to == m ? 1.0f : exp2_fast(m - to);
          m = to;
          l *= f;
#pragma unroll
          for (int db = 0; db < ND; ++db) o[db] *= f;
        }
        const float b = (float)ev + kLift - (m == -__builtin_inff() ? 0.0f : m);
        float sum = 0.0f;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          float w[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            w[e] = exp2_fast(__builtin_fmaf(s[kk / 2][8 * (kk & 1) + e], c, b));
            sum += w[e];
          }
          const f16x8 p = __builtin_bit_cast(f16x8, i32x4{(int)pack_f16x2(w[0], w[1]), (int)pack_f16x2(w[2], w[3]),
                                                          (int)pack_f16x2(w[4], w[5]), (int)pack_f16x2(w[6], w[7])});
#pragma unroll
          for (int db = 0; db < ND; ++db)
            o[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
                __builtin_bit_cast(f16x8, *(const lds_i32x4*)(vread + S * VB + db * 32 * VROW + 32 * kk)), p, o[db], 0, 0, 0);
        }
        // the first values' reads, then the powers of 16 keys beside the product of the
        // 16 before, whose reads are ND ahead
        __builtin_amdgcn_sched_group_barrier(0x100, ND, 0);
        __builtin_amdgcn_sched_group_barrier(0x402, 28, 0);
#pragma unroll
        for (int e = 0; e < 3 * ND; ++e) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x402, 28 / ND, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, ND, 0);
        l += sum * exp2_int(-ev);
      }
      __syncthreads();
    };
    for (int i = 0; i < rounds; i += 2) {
      round(i, std::integral_constant<int, 0>{});
      if (i + 1 < rounds) round(i + 1, std::integral_constant<int, 1>{});
    }
  }

  // the two groups' sums on a common M: group g finishes channels g D / 2 ..
  l += __shfl_xor(l, 32, kWave);
  const int rr = 32 * w + n;
  if (h == 0) {
    row_m[grp][rr] = m;
    row_l[grp][rr] = l;
  }
  __syncthreads();
  const float m1 = row_m[1 - grp][rr], both = fmaxf(m, m1);
  const float f0 = m == both ? 1.0f : exp2_fast(m - both), f1 = m1 == both ? 1.0f : exp2_fast(m1 - both);
  const float total = l * f0 + row_l[1 - grp][rr] * f1;
  const bool none = total == 0.0f;
  const float inv = none ? 0.0f : 1.0f / total, lse = none ? -__builtin_inff() : both - kLift + log2f(total);
  lds_f32* give = (lds_f32*)&smem[0];
#pragma unroll
  for (int d = 0; d < ND / 2; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e)
      give[(((grp * 4 + w) * (ND / 2) + d) * 16 + e) * 64 + lane] = grp == 0 ? o[ND / 2 + d][e] : o[d][e];
  __syncthreads();
  const bool mine = t.r0 + rr < t.rows;
  const int64_t row = t.q.q0 + tok;
#pragma unroll
  for (int d = 0; d < ND / 2; ++d) {
    f32x16 y;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float own = grp == 0 ? o[d][e] : o[ND / 2 + d][e];
      y[e] = (own * f0 + give[((((1 - grp) * 4 + w) * (ND / 2) + d) * 16 + e) * 64 + lane] * f1) * inv;
    }
    const int d0 = 32 * (grp * (ND / 2) + d) + 4 * h;
    if (mine) {
      if (whole) {
        uint8_t* p = a.O + row * a.o_tok + head * a.o_head + 2 * d0;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          *reinterpret_cast<uint2*>(p + 16 * e) = uint2{pack_bf16x2(y[4 * e], y[4 * e + 1]), pack_bf16x2(y[4 * e + 2], y[4 * e + 3])};
      } else {
        float* p = a.part + (((int64_t)split * a.c.tq + row) * a.c.heads + head) * D + d0;
#pragma unroll
        for (int e = 0; e < 4; ++e) *reinterpret_cast<f32x4*>(p + 8 * e) = f32x4{y[4 * e], y[4 * e + 1], y[4 * e + 2], y[4 * e + 3]};
      }
    }
  }
  if (mine && grp == 0 && h == 0) {
    if (!whole) a.part_lse[((int64_t)split * a.c.tq + row) * a.c.heads + head] = lse;
    else if (a.lse != nullptr) a.lse[(int64_t)head * a.c.tq + row] = lse * kLn2;
  }
}

// Joins the parts of the rows that have several: o = sum_p 2^(L_p - L) o_p / sum_p
// 2^(L_p - L).  A block for a row, whose waves read GR parts at a time, 16 bytes per lane,
// four reads in flight; lane l holds the weight of part l for the others.  (A wave for each of
// 128 rows of 64 parts, when there could be as many, took 20 us.)
template <int D>
__global__ __launch_bounds__(256) void kv_join_kernel(KvAttnArgs a) {
  constexpr int GR = 256 / D, STEP = 4 * GR;
  static_assert(kMaxSplits <= 4 * STEP && 4 * STEP <= kWave, "a lane for each part, four reads for all");
  __shared__ f32x4 part[4][D / 4];
  __shared__ float part_sum[4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t at = blockIdx.x;
  const int row = (int)(at / a.c.heads), hd = (int)(at - (int64_t)row * a.c.heads);
  const int64_t step = (int64_t)a.c.tq * a.c.heads;
  // (of all splits: the ones that were not written are left out when the length is known)
  float mine = lane < a.splits ? a.part_lse[lane * step + at] : 0.0f;
  int item;
  const KvSeq q = a.c.q_start == nullptr ? kv_seq(a.c, row) : kv_find(a.c, row, 1, 1, 0, item);
  const int tok = row - q.q0;
  if (tok < 0 || tok >= q.lq) return;                // a token outside every sequence
  const int r = tok * a.c.group + hd % a.c.group;
  const Tile t = tile_at(a, q, r / a.tile_rows);
  if (t.nblk <= a.chunk) return;                     // (written already)
  const int parts = (t.nblk + a.chunk - 1) / a.chunk;
  if (lane >= parts) mine = -__builtin_inff();
  const float all = wave_max(mine), mw = exp2_fast(mine - (all == -__builtin_inff() ? 0.0f : all));
  const int d = 4 * (lane % (D / 4));
  f32x4 y = {0.0f, 0.0f, 0.0f, 0.0f};
  float sum = 0.0f;
  const int p0 = GR * wave + lane / (D / 4);
  f32x4 x[4];
#pragma unroll
  for (int e = 0; e < 4; ++e)
    x[e] = *reinterpret_cast<const f32x4*>(a.part + (min(p0 + e * STEP, parts - 1) * step + at) * D + d);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int p = p0 + e * STEP;
    const float w = __shfl(mw, p, kWave);
    if (p < parts) {
      y += w * x[e];
      sum += w;
    }
  }
#pragma unroll
  for (int x = D / 4; x < kWave; x *= 2) {
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] += __shfl_xor(y[e], x, kWave);
    sum += __shfl_xor(sum, x, kWave);
  }
  if (lane < D / 4) part[wave][lane] = y;
  if (lane == 0) part_sum[wave] = sum;
  __syncthreads();
  if (wave != 0 || lane >= D / 4) return;
  y = part[0][lane];
  sum = part_sum[0];
#pragma unroll
  for (int v = 1; v < 4; ++v) {
    y += part[v][lane];
    sum += part_sum[v];
  }
  const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
  *reinterpret_cast<uint2*>(a.O + row * a.o_tok + hd * a.o_head + 2 * d) = uint2{pack_bf16x2(y[0] * f, y[1] * f), pack_bf16x2(y[2] * f, y[3] * f)};
  if (lane == 0 && a.lse != nullptr) a.lse[(int64_t)hd * a.c.tq + row] = sum == 0.0f ? -__builtin_inff() : (all + log2f(sum)) * kLn2;
}

// The same for many rows of few parts: a wave joins those of 4 heads of a token, four reads
// in flight; lane l holds the weight of part l / 4 of head l % 4.  (A wave for each row,
// two parts of 82000: 247 us with the attention, 227.)
template <int D>
__global__ __launch_bounds__(256) void kv_join_heads_kernel(KvAttnArgs a) {
  constexpr int GR = 256 / D, NP = kWave / 4;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), per = (a.c.heads + 3) / 4;
  const int64_t id = (int64_t)blockIdx.x * 4 + wave;
  if (id >= (int64_t)a.c.tq * per) return;
  const int row = (int)(id / per), hd0 = 4 * (int)(id - (int64_t)row * per), nh = min(4, a.c.heads - hd0);
  const int64_t step = (int64_t)a.c.tq * a.c.heads, at0 = (int64_t)row * a.c.heads + hd0;
  const int hk = min(lane & 3, nh - 1), pl = lane >> 2;
  // (of all splits: the ones that were not written are left out when the length is known)
  float mine = pl < a.splits ? a.part_lse[pl * step + at0 + hk] : 0.0f;
  int item;
  const KvSeq q = a.c.q_start == nullptr ? kv_seq(a.c, row) : kv_find(a.c, row, 1, 1, 0, item);
  const int tok = row - q.q0;
  if (tok < 0 || tok >= q.lq) return;                // a token outside every sequence
  const int r = tok * a.c.group + (hd0 + hk) % a.c.group, nblk = tile_at(a, q, r / a.tile_rows).nblk;
  const int parts = nblk <= a.chunk ? 0 : (nblk + a.chunk - 1) / a.chunk;      // (none: written already)
  const int most = max(max(__builtin_amdgcn_readlane(parts, 0), __builtin_amdgcn_readlane(parts, 1)),
                       max(__builtin_amdgcn_readlane(parts, 2), __builtin_amdgcn_readlane(parts, 3)));
  if (most == 0) return;
  if (pl >= parts) mine = -__builtin_inff();
  float all = mine;
  for (int p = pl + NP; p < parts; p += NP) all = fmaxf(all, a.part_lse[p * step + at0 + hk]);
#pragma unroll
  for (int x = 4; x < kWave; x *= 2) all = fmaxf(all, __shfl_xor(all, x, kWave));
  const float base = all == -__builtin_inff() ? 0.0f : all;
  const int sub = lane / (D / 4), d = 4 * (lane % (D / 4));
  f32x4 y[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) y[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  float sum = 0.0f;
  for (int g = 0; g < most; g += NP) {
    if (g > 0) mine = g + pl < parts ? a.part_lse[(g + pl) * step + at0 + hk] : -__builtin_inff();
    const float mw = exp2_fast(mine - base);
    sum += mw;
    for (int p0 = 0; p0 < NP && g + p0 < most; p0 += GR) {
      f32x4 x[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int n = __builtin_amdgcn_readlane(parts, k);
        x[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if (k < nh && g + p0 + sub < n) x[k] = *reinterpret_cast<const f32x4*>(a.part + ((g + p0 + sub) * step + at0 + k) * D + d);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) y[k] += __shfl(mw, 4 * (p0 + sub) + k, kWave) * x[k];
    }
  }
#pragma unroll
  for (int x = 4; x < kWave; x *= 2) sum += __shfl_xor(sum, x, kWave);
#pragma unroll
  for (int x = D / 4; x < kWave; x *= 2)
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) y[k][e] += __shfl_xor(y[k][e], x, kWave);
#pragma unroll
  for (int k0 = 0; k0 < 4; k0 += GR) {
    const int k = k0 + sub;
    const float f = __shfl(sum == 0.0f ? 0.0f : 1.0f / sum, k, kWave);
    const int n = __shfl(parts, k, kWave);
    f32x4 v = y[k0];
#pragma unroll
    for (int e = 1; e < GR; ++e)
      if (sub == e) v = y[k0 + e];
    if (k < nh && n > 0)
      *reinterpret_cast<uint2*>(a.O + row * a.o_tok + (hd0 + k) * a.o_head + 2 * d) =
          uint2{pack_bf16x2(v[0] * f, v[1] * f), pack_bf16x2(v[2] * f, v[3] * f)};
  }
  if (lane < nh && parts > 0 && a.lse != nullptr)
    a.lse[(int64_t)(hd0 + lane) * a.c.tq + row] = sum == 0.0f ? -__builtin_inff() : (all + log2f(sum)) * kLn2;
}

}  // namespace

// The blocks of a tile size that have rows (when sequences have as many each).
static int64_t kv_blocks(const KvAttnArgs& a, int tile_rows) {
  const int64_t rows = (int64_t)a.c.tq * a.c.group, seqs = a.c.n_seq > 0 ? a.c.n_seq : 1;
  return seqs * ((rows + seqs * tile_rows - 1) / (seqs * tile_rows)) * a.c.kv_heads;
}

// Tile and splits by estimated time in us, fitted to what 120 calls of up to 16 rows a
// sequence and 105 of more took, over 400 to 65000 tokens, with 1 to 64 parts (what up to
// 48 and 64 would pick is level over these calls, 0.1 % better, and slower for the longest: two
// sequences of 30000 and 65000, 82.5 us, 79.6 with 32) and tiles of 32 and 128 rows.  x is the rounds of a block to each of 256
// units; a page costs a block of few rows what it waits for and a share of each round;
// blocks of 128 rows have a unit for themselves, and of unequal lengths fill the last
// round in part; a join costs 6.3 and 1 for 5000 rows of parts.  What is picked takes 3 %
// (up to 16 rows) and 4 % longer than the best of each call.  (8 blocks to a unit whatever
// they hold: 9 % for up to 16 rows; 128 rows from 48 on: two sequences of 243 and 468
// tokens over 484 and 1826, 24 heads of 64, 31 us, 32 rows 18; 32 rows always: 8 chunks of
// 130 to 512 over 457 to 7865, 32 heads on 8, 286 us, 128 rows 196.)
void kv_attn_plan(bool e4m3, KvAttnArgs* a) {
  const int64_t rows = (int64_t)a->c.tq * a->c.group, seqs = a->c.n_seq > 0 ? a->c.n_seq : 1;
  const int64_t pages = a->c.max_len > 0 ? ((int64_t)a->c.max_len + kPage - 1) / kPage : 1;
  const double w = a->c.d / 128.0, joined = (double)rows * a->c.kv_heads * (0.3 + 0.7 * w) / 5000;
  const double wait = 0.15 + 0.85 * w;
  double best = 1e300;
  auto look = [&](int tile_rows) {
    const int64_t blocks = kv_blocks(*a, tile_rows);
    // (parts of whole groups of 4 pages, one for each wave; grids stay far below their limit)
    const int64_t fit = (int64_t(1) << 22) / ((rows + seqs) * a->c.kv_heads), most = fit < 1 ? 1 : fit < kMaxSplits ? fit : kMaxSplits;
    for (int64_t s = 1; s <= most && 4 * (s - 1) < pages; ++s) {
      const int64_t chunk = ((pages + s - 1) / s + 3) / 4 * 4, parts = (pages + chunk - 1) / chunk;
      if (parts < s) continue;
      const double n = (double)(chunk < pages ? chunk : pages), x = blocks * s / 256.0, full = x > 1 ? x : 1;
      double us = parts > 1 ? 6.3 + joined * s : 0;
      if (tile_rows == 16) us += 4.6 + 0.33 * full + n * (0.15 * wait + 0.4 * w * full);
      else if (tile_rows == 32) us += 4.6 + 0.5 * full + n * (e4m3 ? 1 : 1.16) * (0.24 * wait + 0.25 * (0.2 + 0.8 * w) * full);
      else us += 1.6 + (x > 1 ? 0.8 * x + 0.2 * (double)((blocks * s + 255) / 256) : 1) * (3.4 + (0.57 + 0.32 * w) * n);
      if (us < best) {
        best = us;
        a->tile_rows = tile_rows;
        a->chunk = (int)chunk;
        a->splits = (int)parts;
      }
    }
  };
  if (rows <= 16 * seqs) {
    look(16);
  } else {
    look(32);
    look(kTileRows);
  }
  a->tiles = (int)(a->c.q_start == nullptr && a->c.group <= a->tile_rows ? a->c.n_seq : rows / a->tile_rows + a->c.n_seq);
}

hipError_t launch_kv_attn(bool e4m3, const KvAttnArgs& a, hipStream_t s) {
  const dim3 grid((uint32_t)((int64_t)a.tiles * a.c.kv_heads * a.splits));
  LaunchStatus st;
  // Blocks of few sequences are put on one compute unit while others have none: LDS that nothing
  // uses keeps them apart, as many to a unit as there are for each (256 tiles of 32 rows
  // over 4512 tokens, 128-wide heads: 55 -> 38 us).
  const int64_t each = (kv_blocks(a, a.tile_rows) * a.splits + 255) / 256, apart = 160 * 1024 / (each + 1) + 1024;
  const int64_t own = a.tile_rows == kTileRows ? 4 * (kPage * (2 * a.c.d + 16) + a.c.d * (2 * kPage + 16)) + 16 * kTileRows
                                               : 16 * a.tile_rows * (a.c.d + 6);
  const size_t idle = apart > own ? (size_t)(apart - own) : 0;
  auto go = [&](auto k) { st << launch_kernel_lds(k, grid, dim3(a.tile_rows == kTileRows ? 512 : 256), idle, s, a); };
  // each code is read by one block, and there are more than the last-level cache (256 MB)
  // holds from one call to the next: past it (32 tokens over 1 to 8192, 270 MB: 60.2 ->
  // 55.6 us; 79 MB that it may still hold: 28.0 -> 31.4).  Both sides with one cache, read
  // call after call: where a model's other layers read theirs in between, a smaller one
  // is as cold, which the call cannot know.
  const bool once = a.tiles == a.c.n_seq && (int64_t)a.c.n_seq * a.c.max_len * a.c.kv_heads * a.c.d * 2 > (int64_t)256 << 20;
  auto few = [&](auto d, auto fmt, auto nt) {
    constexpr int D = decltype(d)::value, NT = decltype(nt)::value;
    constexpr bool F = decltype(fmt)::value;
    once ? go(kv_attn_kernel<D, F, NT, true>) : go(kv_attn_kernel<D, F, NT, false>);
  };
  auto pick = [&](auto d, auto fmt) {
    constexpr int D = decltype(d)::value;
    constexpr bool F = decltype(fmt)::value;
    if (a.tile_rows == kTileRows) go(kv_tile_kernel<D, F>);
    else if (a.tile_rows == 16) few(d, fmt, std::integral_constant<int, 1>{});
    else few(d, fmt, std::integral_constant<int, 2>{});
  };
  auto width = [&](auto fmt) {
    a.c.d == 128 ? pick(std::integral_constant<int, 128>{}, fmt) : pick(std::integral_constant<int, 64>{}, fmt);
  };
  e4m3 ? width(std::true_type{}) : width(std::false_type{});
  if (a.splits > 1) {
    const int64_t rows = (int64_t)a.c.tq * a.c.heads;
    const bool wide = a.splits > 4 && rows <= 4096;
    const dim3 join((uint32_t)(wide ? rows : ((int64_t)a.c.tq * ((a.c.heads + 3) / 4) + 3) / 4));
    auto j = [&](auto k) { st << launch_kernel(k, join, dim3(256), s, a); };
    if (a.c.d == 128) wide ? j(kv_join_kernel<128>) : j(kv_join_heads_kernel<128>);
    else wide ? j(kv_join_kernel<64>) : j(kv_join_heads_kernel<64>);
  }
  return st.e;
}

}  // namespace dqt
