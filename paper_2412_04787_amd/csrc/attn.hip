// Softmax attention over packed sequences, forward and backward (bf16).
//
// Query i of a sequence of lq queries and lk keys sees key j when j < lk and,
// causal, j <= i + lk - lq.  For one query head h and its key head h / G
// (G = heads / kv_heads query heads share a key head), with c = scale:
//   z_ij = c q_i . k_j,  lse_i = log sum_j exp(z_ij),  p_ij = exp(z_ij - lse_i)
//   o_i = sum_j p_ij v_j
//   dv_j = sum_i p_ij do_i,  g_ij = p_ij (do_i . v_j - do_i . o_i)
//   dq_i = c sum_j g_ij k_j,  dk_j = c sum_i g_ij q_i      (i over all G heads)
// The scores never reach memory: the forward keeps a running maximum and sum
// per row, the backward forms p again from lse.
//
// Rows.  The G query heads of a key head and the tokens of a sequence form
// one list of rows, row r = token r / G, head r % G, so that a tile of rows
// reads the keys and values once for all the heads that share them, a single
// new token fills G rows of a tile, and dk and dv of a shared head are summed
// over its query heads in registers (fixed order, no atomics).
//
// Matrix layout (v_mfma_f32_32x32x16_bf16).  A operand: lane l holds row
// l % 32, 8 values of the reduction from 8 (l / 32); B the same for columns;
// result register i of lane l is row 8 (i / 4) + 4 (l / 32) + i % 4 of column
// l % 32.  The forward and dq form the scores transposed (A = keys, B = rows
// of Q), so that a lane holds scores of one query: the softmax statistics
// need one exchange between lane halves, and the scaling of o is per lane.
// The second product takes the score registers as its B operand as they are:
// registers 8 kk .. 8 kk + 7 of the two lane halves are keys
// 16 kk + 8 (j / 4) + 4 (l / 32) + j % 4, and the order of a reduction is free
// as long as the A operand (V or K, transposed by ds_read_b64_tr_b16) takes
// the same one.  dk/dv run the other way round (A = rows of Q, B = keys).
#include "dqt_launch.h"

namespace dqt {

namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
using lds_i32x4 = __attribute__((address_space(3))) i32x4;
using lds_f32x4 = __attribute__((address_space(3))) f32x4;
using lds_f32 = __attribute__((address_space(3))) float;

constexpr int kBM = 128;      // rows per block of the forward and dq, keys per block of dk/dv
constexpr int kKT = 64;       // keys (forward, dq) or rows (dk/dv) per staged tile
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// A staged tile: kKT rows of D bf16 values, 16-byte chunk c of row r at chunk
// c ^ swz(r).  With swz, the 16 rows that a straight read takes at one chunk,
// and the 4 x 4 chunks that a transposing read takes of 4 rows, each fall on
// all 64 banks once.
template <int D>
__device__ __forceinline__ int swz(int r) {
  return D == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : ((r & 2) << 1) | ((r >> 2) & 3);
}

struct Seq {
  int q0, lq, k0, lk;   // first token and length, of queries and keys
  int tile;             // this block's tile within the sequence
};

__device__ __forceinline__ int clamp_to(int x, int n) { return x < 0 ? 0 : x > n ? n : x; }
// First token and length of sequence s.  Starts are clamped to the tensor: no
// value in them leads out of bounds.
__device__ __forceinline__ void span(const int32_t* p, int n, int s, int& first, int& len) {
  const int b = p == nullptr ? 0 : clamp_to(p[s], n), e = p == nullptr ? n : clamp_to(p[s + 1], n);
  first = b;
  len = e > b ? e - b : 0;
}

// The block's tile: the one of rank p among all sequences' (KEYS: tiles of
// keys, else of rows), the longest first: under a causal mask row tile d of a
// sequence reads about d + 1 tiles of keys, and key tile d from the end as many
// of rows.  False when there are not so many.  (In the order of the sequences
// the last one's long tiles began when all others had ended: dk/dv of 8 x 2048
// tokens left 20 % of the chip idle.)
//
// Up to 64 sequences, one per lane: with n_s tiles each, sum_s max(0, n_s - d)
// tiles have depth d or more; d is found with 64 candidates at a time, one per
// lane.  (Bisection over scalar sums of ballots took 3 to 6 us of each block.)
// More sequences: the list in order, sequence s's tiles from index
// start * mul / kBM + s (rounded down), which leaves room for all of them.
template <bool KEYS>
__device__ __forceinline__ bool find_tile(const AttnArgs& a, int p, Seq& q) {
  const int lane = threadIdx.x & (kWave - 1);
  const int32_t* starts = KEYS ? a.k_start : a.q_start;
  const int n_tok = KEYS ? a.tk : a.tq, mul = KEYS ? 1 : a.group;
  if (a.n_seq <= kWave) {
    Seq v{0, 0, 0, 0, 0};
    if (lane < a.n_seq) {
      span(a.q_start, a.tq, lane, v.q0, v.lq);
      span(a.k_start, a.tk, lane, v.k0, v.lk);
    }
    const int n = (int)(((int64_t)(KEYS ? v.lk : v.lq) * mul + kBM - 1) / kBM);
    int step = 1;                      // 64 steps pass every depth
    for (int64_t most = ((int64_t)n_tok * mul + kBM - 1) / kBM; most > (int64_t)kWave * step;) step *= kWave;
    int d = 0, count;                  // the largest depth with count > p tiles at or below it
    for (;; step /= kWave) {
      const int x = d + lane * step;
      int sum = 0;
      for (int s = 0; s < a.n_seq; s += 8)      // (lanes behind the last sequence hold 0 tiles)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += max(0, __builtin_amdgcn_readlane(n, s + e) - x);
      const unsigned long long more = __ballot(sum > p);
      if (more == 0) return false;
      const int at = __popcll(more) - 1;
      d += at * step;
      count = __builtin_amdgcn_readlane(sum, at);
      if (step == 1) break;
    }
    const unsigned long long deep = __ballot(n > d);
    const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(deep >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)deep, 0));
    const int at = p - (count - __popcll(deep));        // among those of this depth
    const int s = __builtin_ctzll(__ballot(n > d && before == at));
    q.q0 = __builtin_amdgcn_readlane(v.q0, s);
    q.lq = __builtin_amdgcn_readlane(v.lq, s);
    q.k0 = __builtin_amdgcn_readlane(v.k0, s);
    q.lk = __builtin_amdgcn_readlane(v.lk, s);
    q.tile = KEYS ? __builtin_amdgcn_readlane(n, s) - 1 - d : d;
    return true;
  }
  auto first_tile = [&](int s) { return (int64_t)clamp_to(starts[s], n_tok) * mul / kBM + s; };
  int lo = 0, hi = a.n_seq;            // the last sequence whose tiles start at or before p
  while (hi - lo > 1) {
    const int step = (hi - lo + kWave - 1) / kWave;
    const int s = lo + lane * step;
    const int cnt = __popcll(__ballot(s < hi && first_tile(min(s, hi - 1)) <= p));
    if (cnt == 0) return false;
    lo = lo + (cnt - 1) * step;
    hi = min(hi, lo + step);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  int x[4];
  span(a.q_start, a.tq, lo, x[0], x[1]);
  span(a.k_start, a.tk, lo, x[2], x[3]);
  q.q0 = __builtin_amdgcn_readfirstlane(x[0]);
  q.lq = __builtin_amdgcn_readfirstlane(x[1]);
  q.k0 = __builtin_amdgcn_readfirstlane(x[2]);
  q.lk = __builtin_amdgcn_readfirstlane(x[3]);
  q.tile = __builtin_amdgcn_readfirstlane((int)(p - first_tile(lo)));
  return q.tile >= 0;
}

// row r of a sequence -> token and head within the group (r / G, r % G)
__device__ __forceinline__ int row_token(const AttnArgs& a, int r) {
  return (int)((__umulhi((uint32_t)r, a.gmul) + ((uint32_t)r & a.gone)) >> a.gshift);
}

// This lane's byte offsets of the operand reads from a tile.
template <int D>
struct Lanes {
  int sa[D / 16];         // straight: row lane % 32, values 16 ks + 8 (lane / 32) ..
  int ta[2][D / 32];      // transposed: column 32 db + lane % 32, values 8 e + 4 (lane / 32) + 0..3
  __device__ __forceinline__ Lanes() {
    const int l = threadIdx.x & 63, h = l >> 5, i = l & 15;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) sa[ks] = (l & 31) * (2 * D) + (((2 * ks + h) ^ swz<D>(l & 15)) << 4);
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int db = 0; db < D / 32; ++db) {
        const int row = 8 * e + 4 * h + (i >> 2), c = 4 * db + ((l >> 3) & 2) + ((i >> 1) & 1);
        ta[e][db] = row * (2 * D) + ((c ^ swz<D>(row)) << 4) + 8 * (i & 1);
      }
  }
};
template <int D>
__device__ __forceinline__ i32x4 read_straight(const lds_u8* tile, const Lanes<D>& ln, int rb, int ks) {
  return *(const lds_i32x4*)(tile + ln.sa[ks] + rb * (2 * D));
}
// values [kb + {4 h + 0..3, 8 + 4 h + 0..3}] (h = lane half) of column
// 32 db + lane % 32, kb a multiple of 16
template <int D>
__device__ __forceinline__ i32x4 read_transposed(const lds_u8* tile, const Lanes<D>& ln, int kb, int db) {
  auto half = [&](int e) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) s16x4*)(tile + ln.ta[e][db] + kb * (2 * D))));
  };
  const u32x2 lo = half(0), hi = half(1);
  return i32x4{(int)lo[0], (int)lo[1], (int)hi[0], (int)hi[1]};
}
__device__ __forceinline__ f32x16 mfma(i32x4 a, i32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// (not as inline asm, which would read a matrix result before it is written:
// the compiler sees no operands to wait for there)
__device__ __forceinline__ float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
// 8 scores -> B operand of the second products (p for o and dv, g for dq and dk),
// rounded to bf16: the matrix cores take 16-bit values, and operands in fp32 would
// run at a sixteenth of their rate.  Each rounding is off by 2^-8 of its own p or g
// at most, independently of the others (0.0012 of o's norm and 0.0017 of the
// gradients', beside 0.0016 for rounding the results).
__device__ __forceinline__ i32x4 pack8(const f32x16& v, int at) {
  return i32x4{(int)pack_bf16x2(v[at], v[at + 1]), (int)pack_bf16x2(v[at + 2], v[at + 3]),
               (int)pack_bf16x2(v[at + 4], v[at + 5]), (int)pack_bf16x2(v[at + 6], v[at + 7])};
}
__device__ __forceinline__ f32x16 splat(float x) {
  f32x16 v;
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = x;
  return v;
}

// One wave's quarter of a tile of R rows: off(r, c) is the byte offset from
// base of the tile's row r, 16-byte chunk c.
template <int D, int R>
struct Stager {
  static constexpr int CH = D / 8, N = R * CH / 256;       // (the four waves of a group)
  static_assert(N * 256 == R * CH, "whole waves");
  uint32_t off[N];
  template <class F>
  __device__ __forceinline__ void set(F&& f) {
    const int w = (threadIdx.x >> 6) & 3, l = threadIdx.x & 63;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int p = (w * N + n) * 64 + l, row = p / CH;
      off[n] = f(row) + 16 * ((p % CH) ^ swz<D>(row & 15));
    }
  }
  __device__ __forceinline__ void issue(const uint8_t* base, lds_u8* tile) const {
    const int w = (threadIdx.x >> 6) & 3;
    // (the copies take the base from scalar registers)
    const uint64_t b = reinterpret_cast<uint64_t>(base);
    base = reinterpret_cast<const uint8_t*>((uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(b >> 32)) << 32 |
                                            (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)b));
#pragma unroll
    for (int n = 0; n < N; ++n) dma16s(base, off[n], tile + (w * N + n) * 1024);
  }
  // the same from each row's own address
  template <class F>
  static __device__ __forceinline__ void issue_each(lds_u8* tile, F&& row_ptr) {
    const int w = (threadIdx.x >> 6) & 3, l = threadIdx.x & 63;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int p = (w * N + n) * 64 + l, row = p / CH;
      dma16(row_ptr(row) + 16 * ((p % CH) ^ swz<D>(row & 15)), tile + (w * N + n) * 1024);
    }
  }
};
// Keys and values of tile after tile: rows past the last key repeat it.
template <int D, int KT>
struct KeyStream {
  const uint8_t *kp, *vp;
  int64_t k_tok, v_tok;
  int lk;
  Stager<D, KT> ks, vs;
  __device__ __forceinline__ KeyStream(const AttnArgs& a, const Seq& q, int kvh)
      : kp(a.K + (int64_t)q.k0 * a.k_tok + (int64_t)kvh * a.k_head),
        vp(a.V + (int64_t)q.k0 * a.v_tok + (int64_t)kvh * a.v_head), k_tok(a.k_tok), v_tok(a.v_tok), lk(q.lk) {
    ks.set([&](int row) { return (uint32_t)row * (uint32_t)k_tok; });
    vs.set([&](int row) { return (uint32_t)row * (uint32_t)v_tok; });
  }
  __device__ __forceinline__ void issue(const uint8_t* p, int64_t tok, const Stager<D, KT>& st, int k0, lds_u8* tile) const {
    const uint8_t* base = p + (int64_t)k0 * tok;
    if (k0 + KT <= lk) {
      st.issue(base, tile);
    } else {
      Stager<D, KT> e;
      const int last = lk - 1 - k0;
      e.set([&](int row) { return (uint32_t)min(row, last) * (uint32_t)tok; });
      e.issue(base, tile);
    }
  }
  __device__ __forceinline__ void issue_k(int k0, lds_u8* tile) const { issue(kp, k_tok, ks, k0, tile); }
  __device__ __forceinline__ void issue_v(int k0, lds_u8* tile) const { issue(vp, v_tok, vs, k0, tile); }
};
// f(t, stage) for t = 0 .. n - 1 with the stage t % 2 a constant, so that
// tile addresses fold into the reads' offsets
template <class F>
__device__ __forceinline__ void staged_loop(int n, F&& f) {
  for (int t = 0; t < n; t += 2) {
    f(t, std::integral_constant<int, 0>{});
    if (t + 1 < n) f(t + 1, std::integral_constant<int, 1>{});
  }
}

// A wave's result columns (one of 32 rows of the output per lane, N blocks of 32
// values, times f) -> bf16 rows.  Through the wave's 32 x 64 N bytes of LDS, so
// that a store writes whole rows: 8 bytes of 32 rows each kept the block's last
// stores waiting (8 x 2048 tokens, 16 heads of 128: backward 528 -> 506 us,
// forward 180 -> 177).
// Chunks of a row are swizzled over the banks.
template <int N, class F>
__device__ __forceinline__ void store_rows(lds_u8* buf, const f32x16 (&o)[N], float f, int rows, F&& row_ptr) {
  constexpr int CH = 4 * N;
  const int lane = threadIdx.x & 63, h = lane >> 5, r = lane & 31;
  auto at = [](int row, int c) { return row * 16 * CH + ((c ^ ((CH == 16 ? row : row >> 1) & (CH - 1))) << 4); };
#pragma unroll
  for (int db = 0; db < N; ++db)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *(__attribute__((address_space(3))) u32x2*)(buf + at(r, 4 * db + q) + 8 * h) =
          u32x2{pack_bf16x2(o[db][4 * q] * f, o[db][4 * q + 1] * f), pack_bf16x2(o[db][4 * q + 2] * f, o[db][4 * q + 3] * f)};
#pragma unroll
  for (int i = 0; i < CH / 2; ++i) {
    const int p = i * 64 + lane, row = p / CH, c = p % CH;
    const i32x4 v = *(const lds_i32x4*)(buf + at(row, c));
    if (row < rows) *reinterpret_cast<i32x4*>(row_ptr(row) + 16 * c) = v;
  }
}

// the same in fp32, for a sum that is not complete
template <int N>
__device__ __forceinline__ void store_part(float* p, const f32x16 (&o)[N], float f) {
  const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int db = 0; db < N; ++db)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<f32x4*>(p + 32 * db + 8 * q + 4 * h) =
          f32x4{o[db][4 * q] * f, o[db][4 * q + 1] * f, o[db][4 * q + 2] * f, o[db][4 * q + 3] * f};
}

// Two groups of four waves may share a block's rows (GR = 2), each taking every
// second tile of keys: a block is done in half the time, which counts when the
// longest block takes as long as the kernel.  At the end group g
// finishes blocks g ND / 2 .. of the ND (own), with the other group's sums.
constexpr int larger(int a, int b) { return a > b ? a : b; }
constexpr int share_floats(int nd) { return 2 * 4 * (nd / 2) * 16 * 64; }
template <int ND>
__device__ __forceinline__ void join_groups(const f32x16 (&x)[ND], f32x16 (&own)[ND / 2], lds_f32* buf, int g, float f,
                                            float f_other) {
  const int w = (threadIdx.x >> 6) & 3, lane = threadIdx.x & 63;
  constexpr int H = ND / 2;
  __syncthreads();            // (what buf held is read)
#pragma unroll
  for (int d = 0; d < H; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      // (values selected, not places: an index would send the sums to scratch)
      const float give = g == 0 ? x[H + d][i] : x[d][i], keep = g == 0 ? x[d][i] : x[H + d][i];
      buf[(((g * 4 + w) * H + d) * 16 + i) * 64 + lane] = give;
      own[d][i] = keep * f;
    }
  __syncthreads();
#pragma unroll
  for (int d = 0; d < H; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) own[d][i] += buf[((((1 - g) * 4 + w) * H + d) * 16 + i) * 64 + lane] * f_other;
}

// ------------------------------------------------------------------ forward
// A block: 128 rows, 32 per wave; keys and values pass through LDS in tiles of 64,
// two stages, copied while the tile before is worked on.  Scores, powers and sums
// stay in registers.  Bound by matrix and vector work that take turns: 8 x 2048
// tokens, 16 heads of 128, causal, 177 us for the 137 GFLOP that the mask leaves
// (775 TFLOP/s; one sequence of 8192 tokens 930), the matrix cores busy 0.45 and
// the vector units 0.50 of the busy units' cycles at the 1.7 to 1.9 GHz that the
// power limit leaves; a block's first data arrive 4 to 5 us after its start.
// Without the mask 1.53 times the time for twice the work (950 TFLOP/s).  64-wide,
// 4 x 4096 tokens, 16 heads: 160 us; three waves per SIMD (four, at 128 registers: 29.1 -> 31.1 us
// for 8 x 1024, 12 heads).
// New tokens over long contexts are bound by HBM: 32 tokens over 1 to 8192 keys, 8
// key heads: 108 us for 0.54 GB, 5.0 TB/s.
template <int D, int GR>
__global__ __launch_bounds__(256 * GR, GR == 2 || D == 128 ? 2 : 3) void attn_fwd_kernel(AttnArgs a) {
  constexpr int NK = D / 16, ND = D / 32, KT = 64, NB = KT / 32, TB = KT * D * 2;
  constexpr int LDS = GR == 1 ? 4 * TB : larger(8 * TB, share_floats(ND) * 4 + 2048);
  __shared__ __attribute__((aligned(1024))) uint8_t smem[LDS];        // a group's: keys of two tiles, values of two
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w = wave & 3, g = wave >> 2;
  lds_u8* lds = (lds_u8*)&smem[0] + g * 4 * TB;
  // (blocks go to the 8 XCDs in turn: with 8 or 16 key heads each head's keys
  // stay with one XCD's L2)
  const int at_tile = blockIdx.x / a.kv_heads, kvh = blockIdx.x - at_tile * a.kv_heads;
  const int rank = a.splits == 1 ? at_tile : at_tile / a.splits, split = at_tile - rank * a.splits;
  Seq sq;
  if (!find_tile<false>(a, rank, sq)) return;
  const int rows = sq.lq * a.group, r0 = sq.tile * kBM;
  if (r0 >= rows) return;
  const int off = sq.lk - sq.lq;

  // this lane's row
  const int r = r0 + 32 * w + (lane & 31), rc = min(r, rows - 1);
  const int tok = row_token(a, rc), head = kvh * a.group + (rc - tok * a.group);
  // keys of this block: all that its last row sees, of this split
  int kend = sq.lk;
  if (a.causal) kend = min(kend, row_token(a, min(r0 + kBM, rows) - 1) + off + 1);
  int kbeg = 0;
  if (a.splits > 1) {
    // (keys up to the largest count: neither sum fits 31 bits)
    const uint32_t per = (((uint32_t)sq.lk + a.splits - 1) / a.splits + kKT - 1) / kKT * kKT;
    kbeg = (int)min((int64_t)split * per, (int64_t)sq.lk);
    kend = (int)min((int64_t)kend, (int64_t)kbeg + per);
  }
  const int nt = kend > kbeg ? (kend - kbeg + KT - 1) / KT : 0;
  const int lim = min(a.causal ? tok + off : sq.lk - 1, kend - 1);      // last key this row sees
  // (those of the wave's first and last row; a wave without rows sees none)
  const int lim_lo = __builtin_amdgcn_readlane(lim, 0), lim_hi = r0 + 32 * w < rows ? __builtin_amdgcn_readlane(lim, 31) : -1;

  const Lanes<D> ln;
  const KeyStream<D, KT> keys(a, sq, kvh);
  if (g < nt) {
    keys.issue_k(kbeg + g * KT, lds);
    keys.issue_v(kbeg + g * KT, lds + 2 * TB);
  }

  i32x4 qf[NK];
  const uint8_t* qp = a.Q + (int64_t)(sq.q0 + tok) * a.q_tok + (int64_t)head * a.q_head;
#pragma unroll
  for (int ks = 0; ks < NK; ++ks) qf[ks] = *reinterpret_cast<const i32x4*>(qp + 32 * ks + 16 * h);

  f32x16 o[ND];
#pragma unroll
  for (int db = 0; db < ND; ++db) o[db] = splat(0.0f);
  const float c = a.scale * kLog2e;
  // m: what the exponents are relative to, a maximum of c q.k so far; l: their
  // sum.  m moves only when the maximum passes it by 2^8 (the sum of a tile's
  // powers 2^16): large powers lose nothing, and in every tile some row's maximum
  // moves a little (scaling o each time was a fifth of the vector work).
  constexpr float kSlack = 8.0f, kMost = 65536.0f;
  float m = -__builtin_inff(), l = 0.0f;
  // tiles that a row of this wave sees
  const int mine = min(nt, lim_hi < kbeg ? 0 : (lim_hi - kbeg) / KT + 1);

  staged_loop((nt + GR - 1) / GR, [&](int it, auto stage) {
    constexpr int S = decltype(stage)::value;
    const lds_u8 *kt = lds + S * TB, *vt = lds + (2 + S) * TB;
    const int t = it * GR + g, k0 = kbeg + t * KT;
    wait_vm<0>();
    __syncthreads();
    if (t + GR < nt) {
      keys.issue_k(k0 + GR * KT, lds + (1 - S) * TB);
      keys.issue_v(k0 + GR * KT, lds + (3 - S) * TB);
    }
    if (t >= mine) return;
    f32x16 s[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) s[b] = splat(0.0f);
#pragma unroll
    for (int ks = 0; ks < NK; ++ks)
#pragma unroll
      for (int b = 0; b < NB; ++b) s[b] = mfma(read_straight<D>(kt, ln, 32 * b, ks), qf[ks], s[b]);
    if (k0 + KT - 1 > lim_lo) {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int j = k0 + 32 * b + 8 * (i >> 2) + 4 * h + (i & 3);
          s[b][i] = j <= lim ? s[b][i] : -__builtin_inff();
        }
    }
    auto tile_max = [&] {
      float mx = max3(s[0][0], s[0][1], s[0][2]), my = max3(s[0][3], s[0][4], s[0][5]);
#pragma unroll
      for (int i = 6; i < 16 * NB; i += 4) {
        mx = max3(mx, s[i / 16][i % 16], s[i / 16][i % 16 + 1]);
        if (i + 2 < 16 * NB) my = max3(my, s[(i + 2) / 16][(i + 2) % 16], s[(i + 2) / 16][(i + 2) % 16 + 1]);
      }
      mx = fmaxf(mx, my);
      return fmaxf(mx, __shfl_xor(mx, 32, kWave)) * c;
    };
    auto move = [&](float mx) {
      const float mn = fmaxf(m, mx);
      const float f = exp2_fast(m - (mn == -__builtin_inff() ? 0.0f : mn));
      m = mn;
      l *= f;
#pragma unroll
      for (int db = 0; db < ND; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] *= f;
    };
    i32x4 p[2 * NB];
    float sum;
    auto powers = [&] {
      const float mu = m == -__builtin_inff() ? 0.0f : m;
      sum = 0.0f;
#pragma unroll
      for (int kk = 0; kk < 2 * NB; ++kk) {
        float e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          e[i] = exp2_fast(__builtin_fmaf(s[kk >> 1][8 * (kk & 1) + i], c, -mu));
          sum += e[i];          // (in fp32: lse is the sum of the powers themselves)
        }
        p[kk] = i32x4{(int)pack_bf16x2(e[0], e[1]), (int)pack_bf16x2(e[2], e[3]), (int)pack_bf16x2(e[4], e[5]),
                      (int)pack_bf16x2(e[6], e[7])};
      }
    };
    if constexpr (D == 64) {
      // the sums show as well whether m is far behind, and cost nothing: the
      // maxima (a tenth of the vector work) only of the first tile and where the
      // sums ask for them (4 x 4096 tokens, 16 heads 170 -> 164 us)
      if (t == g) move(tile_max());
      powers();
      if (__any(!(sum <= kMost))) {
        move(tile_max());
        powers();
      }
    } else {
      // (128-wide, the matrix products of o take the time of the maxima, and would
      // have to wait for the check of the sums: 5 prompts of 301 to 3001 tokens 185
      // -> 189 us)
      const float mx = tile_max();
      if (__any(mx > m + kSlack)) move(mx);
      powers();
    }
    l += sum;
#pragma unroll
    for (int kk = 0; kk < 2 * NB; ++kk) {
#pragma unroll
      for (int db = 0; db < ND; ++db) o[db] = mfma(read_transposed<D>(vt, ln, 16 * kk, db), p[kk], o[db]);
    }
  });
  l += __shfl_xor(l, 32, kWave);
  // the row's results from block `first` of 32 on
  auto finish = [&](const auto& x, int first) {
    const bool none = l == 0.0f;               // a row that sees no key: zeros
    const float inv = none ? 0.0f : 1.0f / l, lse2 = none ? -__builtin_inff() : m + __log2f(l);
    const int64_t at = (int64_t)head * a.tq + sq.q0 + tok;
    if (a.splits == 1) {
      __syncthreads();            // (the tiles are read)
      constexpr int N = sizeof(x) / sizeof(f32x16);
      const int rw = r0 + 32 * w;
      store_rows<N>((lds_u8*)&smem[0] + wave * 2048 * N, x, inv, rows - rw, [&](int i) {
        const int t = row_token(a, rw + i);
        return a.O + (int64_t)(sq.q0 + t) * a.o_tok + (int64_t)(kvh * a.group + (rw + i - t * a.group)) * a.o_head + 64 * first;
      });
      if (r < rows && h == 0 && first == 0 && a.lse != nullptr) a.lse[at] = lse2 * kLn2;
      return;
    }
    if (r >= rows) return;
    const int64_t all = (int64_t)a.heads * a.tq;
    if (h == 0 && first == 0) a.part_lse[split * all + at] = lse2;
    if (none) return;
    store_part(a.part + (split * all + at) * D + 32 * first, x, inv);
  };
  if constexpr (GR == 2) {
    lds_f32* buf = (lds_f32*)&smem[0];
    lds_f32* ml = buf + share_floats(ND) + (w * 64 + (lane & 31)) * 2;      // [wave][group][row]
    __syncthreads();
    if (h == 0) {
      ml[g * 64] = m;
      ml[g * 64 + 1] = l;
    }
    __syncthreads();
    const float mo = ml[(1 - g) * 64], lo = ml[(1 - g) * 64 + 1];
    const float mn = fmaxf(m, mo), mu = mn == -__builtin_inff() ? 0.0f : mn;
    const float fs = exp2_fast(m - mu), fo = exp2_fast(mo - mu);
    m = mn;
    l = l * fs + lo * fo;
    f32x16 own[ND / 2];
    join_groups<ND>(o, own, buf, g, fs, fo);
    finish(own, g * (ND / 2));
  } else {
    finish(o, 0);
  }
}

// o = sum_s 2^(lse_s - lse) o_s over the splits of a row: one wave per row, up to
// four splits' partials in flight (5 us for 1024 rows of 6 splits, most of it the
// launch).
template <int D>
__global__ __launch_bounds__(256) void attn_combine_kernel(AttnArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t all = (int64_t)a.heads * a.tq;
  const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (at >= all) return;
  const int head = (int)(at / a.tq), tok = (int)(at - (int64_t)head * a.tq);
  if (a.q_start != nullptr && (tok < a.q_start[0] || tok >= a.q_start[a.n_seq])) return;
  float mx = -__builtin_inff();
  for (int s = lane; s < a.splits; s += 64) mx = fmaxf(mx, a.part_lse[s * all + at]);
  mx = wave_max(mx);
  if (mx == -__builtin_inff()) mx = 0.0f;
  constexpr int E = D / 64;
  float o[E] = {}, sum = 0.0f;
  for (int s0 = 0; s0 < a.splits; s0 += 64) {
    const int n = min(64, a.splits - s0);
    // a lane's split: its weight, 0 for one that saw no key (its o was not written)
    const float f = lane < n ? exp2_fast(a.part_lse[(s0 + lane) * all + at] - mx) : 0.0f;
    unsigned long long some = __ballot(f != 0.0f);
    sum += f;
    while (some != 0) {
      // up to 4 splits' partials in flight
      float v[4][E], fs[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int s = some != 0 ? __builtin_ctzll(some) : 0;
        fs[k] = some != 0 ? __shfl(f, s, kWave) : 0.0f;
        const float* p = a.part + ((s0 + s) * all + at) * D + E * lane;
#pragma unroll
        for (int e = 0; e < E; ++e) v[k][e] = some != 0 ? p[e] : 0.0f;
        some &= some - 1;
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] += fs[k] * v[k][e];
    }
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d, kWave);
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  uint8_t* op = a.O + (int64_t)tok * a.o_tok + (int64_t)head * a.o_head;
  if constexpr (E == 2) *reinterpret_cast<uint32_t*>(op + 4 * lane) = pack_bf16x2(o[0] * inv, o[1] * inv);
  else *reinterpret_cast<uint16_t*>(op + 2 * lane) = (uint16_t)f32_to_bf16_bits(o[0] * inv);
  if (lane == 0 && a.lse != nullptr) a.lse[at] = sum == 0.0f ? -__builtin_inff() : (mx + __log2f(sum)) * kLn2;
}

// ------------------------------------------------------------------ backward
// dq, and per row, for dk/dv, in row order [kv head][token * G + head in
// group]: -lse / c, from which a score's accumulator starts (so that the product
// ends as q.k - lse / c), and -do.o, from which do.v starts.  Blocks, tiles and
// groups as in the forward, with three products instead of two: 8 x 2048 tokens,
// 16 heads of 128: 225 us for 206 GFLOP (916 TFLOP/s), the matrix cores busy half
// of all cycles.
template <int D, int GR>
__global__ __launch_bounds__(256 * GR, 2) void attn_dq_kernel(AttnArgs a) {
  constexpr int NK = D / 16, ND = D / 32, TB = kKT * D * 2;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[GR == 1 ? 4 * TB : larger(8 * TB, share_floats(ND) * 4)];
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w = wave & 3, g = wave >> 2;
  lds_u8* lds = (lds_u8*)&smem[0] + g * 4 * TB;
  const int rank = blockIdx.x / a.kv_heads, kvh = blockIdx.x - rank * a.kv_heads;
  Seq sq;
  if (!find_tile<false>(a, rank, sq)) return;
  const int rows = sq.lq * a.group, r0 = sq.tile * kBM;
  if (r0 >= rows) return;
  const int off = sq.lk - sq.lq;
  const int r = r0 + 32 * w + (lane & 31), rc = min(r, rows - 1);
  const int tok = row_token(a, rc), head = kvh * a.group + (rc - tok * a.group);
  const bool active = r0 + 32 * w < rows;
  int kend = sq.lk;
  if (a.causal) kend = min(kend, row_token(a, min(r0 + kBM, rows) - 1) + off + 1);
  const int nt = kend > 0 ? (kend + kKT - 1) / kKT : 0;
  const int lim = min(a.causal ? tok + off : sq.lk - 1, kend - 1);
  const int lim_lo = __builtin_amdgcn_readlane(lim, 0), lim_hi = __builtin_amdgcn_readlane(lim, 31);

  const Lanes<D> ln;
  const KeyStream<D, kKT> keys(a, sq, kvh);
  auto issue = [&](int t, lds_u8* stage) {
    if (t >= nt) return;
    keys.issue_k(t * kKT, stage);
    keys.issue_v(t * kKT, stage + TB);
  };
  const bool exact = nt <= 2;
  issue(exact ? 0 : g, lds);
  i32x4 qf[NK], gf[NK];
  const uint8_t* qp = a.Q + (int64_t)(sq.q0 + tok) * a.q_tok + (int64_t)head * a.q_head;
  const uint8_t* gp = a.dO + (int64_t)(sq.q0 + tok) * a.do_tok + (int64_t)head * a.do_head;
#pragma unroll
  for (int ks = 0; ks < NK; ++ks) {
    qf[ks] = *reinterpret_cast<const i32x4*>(qp + 32 * ks + 16 * h);
    gf[ks] = *reinterpret_cast<const i32x4*>(gp + 32 * ks + 16 * h);
  }
  float nd = 0.0f;
  const uint8_t* op = a.O + (int64_t)(sq.q0 + tok) * a.o_tok + (int64_t)head * a.o_head;
#pragma unroll
  for (int ks = 0; ks < NK; ++ks) {
    const i32x4 x = *reinterpret_cast<const i32x4*>(op + 32 * ks + 16 * h);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      nd -= bf16_bits_to_f32((uint32_t)x[e] & 0xFFFFu) * bf16_bits_to_f32((uint32_t)gf[ks][e] & 0xFFFFu);
      nd -= __uint_as_float((uint32_t)x[e] & 0xFFFF0000u) * __uint_as_float((uint32_t)gf[ks][e] & 0xFFFF0000u);
    }
  }
  nd += __shfl_xor(nd, 32, kWave);
  const float nl = -a.lse[(int64_t)head * a.tq + sq.q0 + tok] / a.scale;
  const float c = a.scale * kLog2e;
  f32x16 dq[ND];
#pragma unroll
  for (int db = 0; db < ND; ++db) dq[db] = splat(0.0f);

  float miss = 0.0f;
  // (tiles t0, t0 + step ..: both groups run the same number of rounds)
  auto pass = [&](auto exact, int t0, int step) {
    staged_loop((nt + step - 1) / step, [&](int it, auto stage) {
      constexpr int S = decltype(stage)::value;
      const int t = t0 + it * step;
      const lds_u8 *kt = lds + S * 2 * TB, *vt = kt + TB;
      wait_vm<0>();
      __syncthreads();
      issue(t + step, lds + (1 - S) * 2 * TB);
      if (t >= nt) return;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int k0 = t * kKT + 32 * b;
        if (!active || k0 > lim_hi) continue;
        f32x16 s = splat(nl);
        int sa = ln.sa[0];
        asm volatile("" : "+v"(sa));
        auto straight = [&](const lds_u8* tile, int ks) { return *(const lds_i32x4*)(tile + (sa ^ (ks << 5)) + 64 * b * D); };
#pragma unroll
        for (int ks = 0; ks < NK; ++ks) s = mfma(straight(kt, ks), qf[ks], s);
        if (k0 + 31 > lim_lo) {
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] = k0 + 8 * (i >> 2) + 4 * h + (i & 3) <= lim ? s[i] : -__builtin_inff();
        }
        // do.v runs while p is formed
        __builtin_amdgcn_sched_barrier(0);
        f32x16 ds = splat(nd);
#pragma unroll
        for (int ks = 0; ks < NK; ++ks) ds = mfma(straight(vt, ks), gf[ks], ds);
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = exp2_fast(s[i] * c);
#pragma unroll
        for (int i = 0; i < 16; ++i) ds[i] *= s[i];
        if constexpr (decltype(exact)::value) {
#pragma unroll
          for (int i = 0; i < 16; ++i) miss += ds[i];
          continue;
        }
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
          const i32x4 p = pack8(ds, 8 * kk);
#pragma unroll
          for (int db = 0; db < ND; ++db) dq[db] = mfma(read_transposed<D>(kt, ln, 32 * b + 16 * kk, db), p, dq[db]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    });
  };
  // do.o is formed from o in bf16.  Where a row sees few keys, its error counts
  // beside do.v - do.o (for one key that is zero): blocks whose rows see no more
  // than 128 keys take a pass of their own that finds sum_j p_ij (do_i.v_j -
  // do_i.o_i), the error itself (relative error of dq and dk of packed documents 0.0025 ->
  // 0.0024, where rounding the exact result to bf16 gives 0.0017 and rounding g
  // as well sqrt(2) of that; no measurable time).
  if (exact) {
    pass(std::true_type{}, 0, 1);
    nd -= miss + __shfl_xor(miss, 32, kWave);
    __syncthreads();
    issue(g, lds);
  }
  if (h == 0 && g == 0 && r < rows) {
    const int64_t at = ((int64_t)kvh * a.tq + sq.q0) * a.group + r;
    a.neg_lse[at] = nl;
    a.neg_delta[at] = nd;
  }
  pass(std::false_type{}, g, GR);
  const int rw = r0 + 32 * w;
  auto finish = [&](const auto& x, int first) {       // from block `first` of 32 on
    constexpr int N = sizeof(x) / sizeof(f32x16);
    __syncthreads();            // (the tiles are read)
    store_rows<N>((lds_u8*)&smem[0] + wave * 2048 * N, x, a.scale, rows - rw, [&](int i) {
      const int t = row_token(a, rw + i);
      return a.dQ + (int64_t)(sq.q0 + t) * a.dq_tok + (int64_t)(kvh * a.group + (rw + i - t * a.group)) * a.dq_head + 64 * first;
    });
  };
  if constexpr (GR == 2) {
    f32x16 own[ND / 2];
    join_groups<ND>(dq, own, (lds_f32*)&smem[0], g, 1.0f, 1.0f);
    finish(own, g * (ND / 2));
  } else {
    finish(dq, 0);
  }
}

// Keys and values stay with the block: those of a wave's 32 keys in registers
// (D = 128: the values in LDS, where the registers of both would not leave room
// for two waves per SIMD), rows of Q and dO pass through LDS.  Four products, dk
// and dv in registers for the whole loop (a pass over the keys by rows would need
// atomics, whose order changes results): 8 x 2048 tokens, 16 heads of 128: 290 us
// for 275 GFLOP (950 TFLOP/s), bound as the forward is, with more reads of LDS
// (active 0.43 of the cycles, 0.02 of them bank conflicts).
template <int D, int GR>
__global__ __launch_bounds__(256 * GR, 2) void attn_dkv_kernel(AttnArgs a) {
  constexpr int NK = D / 16, ND = D / 32;
  constexpr bool VL = D == 128;
  constexpr int RT = D == 128 ? 32 : 64, TB = RT * D * 2;          // rows per staged tile, its bytes
  __shared__ __attribute__((aligned(1024))) uint8_t smem[GR == 1 ? 4 * TB : larger(8 * TB, share_floats(ND) * 4)];
  __shared__ __attribute__((aligned(1024))) uint8_t vtile[VL ? kBM * D * 2 : 16];
  __shared__ __attribute__((aligned(256))) float stat[GR][2][2][64];      // two stages of -lse / c and -do.o
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w = wave & 3, g = wave >> 2;
  lds_u8* lds = (lds_u8*)&smem[0] + g * 4 * TB;        // a group's: two stages of Q and dO
  lds_u8* slds = (lds_u8*)&stat[g][0][0][0];
  lds_u8* vlds = (lds_u8*)&vtile[0];
  const int at_tile = blockIdx.x / a.kv_heads, kvh = blockIdx.x - at_tile * a.kv_heads;
  const int rank = a.bwd_splits == 1 ? at_tile : at_tile / a.bwd_splits, split = at_tile - rank * a.bwd_splits;
  Seq sq;
  if (!find_tile<true>(a, rank, sq)) return;
  const int k0 = sq.tile * kBM;
  if (k0 >= sq.lk) return;
  const int rows = sq.lq * a.group, off = sq.lk - sq.lq;
  const int kw = k0 + 32 * w, j = kw + (lane & 31), jc = min(j, sq.lk - 1);
  // The rows that see key x are a suffix: under a causal mask those from token
  // x - off on.  This block's first; this wave's first and the one from which
  // on all its keys are seen; this lane's.
  auto first_row = [&](int x) { return x >= sq.lk ? 0x7fffffff : a.causal ? max(0, x - off) * a.group : 0; };
  const int rlo = first_row(k0), rw_lo = first_row(kw), rw_hi = first_row(kw + 31), rmin = first_row(j);
  // this split's tiles of rows
  const int all_t = rows > rlo ? (rows - rlo + RT - 1) / RT : 0;
  const int per = a.bwd_splits == 1 ? all_t : (all_t + a.bwd_splits - 1) / a.bwd_splits;
  const int t_lo = min(split * per, all_t), nt = min(per, all_t - t_lo);

  const uint8_t* qp = a.Q + (int64_t)sq.q0 * a.q_tok + (int64_t)kvh * a.group * a.q_head;
  const uint8_t* gp = a.dO + (int64_t)sq.q0 * a.do_tok + (int64_t)kvh * a.group * a.do_head;
  const int64_t at = ((int64_t)kvh * a.tq + sq.q0) * a.group;
  // A tile of rows starts with a token's first head when the group divides RT
  // (rlo is a token's first row): offsets from that token are the same for
  // every tile (where the heads of a group lie within 32 bits of each other).
  const bool even = RT % a.group == 0 && a.group * max(a.q_head, a.do_head) < (int64_t(1) << 31);
  Stager<D, RT> qs, gs;
  auto offs = [&](int row, int64_t tok_s, int64_t head_s) {
    const int tok = row_token(a, row);
    return (uint32_t)tok * (uint32_t)tok_s + (uint32_t)(row - tok * a.group) * (uint32_t)head_s;
  };
  qs.set([&](int row) { return offs(row, a.q_tok, a.q_head); });
  gs.set([&](int row) { return offs(row, a.do_tok, a.do_head); });
  auto each = [&](const uint8_t* p, int64_t tok_s, int64_t head_s, int r0, lds_u8* tile) {
    Stager<D, RT>::issue_each(tile, [&](int row) {
      const int r = min(r0 + row, rows - 1), tok = row_token(a, r);
      return p + tok * tok_s + (r - tok * a.group) * head_s;
    });
  };
  auto issue = [&](int t, int s) {
    if (t >= nt) return;
    lds_u8 *qt = lds + s * 2 * TB, *gt = qt + TB;
    const int r0 = rlo + (t_lo + t) * RT;
    if (even && r0 + RT <= rows) {
      const int64_t t0 = row_token(a, r0);
      qs.issue(qp + t0 * a.q_tok, qt);
      gs.issue(gp + t0 * a.do_tok, gt);
    } else {
      each(qp, a.q_tok, a.q_head, r0, qt);
      each(gp, a.do_tok, a.do_head, r0, gt);
    }
    if (w < 2) {      // (64 statistics; those behind a tile of 32 are not used)
      const float* sp = (w == 0 ? a.neg_lse : a.neg_delta) + at + min(r0 + lane, rows - 1);
      dma4(reinterpret_cast<const uint8_t*>(sp), slds + (s * 2 + w) * 256);
    }
  };
  const Lanes<D> ln;
  issue(g, 0);
  i32x4 kf[NK], vf[VL ? 1 : NK];
  const uint8_t* kp = a.K + (int64_t)(sq.k0 + jc) * a.k_tok + (int64_t)kvh * a.k_head;
#pragma unroll
  for (int ks = 0; ks < NK; ++ks) kf[ks] = *reinterpret_cast<const i32x4*>(kp + 32 * ks + 16 * h);
  if constexpr (VL) {
    const uint8_t* vb = a.V + (int64_t)(sq.k0 + k0) * a.v_tok + (int64_t)kvh * a.v_head;
    Stager<D, kBM> e;
    const int last = sq.lk - 1 - k0;
    e.set([&](int row) { return (uint32_t)min(row, last) * (uint32_t)a.v_tok; });
    if (g == 0) e.issue(vb, vlds);
  } else {
    const uint8_t* vp = a.V + (int64_t)(sq.k0 + jc) * a.v_tok + (int64_t)kvh * a.v_head;
#pragma unroll
    for (int ks = 0; ks < NK; ++ks) vf[ks] = *reinterpret_cast<const i32x4*>(vp + 32 * ks + 16 * h);
  }
  const float c = a.scale * kLog2e;
  f32x16 dk[ND], dv[ND];
#pragma unroll
  for (int db = 0; db < ND; ++db) dk[db] = dv[db] = splat(0.0f);

  staged_loop((nt + GR - 1) / GR, [&](int it, auto stage) {
    constexpr int S = decltype(stage)::value;
    const int t = it * GR + g;
    const lds_u8 *qt = lds + S * 2 * TB, *gt = qt + TB, *st = slds + S * 512;
    wait_vm<0>();
    __syncthreads();
    issue(t + GR, 1 - S);
    if (t >= nt) return;
#pragma unroll
    for (int b = 0; b < RT / 32; ++b) {
      const int r0 = rlo + (t_lo + t) * RT + 32 * b;
      if (r0 >= rows || r0 + 31 < rw_lo) continue;       // (rw_lo is the largest int without a key)
      auto read_stat = [&](int off) {
        f32x16 v;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 x = *(const lds_f32x4*)(st + off + 4 * (32 * b + 8 * q + 4 * h));
#pragma unroll
          for (int e = 0; e < 4; ++e) v[4 * q + e] = x[e];
        }
        return v;
      };
      // (D = 128: a straight read's lane offset is formed again each time; kept
      // for all of them they would take the registers of the keys, whose reload
      // from scratch waits for the copies in flight)
      auto fresh = [&](int x) {
        asm volatile("" : "+v"(x));
        return x;
      };
      auto straight = [&](const lds_u8* tile, int sa, int ks) {
        return *(const lds_i32x4*)(tile + (sa ^ (ks << 5)));
      };
      f32x16 s = read_stat(0);
      const int qsa = fresh(ln.sa[0]);
#pragma unroll
      for (int ks = 0; ks < NK; ++ks) s = mfma(straight(qt + 64 * b * D, qsa, ks), kf[ks], s);
      if (r0 + 31 >= rows || r0 < rw_hi) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int r = r0 + 8 * (i >> 2) + 4 * h + (i & 3);
          s[i] = (r >= rmin && r < rows) ? s[i] : -__builtin_inff();
        }
      }
      const int gsa = fresh(ln.sa[0]), vsa = fresh(ln.sa[0] + w * 64 * D);
      // From here on the matrix cores always have a product that does not wait
      // for the arithmetic beside it: do.v while p is formed, dv while g is, dk.
      __builtin_amdgcn_sched_barrier(0);
      f32x16 ds = read_stat(256);
#pragma unroll
      for (int ks = 0; ks < NK; ++ks) {
        const i32x4 vv = VL ? straight(vlds, vsa, ks) : vf[VL ? 0 : ks];
        ds = mfma(straight(gt + 64 * b * D, gsa, ks), vv, ds);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = exp2_fast(s[i] * c);
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        const i32x4 p = pack8(s, 8 * kk);
#pragma unroll
        for (int db = 0; db < ND; ++db) dv[db] = mfma(read_transposed<D>(gt, ln, 32 * b + 16 * kk, db), p, dv[db]);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) ds[i] *= s[i];
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        const i32x4 gg = pack8(ds, 8 * kk);
#pragma unroll
        for (int db = 0; db < ND; ++db) dk[db] = mfma(read_transposed<D>(qt, ln, 32 * b + 16 * kk, db), gg, dk[db]);
      }
    }
  });
  if (nt == 0) wait_vm<0>();      // (the values' copies, before their LDS is another block's)
  // dk and dv from block `first` of 32 on
  auto finish = [&](const auto& xk, const auto& xv, int first) {
    if (a.bwd_splits == 1) {
      constexpr int N = sizeof(xk) / sizeof(f32x16);
      __syncthreads();            // (the tiles are read)
      lds_u8* buf = (lds_u8*)&smem[0] + wave * 2048 * N;
      store_rows<N>(buf, xk, a.scale, sq.lk - kw,
                    [&](int i) { return a.dK + (int64_t)(sq.k0 + kw + i) * a.dk_tok + (int64_t)kvh * a.dk_head + 64 * first; });
      store_rows<N>(buf, xv, 1.0f, sq.lk - kw,
                    [&](int i) { return a.dV + (int64_t)(sq.k0 + kw + i) * a.dv_tok + (int64_t)kvh * a.dv_head + 64 * first; });
    } else if (j < sq.lk) {
      const int64_t all = (int64_t)a.tk * a.kv_heads * D;
      float* p = a.part + (2 * split) * all + ((int64_t)(sq.k0 + j) * a.kv_heads + kvh) * D + 32 * first;
      store_part(p, xk, a.scale);
      store_part(p + all, xv, 1.0f);
    }
  };
  if constexpr (GR == 2) {
    f32x16 ok[ND / 2], ov[ND / 2];
    join_groups<ND>(dk, ok, (lds_f32*)&smem[0], g, 1.0f, 1.0f);
    join_groups<ND>(dv, ov, (lds_f32*)&smem[0], g, 1.0f, 1.0f);
    finish(ok, ov, g * (ND / 2));
  } else {
    finish(dk, dv, 0);
  }
}

// dk, dv = the sums of the splits, in their order: 4 values per thread (HBM, or
// the cache the partials lie in).
__global__ __launch_bounds__(256) void attn_dkv_sum_kernel(AttnArgs a, int d) {
  const int64_t all = (int64_t)a.tk * a.kv_heads * d;
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= 2 * all) return;
  const bool v = i >= all;
  const int64_t at = v ? i - all : i, row = at / d;
  const int tok = (int)(row / a.kv_heads), kvh = (int)(row - (int64_t)tok * a.kv_heads), c = (int)(at - row * d);
  if (a.k_start != nullptr && (tok < a.k_start[0] || tok >= a.k_start[a.n_seq])) return;
  f32x4 s = *reinterpret_cast<const f32x4*>(a.part + i);
  for (int k = 1; k < a.bwd_splits; ++k) s += *reinterpret_cast<const f32x4*>(a.part + 2 * k * all + i);
  uint8_t* p = v ? a.dV + (int64_t)tok * a.dv_tok + (int64_t)kvh * a.dv_head
                 : a.dK + (int64_t)tok * a.dk_tok + (int64_t)kvh * a.dk_head;
  *reinterpret_cast<uint2*>(p + 2 * c) = make_uint2(pack_bf16x2(s[0], s[1]), pack_bf16x2(s[2], s[3]));
}

}  // namespace

// Tiles of all sequences at most (each has at most one that is not full).
int64_t attn_row_tiles(int64_t tokens, int64_t mul, int64_t n_seq) { return tokens * mul / kBM + n_seq; }

// Splits of the keys.  The partial results are written and read once, at 8
// bytes a value, and joined by another launch, so keys are divided
//  - for balance, to about 6 blocks per CU of at least 128 keys, as far as the
//    partials stay below an eighth of the keys' and values' bytes (new tokens
//    over long contexts).  32 new tokens over 1 to 8192 keys, 8 key heads: not
//    split 150 us, into 4 / 6 / 7 / 10 blocks 124 / 118 / 118 / 119; 4 over 1000 to
//    8192, 4 key heads 114, 23.6 / 23.7 / 22.9 / 23.7.  (Where all are of one
//    length, which the host does not know, not to split is ahead: 32 over 4096 keys
//    103, 108 / 110 / 116 / 118.)
//  - below 96 blocks, to fill the chip, to 2 blocks per CU, where each still gets
//    512 keys (one sequence of 2600 tokens, 4 heads of 128, 84 blocks: without ->
//    with 42.1 -> 38.1 us; from about 100 blocks on two groups of waves in each do
//    better: 1500 tokens, 8 heads, 104 blocks, with splits 32.6 -> two groups 29.0,
//    2 of 1000 and 1500, 12 heads of 64, 250 blocks 32.9 -> 21.1).
int attn_splits(int64_t tq, int64_t tk, int64_t n_seq, int heads, int kv_heads) {
  const int64_t blocks = attn_row_tiles(tq, heads / kv_heads, n_seq) * kv_heads;
  if (tq == 0 || blocks >= 1024) return 1;
  auto least = [](int64_t x, int64_t y) { return x < y ? x : y; };
  const int64_t mean = tk / n_seq;
  const int64_t even = least(least(1600 / blocks, mean / 128), tk * kv_heads / (16 * tq * heads));
  const int64_t fill = blocks < 96 ? least(512 / blocks, mean / 512) : 1;
  const int64_t s = even > fill ? even : fill;
  return s < 1 ? 1 : (int)s;
}

hipError_t launch_attn_fwd(int d, AttnArgs a, hipStream_t stream) {
  const int64_t blocks = (int64_t)a.row_tiles * a.splits * a.kv_heads;
  // Two groups of waves per block up to two blocks per CU (64-wide: one, or two
  // where sequences are long), where a block's own length counts.  One group ->
  // two, 128-wide: 6 sequences of 100 to 2000 tokens, 8 heads on 2 key heads (406
  // blocks) 54.6 -> 45.7 us, 584 blocks 41.2 -> 40.2, 704 blocks 56.9 -> 62.8;
  // 64-wide: one of 2000, 16 heads (256 blocks) 32.6 -> 26.6, 2 of 2000, 12 heads
  // (384) 32.7 -> 27.8, but 8 of 300 to 600, 12 heads (420) 15.3 -> 17.5.  Sequences
  // of fewer than 256 keys on average have nothing to divide: 16 of 128, 2 heads
  // on one 9.7 -> 11.6.
  const bool two = a.splits == 1 && blocks <= 512 && a.tk >= (d == 128 || blocks <= 256 ? 256 : 1024) * (int64_t)a.n_seq;
  auto* k = d == 64 ? (two ? attn_fwd_kernel<64, 2> : attn_fwd_kernel<64, 1>) : two ? attn_fwd_kernel<128, 2> : attn_fwd_kernel<128, 1>;
  LaunchStatus st;
  st << launch_kernel(k, dim3((unsigned)blocks), dim3(two ? 512 : 256), stream, a);
  if (a.splits > 1)
    st << launch_kernel(d == 128 ? attn_combine_kernel<128> : attn_combine_kernel<64>,
                        dim3((unsigned)(((int64_t)a.heads * a.tq + 3) / 4)), dim3(256), stream, a);
  return st.e;
}

// Splits of the rows in dk/dv: few key heads (grouped) over few tokens leave
// the chip empty, so below 192 blocks the rows are divided until there are about
// 2 blocks per CU, with at least 256 rows each on average; the partial sums are
// fp32 and summed by another launch.  Backward without -> with: 2 sequences of
// 1500 and 2500 tokens, 8 heads on one key head 400 -> 90 us; 6 of 100 to 2000,
// 8 on 2 329 -> 148; 3 of 300 to 1200, 32 on 8 214 -> 124.  With 192 blocks or
// more two groups of waves in each do better: 2 of 1000 and 1500, 12 heads of
// their own 62 -> 53 without splits, one of 2000, 16 heads 74 -> 64.
int attn_bwd_splits(int64_t tq, int64_t tk, int64_t n_seq, int heads, int kv_heads) {
  const int64_t blocks = attn_row_tiles(tk, 1, n_seq) * kv_heads;
  if (blocks >= 192) return 1;
  const int64_t want = 512 / blocks, most = tq * (heads / kv_heads) / n_seq / 256;
  const int64_t s = want < most ? want : most;
  return s < 1 ? 1 : (int)s;
}

hipError_t launch_attn_bwd(int d, AttnArgs a, hipStream_t stream) {
  LaunchStatus st;
  // Two groups of waves per block up to two blocks per CU, as in the forward, of
  // both widths, where sequences have 256 keys (rows) or more on average.  One
  // group -> two: 6 sequences of 100 to 2000 tokens, 8 heads of 128 on 2 key heads
  // 159 -> 135 us, 3 of 300 to 1200, 32 on 8 133 -> 123, 2 of 1500 and 2500, 8 heads
  // of 64 on one 92 -> 80; above: 876 blocks 87 -> 114; short sequences: 4 of 30 to
  // 300 23.7 -> 25.8, 8 of 200 to 300 34.4 -> 36.3.
  const int64_t rb = (int64_t)a.row_tiles * a.kv_heads, kb = (int64_t)a.key_tiles * a.bwd_splits * a.kv_heads;
  if (a.tq > 0) {
    const bool two = rb <= 512 && a.tk >= 256 * (int64_t)a.n_seq;
    auto* k = d == 128 ? (two ? attn_dq_kernel<128, 2> : attn_dq_kernel<128, 1>) : (two ? attn_dq_kernel<64, 2> : attn_dq_kernel<64, 1>);
    st << launch_kernel(k, dim3((unsigned)rb), dim3(two ? 512 : 256), stream, a);
  }
  if (a.tk > 0) {
    const bool two = kb <= 512 && (int64_t)a.tq * a.group >= 256 * (int64_t)a.n_seq * a.bwd_splits;
    auto* k = d == 128 ? (two ? attn_dkv_kernel<128, 2> : attn_dkv_kernel<128, 1>) : (two ? attn_dkv_kernel<64, 2> : attn_dkv_kernel<64, 1>);
    st << launch_kernel(k, dim3((unsigned)kb), dim3(two ? 512 : 256), stream, a);
    if (a.bwd_splits > 1)
      st << launch_kernel(attn_dkv_sum_kernel, dim3((unsigned)(((int64_t)a.tk * a.kv_heads * d / 2 + 255) / 256)), dim3(256),
                          stream, a, d);
  }
  return st.e;
}

}  // namespace dqt
