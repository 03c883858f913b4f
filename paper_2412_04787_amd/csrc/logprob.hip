// Log probability of each row's given token, the row's entropy and its most
// probable alternatives, from logits x [M, V], and the gradient:
//   lse = log sum_j exp(x_j),  logp = x_t - lse,  p_j = exp(x_j - lse)
//   entropy = lse - sum_j p_j x_j
//   dx_j = g [j = t] - p_j (g + e (x_j - lse + entropy))
// with g, e the upstream gradients of logp and entropy.
//
// Forward: one pass over the row.  Each thread keeps m, a maximum so far, the
// sum s of exp(x - m) and, for the entropy, w, the sum of exp(x - m) (x - m);
// entropy = log s - w / s.  Rows are split over blocks when there are few; a
// second launch joins them.
//
// Alternatives.  Elements are ordered by value, then by lower index: the key
// (value bits made monotone, ~index) orders them totally, so ties and rows
// with fewer finite logits than alternatives need no care.  The block's
// threads form 64 groups; the k-th largest of the groups' maxima (k <= 32) is
// a bound that at least k elements reach and, unless the row is adverse, few
// more (about 24 of random logits for k = 20): the pieces in whose round a
// thread saw a value that large are read again, from cache, and the elements
// that reach the bound collected in LDS and ranked by comparing all with all.
// If they do not fit, k rounds of a whole-block maximum below the last one take
// their place.
//
// Gradient: one read of the logits and one write.  16384 rows of 32000 bf16 logits:
// 214 us forward (4.9 TB/s, the vector units busy 0.8 of the cycles: an exponential
// a logit; 777 rows of 50001 with entropy and 5 alternatives 26 us, 3.0 TB/s, units
// busy 0.6 of the launch), 350 us backward (6.0 TB/s, HBM).
#include "dqt_launch.h"

namespace dqt {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kCand = 1024;       // candidates held in LDS
constexpr int kMaxSplits = 64;    // blocks per row: a lane each when they are joined
constexpr int kRounds = 16;       // rounds of a row whose maxima are kept (16 KB)

__device__ __forceinline__ float inf() { return __builtin_inff(); }

// fp32 bits as an unsigned integer of the same order, the two zeros as one (by an
// integer select: as x + 0 the compiler may drop it)
__device__ __forceinline__ uint32_t order_bits(float x) {
  uint32_t u = __float_as_uint(x);
  u = u == 0x80000000u ? 0u : u;
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_order(uint32_t o) {
  return __uint_as_float(o ^ ((o >> 31) != 0 ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ __forceinline__ uint64_t key_of(float x, uint32_t i) { return ((uint64_t)order_bits(x) << 32) | (uint32_t)~i; }

template <typename T>
__device__ __forceinline__ float load1(const T* p) {
  if constexpr (sizeof(T) == 2) return bf16_bits_to_f32(*reinterpret_cast<const uint16_t*>(p));
  else return *p;
}
// the 16 bytes at p: 8 bf16 or 4 fp32 values
template <typename T, int E = 16 / sizeof(T)>
__device__ __forceinline__ void unpack(const uint4& u, float (&v)[E]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) {
      v[2 * i] = bf16_bits_to_f32(w[i] & 0xFFFFu);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    } else {
      v[i] = __uint_as_float(w[i]);
    }
  }
}

// A row's elements [lo, hi) as 16-byte pieces from the first aligned element,
// and the elements before and behind them one by one.
template <typename T>
struct Span {
  static constexpr int E = 16 / sizeof(T);
  int body, pieces, tail;       // first element of the body, its pieces, first element behind
  __device__ Span(const T* row, int lo, int hi) {
    const int mis = (int)((reinterpret_cast<uintptr_t>(row + lo) & 15u) / sizeof(T));
    body = min(hi, lo + (mis == 0 ? 0 : E - mis));
    pieces = (hi - body) / E;
    tail = body + pieces * E;
  }
};

// Calls f(values, count <= E, first index) for every piece of [lo, hi) that this
// thread reads: of round r (4 NT pieces of the row) pieces r 4 NT + k NT + tid,
// k = 0 .. 3, if want(r); then, as round -1, up to one element outside the
// body.  after(r) follows a round's pieces.
template <typename T, int NT, class W, class F, class A>
__device__ __forceinline__ void for_row(const T* row, int lo, int hi, W&& want, F&& f, A&& after) {
  constexpr int E = Span<T>::E, U = 4;
  const Span<T> sp(row, lo, hi);
  const int tid = threadIdx.x;
  const uint4* p = reinterpret_cast<const uint4*>(row + sp.body);
  for (int r = 0, c0 = 0; c0 < sp.pieces; ++r, c0 += U * NT) {
    if (!want(r)) continue;
    const int c = c0 + tid;
    float v[E];
    if (c0 + U * NT <= sp.pieces) {
      uint4 u[U];
#pragma unroll
      for (int k = 0; k < U; ++k) u[k] = p[c + k * NT];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        unpack<T>(u[k], v);
        f(v, E, sp.body + (c + k * NT) * E);
      }
    } else {
      for (int k = c; k < sp.pieces; k += NT) {
        unpack<T>(p[k], v);
        f(v, E, sp.body + k * E);
      }
    }
    after(r);
  }
  // up to 2 (E - 1) elements outside the body, one per thread
  const int head = sp.body - lo, n = head + hi - sp.tail;
  if (tid < n) {
    const int i = tid < head ? lo + tid : sp.tail + tid - head;
    float v[E];
    v[0] = load1(row + i);
    f(v, 1, i);
  }
}

// (three at a time; the builtin would first quiet every operand's NaN)
__device__ __forceinline__ float max_of(const float* v, int n) {
  float m = v[0];
  int j = 1;
  for (; j + 1 < n; j += 2) asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(m), "v"(v[j]), "v"(v[j + 1]));
  return j < n ? fmaxf(m, v[j]) : m;
}

// A thread's m moves only when a logit passes it by kSlack: sums of powers up
// to e^8 lose nothing, and among 64 lanes some would move it at every piece
// (and 25 operations each time).
constexpr float kSlack = 8.0f;
struct Stat {
  float m, s, w;
  // joins b into this one: sums relative to the larger maximum
  __device__ void join(const Stat& b) {
    const float mn = fmaxf(m, b.m);
    auto part = [&](const Stat& x, float& ss, float& ww) {
      const float d = x.m == -inf() ? 0.0f : fmaxf(x.m - mn, -1e4f);     // (2^d is 0 long before)
      const float f = __builtin_amdgcn_exp2f(d * kLog2e);
      ss = x.s * f;
      ww = (x.w + d * x.s) * f;
      if (x.s == 0.0f) ww = 0.0f;
    };
    float s0, w0, s1, w1;
    part(*this, s0, w0);
    part(b, s1, w1);
    m = mn;
    s = s0 + s1;
    w = w0 + w1;
  }
};

// The k-th largest key of 64, one per lane (bitonic sort, descending).
__device__ __forceinline__ uint64_t kth_of_wave(uint64_t key, int k) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int size = 2; size <= 64; size <<= 1)
#pragma unroll
    for (int d = size >> 1; d > 0; d >>= 1) {
      const uint64_t other = __shfl_xor(key, d, kWave);
      const bool up = ((lane & size) == 0) == ((lane & d) == 0);       // keep the larger
      key = (key > other) == up ? key : other;
    }
  return __shfl(key, k - 1, kWave);
}

template <int NT>
__device__ __forceinline__ uint64_t block_max(uint64_t key, uint64_t* red) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const uint64_t o = __shfl_xor(key, d, kWave);
    key = o > key ? o : key;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = key;
  __syncthreads();
  key = red[0];
#pragma unroll
  for (int i = 1; i < NT / 64; ++i) key = red[i] > key ? red[i] : key;
  return key;
}

// n candidates (distinct keys): the top largest, in order, by rank
template <int NT, class F>
__device__ __forceinline__ void rank_out(const uint64_t* cand, int n, int top, F&& out) {
  for (int i = threadIdx.x; i < n; i += NT) {
    const uint64_t key = cand[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += cand[j] > key;
    if (rank < top) out(rank, key);
  }
}

template <class A>
__device__ __forceinline__ void write_row(const A& a, int64_t row, const Stat& t, float xt, bool has) {
  const bool none = t.s == 0.0f;          // no finite logit
  const float ls = __log2f(t.s) * kLn2;
  if (a.lse != nullptr) a.lse[row] = none ? -inf() : t.m + ls;
  // (x - m) - log s, not x - lse: large logits would cancel what log s adds
  if (a.logp != nullptr) a.logp[row] = !has ? 0.0f : none ? -inf() : (xt - t.m) - ls;
  if (a.entropy != nullptr) a.entropy[row] = none ? 0.0f : ls - t.w / t.s;
  if (a.stat != nullptr) *reinterpret_cast<float2*>(a.stat + 2 * row) = make_float2(t.m, none ? 0.0f : ls);
}
template <class A>
__device__ __forceinline__ void write_top(const A& a, int64_t row, const Stat& t, int rank, uint64_t key) {
  a.top_ids[row * a.top + rank] = (int64_t)(uint32_t)~(uint32_t)key;
  const float x = from_order((uint32_t)(key >> 32));
  a.top_logp[row * a.top + rank] = x == -inf() ? -inf() : (x - t.m) - __log2f(t.s) * kLn2;
}

template <typename T>
__device__ __forceinline__ float target_logit(const LogprobArgs& a, int64_t row, bool& has) {
  const int64_t t = a.targets == nullptr ? -1 : a.targets[row];
  has = t >= 0 && t < a.V;
  return has ? load1(static_cast<const T*>(a.x) + row * a.stride + t) : 0.0f;
}

template <typename T, int NT, bool ENT, bool TOP>
__global__ __launch_bounds__(NT) void logprob_fwd_kernel(LogprobArgs a) {
  __shared__ Stat red[NT / 64];
  __shared__ uint64_t red64[64];
  __shared__ uint64_t cand[TOP ? kCand : 1];
  __shared__ float round_max[TOP ? kRounds : 1][NT];
  __shared__ int ncand;
  const int tid = threadIdx.x, lane = tid & 63;
  const int64_t row = blockIdx.x / a.splits;
  const int split = (int)(blockIdx.x - row * a.splits);
  const int per = (a.V + a.splits - 1) / a.splits;
  const int lo = split * per, hi = min(a.V, lo + per);
  const T* x = static_cast<const T*>(a.x) + row * a.stride;

  Stat t{-inf(), 0.0f, 0.0f};
  float best = -inf();
  int best_at = -1;            // index behind the piece that holds best; -1: none yet
  const auto every = [](int) { return true; };
  float rm = -inf();           // of this round
  for_row<T, NT>(x, lo, hi, every, [&](const float* v, int n, int first) {
    const float cm = max_of(v, n);
    if constexpr (TOP) {
      rm = fmaxf(rm, cm);
      if (best_at < 0 || cm > best || (cm == best && first + n < best_at)) { best = cm; best_at = first + n; }
    }
    if (cm > t.m + kSlack) t.join(Stat{cm, 0.0f, 0.0f});
    const float m = t.m == -inf() ? 0.0f : t.m;
    for (int j = 0; j < n; ++j) {
      const float d = v[j] - m, e = __builtin_amdgcn_exp2f(d * kLog2e);
      t.s += e;
      if constexpr (ENT) t.w = __builtin_fmaf(e, fmaxf(d, -1e4f), t.w);      // (e is 0 long before; -inf would make it NaN)
    }
  }, [&](int r) {
    if constexpr (TOP) {
      if (r < kRounds) round_max[r][tid] = rm;
      rm = -inf();
    }
  });
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const Stat o{__shfl_xor(t.m, d, kWave), __shfl_xor(t.s, d, kWave), ENT ? __shfl_xor(t.w, d, kWave) : 0.0f};
    t.join(o);
  }
  if (lane == 0) red[tid >> 6] = t;
  if constexpr (TOP) {
    if (tid == 0) ncand = 0;
    // 64 groups of NT / 64 neighbouring threads; the key's index part is the
    // last index of the piece that holds the maximum, so that it lies at or
    // below that element's own key
    uint64_t key = best_at > 0 ? key_of(best, (uint32_t)(best_at - 1)) : 0;
#pragma unroll
    for (int d = 1; d < NT / 64; d <<= 1) {
      const uint64_t o = __shfl_xor(key, d, kWave);
      key = o > key ? o : key;
    }
    if (tid % (NT / 64) == 0) red64[tid / (NT / 64)] = key;
  }
  __syncthreads();
  t = red[0];
#pragma unroll
  for (int i = 1; i < NT / 64; ++i) t.join(red[i]);
  if (a.splits == 1) {
    if (tid == 0) {
      bool has;
      const float xt = target_logit<T>(a, row, has);
      write_row(a, row, t, xt, has);
    }
  } else if (tid == 0) {
    float* p = a.part + (row * a.splits + split) * 4;
    p[0] = t.m;
    p[1] = t.s;
    p[2] = t.w;
  }
  if constexpr (TOP) {
    const int top = min(a.top, hi - lo);
    const uint64_t bound = kth_of_wave(red64[lane], top);
    const float bv = from_order((uint32_t)(bound >> 32));
    for_row<T, NT>(x, lo, hi, [&](int r) { return r >= kRounds || !(round_max[r][tid] < bv); },
                   [&](const float* v, int n, int first) {
      if (max_of(v, n) < bv) return;
      for (int j = 0; j < n; ++j) {
        const uint64_t key = key_of(v[j], (uint32_t)(first + j));
        if (key >= bound) {
          const int at = atomicAdd(&ncand, 1);          // (their order does not matter: ranked below)
          if (at < kCand) cand[at] = key;
        }
      }
    }, [](int) {});
    __syncthreads();
    const int n = ncand;
    auto out = [&](int rank, uint64_t key) {
      if (a.splits == 1) write_top(a, row, t, rank, key);
      else a.part_top[(row * a.splits + split) * a.top + rank] = key;
    };
    if (n >= top && n <= kCand) {       // (n < top: a NaN was a group's maximum)
      rank_out<NT>(cand, n, top, out);
    } else {
      uint64_t last = ~0ull;
      for (int r = 0; r < top; ++r) {
        uint64_t key = 0;
        for_row<T, NT>(x, lo, hi, every, [&](const float* v, int cnt, int first) {
          for (int j = 0; j < cnt; ++j) {
            const uint64_t o = key_of(v[j], (uint32_t)(first + j));
            key = o < last && o > key ? o : key;
          }
        }, [](int) {});
        last = block_max<NT>(key, red64);
        if (tid == 0) out(r, last);
      }
    }
    if (a.splits > 1)
      for (int r = top + tid; r < a.top; r += NT) a.part_top[(row * a.splits + split) * a.top + r] = 0;
  }
}

// Joins the splits of a row (at most 64, a lane each; each wave joins all).
// Each split's alternatives are in order: the k-th largest of the lists' heads
// is reached by k of them, so the elements below it are out; the others are
// ranked as above.
template <typename T>
__global__ __launch_bounds__(256) void logprob_join_kernel(LogprobArgs a) {
  __shared__ uint64_t cand[kMaxSplits * kMaxTop];
  __shared__ int ncand;
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63;
  const bool in = lane < a.splits;
  const float* p = a.part + (row * a.splits + (in ? lane : 0)) * 4;
  Stat t{in ? p[0] : -inf(), in ? p[1] : 0.0f, in ? p[2] : 0.0f};
  const uint64_t* lists = a.part_top + row * a.splits * a.top;
  const uint64_t head = in && a.top > 0 ? lists[lane * a.top] : 0;
  if (tid == 0) ncand = 0;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) t.join(Stat{__shfl_xor(t.m, d, kWave), __shfl_xor(t.s, d, kWave), __shfl_xor(t.w, d, kWave)});
  if (tid == 0) {
    bool has;
    const float xt = target_logit<T>(a, row, has);
    write_row(a, row, t, xt, has);
  }
  if (a.top == 0) return;
  // (fewer lists than k: the bound is 0, which all reach; a list's padding is 0)
  const uint64_t bound = kth_of_wave(head, a.top);
  __syncthreads();
  for (int i = tid; i < a.splits * a.top; i += 256) {
    const uint64_t key = lists[i];
    if (key >= bound && key != 0) cand[atomicAdd(&ncand, 1)] = key;
  }
  __syncthreads();
  rank_out<256>(cand, ncand, a.top, [&](int rank, uint64_t key) { write_top(a, row, t, rank, key); });
}

template <typename T, bool ENT>
__global__ __launch_bounds__(256) void logprob_bwd_kernel(LogprobArgs a, int segs, int64_t tiles) {
  constexpr int E = 16 / sizeof(T), kSeg = 256 * 4 * E;
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t row = tile / segs;
    const T* x = static_cast<const T*>(a.x) + row * a.stride;
    T* dx = static_cast<T*>(a.dx) + row * a.dx_stride;
    const int64_t tgt64 = a.targets == nullptr ? -1 : a.targets[row];
    const bool has = tgt64 >= 0 && tgt64 < a.V;
    const int tgt = has ? (int)tgt64 : -1;
    const float2 st = *reinterpret_cast<const float2*>(a.stat + 2 * row);
    const float m = st.x, ls = st.y;
    const float g = has && a.dlogp != nullptr ? a.dlogp[row] : 0.0f;
    const float e = ENT ? a.dent[row] : 0.0f, eh = ENT ? e * a.entropy[row] : 0.0f;
    // Zeros: a row of nothing but -inf (one of NaN, or of NaN and -inf, has no
    // reference either, but a NaN sum: its gradient is NaN), and a row without a
    // target or an entropy's gradient, whatever its logits are.
    const bool none = (m == -inf() && ls == 0.0f) || (!has && e == 0.0f);
    auto grad = [&](float v, int j) {
      const float d = (v - m) - ls, p = none ? 0.0f : __builtin_amdgcn_exp2f(d * kLog2e);
      float y = g + eh;
      if constexpr (ENT) y += e * fmaxf(d, -1e4f);
      y = none ? 0.0f : -p * y;
      return j == tgt && !none ? y + g : y;
    };
    auto store1 = [&](int i) {
      const float y = grad(load1(x + i), i);
      if constexpr (sizeof(T) == 2) *reinterpret_cast<uint16_t*>(dx + i) = (uint16_t)pack_bf16x2(y, y);
      else dx[i] = y;
    };
    // 16-byte pieces where logits and gradient are aligned alike
    const int mis = (int)((reinterpret_cast<uintptr_t>(x) & 15u) / sizeof(T));
    const int head = min(a.V, mis == 0 ? 0 : E - mis);
    const int lo = (int)(tile - row * segs) * kSeg + (tile == row * segs ? 0 : head);
    const int hi = min(a.V, (int)(tile - row * segs + 1) * kSeg + head);
    if (((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(dx)) & 15u) == 0) {
      const Span<T> sp(x, lo, hi);
      const uint4* p = reinterpret_cast<const uint4*>(x + sp.body);
      uint4* q = reinterpret_cast<uint4*>(dx + sp.body);
      for (int c = threadIdx.x; c < sp.pieces; c += 256) {
        float v[E];
        unpack<T>(p[c], v);
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] = grad(v[j], sp.body + c * E + j);
        if constexpr (sizeof(T) == 2) {
          q[c] = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
        } else {
          q[c] = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        }
      }
      const int before = sp.body - lo, n = before + hi - sp.tail;
      if ((int)threadIdx.x < n) store1((int)threadIdx.x < before ? lo + (int)threadIdx.x : sp.tail + (int)threadIdx.x - before);
    } else {
      for (int i = lo + threadIdx.x; i < hi; i += 256) store1(i);
    }
  }
}

}  // namespace

// Blocks per row.  A row of 128000 fp32 logits takes one block 30 us, and the
// second launch that joins split rows about 6, so rows of 15 x 4096 logits or
// more are split, over about 2 blocks per CU of at least 4096 logits each.  One
// block -> split: 8 rows of 128000 fp32 logits with 20 alternatives 39.0 -> 16.8
// us, 200 with 5 51.2 -> 34.0, 8 rows of 65000 bf16 with 5 17.4 -> 15.7, of
// 100000 bf16 without 14.2 -> 14.3; shorter rows lose: 8 of 50000 fp32 11.6 ->
// 14.3, 64 of 32000 bf16 8.4 -> 13.6.
int logprob_splits(int64_t M, int V) {
  const int64_t want = 512 / (M < 1 ? 1 : M), most = V / 4096;
  if (most < 15) return 1;
  const int64_t s = want < most ? want : most;
  return s < 1 ? 1 : s > kMaxSplits ? kMaxSplits : (int)s;
}

hipError_t launch_logprob_fwd(const LogprobArgs& a, bool bf16, hipStream_t stream) {
  constexpr int NT = 256;
  const bool ent = a.entropy != nullptr, top = a.top > 0;
  auto pick = [&](auto t) {
    using T = decltype(t);
    return ent ? (top ? logprob_fwd_kernel<T, NT, true, true> : logprob_fwd_kernel<T, NT, true, false>)
               : (top ? logprob_fwd_kernel<T, NT, false, true> : logprob_fwd_kernel<T, NT, false, false>);
  };
  LaunchStatus st;
  st << launch_kernel(bf16 ? pick(uint16_t{}) : pick(float{}), dim3((unsigned)(a.M * a.splits)), dim3(NT), stream, a);
  if (a.splits > 1)
    st << launch_kernel(bf16 ? logprob_join_kernel<uint16_t> : logprob_join_kernel<float>, dim3((unsigned)a.M), dim3(256), stream, a);
  return st.e;
}

hipError_t launch_logprob_bwd(const LogprobArgs& a, bool bf16, hipStream_t stream) {
  const int seg = 256 * 4 * (bf16 ? 8 : 4);
  const int segs = (a.V + seg - 1) / seg;
  const int64_t tiles = a.M * segs;
  const bool ent = a.dent != nullptr;
  auto* k = bf16 ? (ent ? logprob_bwd_kernel<uint16_t, true> : logprob_bwd_kernel<uint16_t, false>)
                 : (ent ? logprob_bwd_kernel<float, true> : logprob_bwd_kernel<float, false>);
  return launch_kernel(k, dim3((unsigned)(tiles < (1 << 20) ? tiles : 1 << 20)), dim3(256), stream, a, segs, tiles);
}

}  // namespace dqt
