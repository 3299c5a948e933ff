// Log probabilities of given tokens on gfx950, with the entropy and the top
// alternatives of each row, their gradient, and the gradient's own
// vector-Jacobian product (formulas in diffopt.h).
//
// One workgroup per row, or per slice of one where there are few rows.  One
// pass over a row with a running maximum m gives s = sum e and t = sum e d, with
// d = (x - m) / T and e = exp(d): the entropy is log s - t / s.  Each lane's own
// maximum also says where the alternatives are: the K-th largest maximum of groups
// of lanes is at most the K-th largest logit, so only lanes at or above it look
// at their elements again, and hardly more than K of those pass (of independent
// logits 24 for K = 20 and 64 groups, 177 for K = 128 and 256).  They are ranked by value and lowest
// id in LDS.  A row of so many equal logits that they do not fit there takes
// eight counting passes over the digits of (value, id) instead.  Eight rows of
// 131,072 fp32 logits with 20: slices 7.0 us, join 5.1, both latency.
// The gradient's dense part takes the row from registers where the same call
// has read it (rows of up to 256 KiB), else from memory; the tokens that are
// named are written once more after a barrier.  A few exponentials per element:
// bound by memory.  4,096 rows of 50,021 bf16 logits, a tenth of them padding: results
// and gradient at once 158 us (779 MB, 4.9 TB/s).  2,048 rows with 5 alternatives: 43 us
// (205 MB, 4.8 TB/s).  1,024 rows of 32,000 fp32 logits with 8: forward 38 us where
// earlier results are still on their way to memory, else 28 with its launch (131 MB),
// gradient 43 (262 MB, 6.1 TB/s), its backward 91 (393 MB, 4.3 TB/s).
#include <type_traits>

#include "lm_rows.hpp"

namespace diffopt {
namespace {

constexpr int kLB = 512;     // threads per workgroup of a streamed row
constexpr int kJB = 256;     // ... of a row's joined slices
constexpr int kMaxTop = 128;
constexpr int kCap = 1024;   // candidates that are ranked
// Comparisons of a lane from which on the lowest candidates are left out first: 8,000
// rows of 500 bf16 logits with 64 alternatives 41 us, ranked as they are 247.
constexpr int kRanking = 640;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLow = -256.0f;  // 2^d is 0 from here on: 0 log 0 = 0, whatever d is

struct Rows {
  const void* logits;
  int64_t row_stride, N, V;
  const void* ids;  // or NULL: no token is given, every row counts
  int32_t id_bytes;
  float invT;
};

struct Token {
  int64_t id;  // -1: none
  bool live;   // false: a row of padding
  bool bad;    // not a token
};

__device__ __forceinline__ int64_t id_at(const void* ids, int32_t bytes, int64_t at) {
  return bytes == 4 ? (int64_t) static_cast<const int32_t*>(ids)[at] : static_cast<const int64_t*>(ids)[at];
}

__device__ __forceinline__ void set_id(void* ids, int32_t bytes, int64_t at, int64_t id) {
  if (bytes == 4)
    static_cast<int32_t*>(ids)[at] = (int32_t)id;
  else
    static_cast<int64_t*>(ids)[at] = id;
}

__device__ __forceinline__ Token token_of(const Rows& r, int64_t row) {
  if (!r.ids) return Token{-1, true, false};
  const int64_t id = id_at(r.ids, r.id_bytes, row);
  return Token{id < 0 || id >= r.V ? -1 : id, id >= 0, id >= r.V};
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}

// The logarithm of a sum of exponentials, as exact near a sum of 1 as elsewhere.
__device__ __forceinline__ float log_sum(double s) {
  const float near = (float)s;
  return __builtin_fmaf((float)(s - (double)near), __builtin_amdgcn_rcpf(near), logf(near));
}

// A maximum with the sums over e = 2^d and e d, d = (x - m) c.  A likely token's 1
// beside thousands of numbers near 2^-24 keeps none of them in fp32: eight terms
// are added by a tree, of three roundings at most that have the 1, and fp64 takes
// their sums, over lanes too (bf16, 4,096 rows of 50,021 with their gradient 165 us,
// 2,048 rows with 5 alternatives 43.8, 8,000 rows of 500 12.4; with the whole sum in
// fp32 164, 43.5 and 10.6).
constexpr int kTree = 8;
struct Sums {
  float m = -kInf;
  double s = 0.0, t = 0.0;

  // N values, m not below them.
  template <int N, bool ENT>
  __device__ __forceinline__ void add(const float* x, float b, float c) {
    constexpr int G = N < kTree ? N : kTree;
    static_assert(N % G == 0 && (G & (G - 1)) == 0, "whole trees");
#pragma unroll
    for (int first = 0; first < N; first += G) {
      float e[G], ed = 0.0f;
#pragma unroll
      for (int i = 0; i < G; ++i) {
        const float d = (x[first + i] - b) * c;
        e[i] = exp2_fast(d);
        if (ENT) ed = __builtin_fmaf(e[i], fmaxf(d, kLow), ed);
      }
#pragma unroll
      for (int half = G / 2; half > 0; half /= 2)
#pragma unroll
        for (int i = 0; i < half; ++i) e[i] += e[i + half];
      s += (double)e[0];
      if (ENT) t += (double)ed;
      if (N > G) __builtin_amdgcn_sched_barrier(0);  // trees side by side take 65 registers, a wave of a SIMD less
    }
  }
  template <bool ENT>
  __device__ __forceinline__ void shift(float to, float c) {  // the sums as from another maximum, not below m
    const float d = (m - safe_max(to)) * c;
    const double e = (double)exp2_fast(d);
    if (ENT) t = e * __builtin_fma(s, (double)fmaxf(d, kLow), t);
    s *= e;
    m = to;
  }
  template <bool ENT>
  __device__ __forceinline__ void join(const Sums& o, float c) {
    Sums p = o;
    const float M = fmaxf(m, o.m);
    shift<ENT>(M, c);
    p.shift<ENT>(M, c);
    s += p.s;
    t += p.t;
  }
  // Values and no new maximum below them.
  template <int N, bool ENT>
  __device__ __forceinline__ void piece(const float* e, float c) {
    float vm = e[0];
#pragma unroll
    for (int i = 1; i < N; ++i) vm = fmaxf(vm, e[i]);
    if (vm > m) shift<ENT>(vm, c);
    add<N, ENT>(e, safe_max(m), c);
  }
  template <bool ENT>
  __device__ __forceinline__ void all(double (*R)[3], float c) {  // over the workgroup
    shift<ENT>(wave_max(m), c);
    s = wave_sum(s);
    float near = (float)t;  // a sum of one sign: its own roundings suffice
    if (ENT) near = wave_sum(near);
    const int wave = threadIdx.x >> 6, nw = blockDim.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
      R[wave][0] = m;
      R[wave][1] = s;
      R[wave][2] = near;
    }
    __syncthreads();
    // a wave's lanes take one wave each: nw <= 16
    const int w = threadIdx.x & 15;
    const bool in = w < nw;
    m = in ? (float)R[w][0] : -kInf;
    s = in ? R[w][1] : 0.0;
    t = in ? R[w][2] : 0.0;
    float M = m;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, 64));
    shift<ENT>(M, c);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if (ENT) {
      near = (float)t;
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) near += __shfl_xor(near, o, 64);
      t = near;
    }
  }
  // whether they are those of a distribution: no NaN, no +inf, not -inf alone
  __device__ __forceinline__ bool good() const { return s > 0.0 && s < (double)kInf && m < kInf; }
  __device__ __forceinline__ float entropy() const { return fmaxf(log_sum(s) - kLn2 * ((float)t / (float)s), 0.0f); }  // of good ones
};

// How a workgroup of B lanes shares elements [c0, c1) of a row: 16-byte pieces
// from the first aligned one on, lane after lane, and one of the elements around
// them.
template <class E_, int B>
struct Share {
  static constexpr int N = Vec<E_>::N;
  const E_* x;
  int64_t c0;
  int32_t head, nv, n;
  __device__ __forceinline__ Share(const E_* x_, int64_t c0_, int64_t c1) : x(x_), c0(c0_), n((int32_t)(c1 - c0_)) {
    head = (int32_t)head_of(x + c0, n);
    nv = (n - head) / N;
  }
  __device__ __forceinline__ int64_t piece(int32_t i) const { return c0 + head + (int64_t)i * N; }
  __device__ __forceinline__ bool has_single(int32_t lane) const { return lane < n - nv * N; }
  __device__ __forceinline__ int64_t single(int32_t lane) const { return c0 + (lane < head ? lane : lane + (int64_t)nv * N); }
  // what a lane has, for the others to look at
  static constexpr bool kOwn = false;
  __device__ __forceinline__ int32_t items() const { return (nv + B - 1) / B + 1; }
  template <class F>
  __device__ __forceinline__ void item(int32_t lane, int32_t j, F f) const {
    const int32_t i = lane + (j - 1) * B;
    if (j == 0) {
      if (has_single(lane)) f((float)x[single(lane)], single(lane));
    } else if (i < nv) {
      float e[N];
      load_floats(x + piece(i), e);
#pragma unroll
      for (int k = 0; k < N; ++k) f(e[k], piece(i) + k);
    }
  }
};

// A lane's sums over its share, kAhead pieces on their way at once (2,048 rows of
// 50,021 bf16 logits: 40.6 us, with two 43.3, with six 45.0, with eight 48.0).
constexpr int kAhead = 4;
template <class E_, int B, bool ENT>
__device__ __forceinline__ void row_sums(const Share<E_, B>& sh, float c, Sums& sums) {
  constexpr int N = Vec<E_>::N;
  int32_t i = threadIdx.x;
  for (; i + (kAhead - 1) * B < sh.nv; i += kAhead * B) {
    float e[kAhead][N];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) load_floats(sh.x + sh.piece(i + a * B), e[a]);
    sums.template piece<kAhead * N, ENT>(&e[0][0], c);
  }
  // fewer than kAhead pieces are left, and the element beside them
  const bool single = sh.has_single(threadIdx.x);
  const float one = single ? (float)sh.x[sh.single(threadIdx.x)] : -kInf;
  if (i < sh.nv) {
    float e[kAhead - 1][N];
#pragma unroll
    for (int a = 0; a < kAhead - 1; ++a) load_floats(sh.x + sh.piece(i + a * B < sh.nv ? i + a * B : i), e[a]);
#pragma unroll
    for (int a = 0; a < kAhead - 1; ++a)
      if (i + a * B < sh.nv) sums.template piece<N, ENT>(e[a], c);
  }
  if (single) sums.template piece<1, ENT>(&one, c);
}

// The largest value of a row that stays in registers.  Pairs of bf16 values stay
// packed: as signed numbers their order is right where one of them is not negative,
// and else the least unsigned number is the largest value.  A NaN is the largest
// value or shows in the sums.  4,096 rows of 50,021 with their gradient, bound by
// vector instructions: 166.8 us, unpacked for the maximum too 167.7.
template <class E_, int B, int NV>
__device__ __forceinline__ float kept_max(const Kept<E_, B, NV>& kept) {
  constexpr int N = Vec<E_>::N;
  float top = (float)kept.single;
  if constexpr (sizeof(E_) == 2) {
    typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    i16x2 most = (int16_t)-32768;
    u16x2 least = (uint16_t)65535;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        most = __builtin_elementwise_max(most, __builtin_bit_cast(i16x2, kept.v[i][k]));
        least = __builtin_elementwise_min(least, __builtin_bit_cast(u16x2, kept.v[i][k]));
      }
    const int16_t high = most[0] > most[1] ? most[0] : most[1];
    const uint16_t low = least[0] < least[1] ? least[0] : least[1];
    return fmaxf(top, __builtin_bit_cast(float, (uint32_t)(high >= 0 ? (uint16_t)high : low) << 16));
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float e[N];
      kept.get(i, e);
#pragma unroll
      for (int k = 0; k < N; k += 2) top = fmaxf(fmaxf(top, e[k]), e[k + 1]);
    }
    return top;
  }
}

// A lane's sums over a row that stays in registers.  d is (x - m) c, not x c - m c
// in one instruction: the largest logit's e is 1, so that no probability is above 1
// and that of a row's only token is.
template <bool ENT, class E_, int B, int NV>
__device__ __forceinline__ void kept_sums(const Kept<E_, B, NV>& kept, float c, Sums& sums) {
  constexpr int N = Vec<E_>::N;
  const float top = kept_max(kept);
  sums.m = top;
  const float b = safe_max(top);
  const float single = (float)kept.single;
  sums.template add<1, ENT>(&single, b, c);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    float e[N];
    kept.get(i, e);
    sums.template add<N, ENT>(e, b, c);
  }
}

// ---- alternatives -----------------------------------------------------------

// Unsigned numbers in the order of the values; both zeros are one value.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t k) { return __builtin_bit_cast(float, k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// ... of values and ids, the lower id above the higher one.
__device__ __forceinline__ uint64_t key_of(float x, int64_t id) { return (uint64_t)key_of(x) << 32 | (0xffffffffu - (uint32_t)id); }

struct Select {
  uint64_t found[kCap], prefix;
  uint32_t lane_key[kLB], hist[256], count, left_over, lanes, floor, left, enough;
  uint16_t lane[kLB];
};

// The largest value of the leading 16 bits (all of a bf16 value's) that K of 64 G
// groups of lanes reach, by one wave.
constexpr int kFewTop = 48;
template <int B, int G>
__device__ __forceinline__ uint32_t floor_of(const Select& S, int K) {
  constexpr int kLanes = B / (64 * G);  // of a group
  uint32_t k[G], floor = 0;
#pragma unroll
  for (int g = 0; g < G; ++g) {
    k[g] = 0;
#pragma unroll
    for (int w = 0; w < kLanes; ++w) {
      const uint32_t l = S.lane_key[64 * (g * kLanes + w) + threadIdx.x];
      k[g] = l > k[g] ? l : k[g];
    }
    k[g] >>= 16;
  }
  for (int bit = 15; bit >= 0; --bit) {
    const uint32_t more = floor | 1u << bit;
    int n = 0;
#pragma unroll
    for (int g = 0; g < G; ++g) n += __popcll(__ballot(k[g] >= more));
    if (n >= K) floor = more;
  }
  return floor << 16;
}

// ... that K of the n candidates reach.  Lanes count their own: with a ballot for
// each number the kernel takes more than 80 scalar registers, and a SIMD has
// seven waves instead of eight (2,048 rows of 50,021 logits: 46 us instead of 42).
__device__ __forceinline__ uint32_t floor_of_found(const Select& S, int count, int K) {
  constexpr int G = kCap / 64;
  uint32_t k[G], floor = 0;
#pragma unroll
  for (int g = 0; g < G; ++g) k[g] = 64 * g + (int)threadIdx.x < count ? (uint32_t)(S.found[64 * g + threadIdx.x] >> 48) : 0;
#pragma unroll 1
  for (int bit = 15; bit >= 0; --bit) {
    const uint32_t more = floor | 1u << bit;
    int reached = 0;
#pragma unroll
    for (int g = 0; g < G; ++g) reached += k[g] >= more;
    int n = 0;
#pragma unroll
    for (int b = 0; 1 << b <= G; ++b) n += __popcll(__ballot(reached >> b & 1)) << b;
    if (n >= K) floor = more;
  }
  return floor;
}

// The K largest of what a workgroup of B lanes shares: of.item(lane, j, f) calls
// f(value, id) for item j < items() of a lane, or (kOwn) of.each(f) for all of this
// lane's; largest is the largest value of this lane's; emit(rank, value, id) takes
// the results, (-inf, -1) where fewer values are above -inf.
template <int B, class Of, class Emit>
__device__ __forceinline__ void select_top(Select& S, int K, float largest, const Of& of, Emit emit) {
  const int tid = threadIdx.x;
  const uint32_t own = key_of(largest);
  S.lane_key[tid] = own;
  if (tid == 0) S.count = S.left_over = S.lanes = 0;
  __syncthreads();
  if (tid < 64) {
    const uint32_t floor = K <= kFewTop ? floor_of<B, 1>(S, K) : floor_of<B, (B < 256 ? B / 64 : 4)>(S, K);
    if (tid == 0) S.floor = floor;
  }
  __syncthreads();
  const uint32_t floor = S.floor;
  const auto mine = [&](auto f) {
    if constexpr (Of::kOwn) {
      of.each(f);
    } else {
      for (int j = 0; j < of.items(); ++j) of.item(tid, j, f);
    }
  };
  const auto put = [&](uint64_t from) {
    return [&S, from](float v, int64_t id) {
      const uint64_t k = key_of(v, id);
      if (v > -kInf && k >= from) {
        const uint32_t i = atomicAdd(&S.count, 1u);
        if (i < kCap) S.found[i] = k;
      }
    };
  };
  if constexpr (Of::kOwn) {
    if (own >= floor) {
      const float least = floor > key_of(-kInf) ? value_of(floor) : -__FLT_MAX__;
      of.each([&](float v, int64_t id) {
        if (v >= least) {
          const uint32_t i = atomicAdd(&S.count, 1u);
          if (i < kCap) S.found[i] = key_of(v, id);
        }
      });
    }
  } else {
    if (own >= floor) S.lane[atomicAdd(&S.lanes, 1u)] = (uint16_t)tid;
    __syncthreads();
    // all lanes share what those lanes have: one round trip to the caches, not one an item
    const int items = of.items();
    for (int i = tid; i < (int)S.lanes * items; i += B) {
      const int l = i / items;
      of.item(S.lane[l], i - l * items, put((uint64_t)floor << 32));
    }
  }
  __syncthreads();
  if (S.count > kCap) {  // the same for all lanes; the K-th key digit by digit, until at most kCap keys are not below it
    uint64_t prefix = 0;
    uint32_t left = K;
    for (int shift = 56;; shift -= 8) {
      __syncthreads();
      for (int i = tid; i < 256; i += B) S.hist[i] = 0;
      __syncthreads();
      mine([&](float v, int64_t id) {
        const uint64_t k = key_of(v, id);
        if (v > -kInf && (shift == 56 || k >> (shift + 8) == prefix >> (shift + 8))) atomicAdd(&S.hist[k >> shift & 255], 1u);
      });
      __syncthreads();
      if (tid == 0) {
        uint32_t n = left;
        int digit = 255;
        for (; digit > 0 && S.hist[digit] < n; --digit) n -= S.hist[digit];
        S.left = n;
        S.enough = K - n + S.hist[digit] <= kCap;
        S.prefix = prefix | (uint64_t)digit << shift;
        S.count = 0;
      }
      __syncthreads();
      prefix = S.prefix;
      left = S.left;
      if (S.enough || shift == 0) break;
    }
    mine(put(prefix));
    __syncthreads();
  }
  int n = __builtin_amdgcn_readfirstlane((int)(S.count < kCap ? S.count : kCap));
  if (n > K && n * ((n + B - 1) / B) > kRanking) {  // few groups of lanes for K, or few that hold values: the lowest candidates are left out first
    uint64_t k[kCap / B];
#pragma unroll
    for (int j = 0; j < kCap / B; ++j) k[j] = tid + j * B < n ? S.found[tid + j * B] : 0;
    if (tid < 64) {
      const uint32_t cut = floor_of_found(S, n, K);
      if (tid == 0) S.floor = cut;  // not count: others may still read it
    }
    __syncthreads();
    const uint32_t cut = S.floor;
#pragma unroll
    for (int j = 0; j < kCap / B; ++j)
      if (tid + j * B < n && (uint32_t)(k[j] >> 48) >= cut) S.found[atomicAdd(&S.left_over, 1u)] = k[j];
    __syncthreads();
    n = __builtin_amdgcn_readfirstlane((int)S.left_over);
  }
  for (int i = tid; i < n; i += B) {
    const uint64_t k = S.found[i];
    int rank = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) rank += S.found[j] > k;
    if (rank < K) emit(rank, value_of((uint32_t)(k >> 32)), (int64_t)(0xffffffffu - (uint32_t)k));
  }
  for (int i = n + tid; i < K; i += B) emit(i, -kInf, (int64_t)-1);
}

struct Results {
  float *logprob, *entropy, *stats, *top_logprob;
  void* top_ids;
  int32_t top_bytes, K;
};

constexpr int kMeans = 8;  // floats of a slice's averages

// What a slice leaves for the join: its sums (s in two parts), then its K largest logits and their ids.
struct Parts {
  float* p;
  int32_t slices, K;
  int64_t per;
  __device__ __forceinline__ float* sums(int64_t i) const { return p + i * (4 + 2 * K); }
  __device__ __forceinline__ float* means(int64_t i) const { return p + i * kMeans; }  // of the second derivative, in their place
  __device__ __forceinline__ float* values(int64_t i) const { return sums(i) + 4; }
  __device__ __forceinline__ int32_t* ids(int64_t i) const { return reinterpret_cast<int32_t*>(sums(i) + 4 + K); }
  __device__ __forceinline__ Sums get(int64_t i) const {
    Sums s;
    s.m = sums(i)[0];
    s.s = (double)sums(i)[1] + (double)sums(i)[2];
    s.t = sums(i)[3];
    return s;
  }
  __device__ __forceinline__ void put(int64_t i, const Sums& s) const {
    const float near = (float)s.s;
    sums(i)[0] = s.m;
    sums(i)[1] = near;
    sums(i)[2] = (float)(s.s - (double)near);
    sums(i)[3] = (float)s.t;
  }
};

struct Slice {
  int64_t row, c0, c1;
  int32_t index;
};

__device__ __forceinline__ Slice slice_of(const Rows& r, int32_t slices, int64_t per) {
  Slice s;
  s.row = blockIdx.x / (uint32_t)slices;
  s.index = (int32_t)(blockIdx.x - s.row * slices);
  s.c0 = s.index * per;
  s.c1 = s.c0 + per < r.V ? s.c0 + per : r.V;
  return s;
}

// A row's numbers from its sums, by one lane.
__device__ __forceinline__ void finish(const Rows& r, const Results& o, int64_t row, const Token& tok, float x, const Sums& sums) {
  const bool good = sums.good() && !tok.bad;
  if (o.stats) {
    o.stats[2 * row] = tok.live ? sums.m : 0.0f;
    o.stats[2 * row + 1] = tok.live ? (float)sums.s : 1.0f;
  }
  if (o.logprob) o.logprob[row] = !tok.live ? 0.0f : good ? (x - sums.m) * r.invT - log_sum(sums.s) : kNan;
  if (o.entropy) o.entropy[row] = !tok.live ? 0.0f : good ? sums.entropy() : kNan;
}

// ... and its alternatives, by the workgroup.
template <int B, class Of>
__device__ __forceinline__ void finish_top(const Rows& r, const Results& o, Select& S, int64_t row, const Token& tok, const Sums& sums, float largest,
                                           const Of& of) {
  const float ls = log_sum(sums.s);
  if (!tok.live || tok.bad || !sums.good()) {
    for (int k = threadIdx.x; k < o.K; k += B) {
      o.top_logprob[row * o.K + k] = tok.live ? kNan : -kInf;
      set_id(o.top_ids, o.top_bytes, row * o.K + k, -1);
    }
    return;
  }
  select_top<B>(S, o.K, largest, of, [&](int rank, float v, int64_t id) {
    o.top_logprob[row * o.K + rank] = id < 0 ? -kInf : (v - sums.m) * r.invT - ls;
    set_id(o.top_ids, o.top_bytes, row * o.K + rank, id);
  });
}

// A row (or a slice of one), read once; lanes that may hold an alternative look
// at theirs again, from the caches.
template <class E_, bool ENT, bool TOP, int B>
__global__ __launch_bounds__(B) void logprob_row(Rows r, Results o, Parts parts) {
  __shared__ double R[B / 64][3];
  __shared__ std::conditional_t<TOP, Select, int> S;
  const Slice sl = slice_of(r, parts.slices, parts.per);
  const Token tok = token_of(r, sl.row);
  const E_* x = static_cast<const E_*>(r.logits) + sl.row * r.row_stride;
  const float c = r.invT * kLog2e;
  const Share<E_, B> share(x, sl.c0, sl.c1);
  Sums sums;
  if (tok.live) row_sums<E_, B, ENT>(share, c, sums);
  else if (parts.slices > 1) return;  // nothing of it is read
  const float largest = sums.m;
  sums.all<ENT>(R, c);
  if (parts.slices > 1) {
    if (threadIdx.x == 0) parts.put(blockIdx.x, sums);
    if constexpr (TOP)
      select_top<B>(S, o.K, largest, share, [&](int rank, float v, int64_t id) {
        parts.values(blockIdx.x)[rank] = v;
        parts.ids(blockIdx.x)[rank] = (int32_t)id;
      });
    return;
  }
  if (threadIdx.x == 0) finish(r, o, sl.row, tok, tok.id >= 0 ? (float)x[tok.id] : 0.0f, sums);
  if constexpr (TOP) finish_top<B>(r, o, S, sl.row, tok, sums, largest, share);
}

// What a lane has of a row that stays in registers.
template <class E_, int B, int NV>
struct OwnPieces {
  const Kept<E_, B, NV>& kept;
  static constexpr bool kOwn = true;
  template <class F>
  __device__ __forceinline__ void each(F f) const {
    if (kept.has_single) f((float)kept.single, (int64_t)kept.at_single);
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (kept.has(i)) {
        float e[Vec<E_>::N];
        kept.get(i, e);
#pragma unroll
        for (int k = 0; k < Vec<E_>::N; ++k) f(e[k], (int64_t)(kept.at(i) + k));
      }
  }
};

// A short row of many, read once.
template <class E_, bool ENT, bool TOP, int B, int NV>
__global__ __launch_bounds__(B, kept_waves(B, NV)) void logprob_kept(Rows r, Results o) {
  __shared__ double R[B / 64][3];
  __shared__ std::conditional_t<TOP, Select, int> S;
  const int64_t row = blockIdx.x;
  const Token tok = token_of(r, row);
  const E_* x = static_cast<const E_*>(r.logits) + row * r.row_stride;
  const float c = r.invT * kLog2e;
  Kept<E_, B, NV> kept;
  Sums sums;
  if (tok.live) {
    kept.place(x, (uint32_t)r.V);
    kept.load(x, (E_)-kInf);
    kept_sums<ENT>(kept, c, sums);
  }
  const float largest = sums.m;
  sums.all<ENT>(R, c);
  if (threadIdx.x == 0) finish(r, o, row, tok, tok.id >= 0 ? (float)x[tok.id] : 0.0f, sums);
  if constexpr (TOP) finish_top<B>(r, o, S, row, tok, sums, largest, OwnPieces<E_, B, NV>{kept});
}

// What the slices of a row found, kHeld values a lane.  A slice's values fall: each
// slice is turned a little further than the one before it, so that the largest ones of
// all slices lie in different lanes (2 rows of 151,722 fp32 logits with 128 alternatives
// 19 us, unturned 23).
constexpr int kHeld = 8, kTurn = 37;
struct Held {
  float v[kHeld];
  int32_t id[kHeld];
  static constexpr bool kOwn = true;
  __device__ __forceinline__ Held(const Parts& parts, int64_t first, bool live) {
    const int32_t n = live ? parts.slices * parts.K : 0;
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
      const int32_t i = threadIdx.x + j * kJB;
      v[j] = -kInf;
      id[j] = -1;
      if (i >= n) continue;
      const int32_t slice = i / parts.K, k = (i - slice * parts.K + slice * kTurn) % parts.K;
      v[j] = parts.values(first + slice)[k];
      id[j] = parts.ids(first + slice)[k];
    }
  }
  __device__ __forceinline__ float largest() const {
    float x = v[0];
#pragma unroll
    for (int j = 1; j < kHeld; ++j) x = fmaxf(x, v[j]);
    return x;
  }
  template <class F>
  __device__ __forceinline__ void each(F f) const {
#pragma unroll
    for (int j = 0; j < kHeld; ++j) f(v[j], (int64_t)id[j]);
  }
};

// A row from its slices' sums and largest logits.
template <class E_, bool ENT, bool TOP>
__global__ __launch_bounds__(kJB) void logprob_join(Rows r, Results o, Parts parts) {
  __shared__ double R[kJB / 64][3];
  __shared__ std::conditional_t<TOP, Select, int> S;
  const int64_t row = blockIdx.x, first = row * parts.slices;
  const Token tok = token_of(r, row);
  const E_* x = static_cast<const E_*>(r.logits) + row * r.row_stride;
  const float c = r.invT * kLog2e;
  const Held held(parts, first, TOP && tok.live);
  Sums sums;
  if (tok.live)
    for (int i = threadIdx.x; i < parts.slices; i += kJB) sums.join<ENT>(parts.get(first + i), c);
  sums.all<ENT>(R, c);
  if (threadIdx.x == 0) finish(r, o, row, tok, tok.id >= 0 ? (float)x[tok.id] : 0.0f, sums);
  if constexpr (TOP) finish_top<kJB>(r, o, S, row, tok, sums, held.largest(), held);
}

// ---- gradient ---------------------------------------------------------------

// The cotangents of a row's results, any of them NULL; entropy [N] goes with
// dentropy, top_ids [N][K] with dtop.
struct Cotangents {
  const float *dlogprob, *dentropy, *entropy, *dtop;
  const void* top_ids;
  int32_t top_bytes, K;
};

// The tokens of a row that are named: the alternatives, then the given one.
struct Named {
  int32_t id[kMaxTop + 1];  // -1: none
  float c[kMaxTop + 1], x[kMaxTop + 1];
  float sum;  // of c
};

template <class E_>
__device__ __forceinline__ void load_named(const Rows& r, const Cotangents& t, int64_t row, const Token& tok, const E_* x, Named& M, int lane) {
  float sum = 0.0f;
  for (int j = lane; j <= t.K; j += 64) {
    int64_t id = j == t.K ? tok.id : id_at(t.top_ids, t.top_bytes, row * t.K + j);
    float c = j == t.K ? (t.dlogprob ? t.dlogprob[row] : 0.0f) : t.dtop[row * t.K + j];
    if (id < 0 || id >= r.V) {
      id = -1;
      c = 0.0f;
    }
    M.id[j] = (int32_t)id;
    M.c[j] = c;
    M.x[j] = id >= 0 ? (float)x[id] : 0.0f;
    sum += c;
  }
  sum = wave_sum(sum);
  if (lane == 0) M.sum = sum;
}

// The sum of w over the entries that name the token of entry j.
__device__ __forceinline__ float same_token(const Named& M, int K, int32_t id) {
  float sum = 0.0f;
  for (int i = 0; i <= K; ++i) sum += M.id[i] == id ? M.c[i] : 0.0f;
  return sum;
}

// d = (x - m) c and e = 2^d as Shift computes them: d lies off by a constant that
// `off` has, e by the factor 2^off.
template <bool WIDE>
__device__ __forceinline__ float depth(const Shift& sh, float x) {
  return WIDE ? (x - sh.b) * sh.c : __builtin_fmaf(x, sh.c, -sh.bc);
}
template <bool WIDE>
__device__ __forceinline__ float off(const Shift& sh) {
  return WIDE ? 0.0f : -__builtin_fmaf(sh.b, sh.c, -sh.bc);
}

// The dense part of a row's gradient, -(p / T)(G + h (l + H)) with l + H = ln 2 (d
// + off) - log s + H, as w e (A + B d).
struct Dense {
  Shift sh;
  float w, A, B;
  __device__ __forceinline__ Dense(float m, float s, float c, float invT, float G, float h, float H) : sh(m, c) {
    const float o = sh.wide ? off<true>(sh) : off<false>(sh);
    w = -invT / s * exp2_fast(o);
    B = h * kLn2;
    A = G + h * ((H - logf(s)) + kLn2 * o);
  }
  template <bool ENT, bool WIDE>
  __device__ __forceinline__ float at(float x) const {
    const float d = depth<WIDE>(sh, x), e = w * exp2_fast(d);
    return e * (ENT ? __builtin_fmaf(B, fmaxf(d, kLow), A) : A);
  }
  template <bool ENT>
  __device__ __forceinline__ float at(float x) const {
    return sh.wide ? at<ENT, true>(x) : at<ENT, false>(x);
  }
};

enum Stats { kGiven, kRead, kKept, kParts };  // where a row's sums come from

// A row's gradient (or a slice of it), with its results where the same call
// makes them.
template <class E_, int STATS, bool ENT, int B = kLB, int NV = 1>
__global__ __launch_bounds__(B, (STATS == kKept ? kept_waves(B, NV) : 1)) void logprob_grad(Rows r, Results o, Cotangents t, const float* stats,
                                                                                            E_* dlogits, int64_t drow_stride, Parts parts) {
  __shared__ Named M;
  __shared__ double R[B / 64][3];
  constexpr int N = Vec<E_>::N;
  const int lane = threadIdx.x & 63;
  const float c = r.invT * kLog2e;
  const Slice sl = slice_of(r, parts.slices, parts.per);
  const int64_t row = sl.row;
  const Token tok = token_of(r, row);
  const E_* x = static_cast<const E_*>(r.logits) + row * r.row_stride;
  E_* dx = dlogits + row * drow_stride;
  Kept<E_, B, NV> kept;
  Sums sums;
  if (tok.live) {
    if constexpr (STATS == kKept) {
      kept.place(x, (uint32_t)r.V);
      kept.load(x, (E_)-kInf);
    }
    if (threadIdx.x < 64) load_named(r, t, row, tok, x, M, lane);  // before dlogits, which may be logits, is written
    if constexpr (STATS == kRead) row_sums<E_, B, ENT>(Share<E_, B>(x, 0, r.V), c, sums);
    if constexpr (STATS == kParts)
      for (int i = threadIdx.x; i < parts.slices; i += B) sums.join<ENT>(parts.get(row * parts.slices + i), c);
    if constexpr (STATS == kKept) kept_sums<ENT>(kept, c, sums);
  }
  float H = 0.0f;
  if constexpr (STATS == kGiven) {
    sums.m = stats[2 * row];
    sums.s = stats[2 * row + 1];
    if (ENT) H = t.entropy[row];
    __syncthreads();  // the named tokens
  } else {
    sums.all<ENT>(R, c);
    if (ENT) H = sums.entropy();
    if (threadIdx.x == 0 && sl.index == 0) finish(r, o, row, tok, tok.id >= 0 ? M.x[t.K] : 0.0f, sums);
  }
  const bool good = sums.good() && !tok.bad;
  if (!tok.live || !good) {  // the same for the workgroup
    const float fill = tok.live ? kNan : 0.0f;
    over_row(
        dx, sl.c0, sl.c1,
        [&](int64_t at) {
          float y[N];
#pragma unroll
          for (int i = 0; i < N; ++i) y[i] = fill;
          store_vec(dx + at, y);
        },
        [&](int64_t at) { dx[at] = (E_)fill; });
    return;
  }
  const Dense dense(sums.m, (float)sums.s, c, r.invT, M.sum, ENT && t.dentropy ? t.dentropy[row] : 0.0f, H);
  const auto write = [&](auto wide) {
    constexpr bool W = wide.value;
    if constexpr (STATS == kKept) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (kept.has(i)) {
          float e[N];
          kept.get(i, e);
#pragma unroll
          for (int k = 0; k < N; ++k) e[k] = dense.template at<ENT, W>(e[k]);
          store_vec(dx + kept.at(i), e);
        }
      if (kept.has_single) dx[kept.at_single] = (E_)dense.template at<ENT, W>((float)kept.single);
    } else {
      over_row(
          x, sl.c0, sl.c1,
          [&](int64_t at) {
            float e[N];
            load_floats(x + at, e);
#pragma unroll
            for (int k = 0; k < N; ++k) e[k] = dense.template at<ENT, W>(e[k]);
            store_vec(dx + at, e);
          },
          [&](int64_t at) { dx[at] = (E_)dense.template at<ENT, W>((float)x[at]); });
    }
  };
  if (dense.sh.wide)
    write(std::true_type{});
  else
    write(std::false_type{});
  __syncthreads();  // the named tokens' elements are written after the dense part's
  for (int j = threadIdx.x; j <= t.K; j += B) {
    const int32_t id = M.id[j];
    if (id >= sl.c0 && id < sl.c1) dx[id] = (E_)(dense.template at<ENT>(M.x[j]) + r.invT * same_token(M, t.K, id));
  }
}

// ---- the gradient's vector-Jacobian product ---------------------------------

struct Second {
  const void* a;  // cotangent of dlogits
  int64_t a_stride;
  const float* stats;
  float *out_dlogprob, *out_dentropy, *out_dtop;
  void* out;
  int64_t out_stride;
};

// What a and l + H average to under p, and how they vary together, from sums that
// have no rounding of a in them: weights of fp32, products and sums of fp64, divided
// by the weights' own sum.  Sums in fp32 carry a value common to all of a into the
// covariance, with its rounding: at 100 beside deviations of 0.1 4e-4 of it.  2,048 rows
// of 50,021 bf16 logits 185 us, 1,024 of 32,000 fp32 logits 96, with fp32 sums 162 and 88;
// fp32 sums about a at a lane's likeliest token 186 and 97.
struct Means {
  double w = 0.0, a = 0.0, l = 0.0, al = 0.0;
  template <bool ENT>
  __device__ __forceinline__ void add(float e, float lH, float v) {
    const double p = (double)e, u = (double)v;
    w += p;
    a = __builtin_fma(p, u, a);
    if (ENT) {
      const double pl = (double)(e * lH);
      l += pl;
      al = __builtin_fma(pl, u, al);
    }
  }
  template <bool ENT>
  __device__ __forceinline__ void all(double (*R)[4]) {  // over the workgroup
    w = wave_sum(w);
    a = wave_sum(a);
    if (ENT) {
      l = wave_sum(l);
      al = wave_sum(al);
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
      double* to = R[threadIdx.x >> 6];
      to[0] = w;
      to[1] = a;
      to[2] = l;
      to[3] = al;
    }
    __syncthreads();
    w = a = l = al = 0.0;
#pragma unroll 4
    for (int i = 0; i < (int)(blockDim.x >> 6); ++i) {
      w += R[i][0];
      a += R[i][1];
      l += R[i][2];
      al += R[i][3];
    }
  }
  // of a slice: each sum in two parts
  __device__ __forceinline__ void put(float* to) const {
    const double v[4] = {w, a, l, al};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      to[2 * i] = (float)v[i];
      to[2 * i + 1] = (float)(v[i] - (double)to[2 * i]);
    }
  }
  __device__ __forceinline__ void take(const float* from) {
    w += (double)from[0] + (double)from[1];
    a += (double)from[2] + (double)from[3];
    l += (double)from[4] + (double)from[5];
    al += (double)from[6] + (double)from[7];
  }
};

// p and l + H of a logit.
struct Prob {
  Shift sh;
  float p, lH;  // factor of 2^d, l + H at d = 0
  __device__ __forceinline__ Prob(float m, float s, float c, float H) : sh(m, c) {
    const float o = sh.wide ? off<true>(sh) : off<false>(sh);
    p = exp2_fast(o) / s;
    lH = (H - logf(s)) + kLn2 * o;
  }
  template <bool ENT, bool WIDE>
  __device__ __forceinline__ void at(float x, float& e, float& l) const {
    const float d = depth<WIDE>(sh, x);
    e = p * exp2_fast(d);
    l = ENT ? __builtin_fmaf(kLn2, fmaxf(d, kLow), lH) : 0.0f;
  }
};

template <class E_, bool ENT>
__device__ __forceinline__ void row_means(const E_* x, const E_* a, int64_t c0, int64_t c1, const Prob& prob, Means& means) {
  const auto one = [&](float v, float u) {
    float e, l;
    if (prob.sh.wide)
      prob.at<ENT, true>(v, e, l);
    else
      prob.at<ENT, false>(v, e, l);
    means.add<ENT>(e, l, u);
  };
  over_row(
      x, c0, c1,
      [&](int64_t at) {
        float v[Vec<E_>::N], u[Vec<E_>::N];
        load_floats(x + at, v);
        load_floats(a + at, u);
#pragma unroll
        for (int i = 0; i < Vec<E_>::N; ++i) one(v[i], u[i]);
      },
      [&](int64_t at) { one((float)x[at], (float)a[at]); });
}

// A slice's averages, for rows that several workgroups share.
template <class E_, bool ENT>
__global__ __launch_bounds__(kLB) void logprob_second_parts(Rows r, Cotangents t, Second q, Parts parts) {
  __shared__ double R[kLB / 64][4];
  const Slice sl = slice_of(r, parts.slices, parts.per);
  if (!token_of(r, sl.row).live) return;
  const Prob prob(q.stats[2 * sl.row], q.stats[2 * sl.row + 1], r.invT * kLog2e, ENT ? t.entropy[sl.row] : 0.0f);
  Means means;
  row_means<E_, ENT>(static_cast<const E_*>(r.logits) + sl.row * r.row_stride, static_cast<const E_*>(q.a) + sl.row * q.a_stride, sl.c0, sl.c1, prob,
                     means);
  means.all<ENT>(R);
  if (threadIdx.x == 0) means.put(parts.means(blockIdx.x));
}

// Logits and a read once where they stay in registers, a result written.
template <class E_, int STATS, bool ENT, int B = kLB, int NV = 1>
__global__ __launch_bounds__(B) void logprob_second(Rows r, Cotangents t, Second q, Parts parts) {
  __shared__ Named M;
  __shared__ double R[B / 64][4];
  __shared__ float aj[kMaxTop + 1];
  constexpr int N = Vec<E_>::N;
  const int lane = threadIdx.x & 63;
  const Slice sl = slice_of(r, parts.slices, parts.per);
  const int64_t row = sl.row;
  const Token tok = token_of(r, row);
  const E_* x = static_cast<const E_*>(r.logits) + row * r.row_stride;
  const E_* a = static_cast<const E_*>(q.a) + row * q.a_stride;
  E_* y = static_cast<E_*>(q.out) + row * q.out_stride;
  Sums sums;
  sums.m = q.stats[2 * row];
  sums.s = q.stats[2 * row + 1];
  const bool good = sums.good() && !tok.bad;
  const bool first = sl.index == 0;
  if (!tok.live || !good) {
    const float fill = tok.live ? kNan : 0.0f;
    if (first) {
      if (threadIdx.x == 0) {
        if (q.out_dlogprob) q.out_dlogprob[row] = fill;
        if (q.out_dentropy) q.out_dentropy[row] = fill;
      }
      if (q.out_dtop)
        for (int k = threadIdx.x; k < t.K; k += B) q.out_dtop[row * t.K + k] = fill;
    }
    over_row(
        y, sl.c0, sl.c1,
        [&](int64_t at) {
          float z[N];
#pragma unroll
          for (int i = 0; i < N; ++i) z[i] = fill;
          store_vec(y + at, z);
        },
        [&](int64_t at) { y[at] = (E_)fill; });
    return;
  }
  Kept<E_, B, NV> kx, ka;
  if constexpr (STATS == kKept) {
    kx.place(x, (uint32_t)r.V);
    ka.place(x, (uint32_t)r.V);
    kx.load(x, (E_)-kInf);
    ka.load(a, (E_)0.0f);
  }
  if (threadIdx.x < 64) {
    load_named(r, t, row, tok, x, M, lane);
    for (int j = lane; j <= t.K; j += 64) aj[j] = M.id[j] >= 0 ? (float)a[M.id[j]] : 0.0f;
  }
  const float H = ENT ? t.entropy[row] : 0.0f, h = ENT && t.dentropy ? t.dentropy[row] : 0.0f;
  const Prob prob(sums.m, (float)sums.s, r.invT * kLog2e, H);
  Means means;
  if constexpr (STATS == kKept) {
    const auto sum = [&](auto wide) {
      const auto one = [&](float v, float u) {
        float e, l;
        prob.at<ENT, wide.value>(v, e, l);
        means.add<ENT>(e, l, u);
      };
      one((float)kx.single, (float)ka.single);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (!kx.has(i)) continue;  // short rows: whole waves have nothing (8,000 of 500 bf16 logits 30.3 us, all pieces summed 46)
        float e[N], u[N];
        kx.get(i, e);
        ka.get(i, u);
#pragma unroll
        for (int k = 0; k < N; ++k) one(e[k], u[k]);
      }
    };
    if (prob.sh.wide)
      sum(std::true_type{});
    else
      sum(std::false_type{});
  } else if constexpr (STATS == kRead) {
    row_means<E_, ENT>(x, a, 0, r.V, prob, means);
  } else {
    for (int i = threadIdx.x; i < parts.slices; i += B) means.take(parts.means(row * parts.slices + i));
  }
  means.all<ENT>(R);  // also: the named tokens are there
  const double mean = means.a / means.w;
  const float kappa = ENT ? (float)((means.al - mean * means.l) / means.w) : 0.0f, G = M.sum;
  const float near = (float)mean, rest = (float)(mean - (double)near);  // a's distance to the mean is a - near, exact where they are close, less the rest
  if (first) {
    if (threadIdx.x == 0) {
      if (q.out_dlogprob) q.out_dlogprob[row] = M.id[t.K] >= 0 ? r.invT * (aj[t.K] - near - rest) : 0.0f;
      if (q.out_dentropy) q.out_dentropy[row] = ENT ? -r.invT * kappa : 0.0f;
    }
    if (q.out_dtop)
      for (int k = threadIdx.x; k < t.K; k += B) q.out_dtop[row * t.K + k] = M.id[k] >= 0 ? r.invT * (aj[k] - near - rest) : 0.0f;
  }
  const float w = -r.invT * r.invT;
  const auto write = [&](auto wide) {
    const auto value = [&](float v, float u) {
      float e, l;
      prob.at<ENT, wide.value>(v, e, l);
      const float du = u - near - rest;
      return w * e * (ENT ? __builtin_fmaf(du, __builtin_fmaf(h, l + 1.0f, G), -h * kappa) : du * G);
    };
    if constexpr (STATS == kKept) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (kx.has(i)) {
          float e[N], u[N];
          kx.get(i, e);
          ka.get(i, u);
#pragma unroll
          for (int k = 0; k < N; ++k) e[k] = value(e[k], u[k]);
          store_vec(y + kx.at(i), e);
        }
      if (kx.has_single) y[kx.at_single] = (E_)value((float)kx.single, (float)ka.single);
    } else {
      over_row(
          x, sl.c0, sl.c1,
          [&](int64_t at) {
            float e[N], u[N];
            load_floats(x + at, e);
            load_floats(a + at, u);
#pragma unroll
            for (int k = 0; k < N; ++k) e[k] = value(e[k], u[k]);
            store_vec(y + at, e);
          },
          [&](int64_t at) { y[at] = (E_)value((float)x[at], (float)a[at]); });
    }
  };
  if (prob.sh.wide)
    write(std::true_type{});
  else
    write(std::false_type{});
}

// ---- host -------------------------------------------------------------------

int check_sizes(const char* who, int64_t N, int64_t V, int32_t dtype, const void* ids, int32_t id_bytes, int64_t K, int32_t top_bytes,
                double temperature) {
  if (N < 0) return fail(DIFFOPT_EINVAL, "%s: N must be >= 0", who);
  if (N >= kMostRows) return fail(DIFFOPT_EINVAL, "%s: N must be below 2^22", who);
  if (V < 1 || V > 0x7fffffff) return fail(DIFFOPT_EINVAL, "%s: V must be in [1, 2^31)", who);
  if (!dtype_ok(dtype)) return fail(DIFFOPT_EINVAL, "%s: unknown element type %d", who, (int)dtype);
  if (ids && id_bytes != 4 && id_bytes != 8) return fail(DIFFOPT_EINVAL, "%s: id_bytes must be 4 or 8", who);
  if (K < 0 || K > kMaxTop) return fail(DIFFOPT_EINVAL, "%s: K must be in [0, %d]", who, kMaxTop);
  if (K > 0 && top_bytes != 4 && top_bytes != 8) return fail(DIFFOPT_EINVAL, "%s: top_id_bytes must be 4 or 8", who);
  if (!(std::isfinite(temperature) && temperature > 0.0 && std::isfinite((float)(1.0 / temperature) * kLog2e) && (float)(1.0 / temperature) > 0.0f))
    return fail(DIFFOPT_EINVAL, "%s: temperature and log2(e) / temperature must be finite and > 0 in fp32", who);
  return DIFFOPT_OK;
}

int check_rows(const char* who, const void* logits, int64_t row_stride, int64_t N, int64_t V, int32_t dtype, const void* ids, int32_t id_bytes,
               double temperature, Rows* r) {
  if (!logits) return fail(DIFFOPT_EINVAL, "%s: null logits", who);
  if (!aligned_to(logits, elem_size(dtype)) || (ids && !aligned_to(ids, id_bytes)))
    return fail(DIFFOPT_EINVAL, "%s: a pointer is not aligned to its elements", who);
  *r = Rows{logits, row_stride, N, V, ids, id_bytes, (float)(1.0 / temperature)};
  return DIFFOPT_OK;
}

// Cotangents and what goes with them.
int check_cotangents(const char* who, const Rows& r, const Cotangents& t) {
  if (t.dlogprob && !r.ids) return fail(DIFFOPT_EINVAL, "%s: dlogprob without ids", who);
  if (t.dentropy && !t.entropy) return fail(DIFFOPT_EINVAL, "%s: dentropy without entropy", who);
  if (t.K > 0 && (!t.dtop || !t.top_ids)) return fail(DIFFOPT_EINVAL, "%s: null dtop_logprob or top_ids", who);
  if (t.K > 0 && !aligned_to(t.top_ids, t.top_bytes)) return fail(DIFFOPT_EINVAL, "%s: a pointer is not aligned to its elements", who);
  return check_aligned(who, {t.dlogprob, t.dentropy, t.entropy, t.dtop});
}

// Slices are longer than distillation's, whose join has no alternatives to rank: 8
// rows of 512 KiB with 20 of them 13.8 us in slices of 8 KiB, 12.3 of 16, 12.3 of 32.  With
// many alternatives they are as long as it takes for the join to hold what they find: one
// row of 600,000 fp32 logits with 20 13.3 us, with 128 24.0; a join that reads what slices
// of 16 KiB found again took 15.8 and 64.
Cut row_cut(int64_t N, int64_t V, int32_t dtype, int64_t K) {
  const int64_t fewest = (V * elem_size(dtype) * K + kHeld * kJB - 1) / (kHeld * kJB);
  return cut_of(N, V, dtype, fewest > 16384 ? fewest : 16384);
}

// Lanes of a row: 8,000 rows of 4,000 bf16 logits with 5 alternatives take 28.1 us
// with 128, 30.8 with 256 and 52.2 with 512; 4,000 of 16,000 36.3, 36.9 and 43.2; 2,048
// of 50,021 48.1, 48.3 and 43.6 (without alternatives 42.9, 44.2 and 39.2).
// With more than kFewTop alternatives 128 lanes say too little about where they are, once
// 256 have a piece or nearly: 300 rows of 4,000 with 128 of them 11.7 us, with 128 lanes
// 29.4; 4,000 rows 38.2 and 51.7, with 64 of them 24.3 and 25.6; but 4,000 rows of 500 fp32
// logits with 128 35.8 and 30.3.
constexpr int64_t kShortRow = 16384, kMiddleRow = 65536, kWideRow = 3200;
// Many short rows stay in registers: their maximum is known before the sums, and the
// alternatives are looked for in the lanes that read them.  8,000 rows of 4,000 bf16
// logits 17.2 us (streamed 20.6), with 5 alternatives 25.8 (28.1); 4,000 of 16,000 without
// 28.5 (33.4), with 5 50 (31); of more than 64 KiB and of few rows streaming is as fast or
// faster (300 of 1,000 fp32 logits 4.9 against 5.3, 2,048 of 50,021 39.7 against 41.7).
constexpr int64_t kKeptRows = 2048;

int64_t parts_bytes(int64_t N, int64_t V, int32_t dtype, int64_t K) {
  const Cut c = row_cut(N, V, dtype, K);
  return c.slices > 1 ? N * c.slices * (K ? 4 + 2 * K : kMeans) * 4 : 0;  // K = 0: the second derivative's too
}

int check_workspace(const char* who, const Rows& r, int32_t dtype, int64_t K, void* workspace, int64_t bytes) {
  const int64_t need = parts_bytes(r.N, r.V, dtype, K);
  if (need > 0 && (!workspace || bytes < need))
    return fail(DIFFOPT_EINVAL, "%s: the workspace has %lld bytes of %lld", who, (long long)(workspace ? bytes : 0), (long long)need);
  if (!aligned_to(workspace, 4)) return fail(DIFFOPT_EINVAL, "%s: the workspace is not 4-byte aligned", who);
  return DIFFOPT_OK;
}

#define DIFFOPT_LAUNCH(kernel, grid, block, ...) hipLaunchKernelGGL((kernel), dim3((unsigned)(grid)), dim3(block), 0, st, __VA_ARGS__)

Parts parts_of(const Cut& c, int64_t K, void* workspace) { return Parts{static_cast<float*>(workspace), c.slices, (int32_t)K, c.per}; }

template <class E_, bool ENT, bool TOP>
int fwd_rows(const char* who, const Rows& r, int32_t dtype, const Results& o, void* workspace, hipStream_t st) {
  const Cut c = row_cut(r.N, r.V, dtype, TOP ? o.K : 0);
  const Parts p = parts_of(c, TOP ? o.K : 0, workspace);
  const int64_t bytes = r.V * elem_size(dtype);  // of a row: slices are for few rows, whose time is latency
#define DIFFOPT_KEPT(B, NV)                                                    \
  if (bytes <= (int64_t)B * NV * 16) {                                         \
    DIFFOPT_LAUNCH((logprob_kept<E_, ENT, TOP, B, NV>), r.N, B, r, o);         \
    return launch_status(who);                                                 \
  }
  const bool wide = TOP && o.K > kFewTop && bytes >= kWideRow;
  if (r.N >= kKeptRows && c.slices == 1 && !wide) {
    DIFFOPT_KEPT(128, 2)
    DIFFOPT_KEPT(128, 4)
    if constexpr (!TOP) {
      DIFFOPT_KEPT(128, 8)
      DIFFOPT_KEPT(256, 8)
      DIFFOPT_KEPT(256, 16)
    }
  }
#undef DIFFOPT_KEPT
  if (bytes <= kShortRow && !wide) DIFFOPT_LAUNCH((logprob_row<E_, ENT, TOP, 128>), r.N * c.slices, 128, r, o, p);
  else if (bytes <= kMiddleRow) DIFFOPT_LAUNCH((logprob_row<E_, ENT, TOP, 256>), r.N * c.slices, 256, r, o, p);
  else DIFFOPT_LAUNCH((logprob_row<E_, ENT, TOP, kLB>), r.N * c.slices, kLB, r, o, p);
  if (c.slices > 1) DIFFOPT_LAUNCH((logprob_join<E_, ENT, TOP>), r.N, kJB, r, o, p);
  return launch_status(who);
}

template <class E_, bool ENT>
int bwd_rows(const char* who, const Rows& r, int32_t dtype, const Cotangents& t, const float* stats, void* dx, int64_t dstride, hipStream_t st) {
  // over the logits in place, a row's workgroups would overwrite one another's named tokens
  const Cut c = dx == r.logits ? Cut{1, r.V} : row_cut(r.N, r.V, dtype, 0);
  DIFFOPT_LAUNCH((logprob_grad<E_, kGiven, ENT>), r.N * c.slices, kLB, r, Results{}, t, stats, static_cast<E_*>(dx), dstride, parts_of(c, 0, nullptr));
  return launch_status(who);
}

template <class E_, bool ENT>
int both_rows(const char* who, const Rows& r, int32_t dtype, const Results& o, const Cotangents& t, void* dlogits, int64_t dstride, void* workspace,
              hipStream_t st) {
  const Cut c = row_cut(r.N, r.V, dtype, 0);
  const Parts p = parts_of(c, 0, workspace);
  E_* dx = static_cast<E_*>(dlogits);
  const float* none = nullptr;
  if (c.slices > 1) {
    DIFFOPT_LAUNCH((logprob_row<E_, ENT, false, kLB>), r.N * c.slices, kLB, r, o, p);
    DIFFOPT_LAUNCH((logprob_grad<E_, kParts, ENT>), r.N * c.slices, kLB, r, o, t, none, dx, dstride, p);
    return launch_status(who);
  }
  const int64_t bytes = r.V * elem_size(dtype);
#define DIFFOPT_KEPT(B, NV)                                                                          \
  if (bytes <= (int64_t)B * NV * 16) {                                                               \
    DIFFOPT_LAUNCH((logprob_grad<E_, kKept, ENT, B, NV>), r.N, B, r, o, t, none, dx, dstride, p);    \
    return launch_status(who);                                                                       \
  }
  DIFFOPT_KEPT(256, 2)
  DIFFOPT_KEPT(256, 4)
  DIFFOPT_KEPT(256, 8)
  DIFFOPT_KEPT(512, 8)
  DIFFOPT_KEPT(512, 13)
  DIFFOPT_KEPT(512, 16)
  DIFFOPT_KEPT(1024, 16)
#undef DIFFOPT_KEPT
  DIFFOPT_LAUNCH((logprob_grad<E_, kRead, ENT>), r.N, kLB, r, o, t, none, dx, dstride, p);
  return launch_status(who);
}

template <class E_, bool ENT>
int second_rows(const char* who, const Rows& r, int32_t dtype, const Cotangents& t, const Second& q, void* workspace, hipStream_t st) {
  const Cut c = row_cut(r.N, r.V, dtype, 0);
  const Parts p = parts_of(c, 0, workspace);
  if (c.slices > 1) {
    DIFFOPT_LAUNCH((logprob_second_parts<E_, ENT>), r.N * c.slices, kLB, r, t, q, p);
    DIFFOPT_LAUNCH((logprob_second<E_, kParts, ENT>), r.N * c.slices, kLB, r, t, q, p);
    return launch_status(who);
  }
  const int64_t bytes = r.V * elem_size(dtype);
#define DIFFOPT_KEPT(B, NV)                                                        \
  if (bytes <= (int64_t)B * NV * 16) {                                             \
    DIFFOPT_LAUNCH((logprob_second<E_, kKept, ENT, B, NV>), r.N, B, r, t, q, p);   \
    return launch_status(who);                                                     \
  }
  DIFFOPT_KEPT(256, 4)
  DIFFOPT_KEPT(512, 4)
  DIFFOPT_KEPT(512, 8)
  DIFFOPT_KEPT(1024, 8)
#undef DIFFOPT_KEPT
  DIFFOPT_LAUNCH((logprob_second<E_, kRead, ENT>), r.N, kLB, r, t, q, p);
  return launch_status(who);
}

}  // namespace
}  // namespace diffopt

using namespace diffopt;

extern "C" int64_t diffopt_logprob_workspace(int64_t N, int64_t V, int32_t dtype, int64_t K) {
  if (N < 0 || N >= kMostRows || V < 1 || V > 0x7fffffff || !dtype_ok(dtype) || K < 0 || K > kMaxTop) return -1;
  return parts_bytes(N, V, dtype, K);
}

extern "C" int diffopt_logprob_fwd(const void* logits, int64_t row_stride, int64_t N, int64_t V, int32_t dtype, const void* ids, int32_t id_bytes,
                                   double temperature, float* logprob, float* entropy, float* stats, float* top_logprob, void* top_ids,
                                   int32_t top_id_bytes, int64_t K, void* workspace, int64_t workspace_bytes, void* stream) {
  clear_error();
  static const char* who = "diffopt_logprob_fwd";
  int rc = check_sizes(who, N, V, dtype, ids, id_bytes, K, top_id_bytes, temperature);
  if (rc || N == 0) return rc;
  Rows r;
  rc = check_rows(who, logits, row_stride, N, V, dtype, ids, id_bytes, temperature, &r);
  if (rc) return rc;
  if (!stats || (ids && !logprob)) return fail(DIFFOPT_EINVAL, "%s: null stats or logprob", who);
  if (!ids && logprob) return fail(DIFFOPT_EINVAL, "%s: logprob without ids", who);
  if (K > 0 && (!top_logprob || !top_ids)) return fail(DIFFOPT_EINVAL, "%s: null top_logprob or top_ids", who);
  if (K > 0 && !aligned_to(top_ids, top_id_bytes)) return fail(DIFFOPT_EINVAL, "%s: a pointer is not aligned to its elements", who);
  rc = check_aligned(who, {logprob, entropy, stats, top_logprob});
  if (!rc) rc = check_workspace(who, r, dtype, K, workspace, workspace_bytes);
  const float* tops = static_cast<const float*>(top_ids);
  if (!rc)
    rc = check_apart(who, {{logprob, N}, {entropy, N}, {stats, 2 * N}, {K ? top_logprob : nullptr, N * K}, {K ? tops : nullptr, N * K * (top_id_bytes / 4)}},
                     {{static_cast<const float*>(ids), N * (id_bytes / 4)}});
  if (rc) return rc;
  const Results o{logprob, entropy, stats, top_logprob, top_ids, top_id_bytes, (int32_t)K};
  const hipStream_t st = as_stream(stream);
  const auto go = [&](auto e, auto ent, auto top) {
    return fwd_rows<decltype(e), decltype(ent)::value, decltype(top)::value>(who, r, dtype, o, workspace, st);
  };
  const auto with = [&](auto e) {
    if (entropy) return K ? go(e, std::true_type{}, std::true_type{}) : go(e, std::true_type{}, std::false_type{});
    return K ? go(e, std::false_type{}, std::true_type{}) : go(e, std::false_type{}, std::false_type{});
  };
  return dtype == DIFFOPT_F32 ? with(0.0f) : with((bf16)0.0f);
}

extern "C" int diffopt_logprob_bwd(const float* dlogprob, const float* dentropy, const float* entropy, const float* dtop_logprob, const void* top_ids,
                                   int32_t top_id_bytes, int64_t K, const void* logits, int64_t row_stride, int64_t N, int64_t V, int32_t dtype,
                                   const void* ids, int32_t id_bytes, double temperature, const float* stats, void* dlogits, int64_t drow_stride,
                                   void* stream) {
  clear_error();
  static const char* who = "diffopt_logprob_bwd";
  int rc = check_sizes(who, N, V, dtype, ids, id_bytes, K, top_id_bytes, temperature);
  if (rc || N == 0) return rc;
  Rows r;
  rc = check_rows(who, logits, row_stride, N, V, dtype, ids, id_bytes, temperature, &r);
  const Cotangents t{dlogprob, dentropy, entropy, dtop_logprob, top_ids, top_id_bytes, (int32_t)K};
  if (!rc) rc = check_cotangents(who, r, t);
  if (!rc && !stats) rc = fail(DIFFOPT_EINVAL, "%s: null stats", who);
  if (!rc) rc = check_aligned(who, {stats});
  if (!rc) rc = check_out_rows(who, dlogits, drow_stride, V, N, dtype);
  if (rc) return rc;
  if (dlogits == logits && N > 1 && drow_stride != row_stride)
    return fail(DIFFOPT_EINVAL, "%s: dlogits in the logits' place must have their row stride", who);
  const hipStream_t st = as_stream(stream);
  if (dtype == DIFFOPT_F32)
    return dentropy ? bwd_rows<float, true>(who, r, dtype, t, stats, dlogits, drow_stride, st)
                    : bwd_rows<float, false>(who, r, dtype, t, stats, dlogits, drow_stride, st);
  return dentropy ? bwd_rows<bf16, true>(who, r, dtype, t, stats, dlogits, drow_stride, st)
                  : bwd_rows<bf16, false>(who, r, dtype, t, stats, dlogits, drow_stride, st);
}

extern "C" int diffopt_logprob_fwd_bwd(const float* dlogprob, const float* dentropy, const void* logits, int64_t row_stride, int64_t N, int64_t V,
                                       int32_t dtype, const void* ids, int32_t id_bytes, double temperature, float* logprob, float* entropy, float* stats,
                                       void* dlogits, int64_t drow_stride, void* workspace, int64_t workspace_bytes, void* stream) {
  clear_error();
  static const char* who = "diffopt_logprob_fwd_bwd";
  int rc = check_sizes(who, N, V, dtype, ids, id_bytes, 0, 0, temperature);
  if (rc || N == 0) return rc;
  Rows r;
  rc = check_rows(who, logits, row_stride, N, V, dtype, ids, id_bytes, temperature, &r);
  if (rc) return rc;
  if (!stats || !ids || !logprob || !dlogprob) return fail(DIFFOPT_EINVAL, "%s: null required pointer", who);
  rc = check_aligned(who, {dlogprob, dentropy, logprob, entropy, stats});
  if (!rc) rc = check_out_rows(who, dlogits, drow_stride, V, N, dtype);
  if (rc) return rc;
  if (dlogits == logits) return fail(DIFFOPT_EINVAL, "%s: dlogits must not be logits", who);
  rc = check_workspace(who, r, dtype, 0, workspace, workspace_bytes);
  if (!rc)
    rc = check_apart(who, {{logprob, N}, {entropy, N}, {stats, 2 * N}},
                     {{dlogprob, N}, {dentropy, N}, {static_cast<const float*>(ids), N * (id_bytes / 4)}});
  if (rc) return rc;
  const Cotangents t{dlogprob, dentropy, entropy, nullptr, nullptr, 0, 0};
  const Results o{logprob, entropy, stats, nullptr, nullptr, 0, 0};
  const hipStream_t st = as_stream(stream);
  if (dtype == DIFFOPT_F32)
    return dentropy || entropy ? both_rows<float, true>(who, r, dtype, o, t, dlogits, drow_stride, workspace, st)
                               : both_rows<float, false>(who, r, dtype, o, t, dlogits, drow_stride, workspace, st);
  return dentropy || entropy ? both_rows<bf16, true>(who, r, dtype, o, t, dlogits, drow_stride, workspace, st)
                             : both_rows<bf16, false>(who, r, dtype, o, t, dlogits, drow_stride, workspace, st);
}

extern "C" int diffopt_logprob_bwd_bwd(const void* ddlogits, int64_t ddrow_stride, const float* dlogprob, const float* dentropy, const float* entropy,
                                       const float* dtop_logprob, const void* top_ids, int32_t top_id_bytes, int64_t K, const void* logits,
                                       int64_t row_stride, int64_t N, int64_t V, int32_t dtype, const void* ids, int32_t id_bytes, double temperature,
                                       const float* stats, float* out_dlogprob, float* out_dentropy, float* out_dtop_logprob, void* out_logits,
                                       int64_t out_row_stride, void* workspace, int64_t workspace_bytes, void* stream) {
  clear_error();
  static const char* who = "diffopt_logprob_bwd_bwd";
  int rc = check_sizes(who, N, V, dtype, ids, id_bytes, K, top_id_bytes, temperature);
  if (rc || N == 0) return rc;
  Rows r;
  rc = check_rows(who, logits, row_stride, N, V, dtype, ids, id_bytes, temperature, &r);
  const Cotangents t{dlogprob, dentropy, entropy, dtop_logprob, top_ids, top_id_bytes, (int32_t)K};
  if (!rc) rc = check_cotangents(who, r, t);
  if (!rc && (!stats || !ddlogits)) rc = fail(DIFFOPT_EINVAL, "%s: null stats or ddlogits", who);
  if (!rc) rc = check_aligned(who, {stats, out_dlogprob, out_dentropy, out_dtop_logprob});
  if (!rc && !aligned_to(ddlogits, elem_size(dtype))) rc = fail(DIFFOPT_EINVAL, "%s: a pointer is not aligned to its elements", who);
  if (!rc) rc = check_out_rows(who, out_logits, out_row_stride, V, N, dtype);
  if (rc) return rc;
  if (out_logits == logits || out_logits == ddlogits) return fail(DIFFOPT_EINVAL, "%s: out_logits must be neither logits nor ddlogits", who);
  rc = check_workspace(who, r, dtype, 0, workspace, workspace_bytes);
  const int64_t NK = N * K;
  if (!rc)
    rc = check_apart(who, {{out_dlogprob, N}, {out_dentropy, N}, {K ? out_dtop_logprob : nullptr, NK}},
                     {{dlogprob, N}, {dentropy, N}, {entropy, N}, {K ? dtop_logprob : nullptr, NK}, {stats, 2 * N},
                      {static_cast<const float*>(ids), ids ? N * (id_bytes / 4) : 0},
                      {K ? static_cast<const float*>(top_ids) : nullptr, K ? NK * (top_id_bytes / 4) : 0}});
  if (rc) return rc;
  if (out_dlogprob && !ids) return fail(DIFFOPT_EINVAL, "%s: out_dlogprob without ids", who);
  if (out_dentropy && !entropy) return fail(DIFFOPT_EINVAL, "%s: out_dentropy without entropy", who);
  const Second q{ddlogits, ddrow_stride, stats, out_dlogprob, out_dentropy, K ? out_dtop_logprob : nullptr, out_logits, out_row_stride};
  const hipStream_t st = as_stream(stream);
  if (dtype == DIFFOPT_F32)
    return entropy ? second_rows<float, true>(who, r, dtype, t, q, workspace, st) : second_rows<float, false>(who, r, dtype, t, q, workspace, st);
  return entropy ? second_rows<bf16, true>(who, r, dtype, t, q, workspace, st) : second_rows<bf16, false>(who, r, dtype, t, q, workspace, st);
}
