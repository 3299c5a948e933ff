// Rows of logits, for the operators that take them (distill, logprob): a row's
// maximum and sum of exponentials, by one pass with a running maximum or from
// registers; how rows are cut into slices; the rows' checks.
#pragma once

#include <initializer_list>

#include "lm_common.hpp"

namespace diffopt {

constexpr int64_t kMostRows = int64_t(1) << 22;  // a launch has fewer than 2^32 threads, a workgroup of up to 1024 for each row
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// (x - m) / T in units of log 2; a row of -inf alone keeps m = -inf, s = 0.
__device__ __forceinline__ float safe_max(float m) { return m == -kInf ? 0.0f : m; }

// exp((x - b) / T) for many x and one b: 2^(x c - b c) by one multiply-add, with
// what the rounding of b c leaves out as a factor of its own.  That factor and what
// it corrects are 2^-+r with |r| up to half a last place of b c: harmless while |b c|
// stays below 2^24 (|r| <= 1/2), infinite times zero from about 2^31 on.  `wide` takes
// the difference first; the factor goes with the form that a wave has taken.
struct Shift {
  float b, c, bc;
  bool wide;
  __device__ __forceinline__ Shift(float b_, float c_) : b(b_), c(c_), bc(b_ * c_), wide(!(__builtin_fabsf(bc) < 0x1p24f)) {}
  template <bool WIDE>
  __device__ __forceinline__ float factor() const {
    return WIDE ? 1.0f : exp2_fast(-__builtin_fmaf(b, c, -bc));
  }
  template <bool WIDE>
  __device__ __forceinline__ float part(float x) const {
    return exp2_fast(WIDE ? (x - b) * c : __builtin_fmaf(x, c, -bc));
  }
};

__device__ __forceinline__ void join(float& m, float& s, float m2, float s2, float c) {
  const float M = fmaxf(m, m2), b = safe_max(M);
  s = s * exp2_fast((m - b) * c) + s2 * exp2_fast((m2 - b) * c);
  m = M;
}

// Elements before the first 16-byte boundary of x, at most n.
template <class E_>
__device__ __forceinline__ int64_t head_of(const E_* x, int64_t n) {
  const int64_t off = (int64_t)((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / (int)sizeof(E_);
  return off < n ? off : n;
}

// f(first element) over the aligned 16-byte pieces of elements [c0, c1) of a
// row, g(element) over the elements before and after them.
template <class E_, class F, class G>
__device__ __forceinline__ void over_row(const E_* x, int64_t c0, int64_t c1, F f, G g) {
  constexpr int NV = Vec<E_>::N;
  const int64_t n = c1 - c0, head = head_of(x + c0, n), nv = (n - head) / NV;
  for (int64_t i = threadIdx.x; i < nv; i += blockDim.x) f(c0 + head + i * NV);
  const int64_t rest = n - nv * NV;  // head and tail elements
  if ((int64_t)threadIdx.x < rest) g(c0 + ((int64_t)threadIdx.x < head ? (int64_t)threadIdx.x : threadIdx.x + nv * NV));
}

constexpr int kMaxWaves = 16;
struct Reduce {
  float m[kMaxWaves], s[kMaxWaves];
};

// One lane's running max and sum.
struct Running {
  float m = -kInf, s = 0.0f;
  template <int N>
  __device__ __forceinline__ void piece(const float* e, float c) {
    float vm = e[0];
#pragma unroll
    for (int i = 1; i < N; ++i) vm = fmaxf(vm, e[i]);
    if (vm > m) {
      s *= exp2_fast((m - vm) * c);
      m = vm;
    }
    const float b = safe_max(m);
#pragma unroll
    for (int i = 0; i < N; ++i) s += exp2_fast((e[i] - b) * c);
  }
  __device__ __forceinline__ void one(float e, float c) { join(m, s, e, e == -kInf ? 0.0f : (e - e == 0.0f ? 1.0f : kNan), c); }
  // over the workgroup
  __device__ __forceinline__ void all(Reduce& R, float c) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const float m2 = __shfl_xor(m, o, 64), s2 = __shfl_xor(s, o, 64);
      join(m, s, m2, s2, c);
    }
    const int wave = threadIdx.x >> 6, nw = blockDim.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
      R.m[wave] = m;
      R.s[wave] = s;
    }
    __syncthreads();
    m = R.m[0];
    s = R.s[0];
    for (int w = 1; w < nw; ++w) join(m, s, R.m[w], R.s[w], c);
  }
};

template <class E_>
__device__ __forceinline__ void row_stats(const E_* x, int64_t c0, int64_t c1, float c, Running& run) {
  over_row(
      x, c0, c1,
      [&](int64_t at) {
        const auto v = load_vec(x + at);
        float e[Vec<E_>::N];
#pragma unroll
        for (int i = 0; i < Vec<E_>::N; ++i) e[i] = (float)v[i];
        run.template piece<Vec<E_>::N>(e, c);
      },
      [&](int64_t at) { run.one((float)x[at], c); });
}

// A row in registers: NV pieces of every lane of a workgroup of B, and one of
// the elements around them.  Where the pieces lie goes by one array's alignment,
// another array's are taken at the same elements.  Offsets are 32 bits from the
// row, which a wave's registers hold once.
template <class E_, int B, int NV>
struct Kept {
  static constexpr int N = Vec<E_>::N;
  uint32_t v[NV][4];  // the pieces as memory holds them
  E_ single;
  uint32_t first, nv, at_single;
  bool has_single;

  __device__ __forceinline__ void place(const E_* x, uint32_t n) {
    const uint32_t head = (uint32_t)head_of(x, n), rest = n - (n - head) / N * N;
    nv = (n - head) / N;
    first = head + threadIdx.x * N;
    has_single = threadIdx.x < rest;
    at_single = threadIdx.x < head ? threadIdx.x : threadIdx.x + nv * N;
  }
  __device__ __forceinline__ bool has(int i) const { return threadIdx.x + i * B < nv; }
  __device__ __forceinline__ uint32_t at(int i) const { return first + i * (B * N); }
  // pieces that are not there hold `none`
  __device__ __forceinline__ void load(const E_* x, E_ none) {
    typename Vec<E_>::type fill;
#pragma unroll
    for (int k = 0; k < N; ++k) fill[k] = none;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      typename Vec<E_>::type y = fill;
      if (has(i)) y = load_vec(x + at(i));
      __builtin_memcpy(v[i], &y, 16);
    }
    single = none;
    if (has_single) single = x[at_single];
  }
  // A piece's values.  The compiler would keep what one pass unpacked for the
  // next, twice the registers of the row itself: it is made to unpack anew.
  __device__ __forceinline__ void get(int i, float* e) const {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      uint32_t x = v[i][k];
      asm volatile("" : "+v"(x));
      if constexpr (sizeof(E_) == 2) {
        e[2 * k] = __builtin_bit_cast(float, x << 16);
        e[2 * k + 1] = __builtin_bit_cast(float, x & 0xffff0000u);
      } else {
        e[k] = __builtin_bit_cast(float, x);
      }
    }
  }
};

// The sum over the workgroup, the same in every lane.
__device__ __forceinline__ float block_sum(float x, Reduce& R) {
  x = wave_sum(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) R.s[threadIdx.x >> 6] = x;
  __syncthreads();
  x = 0.0f;
  for (int w = 0; w < (int)(blockDim.x >> 6); ++w) x += R.s[w];
  return x;
}

// Waves of a SIMD that the compiler has to leave room for where rows stay in
// registers: rows of 104 KiB at three workgroups a compute unit (80 registers, 52
// of them the row's) took 175 us for 4096 rows of 50,021 bf16 logits, at two 186,
// at four (with spills) 199.  Elsewhere its own choice stands: made to leave room for
// more, rows of 64 KiB (4,096 of 32,001 bf16 logits) take 115 us instead of 118, those of
// up to 32 KiB the same within 1%, of 125 KiB 71 instead of 62 (1,024 of 32,000 fp32
// logits) and of 254 KiB 223 instead of 125 (spills).
constexpr int kept_waves(int B, int NV) { return B == 512 && NV == 13 ? 6 : 1; }

// ---- host -------------------------------------------------------------------

inline int check_aligned(const char* who, std::initializer_list<const void*> floats) {
  for (const void* p : floats)
    if (!aligned_to(p, 4)) return fail(DIFFOPT_EINVAL, "%s: pointer %p is not 4-byte aligned", who, p);
  return DIFFOPT_OK;
}

inline int check_out_rows(const char* who, const void* out, int64_t stride, int64_t V, int64_t N, int32_t dtype) {
  if (!out) return fail(DIFFOPT_EINVAL, "%s: null required pointer", who);
  if (!aligned_to(out, elem_size(dtype))) return fail(DIFFOPT_EINVAL, "%s: a pointer is not aligned to its elements", who);
  if (N > 1 && stride < V && stride > -V) return fail(DIFFOPT_EINVAL, "%s: rows of the result overlap", who);
  return DIFFOPT_OK;
}

// fp32 arrays of a call: a result of a row is written while other waves, or the
// row's other workgroups, still read its operands.
struct Floats {
  const float* p;
  int64_t n;
};

inline int check_apart(const char* who, std::initializer_list<Floats> results, std::initializer_list<Floats> operands) {
  for (auto r = results.begin(); r != results.end(); ++r) {
    for (const Floats& o : operands)
      if (overlap(r->p, r->n * 4, o.p, o.n * 4)) return fail(DIFFOPT_EINVAL, "%s: a result must not be an operand", who);
    for (auto t = results.begin(); t != r; ++t)
      if (overlap(r->p, r->n * 4, t->p, t->n * 4)) return fail(DIFFOPT_EINVAL, "%s: two results must not be one array", who);
  }
  return DIFFOPT_OK;
}

// Workgroups of a row: with fewer rows than kFewRows long ones are cut into slices
// of at least kSliceBytes until kFillRows workgroups run.  fp32, the loss alone, cut
// and whole: 8 rows of 512 KiB 8.4 and 15.4 us, 200 of them 23.6 and 28.7, 512 of
// them 47.1 and 42.6.  Rows that a workgroup keeps in registers (up to 256 KiB) are
// cut where there are fewer than kVeryFewRows (8 of 256 KiB 7.6 and 10.0, with the
// gradient 10.7 and 13.0; 64 of them 10.4 and 10.2, with the gradient 18.3 and 15.5)
// and longer than kShortBytes (8 of 125 KiB 7.6 and 7.3, with the gradient 10.8 and
// 9.4).
constexpr int64_t kFewRows = 256, kFillRows = 1024, kSliceBytes = 8192;
constexpr int64_t kVeryFewRows = 32, kShortBytes = 128 * 1024, kLongBytes = 256 * 1024;

struct Cut {
  int32_t slices;
  int64_t per;
};

inline Cut cut_of(int64_t N, int64_t V, int32_t dtype, int64_t slice_bytes = kSliceBytes) {
  if (N >= kFewRows || N == 0 || V * elem_size(dtype) <= (N < kVeryFewRows ? kShortBytes : kLongBytes)) return Cut{1, V};
  int64_t n = kFillRows / N;
  const int64_t most = V * elem_size(dtype) / slice_bytes;
  n = n > most ? most : n;
  if (n < 2) return Cut{1, V};
  int64_t per = (V + n - 1) / n;
  per = (per + 63) / 64 * 64;
  return Cut{(int32_t)((V + per - 1) / per), per};
}

}  // namespace diffopt
