// Distillation from a teacher's top logits on gfx950: the loss, its gradient,
// and the gradient's own vector-Jacobian product (formulas in diffopt.h).
//
// One workgroup per row, or per slice of one where there are few rows.  The
// row's max m and sum s = sum exp((x - m)/T) come from one pass with a running
// max (a lane rescales its sum once per 16 bytes); wave 0 forms the teacher's
// softmax over the K entries meanwhile.  The gradient's dense part g T p takes
// the row again: where the same call has just read it, from registers (rows of
// up to 256 KiB), else from memory.  The K entries are then written once more
// by the same workgroup after a barrier, each with the sum of q over the entries
// of its token, so nothing is added atomically and equal ids need no order.
// A few exponentials per element: bound by memory.
#include <type_traits>

#include "lm_rows.hpp"

namespace diffopt {
namespace {

constexpr int kDB = 512;       // threads per workgroup
constexpr int kMaxK = 1024;    // entries of a row
struct Rows {
  const void* logits;
  int64_t row_stride, N, V;
  const void* ids;
  int32_t id_bytes;
  const float* teacher;
  int32_t K;
  float T, invT;
};

// What the entries of one row need to stay in LDS.
struct Entries {
  int64_t id[kMaxK];
  float q[kMaxK];
  float lq[kMaxK];  // T log q, then T l = T (log q - log p)
  float x[kMaxK];   // the token's logit
  int some;         // the row has an entry
  int bad;          // one of its ids is >= V
};

__device__ __forceinline__ int64_t id_at(const Rows& r, int64_t at) {
  return r.id_bytes == 4 ? (int64_t) static_cast<const int32_t*>(r.ids)[at] : static_cast<const int64_t*>(r.ids)[at];
}

// The teacher's softmax over one row's entries, by one wave.
__device__ void teacher_softmax(const Rows& r, int64_t row, Entries& E, int lane) {
  float top = -kInf;
  bool some = false, bad = false;
  for (int j = lane; j < r.K; j += 64) {
    int64_t id = id_at(r, row * r.K + j);
    const float t = r.teacher[row * r.K + j];
    if (id < 0 || t == -kInf) id = -1;
    bad |= id >= r.V;
    if (id >= r.V) id = -1;
    else if (id >= 0) {
      some = true;
      top = fmaxf(top, t);
    }
    E.id[j] = id;
    E.lq[j] = t;
  }
  top = safe_max(wave_max(top));
  some = __any(some);
  bad = __any(bad);
  float sum = 0.0f;
  for (int j = lane; j < r.K; j += 64)
    if (E.id[j] >= 0) sum += exp2_fast((E.lq[j] - top) * (r.invT * kLog2e));
  sum = wave_sum(sum);
  const float lsum = r.T * logf(sum), inv = 1.0f / sum;
  for (int j = lane; j < r.K; j += 64) {
    const float d = E.lq[j] - top;
    const bool in = E.id[j] >= 0;
    E.q[j] = in ? exp2_fast(d * (r.invT * kLog2e)) * inv : 0.0f;
    E.lq[j] = in ? d - lsum : 0.0f;
  }
  if (lane == 0) {
    E.some = some || bad;
    E.bad = bad;
  }
}

// The logits (or another array's values) at the entries' tokens, by one wave.
template <class E_>
__device__ __forceinline__ void gather(const E_* x, const Entries& E, int K, float* to, int lane) {
  for (int j = lane; j < K; j += 64) to[j] = E.id[j] >= 0 ? (float)x[E.id[j]] : 0.0f;
}

// T l_j = T (log q_j - log p[ids_j]) in place of T log q; its mean under q.  In
// units of the logits: (x - m) / T alone may overflow where the loss does not.
__device__ float entry_terms(const Rows& r, Entries& E, float m, float s, int lane) {
  const float ls = r.T * logf(s);
  float mean = 0.0f;
  for (int j = lane; j < r.K; j += 64) {
    float l = 0.0f;
    if (E.id[j] >= 0 && E.q[j] != 0.0f) {  // 0 log 0 = 0
      l = E.lq[j] - ((E.x[j] - m) - ls);
      mean += E.q[j] * l;
    }
    E.lq[j] = l;
  }
  return wave_sum(mean);
}

// What a workgroup takes of a launch of `slices` per row.
struct Slice {
  int64_t row, c0, c1;
  int32_t index;
};

__device__ __forceinline__ Slice slice_of(const Rows& r, int64_t block, int32_t slices, int64_t per) {
  Slice s;
  s.row = block / slices;
  s.index = (int32_t)(block - s.row * slices);
  s.c0 = s.index * per;
  s.c1 = s.c0 + per < r.V ? s.c0 + per : r.V;
  return s;
}

// A slice's max and sum, for rows that several workgroups share.  One read of the
// row, bound by latency for few of them (8 rows of 512 KiB: 4.5 us).
template <class E_>
__global__ __launch_bounds__(kDB) void distill_parts(Rows r, float* parts, int32_t slices, int64_t per) {
  __shared__ Reduce R;
  const Slice sl = slice_of(r, blockIdx.x, slices, per);
  const float c = r.invT * kLog2e;
  Running run;
  row_stats(static_cast<const E_*>(r.logits) + sl.row * r.row_stride, sl.c0, sl.c1, c, run);
  run.all(R, c);
  if (threadIdx.x == 0) {
    parts[2 * (int64_t)blockIdx.x] = run.m;
    parts[2 * (int64_t)blockIdx.x + 1] = run.s;
  }
}

// The row's max and sum from its slices'.
__device__ __forceinline__ void join_parts(const float* parts, int64_t row, int32_t slices, float c, Running& run, Reduce& R) {
  for (int i = threadIdx.x; i < slices; i += blockDim.x) join(run.m, run.s, parts[2 * (row * slices + i)], parts[2 * (row * slices + i) + 1], c);
  run.all(R, c);
}

// The sum of q over the entries that name the token of entry j.
__device__ __forceinline__ float same_token(const float* w, const Entries& E, int K, int64_t id) {
  float sum = 0.0f;
  for (int i = 0; i < K; ++i) sum += E.id[i] == id ? w[i] : 0.0f;
  return sum;
}

// Where a row's max and sum come from.
enum Stats {
  kGiven,  // the caller
  kRead,   // this workgroup's pass over the row
  kKept,   // the same, the row staying in registers
  kParts   // slices of the row
};

// A row (or a slice of one): the loss, with BWD its gradients.  Bound by memory, each
// logit read once and each gradient written once: 4,096 rows of 50,021 bf16 logits,
// 820 MB, take 174 us (4.7 TB/s; a copy of that size reaches 4.9 to 5.3), 1,024 rows
// of 32,000 fp32 ones 54 us (4.9 TB/s).  With the exponentials kept in fp32 rather
// than the packed logits half as many rows are in flight and it takes 192 us.
template <class E_, int STATS, bool BWD, int B = kDB, int NV = 1>
__global__ __launch_bounds__(B, (STATS == kKept ? kept_waves(B, NV) : 1)) void distill_row(
    Rows r, const float* dloss, float* loss, float* stats, E_* dlogits, int64_t drow_stride, float* dteacher, const float* parts,
    int32_t slices, int64_t per) {
  constexpr bool FWD = STATS != kGiven;
  __shared__ Entries E;
  __shared__ Reduce R;
  const int lane = threadIdx.x & 63;
  const float c = r.invT * kLog2e;
  const Slice sl = slice_of(r, blockIdx.x, BWD ? slices : 1, BWD ? per : r.V);
  const int64_t row = sl.row;
  const E_* x = static_cast<const E_*>(r.logits) + row * r.row_stride;
  Kept<E_, B, NV> kept;
  if (STATS == kKept) {
    kept.place(x, (uint32_t)r.V);
    kept.load(x, (E_)-kInf);
  }
  if (threadIdx.x < 64) {
    teacher_softmax(r, row, E, lane);
    gather(x, E, r.K, E.x, lane);  // before dlogits, which may be logits, is written
  }
  Running run;
  if (STATS == kRead) row_stats(x, 0, r.V, c, run);
  if (STATS == kKept) {
    constexpr int N = Vec<E_>::N;
    float top = (float)kept.single;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float e[N];
      kept.get(i, e);
#pragma unroll
      for (int k = 0; k < N; k += 2) top = fmaxf(fmaxf(top, e[k]), e[k + 1]);
    }
    run.m = top;
    const Shift sh(safe_max(top), c);
    auto sum = [&](auto wide) {
      run.s = sh.part<wide.value>((float)kept.single);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        float e[N];
        kept.get(i, e);
#pragma unroll
        for (int k = 0; k < N; ++k) run.s += sh.part<wide.value>(e[k]);
      }
      run.s *= sh.factor<wide.value>();
    };
    if (__any(sh.wide))
      sum(std::true_type{});
    else
      sum(std::false_type{});
  }
  if (STATS == kRead || STATS == kKept) run.all(R, c);
  if (STATS == kParts) join_parts(parts, row, slices, c, run, R);
  if (STATS == kGiven) {
    run.m = stats[2 * row];
    run.s = stats[2 * row + 1];
  } else if (threadIdx.x == 0 && sl.index == 0) {
    stats[2 * row] = run.m;
    stats[2 * row + 1] = run.s;
  }
  const float m = run.m, s = run.s;
  __syncthreads();
  const bool some = E.some, bad = E.bad;
  const float g = BWD ? (bad ? kNan : dloss[row]) : 0.0f, gT = g * r.T;
  if (threadIdx.x < 64 && sl.index == 0 && (FWD || dteacher)) {
    const float mean = entry_terms(r, E, m, s, lane);
    if (FWD && lane == 0) loss[row] = bad ? kNan : some ? r.T * mean : 0.0f;
    if (BWD && dteacher)
      for (int j = lane; j < r.K; j += 64)
        dteacher[row * r.K + j] = E.q[j] != 0.0f ? g * E.q[j] * (E.lq[j] - mean) : bad ? kNan : 0.0f;
  }
  if (!BWD) return;
  E_* dx = dlogits + row * drow_stride;
  const float w = some ? gT / s : 0.0f;
  auto piece = [&](int64_t at, const float* e) {
    float y[Vec<E_>::N];
#pragma unroll
    for (int i = 0; i < Vec<E_>::N; ++i) y[i] = some ? w * exp2_fast((e[i] - m) * c) : 0.0f;
    store_vec(dx + at, y);
  };
  auto one = [&](int64_t at, float e) { dx[at] = (E_)(some ? w * exp2_fast((e - m) * c) : 0.0f); };
  if (STATS == kKept) {
    const Shift sh(m, c);
    auto write = [&](auto value) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (kept.has(i)) {
          float e[Vec<E_>::N];
          kept.get(i, e);
#pragma unroll
          for (int k = 0; k < Vec<E_>::N; ++k) e[k] = value(e[k]);
          store_vec(dx + kept.at(i), e);
        }
      if (kept.has_single) dx[kept.at_single] = (E_)value((float)kept.single);
    };
    if (!some)
      write([](float) { return 0.0f; });
    else if (sh.wide)
      write([&](float e) { return w * sh.part<true>(e); });
    else
      write([&, f = w * sh.factor<false>()](float e) { return f * sh.part<false>(e); });
  } else {
    over_row(
        x, sl.c0, sl.c1,
        [&](int64_t at) {
          float e[Vec<E_>::N];
          load_floats(x + at, e);
          piece(at, e);
        },
        [&](int64_t at) { one(at, (float)x[at]); });
  }
  __syncthreads();  // the entries' elements are written after the dense part's
  for (int j = threadIdx.x; j < r.K; j += blockDim.x)
    if (E.id[j] >= sl.c0 && E.id[j] < sl.c1)
      dx[E.id[j]] = (E_)(w * exp2_fast((E.x[j] - m) * c) - gT * same_token(E.q, E, r.K, E.id[j]));
}

// ---- the gradient's vector-Jacobian product ---------------------------------

struct Second {
  const void* a;  // cotangent of dlogits or NULL
  int64_t a_stride;
  const float *c, *dloss, *stats;
  float *out_dloss, *out_teacher;
  void* out;
  int64_t out_stride;
};

// A lane's sum of p a (times s), over elements [c0, c1).
template <class E_>
__device__ __forceinline__ float weighted(const E_* x, const E_* a, int64_t c0, int64_t c1, float m, float c) {
  float pa = 0.0f;
  over_row(
      x, c0, c1,
      [&](int64_t at) {
        const auto v = load_vec(x + at);
        const auto u = load_vec(a + at);
#pragma unroll
        for (int i = 0; i < Vec<E_>::N; ++i) pa += exp2_fast(((float)v[i] - m) * c) * (float)u[i];
      },
      [&](int64_t at) { pa += exp2_fast(((float)x[at] - m) * c) * (float)a[at]; });
  return pa;
}

// A slice's sum of p a, for rows that several workgroups share.
template <class E_>
__global__ __launch_bounds__(kDB) void distill_second_parts(Rows r, Second t, float* parts, int32_t slices, int64_t per) {
  __shared__ Reduce R;
  const Slice sl = slice_of(r, blockIdx.x, slices, per);
  const float pa = block_sum(weighted(static_cast<const E_*>(r.logits) + sl.row * r.row_stride, static_cast<const E_*>(t.a) + sl.row * t.a_stride,
                                      sl.c0, sl.c1, t.stats[2 * sl.row], r.invT * kLog2e), R);
  if (threadIdx.x == 0) parts[blockIdx.x] = pa;
}

// The gradient's own vector-Jacobian product for a row (or a slice of one): logits
// and a read once, a result written.  Bound by memory: 1,024 rows of 32,000 fp32
// logits, 393 MB, take 86 us (4.6 TB/s).
template <class E_, int STATS, int B = kDB, int NV = 1>
__global__ __launch_bounds__(B) void distill_second(Rows r, Second t, const float* parts, int32_t slices, int64_t per) {
  __shared__ Entries E;
  __shared__ float aj[kMaxK], cj[kMaxK];
  __shared__ Reduce R;
  const int lane = threadIdx.x & 63;
  const float c = r.invT * kLog2e;
  const Slice sl = slice_of(r, blockIdx.x, slices, per);
  const int64_t row = sl.row;
  const E_* x = static_cast<const E_*>(r.logits) + row * r.row_stride;
  const E_* a = t.a ? static_cast<const E_*>(t.a) + row * t.a_stride : nullptr;
  E_* y = static_cast<E_*>(t.out) + row * t.out_stride;
  Kept<E_, B, NV> kx, ka;
  if (STATS == kKept && a) {
    kx.place(x, (uint32_t)r.V);
    ka.place(x, (uint32_t)r.V);
    kx.load(x, (E_)-kInf);
    ka.load(a, (E_)0.0f);
  }
  const float m = t.stats[2 * row], s = t.stats[2 * row + 1], inv = 1.0f / s;
  if (threadIdx.x < 64) {
    teacher_softmax(r, row, E, lane);
    gather(x, E, r.K, E.x, lane);
    for (int j = lane; j < r.K; j += 64) {
      aj[j] = a && E.id[j] >= 0 ? (float)a[E.id[j]] : 0.0f;
      cj[j] = t.c && E.q[j] != 0.0f ? t.c[row * r.K + j] : 0.0f;
    }
  }
  float pa = 0.0f;
  const Shift sh(m, c);
  if (STATS == kKept && a) {
    auto sum = [&](auto wide) {
      pa = sh.part<wide.value>((float)kx.single) * (float)ka.single;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        float e[Vec<E_>::N], u[Vec<E_>::N];
        kx.get(i, e);
        ka.get(i, u);
#pragma unroll
        for (int k = 0; k < Vec<E_>::N; ++k) pa += sh.part<wide.value>(e[k]) * u[k];
      }
      pa *= sh.factor<wide.value>();
    };
    if (sh.wide)
      sum(std::true_type{});
    else
      sum(std::false_type{});
  } else if (STATS == kRead && a) {
    pa = weighted(x, a, 0, r.V, m, c);
  } else if (STATS == kParts && a) {
    for (int i = threadIdx.x; i < slices; i += blockDim.x) pa += parts[row * slices + i];
  }
  pa = block_sum(pa, R) * inv;
  const bool some = E.some, bad = E.bad;
  const float g = bad ? kNan : t.dloss[row];
  if (threadIdx.x < 64) {
    const float mean = entry_terms(r, E, m, s, lane);
    float abar = 0.0f, cbar = 0.0f, cov = 0.0f;  // means of a and c, covariance of c and T l under q
    for (int j = lane; j < r.K; j += 64) {
      const float q = E.q[j];
      if (q == 0.0f) continue;
      abar += q * aj[j];
      cbar += q * cj[j];
    }
    abar = wave_sum(abar);
    cbar = wave_sum(cbar);
    for (int j = lane; j < r.K; j += 64) cov += E.q[j] * (cj[j] - cbar) * (E.lq[j] - mean);
    cov = wave_sum(cov);
    if (t.out_dloss && sl.index == 0 && lane == 0) t.out_dloss[row] = bad ? kNan : some ? r.T * (pa - abar) + cov : 0.0f;
    for (int j = lane; j < r.K; j += 64) {
      const float q = E.q[j], cc = cj[j], l = E.lq[j];
      if (t.out_teacher && sl.index == 0)
        t.out_teacher[row * r.K + j] =
            q != 0.0f ? g * q * ((abar - aj[j]) + (cc - cbar) + r.invT * ((cc - cbar) * (l - mean) - cov)) : bad ? kNan : 0.0f;
      E.q[j] = q * (cc - cbar);  // what the entry takes from its token's element
    }
  }
  const float w = some ? g * inv : 0.0f;
  const bool dense = a && some;
  const float rest = bad ? kNan : 0.0f;  // where no cotangent of dlogits is given
  auto piece = [&](int64_t at, const float* e, const float* u) {
    float z[Vec<E_>::N];
#pragma unroll
    for (int i = 0; i < Vec<E_>::N; ++i) z[i] = dense ? w * exp2_fast((e[i] - m) * c) * (u[i] - pa) : rest;
    store_vec(y + at, z);
  };
  auto one = [&](int64_t at, float v, float u) { y[at] = (E_)(dense ? w * exp2_fast((v - m) * c) * (u - pa) : rest); };
  if (STATS == kKept && a) {
    auto write = [&](auto value) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (kx.has(i)) {
          float e[Vec<E_>::N], u[Vec<E_>::N];
          kx.get(i, e);
          ka.get(i, u);
#pragma unroll
          for (int k = 0; k < Vec<E_>::N; ++k) e[k] = value(e[k], u[k]);
          store_vec(y + kx.at(i), e);
        }
      if (kx.has_single) y[kx.at_single] = (E_)value((float)kx.single, (float)ka.single);
    };
    if (!some)
      write([](float, float) { return 0.0f; });
    else if (sh.wide)
      write([&](float e, float u) { return w * sh.part<true>(e) * (u - pa); });
    else
      write([&, f = w * sh.factor<false>()](float e, float u) { return f * sh.part<false>(e) * (u - pa); });
  } else {
    const E_* b = a ? a : x;
    over_row(
        x, sl.c0, sl.c1,
        [&](int64_t at) {
          float e[Vec<E_>::N], u[Vec<E_>::N];
          load_floats(x + at, e);
          load_floats(b + at, u);
          piece(at, e, u);
        },
        [&](int64_t at) { one(at, (float)x[at], (float)b[at]); });
  }
  __syncthreads();
  for (int j = threadIdx.x; j < r.K; j += blockDim.x)
    if (E.id[j] >= sl.c0 && E.id[j] < sl.c1) {
      const float d = a ? w * exp2_fast((E.x[j] - m) * c) * (aj[j] - pa) : 0.0f;
      y[E.id[j]] = (E_)(d - g * same_token(E.q, E, r.K, E.id[j]));
    }
}

// ---- host -------------------------------------------------------------------

int check_rows(const char* who, const void* logits, int64_t row_stride, int64_t N, int64_t V, int32_t dtype,
               const void* ids, int32_t id_bytes, const float* teacher, int64_t K, double temperature, Rows* r) {
  if (N < 0) return fail(DIFFOPT_EINVAL, "%s: N must be >= 0", who);
  if (N >= kMostRows) return fail(DIFFOPT_EINVAL, "%s: N must be below 2^22", who);
  if (V < 1 || V > 0x7fffffff) return fail(DIFFOPT_EINVAL, "%s: V must be in [1, 2^31)", who);
  if (!dtype_ok(dtype)) return fail(DIFFOPT_EINVAL, "%s: unknown element type %d", who, (int)dtype);
  if (id_bytes != 4 && id_bytes != 8) return fail(DIFFOPT_EINVAL, "%s: id_bytes must be 4 or 8", who);
  if (K < 1 || K > kMaxK) return fail(DIFFOPT_EINVAL, "%s: K must be in [1, %d]", who, kMaxK);
  if (!(std::isfinite(temperature) && temperature > 0.0 && std::isfinite((float)(1.0 / temperature) * kLog2e) && (float)temperature > 0.0f &&
        std::isfinite((float)temperature)))
    return fail(DIFFOPT_EINVAL, "%s: temperature and log2(e) / temperature must be finite and > 0 in fp32", who);
  if (N == 0) return DIFFOPT_OK;
  if (!logits || !ids || !teacher) return fail(DIFFOPT_EINVAL, "%s: null required pointer", who);
  if (!aligned_to(logits, elem_size(dtype)) || !aligned_to(ids, id_bytes) || !aligned_to(teacher, 4))
    return fail(DIFFOPT_EINVAL, "%s: a pointer is not aligned to its elements", who);
  *r = Rows{logits, row_stride, N, V, ids, id_bytes, teacher, (int32_t)K, (float)temperature, (float)(1.0 / temperature)};
  return DIFFOPT_OK;
}

#define DIFFOPT_LAUNCH(kernel, grid, block, ...) hipLaunchKernelGGL((kernel), dim3((unsigned)(grid)), dim3(block), 0, st, __VA_ARGS__)

template <class E_>
int fwd_rows(const char* who, const Rows& r, int32_t dtype, float* loss, float* stats, float* parts, hipStream_t st) {
  const Cut c = cut_of(r.N, r.V, dtype);
  E_* none = nullptr;
  if (c.slices > 1) {
    DIFFOPT_LAUNCH(distill_parts<E_>, r.N * c.slices, kDB, r, parts, c.slices, c.per);
    DIFFOPT_LAUNCH((distill_row<E_, kParts, false, 64>), r.N, 64, r, nullptr, loss, stats, none, 0, nullptr, parts, c.slices, c.per);
  } else {
    DIFFOPT_LAUNCH((distill_row<E_, kRead, false>), r.N, kDB, r, nullptr, loss, stats, none, 0, nullptr, nullptr, 1, r.V);
  }
  return launch_status(who);
}

template <class E_>
int bwd_rows(const char* who, const Rows& r, int32_t dtype, const float* dloss, const float* stats, void* dx, int64_t dstride, float* dt,
             hipStream_t st) {
  // over the logits in place, a row's workgroups would overwrite one another's entries
  const Cut c = dx == r.logits ? Cut{1, r.V} : cut_of(r.N, r.V, dtype);
  DIFFOPT_LAUNCH((distill_row<E_, kGiven, true>), r.N * c.slices, kDB, r, dloss, nullptr, const_cast<float*>(stats), static_cast<E_*>(dx), dstride,
                 dt, nullptr, c.slices, c.per);
  return launch_status(who);
}

template <class E_>
int both_rows(const char* who, const Rows& r, int32_t dtype, const float* dloss, float* loss, float* stats, void* dlogits, int64_t dstride,
              float* dt, float* parts, hipStream_t st) {
  const Cut c = cut_of(r.N, r.V, dtype);
  E_* dx = static_cast<E_*>(dlogits);
  if (c.slices > 1) {
    DIFFOPT_LAUNCH(distill_parts<E_>, r.N * c.slices, kDB, r, parts, c.slices, c.per);
    DIFFOPT_LAUNCH((distill_row<E_, kParts, true>), r.N * c.slices, kDB, r, dloss, loss, stats, dx, dstride, dt, parts, c.slices, c.per);
    return launch_status(who);
  }
  const int64_t bytes = r.V * elem_size(dtype);
#define DIFFOPT_KEPT(B, NV)                                                                                                       \
  if (bytes <= (int64_t)B * NV * 16) {                                                                                            \
    DIFFOPT_LAUNCH((distill_row<E_, kKept, true, B, NV>), r.N, B, r, dloss, loss, stats, dx, dstride, dt, nullptr, 1, r.V);       \
    return launch_status(who);                                                                                                    \
  }
  DIFFOPT_KEPT(256, 2)
  DIFFOPT_KEPT(256, 4)
  DIFFOPT_KEPT(256, 8)
  DIFFOPT_KEPT(512, 8)
  DIFFOPT_KEPT(512, 13)
  DIFFOPT_KEPT(512, 16)
  DIFFOPT_KEPT(1024, 16)
#undef DIFFOPT_KEPT
  DIFFOPT_LAUNCH((distill_row<E_, kRead, true>), r.N, kDB, r, dloss, loss, stats, dx, dstride, dt, nullptr, 1, r.V);
  return launch_status(who);
}

template <class E_>
int second_rows(const char* who, const Rows& r, int32_t dtype, const Second& t, float* parts, hipStream_t st) {
  const Cut c = cut_of(r.N, r.V, dtype);
  if (c.slices > 1) {
    if (t.a) DIFFOPT_LAUNCH(distill_second_parts<E_>, r.N * c.slices, kDB, r, t, parts, c.slices, c.per);
    DIFFOPT_LAUNCH((distill_second<E_, kParts>), r.N * c.slices, kDB, r, t, parts, c.slices, c.per);
    return launch_status(who);
  }
  const int64_t bytes = r.V * elem_size(dtype);
#define DIFFOPT_KEPT(B, NV)                                                                  \
  if (bytes <= (int64_t)B * NV * 16) {                                                       \
    DIFFOPT_LAUNCH((distill_second<E_, kKept, B, NV>), r.N, B, r, t, nullptr, 1, r.V);       \
    return launch_status(who);                                                               \
  }
  DIFFOPT_KEPT(256, 4)
  DIFFOPT_KEPT(512, 4)
  DIFFOPT_KEPT(512, 8)
  DIFFOPT_KEPT(1024, 8)
#undef DIFFOPT_KEPT
  DIFFOPT_LAUNCH((distill_second<E_, kRead>), r.N, kDB, r, t, nullptr, 1, r.V);
  return launch_status(who);
}

int check_workspace(const char* who, const Rows& r, int32_t dtype, void* workspace, int64_t bytes) {
  const Cut c = cut_of(r.N, r.V, dtype);
  const int64_t need = c.slices > 1 ? r.N * c.slices * 8 : 0;
  if (need > 0 && (!workspace || bytes < need))
    return fail(DIFFOPT_EINVAL, "%s: the workspace has %lld bytes of %lld", who, (long long)(workspace ? bytes : 0), (long long)need);
  if (!aligned_to(workspace, 4)) return fail(DIFFOPT_EINVAL, "%s: the workspace is not 4-byte aligned", who);
  return DIFFOPT_OK;
}

}  // namespace
}  // namespace diffopt

using namespace diffopt;

extern "C" int64_t diffopt_distill_workspace(int64_t N, int64_t V, int32_t dtype, int64_t K) {
  if (N < 0 || N >= kMostRows || V < 1 || V > 0x7fffffff || !dtype_ok(dtype) || K < 1 || K > kMaxK) return -1;
  const Cut c = cut_of(N, V, dtype);
  return c.slices > 1 ? N * c.slices * 8 : 0;
}

extern "C" int diffopt_distill_fwd(const void* logits, int64_t row_stride, int64_t N, int64_t V, int32_t dtype,
                                   const void* ids, int32_t id_bytes, const float* teacher, int64_t K,
                                   double temperature, float* loss, float* stats, void* workspace,
                                   int64_t workspace_bytes, void* stream) {
  clear_error();
  static const char* who = "diffopt_distill_fwd";
  Rows r;
  int rc = check_rows(who, logits, row_stride, N, V, dtype, ids, id_bytes, teacher, K, temperature, &r);
  if (rc || N == 0) return rc;
  if (!loss || !stats) return fail(DIFFOPT_EINVAL, "%s: null required pointer", who);
  rc = check_aligned(who, {loss, stats});
  if (rc) return rc;
  rc = check_workspace(who, r, dtype, workspace, workspace_bytes);
  if (!rc) rc = check_apart(who, {{loss, N}, {stats, 2 * N}}, {{teacher, N * K}});
  if (rc) return rc;
  float* parts = static_cast<float*>(workspace);
  return dtype == DIFFOPT_F32 ? fwd_rows<float>(who, r, dtype, loss, stats, parts, as_stream(stream))
                              : fwd_rows<bf16>(who, r, dtype, loss, stats, parts, as_stream(stream));
}

extern "C" int diffopt_distill_bwd(const float* dloss, const void* logits, int64_t row_stride, int64_t N, int64_t V,
                                   int32_t dtype, const void* ids, int32_t id_bytes, const float* teacher, int64_t K,
                                   double temperature, const float* stats, void* dlogits, int64_t drow_stride,
                                   float* dteacher, void* stream) {
  clear_error();
  static const char* who = "diffopt_distill_bwd";
  Rows r;
  int rc = check_rows(who, logits, row_stride, N, V, dtype, ids, id_bytes, teacher, K, temperature, &r);
  if (rc || N == 0) return rc;
  if (!dloss || !stats) return fail(DIFFOPT_EINVAL, "%s: null required pointer", who);
  rc = check_aligned(who, {dloss, stats, dteacher});
  if (!rc) rc = check_out_rows(who, dlogits, drow_stride, V, N, dtype);
  if (!rc && dlogits == logits && N > 1 && drow_stride != row_stride)
    rc = fail(DIFFOPT_EINVAL, "%s: dlogits in the logits' place must have their row stride", who);
  if (!rc) rc = check_apart(who, {{dteacher, N * K}}, {{dloss, N}, {teacher, N * K}, {stats, 2 * N}});
  if (rc) return rc;
  return dtype == DIFFOPT_F32 ? bwd_rows<float>(who, r, dtype, dloss, stats, dlogits, drow_stride, dteacher, as_stream(stream))
                              : bwd_rows<bf16>(who, r, dtype, dloss, stats, dlogits, drow_stride, dteacher, as_stream(stream));
}

extern "C" int diffopt_distill_fwd_bwd(const float* dloss, const void* logits, int64_t row_stride, int64_t N, int64_t V,
                                       int32_t dtype, const void* ids, int32_t id_bytes, const float* teacher,
                                       int64_t K, double temperature, float* loss, float* stats, void* dlogits,
                                       int64_t drow_stride, float* dteacher, void* workspace, int64_t workspace_bytes,
                                       void* stream) {
  clear_error();
  static const char* who = "diffopt_distill_fwd_bwd";
  Rows r;
  int rc = check_rows(who, logits, row_stride, N, V, dtype, ids, id_bytes, teacher, K, temperature, &r);
  if (rc || N == 0) return rc;
  if (!dloss || !loss || !stats) return fail(DIFFOPT_EINVAL, "%s: null required pointer", who);
  rc = check_aligned(who, {dloss, loss, stats, dteacher});
  if (!rc) rc = check_out_rows(who, dlogits, drow_stride, V, N, dtype);
  if (rc) return rc;
  if (dlogits == logits) return fail(DIFFOPT_EINVAL, "%s: dlogits must not be logits", who);
  rc = check_workspace(who, r, dtype, workspace, workspace_bytes);
  if (!rc) rc = check_apart(who, {{loss, N}, {stats, 2 * N}, {dteacher, N * K}}, {{dloss, N}, {teacher, N * K}});
  if (rc) return rc;
  float* parts = static_cast<float*>(workspace);
  return dtype == DIFFOPT_F32
             ? both_rows<float>(who, r, dtype, dloss, loss, stats, dlogits, drow_stride, dteacher, parts, as_stream(stream))
             : both_rows<bf16>(who, r, dtype, dloss, loss, stats, dlogits, drow_stride, dteacher, parts, as_stream(stream));
}

extern "C" int diffopt_distill_bwd_bwd(const void* ddlogits, int64_t ddrow_stride, const float* ddteacher,
                                       const float* dloss, const void* logits, int64_t row_stride, int64_t N,
                                       int64_t V, int32_t dtype, const void* ids, int32_t id_bytes,
                                       const float* teacher, int64_t K, double temperature, const float* stats,
                                       float* out_dloss, void* out_logits, int64_t out_row_stride, float* out_teacher,
                                       void* workspace, int64_t workspace_bytes, void* stream) {
  clear_error();
  static const char* who = "diffopt_distill_bwd_bwd";
  Rows r;
  int rc = check_rows(who, logits, row_stride, N, V, dtype, ids, id_bytes, teacher, K, temperature, &r);
  if (rc || N == 0) return rc;
  if (!dloss || !stats) return fail(DIFFOPT_EINVAL, "%s: null required pointer", who);
  rc = check_aligned(who, {ddteacher, dloss, stats, out_dloss, out_teacher});
  if (!rc && !aligned_to(ddlogits, elem_size(dtype)))
    rc = fail(DIFFOPT_EINVAL, "%s: a pointer is not aligned to its elements", who);
  if (!rc) rc = check_out_rows(who, out_logits, out_row_stride, V, N, dtype);
  if (rc) return rc;
  if (out_logits == logits || out_logits == ddlogits)
    return fail(DIFFOPT_EINVAL, "%s: out_logits must be neither logits nor ddlogits", who);
  rc = check_workspace(who, r, dtype, workspace, workspace_bytes);
  if (!rc)
    rc = check_apart(who, {{out_dloss, N}, {out_teacher, N * K}}, {{ddteacher, N * K}, {dloss, N}, {teacher, N * K}, {stats, 2 * N}});
  if (rc) return rc;
  const Second t{ddlogits, ddrow_stride, ddteacher, dloss, stats, out_dloss, out_teacher, out_logits, out_row_stride};
  float* parts = static_cast<float*>(workspace);
  return dtype == DIFFOPT_F32 ? second_rows<float>(who, r, dtype, t, parts, as_stream(stream))
                              : second_rows<bf16>(who, r, dtype, t, parts, as_stream(stream));
}
