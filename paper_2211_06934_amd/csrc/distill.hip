// Distillation from a teacher's top logits on gfx950: the loss, its gradient,
// and the gradient's own vector-Jacobian product (formulas in diffopt.h).
//
// One workgroup per row.  The row's max m and sum s = sum exp((x - m)/T) come
// from one pass with a running max (a lane rescales its sum once per 16 bytes);
// wave 0 forms the teacher's softmax over the K entries meanwhile.  The
// gradient's dense part g T p is one more pass over the row; the K entries are
// then written once more by the same workgroup after a barrier, each with the
// sum of q over the entries of its token, so nothing is added atomically and
// equal ids need no order.  A few exponentials per element: bound by memory.
#include <initializer_list>

#include "lm_common.hpp"

namespace diffopt {
namespace {

constexpr int kDB = 512;       // threads per workgroup
constexpr int kMaxK = 1024;    // entries of a row
constexpr float kLog2e = 1.4426950408889634f;

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

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// (x - m) / T in units of log 2; a row of -inf alone keeps m = -inf, s = 0.
__device__ __forceinline__ float safe_max(float m) { return m == -kInf ? 0.0f : m; }

__device__ __forceinline__ void join(float& m, float& s, float m2, float s2, float c) {
  const float M = fmaxf(m, m2), b = safe_max(M);
  s = s * exp2_fast((m - b) * c) + s2 * exp2_fast((m2 - b) * c);
  m = M;
}

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

// f(first element, 16 bytes of x from there) over a row's aligned vectors,
// g(element) over the elements before and after them.
template <class E_, class F, class G>
__device__ __forceinline__ void over_row(const E_* x, int64_t n, F f, G g) {
  constexpr int NV = Vec<E_>::N;
  const int64_t off = (int64_t)((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / (int)sizeof(E_);
  const int64_t head = off < n ? off : n;
  const int64_t nv = (n - head) / NV;
  for (int64_t i = threadIdx.x; i < nv; i += blockDim.x) f(head + i * NV);
  const int64_t rest = n - nv * NV;  // head and tail elements
  if ((int64_t)threadIdx.x < rest) g((int64_t)threadIdx.x < head ? (int64_t)threadIdx.x : threadIdx.x + nv * NV);
}

struct Reduce {
  float m[kDB / 64], s[kDB / 64];
};

template <class E_>
__device__ void row_stats(const E_* x, int64_t V, float c, Reduce& R, float& m, float& s) {
  m = -kInf;
  s = 0.0f;
  over_row(
      x, V,
      [&](int64_t at) {
        const auto v = load_vec(x + at);
        float e[Vec<E_>::N], vm = -kInf;
#pragma unroll
        for (int i = 0; i < Vec<E_>::N; ++i) {
          e[i] = (float)v[i];
          vm = fmaxf(vm, e[i]);
        }
        if (vm > m) {
          s *= exp2_fast((m - vm) * c);
          m = vm;
        }
        const float b = safe_max(m);
#pragma unroll
        for (int i = 0; i < Vec<E_>::N; ++i) s += exp2_fast((e[i] - b) * c);
      },
      [&](int64_t at) {
        const float e = (float)x[at];
        join(m, s, e, e == -kInf ? 0.0f : (e - e == 0.0f ? 1.0f : kNan), c);
      });
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

// The sum of q over the entries that name the token of entry j.
__device__ __forceinline__ float same_token(const float* w, const Entries& E, int K, int64_t id) {
  float sum = 0.0f;
  for (int i = 0; i < K; ++i) sum += E.id[i] == id ? w[i] : 0.0f;
  return sum;
}

// The row's results from its statistics on: loss, gradients.
template <class E_, bool FWD, bool BWD>
__global__ __launch_bounds__(kDB) void distill_row(Rows r, const float* dloss, float* loss, float* stats, E_* dlogits,
                                                   int64_t drow_stride, float* dteacher) {
  __shared__ Entries E;
  __shared__ Reduce R;
  const int lane = threadIdx.x & 63;
  const float c = r.invT * kLog2e;
  for (int64_t row = blockIdx.x; row < r.N; row += gridDim.x) {
    const E_* x = static_cast<const E_*>(r.logits) + row * r.row_stride;
    __syncthreads();
    if (threadIdx.x < 64) {
      teacher_softmax(r, row, E, lane);
      gather(x, E, r.K, E.x, lane);  // before dlogits, which may be logits, is written
    }
    float m, s;
    if (FWD) {
      row_stats(x, r.V, c, R, m, s);
      if (threadIdx.x == 0) {
        stats[2 * row] = m;
        stats[2 * row + 1] = s;
      }
    } else {
      m = stats[2 * row];
      s = stats[2 * row + 1];
    }
    __syncthreads();
    const bool some = E.some, bad = E.bad;
    const float g = BWD ? (bad ? kNan : dloss[row]) : 0.0f, gT = g * r.T;
    if (threadIdx.x < 64 && (FWD || dteacher)) {
      const float mean = entry_terms(r, E, m, s, lane);
      if (FWD && lane == 0) loss[row] = bad ? kNan : some ? r.T * mean : 0.0f;
      if (BWD && dteacher)
        for (int j = lane; j < r.K; j += 64)
          dteacher[row * r.K + j] = E.q[j] != 0.0f ? g * E.q[j] * (E.lq[j] - mean) : bad ? kNan : 0.0f;
    }
    if (!BWD) continue;
    E_* dx = dlogits + row * drow_stride;
    const float w = some ? gT / s : 0.0f;
    over_row(
        x, r.V,
        [&](int64_t at) {
          float y[Vec<E_>::N];
          const auto v = load_vec(x + at);
#pragma unroll
          for (int i = 0; i < Vec<E_>::N; ++i) y[i] = some ? w * exp2_fast(((float)v[i] - m) * c) : 0.0f;
          store_vec(dx + at, y);
        },
        [&](int64_t at) { dx[at] = (E_)(some ? w * exp2_fast(((float)x[at] - m) * c) : 0.0f); });
    __syncthreads();  // the entries' elements are written after the dense part's
    for (int j = threadIdx.x; j < r.K; j += kDB)
      if (E.id[j] >= 0)
        dx[E.id[j]] = (E_)(w * exp2_fast((E.x[j] - m) * c) - gT * same_token(E.q, E, r.K, E.id[j]));
  }
}

template <class E_>
__global__ __launch_bounds__(kDB) void distill_second(Rows r, const E_* dd, int64_t ddrow_stride, const float* ddteacher,
                                                      const float* dloss, const float* stats, float* out_dloss,
                                                      E_* out, int64_t out_stride, float* out_teacher) {
  __shared__ Entries E;
  __shared__ float aj[kMaxK], cj[kMaxK];
  __shared__ float part[kDB / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float c = r.invT * kLog2e;
  for (int64_t row = blockIdx.x; row < r.N; row += gridDim.x) {
    const E_* x = static_cast<const E_*>(r.logits) + row * r.row_stride;
    const E_* a = dd ? dd + row * ddrow_stride : nullptr;
    E_* y = out + row * out_stride;
    const float m = stats[2 * row], s = stats[2 * row + 1], inv = 1.0f / s;
    __syncthreads();
    if (threadIdx.x < 64) {
      teacher_softmax(r, row, E, lane);
      gather(x, E, r.K, E.x, lane);
      for (int j = lane; j < r.K; j += 64) {
        aj[j] = a && E.id[j] >= 0 ? (float)a[E.id[j]] : 0.0f;
        cj[j] = ddteacher && E.q[j] != 0.0f ? ddteacher[row * r.K + j] : 0.0f;
      }
    }
    float pa = 0.0f;
    if (a)
      over_row(
          x, r.V,
          [&](int64_t at) {
            const auto v = load_vec(x + at);
            const auto u = load_vec(a + at);
#pragma unroll
            for (int i = 0; i < Vec<E_>::N; ++i) pa += exp2_fast(((float)v[i] - m) * c) * (float)u[i];
          },
          [&](int64_t at) { pa += exp2_fast(((float)x[at] - m) * c) * (float)a[at]; });
    pa = wave_sum(pa);
    if (lane == 0) part[wave] = pa;
    __syncthreads();
    pa = 0.0f;
    for (int w = 0; w < kDB / 64; ++w) pa += part[w];
    pa *= inv;
    const bool some = E.some, bad = E.bad;
    const float g = bad ? kNan : dloss[row];
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
      if (out_dloss && lane == 0) out_dloss[row] = bad ? kNan : some ? r.T * (pa - abar) + cov : 0.0f;
      for (int j = lane; j < r.K; j += 64) {
        const float q = E.q[j], cc = cj[j], l = E.lq[j];
        if (out_teacher)
          out_teacher[row * r.K + j] =
              q != 0.0f ? g * q * ((abar - aj[j]) + (cc - cbar) + r.invT * ((cc - cbar) * (l - mean) - cov))
                        : bad ? kNan : 0.0f;
        E.q[j] = q * (cc - cbar);  // what the entry takes from its token's element
      }
    }
    const float w = some ? g * inv : 0.0f;
    over_row(
        x, r.V,
        [&](int64_t at) {
          float z[Vec<E_>::N];
          if (a && some) {
            const auto v = load_vec(x + at);
            const auto u = load_vec(a + at);
#pragma unroll
            for (int i = 0; i < Vec<E_>::N; ++i) z[i] = w * exp2_fast(((float)v[i] - m) * c) * ((float)u[i] - pa);
          } else {
#pragma unroll
            for (int i = 0; i < Vec<E_>::N; ++i) z[i] = 0.0f;
          }
          store_vec(y + at, z);
        },
        [&](int64_t at) {
          y[at] = (E_)(a && some ? w * exp2_fast(((float)x[at] - m) * c) * ((float)a[at] - pa) : 0.0f);
        });
    __syncthreads();
    for (int j = threadIdx.x; j < r.K; j += kDB)
      if (E.id[j] >= 0) {
        const float dense = a ? w * exp2_fast((E.x[j] - m) * c) * (aj[j] - pa) : 0.0f;
        y[E.id[j]] = (E_)(dense - g * same_token(E.q, E, r.K, E.id[j]));
      }
  }
}

// ---- host -------------------------------------------------------------------

int check_rows(const char* who, const void* logits, int64_t row_stride, int64_t N, int64_t V, int32_t dtype,
               const void* ids, int32_t id_bytes, const float* teacher, int64_t K, double temperature, Rows* r) {
  if (N < 0) return fail(DIFFOPT_EINVAL, "%s: N must be >= 0", who);
  if (V < 1) return fail(DIFFOPT_EINVAL, "%s: V must be >= 1", who);
  if (!dtype_ok(dtype)) return fail(DIFFOPT_EINVAL, "%s: unknown element type %d", who, (int)dtype);
  if (id_bytes != 4 && id_bytes != 8) return fail(DIFFOPT_EINVAL, "%s: id_bytes must be 4 or 8", who);
  if (K < 1 || K > kMaxK) return fail(DIFFOPT_EINVAL, "%s: K must be in [1, %d]", who, kMaxK);
  if (!(std::isfinite(temperature) && temperature > 0.0 && std::isfinite((float)(1.0 / temperature)) && (float)temperature > 0.0f &&
        std::isfinite((float)temperature)))
    return fail(DIFFOPT_EINVAL, "%s: temperature must be finite and > 0", who);
  if (N == 0) return DIFFOPT_OK;
  if (!logits || !ids || !teacher) return fail(DIFFOPT_EINVAL, "%s: null required pointer", who);
  if (!aligned_to(logits, elem_size(dtype)) || !aligned_to(ids, id_bytes) || !aligned_to(teacher, 4))
    return fail(DIFFOPT_EINVAL, "%s: a pointer is not aligned to its elements", who);
  *r = Rows{logits, row_stride, N, V, ids, id_bytes, teacher, (int32_t)K, (float)temperature, (float)(1.0 / temperature)};
  return DIFFOPT_OK;
}

int check_aligned(const char* who, std::initializer_list<const void*> floats) {
  for (const void* p : floats)
    if (!aligned_to(p, 4)) return fail(DIFFOPT_EINVAL, "%s: pointer %p is not 4-byte aligned", who, p);
  return DIFFOPT_OK;
}

int check_out_rows(const char* who, const void* out, int64_t stride, int64_t V, int64_t N, int32_t dtype) {
  if (!out) return fail(DIFFOPT_EINVAL, "%s: null required pointer", who);
  if (!aligned_to(out, elem_size(dtype))) return fail(DIFFOPT_EINVAL, "%s: a pointer is not aligned to its elements", who);
  if (N > 1 && stride < V && stride > -V) return fail(DIFFOPT_EINVAL, "%s: rows of the result overlap", who);
  return DIFFOPT_OK;
}

dim3 row_grid(int64_t N) { return dim3((unsigned)(N < 0x7fffffff ? N : 0x7fffffff)); }

template <bool FWD, bool BWD>
int launch_rows(const char* who, const Rows& r, int32_t dtype, const float* dloss, float* loss, float* stats,
                void* dlogits, int64_t drow_stride, float* dteacher, hipStream_t st) {
  if (dtype == DIFFOPT_F32)
    hipLaunchKernelGGL((distill_row<float, FWD, BWD>), row_grid(r.N), dim3(kDB), 0, st, r, dloss, loss, stats,
                       static_cast<float*>(dlogits), drow_stride, dteacher);
  else
    hipLaunchKernelGGL((distill_row<bf16, FWD, BWD>), row_grid(r.N), dim3(kDB), 0, st, r, dloss, loss, stats,
                       static_cast<bf16*>(dlogits), drow_stride, dteacher);
  return launch_status(who);
}

}  // namespace
}  // namespace diffopt

using namespace diffopt;

extern "C" int64_t diffopt_distill_workspace(int64_t N, int64_t V, int32_t dtype, int64_t K) {
  if (N < 0 || V < 1 || !dtype_ok(dtype) || K < 1 || K > kMaxK) return -1;
  return 0;
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
  (void)workspace;
  (void)workspace_bytes;
  return launch_rows<true, false>(who, r, dtype, nullptr, loss, stats, nullptr, 0, nullptr, as_stream(stream));
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
  if (rc) return rc;
  return launch_rows<false, true>(who, r, dtype, dloss, nullptr, const_cast<float*>(stats), dlogits, drow_stride,
                                  dteacher, as_stream(stream));
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
  (void)workspace;
  (void)workspace_bytes;
  return launch_rows<true, true>(who, r, dtype, dloss, loss, stats, dlogits, drow_stride, dteacher, as_stream(stream));
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
  (void)workspace;
  (void)workspace_bytes;
  hipStream_t st = as_stream(stream);
  if (dtype == DIFFOPT_F32)
    hipLaunchKernelGGL((distill_second<float>), row_grid(N), dim3(kDB), 0, st, r, static_cast<const float*>(ddlogits),
                       ddrow_stride, ddteacher, dloss, stats, out_dloss, static_cast<float*>(out_logits),
                       out_row_stride, out_teacher);
  else
    hipLaunchKernelGGL((distill_second<bf16>), row_grid(N), dim3(kDB), 0, st, r, static_cast<const bf16*>(ddlogits),
                       ddrow_stride, ddteacher, dloss, stats, out_dloss, static_cast<bf16*>(out_logits),
                       out_row_stride, out_teacher);
  return launch_status(who);
}
