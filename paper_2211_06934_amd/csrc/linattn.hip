// Linear attention with a decay for each head on gfx950 (formulas in
// diffopt.h).  The forward and each of the three gradients are one scan over
// tokens with a matrix state S in fp32,
//   S = g S + sum_j ks k_j v_j^T,   o_i = qs S^T q_i,
// on permuted operands (dq: q = dout, k = v, v = k, the state transposed; dk
// and dv: back in time, the k/v heads of a state being the query heads that
// share it), so every direction is one `Scan` run by the same kernels.
#include <initializer_list>

#include "lm_common.hpp"

namespace diffopt {
namespace {

struct HeadArr {
  void* p;
  int64_t sb, st, sh;
};

// One scan: state head j of sequence b reads query heads j nq .. + nq and k/v
// heads j nk .. + nk (one of nq, nk is 1).
struct Scan {
  HeadArr q, k, v, o;
  const float* s0;  // initial state or NULL; element (r, c) at r s_r + c s_c of its [Dk][Dv] block
  float* s1;        // final state or NULL, laid out alike
  int64_t s_r, s_c;
  int32_t nq, nk, Dk, Dv;
  int32_t back;     // tokens run from the last to the first; the state meets a token undecayed
  float qs, ks;     // scale of the outputs, of the update
};

struct Shape {
  int64_t B, T;
  int32_t Hs;  // states per sequence
  const float* log_decay;
  const int32_t* lengths;
};

__device__ __forceinline__ int64_t length_of(const Shape& s, int64_t b) {
  if (!s.lengths) return s.T;
  const int64_t n = s.lengths[b];
  return n < 0 ? 0 : n > s.T ? s.T : n;
}

template <class E>
__device__ __forceinline__ E* at(const HeadArr& h, int64_t b, int64_t t, int64_t head) {
  return static_cast<E*>(h.p) + b * h.sb + t * h.st + head * h.sh;
}

// Token after token: a workgroup holds 64 columns of one state, a lane R rows
// by 4 columns of them.  For single tokens and short sequences.
constexpr int kTokenB = 256, kTokenCols = 64;

template <class E, int R>
__global__ __launch_bounds__(kTokenB) void linattn_tokens(Shape s, Scan a, int32_t col_tiles) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int rg = lane >> 2;
  const int64_t state = blockIdx.x / col_tiles, b = state / s.Hs;
  const int j = (int)(state - b * s.Hs);
  const int c0 = (int)(blockIdx.x % col_tiles) * kTokenCols + wave * 16 + (lane & 3) * 4;
  // the decay to 48 bits: one rounding of it would grow with every token
  const double gd = exp((double)s.log_decay[j]);
  const float g = (float)gd, g_lo = (float)(gd - (double)g);
  const int64_t L = length_of(s, b), block = state * a.Dk * a.Dv;
  float S[R][4];
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int r = rg + 16 * i;
      S[i][c] = a.s0 && r < a.Dk && c0 + c < a.Dv ? a.s0[block + r * a.s_r + (c0 + c) * a.s_c] : 0.0f;
    }
  for (int64_t n = 0; n < L; ++n) {
    const int64_t t = a.back ? L - 1 - n : n;
    if (!a.back || n > 0)
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) S[i][c] = fmaf(S[i][c], g, S[i][c] * g_lo);
    for (int h = 0; h < a.nk; ++h) {
      const E *k = at<E>(a.k, b, t, j * a.nk + h), *v = at<E>(a.v, b, t, j * a.nk + h);
      float vv[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) vv[c] = c0 + c < a.Dv ? (float)v[c0 + c] * a.ks : 0.0f;
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const int r = rg + 16 * i;
        const float kk = r < a.Dk ? (float)k[r] : 0.0f;
#pragma unroll
        for (int c = 0; c < 4; ++c) S[i][c] = fmaf(kk, vv[c], S[i][c]);
      }
    }
    if (!a.o.p) continue;
    for (int h = 0; h < a.nq; ++h) {
      const E* q = at<E>(a.q, b, t, j * a.nq + h);
      float o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const int r = rg + 16 * i;
        const float qq = r < a.Dk ? (float)q[r] : 0.0f;
#pragma unroll
        for (int c = 0; c < 4; ++c) o[c] = fmaf(qq, S[i][c], o[c]);
      }
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int m = 4; m < 64; m <<= 1) o[c] += __shfl_xor(o[c], m, 64);
      if (rg == 0) {
        E* out = at<E>(a.o, b, t, j * a.nq + h);
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (c0 + c < a.Dv) out[c0 + c] = (E)(o[c] * a.qs);
      }
    }
  }
  if (a.o.p && rg == 0)
    for (int64_t t = L; t < s.T; ++t)
      for (int h = 0; h < a.nq; ++h)
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (c0 + c < a.Dv) at<E>(a.o, b, t, j * a.nq + h)[c0 + c] = (E)0.0f;
  if (a.s1) {
    const float last = a.back && L > 0 ? g : 1.0f;
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int r = rg + 16 * i;
        if (r < a.Dk && c0 + c < a.Dv) a.s1[block + r * a.s_r + (c0 + c) * a.s_c] = S[i][c] * last;
      }
  }
}

// ---- host -------------------------------------------------------------------

constexpr int kMaxWidth = 256;

template <class E>
void launch_tokens(const Shape& s, const Scan& a, hipStream_t st) {
  const int tiles = (a.Dv + kTokenCols - 1) / kTokenCols;
  const dim3 grid((unsigned)(s.B * s.Hs * tiles)), block(kTokenB);
  if (a.Dk <= 64)
    hipLaunchKernelGGL((linattn_tokens<E, 4>), grid, block, 0, st, s, a, tiles);
  else if (a.Dk <= 128)
    hipLaunchKernelGGL((linattn_tokens<E, 8>), grid, block, 0, st, s, a, tiles);
  else
    hipLaunchKernelGGL((linattn_tokens<E, 16>), grid, block, 0, st, s, a, tiles);
}

int run_scan(const char* who, const Shape& s, const Scan& a, int32_t dtype, hipStream_t st) {
  if (dtype == DIFFOPT_F32)
    launch_tokens<float>(s, a, st);
  else
    launch_tokens<bf16>(s, a, st);
  return launch_status(who);
}

const char* sizes_wrong(int64_t B, int64_t T, int64_t H, int64_t Hk, int64_t Dk, int64_t Dv, int32_t dtype) {
  if (B < 0 || T < 0 || H < 0 || Hk < 0) return "B, T, H and Hk must be >= 0";
  if ((H == 0) != (Hk == 0) || (Hk > 0 && H % Hk)) return "H must be a multiple of Hk";
  if (Dk < 1 || Dk > kMaxWidth || Dv < 1 || Dv > kMaxWidth) return "Dk and Dv must be in [1, 256]";
  if (!dtype_ok(dtype)) return "unknown element type";
  if (H > 65536 || B > (int64_t(1) << 24) || B * Hk > (int64_t(1) << 24) || T > (int64_t(1) << 40)) return "too many heads, sequences or tokens";
  return nullptr;
}

int check_heads(const char* who, const char* what, const diffopt_heads* h, int32_t dtype, HeadArr* out) {
  if (!h || !h->data) return fail(DIFFOPT_EINVAL, "%s: null %s", who, what);
  if (!aligned_to(h->data, elem_size(dtype))) return fail(DIFFOPT_EINVAL, "%s: %s is not aligned to its elements", who, what);
  *out = HeadArr{h->data, h->stride_b, h->stride_t, h->stride_h};
  return DIFFOPT_OK;
}

int check_call(const char* who, int64_t B, int64_t T, int64_t H, int64_t Hk, int64_t Dk, int64_t Dv, int32_t dtype, double scale,
               const float* log_decay, const int32_t* lengths, std::initializer_list<const float*> states) {
  if (const char* w = sizes_wrong(B, T, H, Hk, Dk, Dv, dtype)) return fail(DIFFOPT_EINVAL, "%s: %s", who, w);
  if (!std::isfinite(scale) || !std::isfinite((float)scale)) return fail(DIFFOPT_EINVAL, "%s: scale must be finite", who);
  if (B * Hk > 0 && !log_decay) return fail(DIFFOPT_EINVAL, "%s: null log_decay", who);
  if (!aligned_to(log_decay, 4) || !aligned_to(lengths, 4))
    return fail(DIFFOPT_EINVAL, "%s: log_decay or lengths is not 4-byte aligned", who);
  for (const float* p : states)
    if (!aligned_to(p, 4)) return fail(DIFFOPT_EINVAL, "%s: a state is not 4-byte aligned", who);
  return DIFFOPT_OK;
}

}  // namespace
}  // namespace diffopt

using namespace diffopt;

extern "C" int64_t diffopt_linattn_workspace(int64_t B, int64_t T, int64_t H, int64_t Hk, int64_t Dk, int64_t Dv,
                                             int32_t dtype, int32_t backward) {
  (void)backward;
  return sizes_wrong(B, T, H, Hk, Dk, Dv, dtype) ? -1 : 0;
}

extern "C" int diffopt_linattn_fwd(const diffopt_heads* q, const diffopt_heads* k, const diffopt_heads* v,
                                   const float* log_decay, const int32_t* lengths, const float* state, int64_t B,
                                   int64_t T, int64_t H, int64_t Hk, int64_t Dk, int64_t Dv, int32_t dtype, double scale,
                                   const diffopt_heads* out, float* state_out, void* workspace, int64_t workspace_bytes,
                                   void* stream) {
  clear_error();
  static const char* who = "diffopt_linattn_fwd";
  int rc = check_call(who, B, T, H, Hk, Dk, Dv, dtype, scale, log_decay, lengths, {state, state_out});
  if (rc || B == 0 || Hk == 0) return rc;
  Scan a{};
  if (T > 0) {
    rc = check_heads(who, "q", q, dtype, &a.q);
    if (!rc) rc = check_heads(who, "k", k, dtype, &a.k);
    if (!rc) rc = check_heads(who, "v", v, dtype, &a.v);
    if (!rc) rc = check_heads(who, "out", out, dtype, &a.o);
    if (rc) return rc;
  } else if (!state_out) {
    return DIFFOPT_OK;
  }
  (void)workspace;
  (void)workspace_bytes;
  a.s0 = state;
  a.s1 = state_out;
  a.s_r = Dv;
  a.s_c = 1;
  a.nq = (int32_t)(H / Hk);
  a.nk = 1;
  a.Dk = (int32_t)Dk;
  a.Dv = (int32_t)Dv;
  a.qs = (float)scale;
  a.ks = 1.0f;
  const Shape s{B, T, (int32_t)Hk, log_decay, lengths};
  return run_scan(who, s, a, dtype, as_stream(stream));
}

extern "C" int diffopt_linattn_bwd(const diffopt_heads* dout, const float* dstate_out, const diffopt_heads* q,
                                   const diffopt_heads* k, const diffopt_heads* v, const float* log_decay,
                                   const int32_t* lengths, const float* state, int64_t B, int64_t T, int64_t H,
                                   int64_t Hk, int64_t Dk, int64_t Dv, int32_t dtype, double scale,
                                   const diffopt_heads* dq, const diffopt_heads* dk, const diffopt_heads* dv,
                                   float* dstate, void* workspace, int64_t workspace_bytes, void* stream) {
  clear_error();
  static const char* who = "diffopt_linattn_bwd";
  int rc = check_call(who, B, T, H, Hk, Dk, Dv, dtype, scale, log_decay, lengths, {state, dstate_out, dstate});
  if (rc || B == 0 || Hk == 0) return rc;
  HeadArr Q{}, K{}, V{}, DO{}, DQ{}, DK{}, DV{};
  if (T > 0) {
    rc = check_heads(who, "q", q, dtype, &Q);
    if (!rc) rc = check_heads(who, "k", k, dtype, &K);
    if (!rc) rc = check_heads(who, "v", v, dtype, &V);
    if (!rc) rc = check_heads(who, "dout", dout, dtype, &DO);
    if (!rc && dq) rc = check_heads(who, "dq", dq, dtype, &DQ);
    if (!rc && dk) rc = check_heads(who, "dk", dk, dtype, &DK);
    if (!rc && dv) rc = check_heads(who, "dv", dv, dtype, &DV);
    if (rc) return rc;
  }
  if (dstate && (dstate == dstate_out || dstate == state))
    return fail(DIFFOPT_EINVAL, "%s: dstate must be neither dstate_out nor state", who);
  (void)workspace;
  (void)workspace_bytes;
  const Shape s{B, T, (int32_t)Hk, log_decay, lengths};
  const int32_t G = (int32_t)(H / Hk), dk_ = (int32_t)Dk, dv_ = (int32_t)Dv;
  const float sc = (float)scale;
  hipStream_t st = as_stream(stream);
  if (DQ.p) {
    rc = run_scan(who, s, Scan{DO, V, K, DQ, state, nullptr, 1, Dv, G, 1, dv_, dk_, 0, sc, 1.0f}, dtype, st);
    if (rc) return rc;
  }
  // dv's scan holds the state's gradient as [Dk][Dv], dk's its transpose
  if (DV.p || dstate) {
    rc = run_scan(who, s, Scan{K, Q, DO, DV, dstate_out, dstate, Dv, 1, 1, G, dk_, dv_, 1, 1.0f, sc}, dtype, st);
    if (rc) return rc;
  }
  if (DK.p) rc = run_scan(who, s, Scan{V, DO, Q, DK, dstate_out, nullptr, 1, Dv, 1, G, dv_, dk_, 1, 1.0f, sc}, dtype, st);
  return rc;
}

extern "C" int diffopt_linattn_step(const diffopt_heads* q, const diffopt_heads* k, const diffopt_heads* v,
                                    const float* log_decay, int64_t B, int64_t H, int64_t Hk, int64_t Dk, int64_t Dv,
                                    int32_t dtype, double scale, float* state, const diffopt_heads* out, void* stream) {
  clear_error();
  static const char* who = "diffopt_linattn_step";
  int rc = check_call(who, B, 1, H, Hk, Dk, Dv, dtype, scale, log_decay, nullptr, {state});
  if (rc || B == 0 || Hk == 0) return rc;
  if (!state) return fail(DIFFOPT_EINVAL, "%s: null state", who);
  Scan a{};
  rc = check_heads(who, "q", q, dtype, &a.q);
  if (!rc) rc = check_heads(who, "k", k, dtype, &a.k);
  if (!rc) rc = check_heads(who, "v", v, dtype, &a.v);
  if (!rc) rc = check_heads(who, "out", out, dtype, &a.o);
  if (rc) return rc;
  a.s0 = state;
  a.s1 = state;
  a.s_r = Dv;
  a.s_c = 1;
  a.nq = (int32_t)(H / Hk);
  a.nk = 1;
  a.Dk = (int32_t)Dk;
  a.Dv = (int32_t)Dv;
  a.qs = (float)scale;
  a.ks = 1.0f;
  const Shape s{B, 1, (int32_t)Hk, log_decay, nullptr};
  return run_scan(who, s, a, dtype, as_stream(stream));
}
