// A gated linear recurrence over sequences on gfx950 and its derivatives
// (formulas in diffopt.h): h_t = a_t h_{t-1} + x_t for each channel, a = exp(log_gate).
//
// A run of tokens maps the state that enters it linearly: h -> A h + X with
// A = exp(sum of its log gates) and X its own state from zero.  The adjoint e
// runs the other way through the same gates, e -> A e + E, and the two
// recurrences of the second derivative are coupled to them by r alone:
// y -> A (y + rho h) + Y and f -> A (f + rho e) + F with rho the sum of r.  So
// a run is known by A and one to five numbers a channel.  The logarithm of A is
// kept, not A: a sum's rounding does not drift where a long product's does.
//
// A workgroup of kW waves holds a chunk of kW U tokens of 64 VEC channels in
// registers, each wave U tokens of it, so that an operand is read once for both
// directions.  Waves tell one another their runs through LDS.  Longer
// sequences are cut into one chunk a workgroup: a first launch writes each
// chunk's run, a small one turns runs into the states that enter each chunk, a
// third walks the chunks.  A token past its sequence's end maps every state to
// itself.  With enough columns of 64 channels, or in short sequences, a workgroup
// takes its column through the whole sequence instead (sweeps, below).
//
// An element costs an exponential, a few multiply-adds and its share of a run:
// memory bounds it, and that chunks read their operands twice, which they could
// only avoid by waiting for one another.  4 x 4,096 tokens of 2,048 bf16 channels: the
// sweep 62 us (201 MB, 3.2 TB/s), backward runs 35 (201 MB, 5.8 TB/s), join 8, walk
// 58 (336 MB, 5.8 TB/s).  16,384 tokens in one sequence: runs 27 (134 MB, 5.0 TB/s),
// join 7, walk 33 (201 MB, 6.1 TB/s).
#include <initializer_list>
#include <type_traits>

#include "lm_common.hpp"

namespace diffopt {
namespace {

constexpr int kW = 8;  // waves of a chunk, and the most chunks whose runs the walk joins itself
constexpr float kLog2e = 1.4426950408889634f;
constexpr int64_t kMostGroups = (int64_t(1) << 32) / (64 * kW) - 1;  // a launch has fewer than 2^32 threads

enum Mode { kFwd, kBwd, kSecond };

// What a run is known by: kL, kX always, kE for the adjoint, the others for the second derivative.
enum Field { kL, kX, kE, kRho, kY, kF };
constexpr int fields(int mode) { return mode == kFwd ? 2 : mode == kBwd ? 3 : 6; }

struct Scan {
  HeadArr lg, x, dh, r, p;                  // operands
  HeadArr out[3];                           // h / dlog_gate, dx / out_dh, out_log_gate, out_x
  const int32_t* lengths;
  const float *state, *dstate_out, *ddstate;
  float *end, *begin, *end2;                // the state (or y) after the last token, the adjoint (or f) before the first
  float* parts;                             // [B][S][fields][C]: chunks' runs, then the states that enter them
  int64_t T, C, S;
  int32_t cols;
  bool from_end;  // the walk's order of chunks
  bool together;  // neighbouring columns share a chip
};

// What a workgroup works on.  Workgroups go to the eight chips in turn: from the last to
// the first in eights, each chip's L2 meets its own again; together, a chip has the
// columns beside one another, whose rows end within a line.
__device__ __forceinline__ uint32_t place_of(const Scan& s, bool from_end) {
  const uint32_t eights = gridDim.x / 8, eight = blockIdx.x / 8, chip = blockIdx.x % 8;
  if (eight >= eights) return blockIdx.x;
  const uint32_t at = from_end ? eights - 1 - eight : eight;
  return s.together ? chip * eights + at : at * 8 + chip;
}

template <class E, int VEC>
struct Pack {
  typedef E type __attribute__((ext_vector_type(VEC), aligned(alignof(E))));
};
template <class E>
struct Pack<E, 1> {
  typedef E type;
};

template <class E, int VEC>
__device__ __forceinline__ void load_pack(const E* at, float* v) {
  const auto x = *reinterpret_cast<const typename Pack<E, VEC>::type*>(at);
  if constexpr (VEC == 1) {
    v[0] = (float)x;
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = (float)x[i];
  }
}

template <class E, int VEC>
__device__ __forceinline__ void store_pack(E* at, const float* v) {
  if constexpr (VEC == 1) {
    *at = (E)v[0];
  } else {
    typedef float wide __attribute__((ext_vector_type(VEC)));
    typedef E whole __attribute__((ext_vector_type(VEC)));
    wide w;
#pragma unroll
    for (int i = 0; i < VEC; ++i) w[i] = v[i];
    *reinterpret_cast<typename Pack<E, VEC>::type*>(at) = __builtin_convertvector(w, whole);
  }
}

// The wave, as a number that its lanes share: rows' addresses are scalars.
__device__ __forceinline__ int wave_of() { return __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)); }

// A barrier for what is in LDS: loads from memory stay on their way.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

__device__ __forceinline__ float gate(float lg) { return __builtin_amdgcn_exp2f(lg * kLog2e); }

// States of VEC channels that pass through a run forwards (h, y) and backwards (e, f).
template <int VEC>
struct States {
  float h[VEC], y[VEC], e[VEC], f[VEC];
};

// f(channel, field) gives the run.
template <int MODE, class R>
__device__ __forceinline__ void pass_fwd(float& h, float& y, const R& run) {
  const float A = gate(run(kL));
  if (MODE == kSecond) y = A * (y + run(kRho) * h) + run(kY);
  h = A * h + run(kX);
}

template <int MODE, class R>
__device__ __forceinline__ void pass_bwd(float& e, float& f, const R& run) {
  const float A = gate(run(kL));
  if (MODE == kSecond) f = A * (f + run(kRho) * e) + run(kF);
  e = A * e + run(kE);
}

// Where a workgroup, a wave and a lane work.
template <int VEC>
struct Place {
  int64_t b, seg, len;
  uint32_t c;
  bool on;  // the lane has channels; the last one's may be the neighbour's too, with the same values
  __device__ __forceinline__ Place(const Scan& s, bool from_end = false) {
    const uint32_t id = place_of(s, from_end);
    const uint32_t row = id / (uint32_t)s.cols, col = id - row * s.cols;
    b = row / (uint32_t)s.S;
    seg = row - b * s.S;
    c = (col * 64 + (threadIdx.x & 63)) * VEC;  // below 2^32: C is at most 2^31
    on = c < s.C;
    if (c + VEC > s.C) c = (uint32_t)s.C - VEC;  // C >= VEC
    len = s.T;
    if (s.lengths) {
      const int64_t n = s.lengths[b];
      len = n < 0 ? 0 : n < len ? n : len;
    }
  }
};

// A wave's tokens [t0, t0 + U) of VEC channels.
template <class E, int MODE, int VEC, int U>
struct Tokens {
  float a[U][VEC], x[U][VEC], dh[MODE >= kBwd ? U : 1][VEC], r[MODE == kSecond ? U : 1][VEC], p[MODE == kSecond ? U : 1][VEC];
  float run[fields(MODE)][VEC];

  static __device__ __forceinline__ void rows(const HeadArr& h, const Place<VEC>& at, int64_t t0, float (*v)[VEC]) {
    const E* row = static_cast<const E*>(h.p) + at.b * h.sb + t0 * h.st;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      load_pack<E, VEC>(row + at.c, v[u]);
      if (t0 + u + 1 < at.len) row += h.st;  // else once more the last one
    }
  }
  static __device__ __forceinline__ void no_rows(float (*v)[VEC]) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[u][i] = 0.0f;
  }

  // All of the tokens' operands on their way at once.
  __device__ __forceinline__ void load(const Scan& s, const Place<VEC>& at, int64_t t0) {
    if (t0 < at.len) {
      rows(s.lg, at, t0, a);
      rows(s.x, at, t0, x);
      if constexpr (MODE >= kBwd) rows(s.dh, at, t0, dh);
      if constexpr (MODE == kSecond) {
        rows(s.r, at, t0, r);
        rows(s.p, at, t0, p);
      }
    } else {
      no_rows(a);
      no_rows(x);
      if constexpr (MODE >= kBwd) no_rows(dh);
      if constexpr (MODE == kSecond) {
        no_rows(r);
        no_rows(p);
      }
    }
  }

  // Log gates become gates; tokens past the end the identity; the run of the rest.
  __device__ __forceinline__ void finish(const Place<VEC>& at, int64_t t0) {
    if (t0 + U > at.len) {  // the same for the wave
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (t0 + u >= at.len)
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            a[u][i] = x[u][i] = 0.0f;
            if constexpr (MODE >= kBwd) dh[u][i] = 0.0f;
            if constexpr (MODE == kSecond) r[u][i] = p[u][i] = 0.0f;
          }
    }
#pragma unroll
    for (int f = 0; f < fields(MODE); ++f)
#pragma unroll
      for (int i = 0; i < VEC; ++i) run[f][i] = 0.0f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        run[kL][i] += a[u][i];
        a[u][i] = gate(a[u][i]);
        if constexpr (MODE == kSecond) {
          run[kRho][i] += r[u][i];
          run[kY][i] = a[u][i] * (run[kY][i] + r[u][i] * run[kX][i]) + p[u][i];
        }
        run[kX][i] = a[u][i] * run[kX][i] + x[u][i];
      }
    if constexpr (MODE >= kBwd)
#pragma unroll
      for (int u = U - 1; u >= 0; --u)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const float g = dh[u][i] + run[kE][i];
          if constexpr (MODE == kSecond) run[kF][i] = a[u][i] * (r[u][i] * g + run[kF][i]);
          run[kE][i] = a[u][i] * g;
        }
  }
};

// Waves' runs: channel i of a lane's VEC lies 64 floats on, so that a wave's
// lanes read neighbouring words.
template <int MODE, int VEC>
struct Runs {
  float v[kW][fields(MODE)][VEC][64];
  template <class Tok>
  __device__ __forceinline__ void put(int wave, int lane, const Tok& t) {
#pragma unroll
    for (int f = 0; f < fields(MODE); ++f)
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[wave][f][i][lane] = t.run[f][i];
  }
};

__device__ __forceinline__ float* part_of(const Scan& s, int nf, int64_t b, int64_t seg) { return s.parts + (b * s.S + seg) * nf * s.C; }

// A chunk's run, for sequences of more than one chunk.
template <class E, int MODE, int VEC, int U>
__global__ __launch_bounds__(64 * kW) void gscan_runs(Scan s) {
  __shared__ Runs<MODE, VEC> R;
  constexpr int NF = fields(MODE);
  const Place<VEC> at(s);
  const int lane = threadIdx.x & 63, wave = wave_of();
  const int64_t t0 = (at.seg * kW + wave) * U;
  Tokens<E, MODE, VEC, U> tok;
  tok.load(s, at, t0);
  tok.finish(at, t0);
  R.put(wave, lane, tok);
  __syncthreads();
  if (wave != 0 || !at.on) return;
  float* to = part_of(s, NF, at.b, at.seg) + at.c;
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    float L = 0.0f, rho = 0.0f, h = 0.0f, y = 0.0f, e = 0.0f, f = 0.0f;
#pragma unroll
    for (int w = 0; w < kW; ++w) {
      L += R.v[w][kL][i][lane];
      if constexpr (MODE == kSecond) rho += R.v[w][kRho][i][lane];
      pass_fwd<MODE>(h, y, [&](int k) { return R.v[w][k][i][lane]; });
    }
    if constexpr (MODE >= kBwd)
#pragma unroll
      for (int w = kW - 1; w >= 0; --w) pass_bwd<MODE>(e, f, [&](int k) { return R.v[w][k][i][lane]; });
    to[i] = L;
    to[s.C + i] = h;
    if constexpr (MODE >= kBwd) to[2 * s.C + i] = e;
    if constexpr (MODE == kSecond) {
      to[3 * s.C + i] = rho;
      to[4 * s.C + i] = y;
      to[5 * s.C + i] = f;
    }
  }
}

// Chunks' runs become the states that enter each chunk: kX holds h, kY y, kE e
// and kF f.  A workgroup has 64 channels of a sequence, its waves share the
// chunks, and hold 16 of them forwards (256 chunks 8.2 us, in two batches of 8 9.5; 128
// chunks 7.1).
constexpr int kJW = 16;
template <int MODE>
__global__ __launch_bounds__(64 * kJW) void gscan_join(Scan s) {
  constexpr int NF = fields(MODE), kBatch = MODE == kFwd ? 16 : 8;
  __shared__ float v[kJW][NF][64];
  const int64_t cols = (s.C + 63) / 64, b = blockIdx.x / cols;
  const int lane = threadIdx.x & 63, wave = wave_of();
  const int64_t c0 = (blockIdx.x - b * cols) * 64 + lane, c = c0 < s.C ? c0 : s.C - 1;
  const int64_t per = (s.S + kJW - 1) / kJW, s0 = wave * per < s.S ? wave * per : s.S, s1 = s0 + per < s.S ? s0 + per : s.S;
  float L = 0.0f, rho = 0.0f, h = 0.0f, y = 0.0f, e = 0.0f, f = 0.0f;
  float run[kBatch][NF];
  // chunks [first, first + kBatch) of the wave's, all loads at once
  const auto load = [&](int64_t first) {
#pragma unroll
    for (int n = 0; n < kBatch; ++n) {
      const int64_t seg = first + n < s1 ? first + n : s1 - 1;
      const float* at = part_of(s, NF, b, seg) + c;
#pragma unroll
      for (int k = 0; k < NF; ++k) run[n][k] = at[k * s.C];
    }
  };
  const int64_t batches = (s1 - s0 + kBatch - 1) / kBatch;
  for (int64_t n0 = 0; n0 < batches; ++n0) {
    load(s0 + n0 * kBatch);
#pragma unroll
    for (int n = 0; n < kBatch; ++n)
      if (s0 + n0 * kBatch + n < s1) {
        L += run[n][kL];
        if constexpr (MODE == kSecond) rho += run[n][kRho];
        pass_fwd<MODE>(h, y, [&](int k) { return run[n][k]; });
      }
  }
  if constexpr (MODE >= kBwd)
    for (int64_t n0 = batches - 1; n0 >= 0; --n0) {
      if (batches > 1) load(s0 + n0 * kBatch);
#pragma unroll
      for (int n = kBatch - 1; n >= 0; --n)
        if (s0 + n0 * kBatch + n < s1) pass_bwd<MODE>(e, f, [&](int k) { return run[n][k]; });
    }
  v[wave][kL][lane] = L;
  v[wave][kX][lane] = h;
  if constexpr (MODE >= kBwd) v[wave][kE][lane] = e;
  if constexpr (MODE == kSecond) {
    v[wave][kRho][lane] = rho;
    v[wave][kY][lane] = y;
    v[wave][kF][lane] = f;
  }
  h = s.state ? s.state[b * s.C + c] : 0.0f;
  y = MODE == kSecond && s.ddstate ? s.ddstate[b * s.C + c] : 0.0f;
  e = MODE >= kBwd && s.dstate_out ? s.dstate_out[b * s.C + c] : 0.0f;
  f = 0.0f;
  __syncthreads();
  for (int w = 0; w < wave; ++w) pass_fwd<MODE>(h, y, [&](int k) { return v[w][k][lane]; });
  if constexpr (MODE >= kBwd)
    for (int w = kJW - 1; w > wave; --w) pass_bwd<MODE>(e, f, [&](int k) { return v[w][k][lane]; });
  if (c0 >= s.C) return;
  // the adjoint's way first: the forward way reads nothing that it writes
  if constexpr (MODE >= kBwd)
    for (int64_t n0 = batches - 1; n0 >= 0; --n0) {
      if (batches > 1) load(s0 + n0 * kBatch);
#pragma unroll
      for (int n = kBatch - 1; n >= 0; --n) {
        const int64_t seg = s0 + n0 * kBatch + n;
        if (seg >= s1) continue;
        float* at = part_of(s, NF, b, seg) + c;
        at[kE * s.C] = e;
        if constexpr (MODE == kSecond) at[kF * s.C] = f;
        pass_bwd<MODE>(e, f, [&](int k) { return run[n][k]; });
      }
    }
  for (int64_t n0 = 0; n0 < batches; ++n0) {
    if (batches > 1) load(s0 + n0 * kBatch);
#pragma unroll
    for (int n = 0; n < kBatch; ++n) {
      const int64_t seg = s0 + n0 * kBatch + n;
      if (seg >= s1) continue;
      float* at = part_of(s, NF, b, seg) + c;
      at[kX * s.C] = h;
      if constexpr (MODE == kSecond) at[kY * s.C] = y;
      pass_fwd<MODE>(h, y, [&](int k) { return run[n][k]; });
    }
  }
}

// The states that enter a chunk, from both sides: from the join, or those that
// enter the sequence.
template <int MODE, int VEC, bool JOIN>
__device__ __forceinline__ void enter(const Scan& s, const Place<VEC>& at, States<VEC>& st) {
  constexpr int NF = fields(MODE);
  const int64_t first = at.b * s.C + at.c;
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    if constexpr (!JOIN) {
      const float* from = part_of(s, NF, at.b, at.seg) + at.c + i;
      st.h[i] = from[kX * s.C];
      if constexpr (MODE >= kBwd) st.e[i] = from[kE * s.C];
      if constexpr (MODE == kSecond) {
        st.y[i] = from[kY * s.C];
        st.f[i] = from[kF * s.C];
      }
    } else {
      st.h[i] = s.state ? s.state[first + i] : 0.0f;
      st.y[i] = MODE == kSecond && s.ddstate ? s.ddstate[first + i] : 0.0f;
      st.e[i] = MODE >= kBwd && s.dstate_out ? s.dstate_out[first + i] : 0.0f;
      st.f[i] = 0.0f;
    }
  }
}

template <class E, int VEC, int U>
__device__ __forceinline__ void store_rows(const Scan& s, const HeadArr& h, const Place<VEC>& at, int64_t t0, float (*v)[VEC]) {
  E* row = static_cast<E*>(h.p) + at.b * h.sb + t0 * h.st;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (t0 + u >= at.len) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[u][i] = 0.0f;
    }
    if (t0 + u < s.T) store_pack<E, VEC>(row + at.c, v[u]);
    row += h.st;
  }
}

// A chunk's results.  JOIN: the sequence has at most kW chunks, whose runs the
// workgroup joins itself.
template <class E, int MODE, int VEC, int U, bool JOIN>
__global__ __launch_bounds__(64 * kW) void gscan_walk(Scan s) {
  __shared__ Runs<MODE, VEC> R;
  __shared__ std::conditional_t<JOIN, Runs<MODE, VEC>, char> J;
  const Place<VEC> at(s, s.from_end);
  const int lane = threadIdx.x & 63, wave = wave_of();
  const int64_t t0 = (at.seg * kW + wave) * U;
  Tokens<E, MODE, VEC, U> tok;
  tok.load(s, at, t0);
  States<VEC> st;
  enter<MODE, VEC, JOIN>(s, at, st);
  if constexpr (JOIN)
    if (s.S > 1 && wave < s.S) {  // a wave brings one chunk's run
      const float* run = part_of(s, fields(MODE), at.b, wave) + at.c;
#pragma unroll
      for (int f = 0; f < fields(MODE); ++f)
#pragma unroll
        for (int i = 0; i < VEC; ++i) J.v[wave][f][i][lane] = run[f * s.C + i];
    }
  tok.finish(at, t0);
  R.put(wave, lane, tok);
  __syncthreads();  // also: every wave has read the state that the last one may now overwrite
  if (!at.on) return;
  if constexpr (JOIN) {
    for (int c = 0; c < (int)at.seg; ++c)
#pragma unroll
      for (int i = 0; i < VEC; ++i) pass_fwd<MODE>(st.h[i], st.y[i], [&](int k) { return J.v[c][k][i][lane]; });
    if constexpr (MODE >= kBwd)
      for (int c = (int)s.S - 1; c > (int)at.seg; --c)
#pragma unroll
        for (int i = 0; i < VEC; ++i) pass_bwd<MODE>(st.e[i], st.f[i], [&](int k) { return J.v[c][k][i][lane]; });
  }
  for (int w = 0; w < wave; ++w)
#pragma unroll
    for (int i = 0; i < VEC; ++i) pass_fwd<MODE>(st.h[i], st.y[i], [&](int k) { return R.v[w][k][i][lane]; });
  if constexpr (MODE >= kBwd)
    for (int w = kW - 1; w > wave; --w)
#pragma unroll
      for (int i = 0; i < VEC; ++i) pass_bwd<MODE>(st.e[i], st.f[i], [&](int k) { return R.v[w][k][i][lane]; });
  const bool last = at.seg == s.S - 1 && wave == kW - 1, first = at.seg == 0 && wave == 0;
  const int64_t state = at.b * s.C + at.c;
  if constexpr (MODE == kFwd) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < VEC; ++i) tok.x[u][i] = st.h[i] = tok.a[u][i] * st.h[i] + tok.x[u][i];
    store_rows<E, VEC, U>(s, s.out[0], at, t0, tok.x);
    if (last && s.end)
#pragma unroll
      for (int i = 0; i < VEC; ++i) s.end[state + i] = st.h[i];
  } else if constexpr (MODE == kBwd) {
    float dlg[U][VEC];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        dlg[u][i] = st.h[i];
        st.h[i] = tok.a[u][i] * st.h[i] + tok.x[u][i];
      }
#pragma unroll
    for (int u = U - 1; u >= 0; --u)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float g = tok.dh[u][i] + st.e[i];
        st.e[i] = tok.a[u][i] * g;
        dlg[u][i] *= st.e[i];
        tok.dh[u][i] = g;
      }
    if (s.out[0].p) store_rows<E, VEC, U>(s, s.out[0], at, t0, dlg);
    if (s.out[1].p) store_rows<E, VEC, U>(s, s.out[1], at, t0, tok.dh);
    if (first && s.begin)
#pragma unroll
      for (int i = 0; i < VEC; ++i) s.begin[state + i] = st.e[i];
  } else {
    float hp[U][VEC], yp[U][VEC];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        hp[u][i] = st.h[i];
        yp[u][i] = st.y[i];
        tok.p[u][i] = st.y[i] = tok.a[u][i] * (st.y[i] + tok.r[u][i] * st.h[i]) + tok.p[u][i];
        st.h[i] = tok.a[u][i] * st.h[i] + tok.x[u][i];
      }
    store_rows<E, VEC, U>(s, s.out[0], at, t0, tok.p);
    if (last && s.end)
#pragma unroll
      for (int i = 0; i < VEC; ++i) s.end[state + i] = st.y[i];
#pragma unroll
    for (int u = U - 1; u >= 0; --u)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float a = tok.a[u][i], g = tok.dh[u][i] + st.e[i], v = tok.r[u][i] * g + st.f[i];
        tok.x[u][i] = st.f[i];
        hp[u][i] = a * (g * yp[u][i] + hp[u][i] * v);
        st.e[i] = a * g;
        st.f[i] = a * v;
      }
    store_rows<E, VEC, U>(s, s.out[1], at, t0, hp);
    store_rows<E, VEC, U>(s, s.out[2], at, t0, tok.x);
    if (first && s.begin)
#pragma unroll
      for (int i = 0; i < VEC; ++i) s.begin[state + i] = st.f[i];
  }
}

// ---- sweeps: many channels --------------------------------------------------
// With enough columns of 64 channels a workgroup takes its column through the
// whole sequence, kSweepWaves U tokens at a time, the next ones on their way: a
// forward sweep reads its operands once, where chunks of their own read them
// twice.  The backward sweep needs the states from before: a forward sweep that
// stores nothing else leaves one for each chunk.
// 128 columns occupy half of the compute units, and 16 waves each with 32 loads a lane
// on their way bring 3.2 TB/s of operands that lie in no cache (a plain copy of the same
// columns by the same workgroups is no faster); 256 columns of 2,048 tokens 6.1 TB/s.

constexpr int kSweepWaves = 16;
constexpr int kSweepU = 16, kBackU = 8;              // tokens of a wave
constexpr int kBackChunk = kSweepWaves * kBackU;     // tokens for which a state is left

struct Sweep {
  int64_t b, len, T, nk;  // nk: chunks
  uint32_t c;             // lanes past the last channel take the last one, and write what its own lane writes
  int lane, wave;
  __device__ __forceinline__ Sweep(const Scan& s, int tokens) {
    lane = threadIdx.x & 63;
    wave = wave_of();
    const uint32_t id = place_of(s, false);
    b = id / (uint32_t)s.cols;
    c = (uint32_t)(id - b * s.cols) * 64 + lane;
    if (c >= s.C) c = (uint32_t)s.C - 1;
    T = s.T;
    len = T;
    if (s.lengths) {
      const int64_t n = s.lengths[b];
      len = n < 0 ? 0 : n < len ? n : len;
    }
    nk = (T + tokens - 1) / tokens;
  }
};

// A wave's tokens of one channel a lane, as memory holds them.  FULL: all of
// them are there.
template <class E, int U>
struct Raw {
  E v[U];
  template <bool FULL>
  __device__ __forceinline__ void load(const HeadArr& h, const Sweep& w, int64_t t0) {
    const E* row = static_cast<const E*>(h.p) + w.b * h.sb + t0 * h.st;
    if (FULL || t0 < w.len) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        v[u] = row[w.c];
        if (FULL || t0 + u + 1 < w.len) row += h.st;  // else once more the last one
      }
    }
  }
  // tokens past the end are 0
  template <bool FULL>
  __device__ __forceinline__ void get(const Sweep& w, int64_t t0, float* to) const {
#pragma unroll
    for (int u = 0; u < U; ++u) to[u] = FULL || t0 + u < w.len ? (float)v[u] : 0.0f;
  }
};

template <bool FULL, class E, int U>
__device__ __forceinline__ void put_rows(const HeadArr& h, const Sweep& w, int64_t t0, const float* v) {
  E* row = static_cast<E*>(h.p) + w.b * h.sb + t0 * h.st;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (FULL || t0 + u < w.T) row[w.c] = (E)(FULL || t0 + u < w.len ? v[u] : 0.0f);
    row += h.st;
  }
}

// Forward: h and the last state, or (STATES) the state before each kBackChunk
// tokens.  Whole chunks are pipelined: their code has no condition around a load
// or a store, so that the wait for the next chunk's loads counts the stores after
// them and does not wait for those too.
template <class E, bool STATES>
struct SweepFwd {
  static constexpr int U = kSweepU, W = kSweepWaves;
  const Scan& s;
  const Sweep w;
  float h;
  Raw<E, U> lg, x;

  template <bool FULL>
  __device__ __forceinline__ void load(int64_t k) {
    const int64_t t0 = (k * W + w.wave) * U;
    lg.template load<FULL>(s.lg, w, t0);
    x.template load<FULL>(s.x, w, t0);
  }
  template <bool FULL>
  __device__ __forceinline__ void step(int64_t k, int64_t next, float (*r)[2][64]) {
    const int64_t t0 = (k * W + w.wave) * U;
    float a[U], v[U], L = 0.0f, X = 0.0f;
    lg.template get<FULL>(w, t0, a);
    x.template get<FULL>(w, t0, v);
    if (FULL) load<FULL>(next);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      L += a[u];
      a[u] = gate(a[u]);
      X = a[u] * X + v[u];
    }
    r[w.wave][0][w.lane] = gate(L);
    r[w.wave][1][w.lane] = X;
    asm volatile("" : "+v"(h));  // the state has arrived: past the barrier its place may be written
    lds_barrier();               // the other half is written only after the next one
    float mine = h;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      if (i == w.wave) mine = h;
      h = r[i][0][w.lane] * h + r[i][1][w.lane];
    }
    if constexpr (STATES) {
      if (w.wave * U % kBackChunk == 0 && t0 < w.T) s.parts[(w.b * s.S + t0 / kBackChunk) * s.C + w.c] = mine;
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = mine = a[u] * mine + v[u];
      put_rows<FULL, E, U>(s.out[0], w, t0, v);
    }
  }
};

template <class E, bool STATES>
__global__ __launch_bounds__(64 * kSweepWaves) void gscan_sweep(Scan s) {
  using F = SweepFwd<E, STATES>;
  __shared__ float R[2][F::W][2][64];
  F f{s, Sweep(s, F::W * F::U), 0.0f, {}, {}};
  const int64_t st = f.w.b * s.C + f.w.c;
  if (s.state) f.h = s.state[st];
  const int64_t full = f.w.len / (F::W * F::U);
  if (full > 0) {
    f.template load<true>(0);
    f.template step<true>(0, full > 1 ? 1 : 0, R[0]);
    for (int64_t k = 1; k < full; ++k) f.template step<true>(k, k + 1 < full ? k + 1 : k, R[k & 1]);
  }
  for (int64_t k = full; k < f.w.nk; ++k) {
    f.template load<false>(k);
    f.template step<false>(k, k, R[k & 1]);
  }
  if (!STATES && s.end && f.w.wave == 0) s.end[st] = f.h;
}

// Backward, from the last chunk to the first.
template <class E, bool DLG, bool DX>
struct SweepBwd {
  static constexpr int U = kBackU, W = kSweepWaves;
  const Scan& s;
  const Sweep w;
  float e, before;
  Raw<E, U> lg, x, dh;

  template <bool FULL>
  __device__ __forceinline__ void load(int64_t k) {
    const int64_t t0 = (k * W + w.wave) * U;
    lg.template load<FULL>(s.lg, w, t0);
    x.template load<FULL>(s.x, w, t0);
    dh.template load<FULL>(s.dh, w, t0);
    before = s.parts[(w.b * s.S + k) * s.C + w.c];
  }
  template <bool FULL>
  __device__ __forceinline__ void step(int64_t k, int64_t next, float (*r)[3][64]) {
    const int64_t t0 = (k * W + w.wave) * U;
    float a[U], v[U], g[U], L = 0.0f, X = 0.0f, E0 = 0.0f, h = before;
    lg.template get<FULL>(w, t0, a);
    x.template get<FULL>(w, t0, v);
    dh.template get<FULL>(w, t0, g);
    if (FULL) load<FULL>(next);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      L += a[u];
      a[u] = gate(a[u]);
      X = a[u] * X + v[u];
    }
#pragma unroll
    for (int u = U - 1; u >= 0; --u) E0 = a[u] * (g[u] + E0);
    r[w.wave][0][w.lane] = gate(L);
    r[w.wave][1][w.lane] = X;
    r[w.wave][2][w.lane] = E0;
    lds_barrier();  // the other half is written only after the next one
    float mine = h, back = e;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      if (i == w.wave) mine = h;
      h = r[i][0][w.lane] * h + r[i][1][w.lane];
    }
#pragma unroll
    for (int i = W - 1; i >= 0; --i) {
      if (i == w.wave) back = e;
      e = r[i][0][w.lane] * e + r[i][2][w.lane];
    }
    float dlg[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      dlg[u] = mine;
      mine = a[u] * mine + v[u];
    }
    {
#pragma clang fp contract(off)  // the same roundings whichever results are wanted
#pragma unroll
      for (int u = U - 1; u >= 0; --u) {
        g[u] = g[u] + back;
        back = a[u] * g[u];
        dlg[u] = dlg[u] * back;
      }
    }
    if constexpr (DLG) put_rows<FULL, E, U>(s.out[0], w, t0, dlg);
    if constexpr (DX) put_rows<FULL, E, U>(s.out[1], w, t0, g);
  }
};

template <class E, bool DLG, bool DX>
__global__ __launch_bounds__(64 * kSweepWaves) void gscan_back(Scan s) {
  using F = SweepBwd<E, DLG, DX>;
  __shared__ float R[2][F::W][3][64];
  F f{s, Sweep(s, F::W * F::U), 0.0f, 0.0f, {}, {}, {}};
  const int64_t st = f.w.b * s.C + f.w.c;
  if (s.dstate_out) f.e = s.dstate_out[st];
  const int64_t full = f.w.len / (F::W * F::U);
  for (int64_t k = f.w.nk - 1; k >= full; --k) {
    f.template load<false>(k);
    f.template step<false>(k, k, R[k & 1]);
  }
  if (full > 0) {
    f.template load<true>(full - 1);
    f.template step<true>(full - 1, full > 1 ? full - 2 : 0, R[(full - 1) & 1]);
    for (int64_t k = full - 2; k >= 0; --k) f.template step<true>(k, k > 0 ? k - 1 : 0, R[k & 1]);
  }
  if (s.begin && f.w.wave == 0) s.begin[st] = f.e;
}

// One token of every sequence, the state in place: the state's traffic (512 sequences of
// 4,096 channels 5.2 us, 29 MB), or the launch (2,048 channels 1.6 us).
template <class E, int VEC>
__global__ __launch_bounds__(kBlock) void gscan_one(HeadArr lg, HeadArr x, HeadArr out, float* state, int64_t C, int64_t cols, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
  if (i >= n) return;
  const int64_t b = i / cols;
  const int64_t c = (i - b * cols) * VEC;
  float g[VEC], v[VEC], h[VEC];
  float* const at = state + b * C + c;
  load_pack<float, VEC>(at, h);
  load_pack<E, VEC>(static_cast<const E*>(lg.p) + b * lg.sb + c, g);
  load_pack<E, VEC>(static_cast<const E*>(x.p) + b * x.sb + c, v);
#pragma unroll
  for (int k = 0; k < VEC; ++k) h[k] = gate(g[k]) * h[k] + v[k];
  store_pack<float, VEC>(at, h);
  store_pack<E, VEC>(static_cast<E*>(out.p) + b * out.sb + c, h);
}

// ---- host -------------------------------------------------------------------

// Tokens of a wave in sequences of one chunk, and in longer ones.  Forward in bf16 a
// lane has more of its two operands on their way: 16,384 x 2,048 channels 69.5 us, with
// 8 tokens 74.0, 12 70.8, 24 70.7 (in fp32 131.1 and 128.6; 64 tokens 5.5 and 5.2).
constexpr int kU = 8;
constexpr int long_tokens(int mode, int32_t dtype) { return mode == kFwd && dtype == DIFFOPT_BF16 ? 16 : kU; }
constexpr int64_t kChunk = kW * kU;
int64_t chunks_of(int64_t T, int mode, int32_t dtype) {
  const int64_t chunk = kW * long_tokens(mode, dtype);
  return T <= kChunk ? 1 : (T + chunk - 1) / chunk;
}

// Sweeps or chunks.  A forward sweep's step of 256 tokens takes 2.4 us until memory
// bounds it, a backward one's of 128 3.5: sweeps are for sequences of few steps, or
// enough columns of 64 channels to keep the memory busy.  bf16, columns x tokens, sweep
// and chunks: forward 1 x 256 4.9 and 7.7 us, 1 x 1024 11.0 and 11.9, 1 x 2048 19.2 and
// 11.5, 32 x 2048 19.9 and 17.6, 64 x 2048 20.5 and 24.3, 64 x 8192 69 and 66, 128 x 4096
// 40 and 68, 256 x 2048 33 and 63; backward 128 x 2048 57 and 52, 128 x 8192 282 and 231,
// 192 x 256 13.7 and 13.9, 192 x 2048 62 and 73, 256 x 1024 40 and 53, 512 x 2048 205 and 233.
// With operands that lie in no cache 128 x 4096 forward takes 62 and 71.
constexpr int64_t kSweepTokens = 1024, kSweepColumns = 64, kBackTokens = 256, kBackColumns = 192;
bool sweeps(int64_t B, int64_t T, int64_t C, int mode) {
  const int64_t cols = B * ((C + 63) / 64);
  if (mode == kFwd) return T > kChunk && (T <= kSweepTokens || cols >= kSweepColumns);
  return mode == kBwd && T >= kBackTokens && cols >= kBackColumns;
}

int64_t workspace_bytes(int64_t B, int64_t T, int64_t C, int32_t dtype, int mode) {
  if (B == 0 || C == 0) return 0;
  if (sweeps(B, T, C, mode)) return mode == kFwd ? 0 : B * ((T + kBackChunk - 1) / kBackChunk) * C * 4;
  const int64_t S = chunks_of(T, mode, dtype);
  return S == 1 ? 0 : B * S * fields(mode) * C * 4;
}

bool sizes_ok(int64_t B, int64_t T, int64_t C) {
  if (B < 0 || T < 0 || C < 0) return false;
  if (B == 0 || C == 0) return true;
  if (T > (int64_t(1) << 35) || C > (int64_t(1) << 31) || B > (int64_t(1) << 31)) return false;
  const int64_t cols = (C + 63) / 64, S = chunks_of(T, kBwd, DIFFOPT_F32);  // the most: at most 2^25, 2^29
  return cols <= kMostGroups / S && B <= kMostGroups / (cols * S);
}

// The walk begins with the chunks whose operands the runs read last, which the caches
// still hold: 1 x 16,384 x 2,048 channels forward 67.6 us, in the runs' order 69.9; second
// derivative of 4 x 2,048 x 1,024 55.1 and 57.8; backward 4 x 8,192 x 2,048 (bf16) 211 and
// 234, but where the Infinity Cache has all of them the runs' order is as fast or faster
// (2 x 4,096 x 2,048 62.3 and 57.5, 4 x 4,096 x 2,048 113.6 both).
constexpr int64_t kInfinityCache = int64_t(256) << 20;
template <class E, int MODE, int VEC>
int launch(const char* who, Scan s, int64_t B, hipStream_t st) {
  s.from_end = MODE != kBwd || 3 * B * s.T * s.C * (int64_t)sizeof(E) > kInfinityCache;
  s.cols = (int32_t)((s.C + 64 * VEC - 1) / (64 * VEC));
  const dim3 grid((unsigned)(B * s.S * s.cols)), block(64 * kW);
  if (s.S == 1 || (MODE != kFwd && s.S <= kW)) {  // forward, sweeps take what has two to eight chunks
    if constexpr (MODE != kFwd)
      if (s.S > 1) hipLaunchKernelGGL((gscan_runs<E, MODE, VEC, kU>), grid, block, 0, st, s);
    hipLaunchKernelGGL((gscan_walk<E, MODE, VEC, kU, true>), grid, block, 0, st, s);
  } else {
    constexpr int U = long_tokens(MODE, sizeof(E) == 2 ? DIFFOPT_BF16 : DIFFOPT_F32);
    hipLaunchKernelGGL((gscan_runs<E, MODE, VEC, U>), grid, block, 0, st, s);
    hipLaunchKernelGGL((gscan_join<MODE>), dim3((unsigned)(B * ((s.C + 63) / 64))), dim3(64 * kJW), 0, st, s);
    hipLaunchKernelGGL((gscan_walk<E, MODE, VEC, U, false>), grid, block, 0, st, s);
  }
  return launch_status(who);
}

template <class E, int MODE>
int launch_sweeps(const char* who, Scan s, int64_t B, hipStream_t st) {
  s.cols = (int32_t)((s.C + 63) / 64);
  s.S = (s.T + kBackChunk - 1) / kBackChunk;
  const dim3 grid((unsigned)(B * s.cols)), block(64 * kSweepWaves);
  hipLaunchKernelGGL((gscan_sweep<E, MODE == kBwd>), grid, block, 0, st, s);
  if constexpr (MODE == kBwd) {
    if (s.out[0].p && s.out[1].p) hipLaunchKernelGGL((gscan_back<E, true, true>), grid, block, 0, st, s);
    else if (s.out[0].p) hipLaunchKernelGGL((gscan_back<E, true, false>), grid, block, 0, st, s);
    else if (s.out[1].p) hipLaunchKernelGGL((gscan_back<E, false, true>), grid, block, 0, st, s);
    else hipLaunchKernelGGL((gscan_back<E, false, false>), grid, block, 0, st, s);
  }
  return launch_status(who);
}

// Two channels a lane for the second derivative in bf16, where workgroups for all compute
// units are left: 4 x 2,048 x 1,024 channels 57.9 us against 62.0, 16 x 128 x 1,024 14.8
// against 15.4, but 1 x 509 x 1,000 13.5 against 12.0; in fp32 one is as fast or faster
// (8 x 509 x 1,034 57.5 against 56.4, 2 x 300 x 512 14.3 against 11.1).
constexpr int64_t kPairGroups = 256;

// Where rows of 64 channels begin within lines of 128 bytes, workgroups of neighbouring
// columns write parts of one line, which one L2 puts together: bf16, forward and backward,
// 2 x 4,750 x 1,167 channels 32.4 and 49.7 us, over all chips 41.6 and 64.9; but 4 x 4,096
// x 2,048 backward 121 and 113.
bool within_lines(const Scan& s, int32_t dtype) {
  const int64_t size = elem_size(dtype);
  for (const HeadArr* h : {&s.lg, &s.x, &s.dh, &s.out[0], &s.out[1], &s.out[2]})
    if (h->p && (reinterpret_cast<uintptr_t>(h->p) % 128 || h->sb * size % 128 || h->st * size % 128)) return true;
  return false;
}

template <int MODE>
int run(const char* who, Scan s, int64_t B, int32_t dtype, hipStream_t st) {
  s.together = within_lines(s, dtype);
  if constexpr (MODE != kSecond)
    if (sweeps(B, s.T, s.C, MODE)) return dtype == DIFFOPT_F32 ? launch_sweeps<float, MODE>(who, s, B, st) : launch_sweeps<bf16, MODE>(who, s, B, st);
  if (dtype == DIFFOPT_F32) return launch<float, MODE, 1>(who, s, B, st);
  if constexpr (MODE == kSecond)
    if (s.C >= 128 && B * s.S * ((s.C + 127) / 128) >= kPairGroups) return launch<bf16, MODE, 2>(who, s, B, st);
  return launch<bf16, MODE, 1>(who, s, B, st);
}

struct Operand {
  const char* name;
  const diffopt_heads* given;
  HeadArr* to;
  bool optional = false;
};

// The [B][T][C] operands and results of a call: there, aligned, no result where an operand or another result begins.
int check_arrays(const char* who, int32_t dtype, std::initializer_list<Operand> operands, std::initializer_list<Operand> results) {
  for (const Operand& o : operands)
    if (int rc = check_heads(who, o.name, o.given, dtype, o.to)) return rc;
  for (const Operand& o : results)
    if (!o.optional || o.given)
      if (int rc = check_heads(who, o.name, o.given, dtype, o.to)) return rc;
  for (auto r = results.begin(); r != results.end(); ++r) {
    if (!r->to->p) continue;
    for (const Operand& o : operands)
      if (r->to->p == o.to->p) return fail(DIFFOPT_EINVAL, "%s: %s must not be %s", who, r->name, o.name);
    for (auto t = results.begin(); t != r; ++t)
      if (r->to->p == t->to->p) return fail(DIFFOPT_EINVAL, "%s: %s must not be %s", who, r->name, t->name);
  }
  return DIFFOPT_OK;
}

// An array of a call: B x T rows of `bytes` bytes, or one piece (B and T 1).
struct Extent {
  const char* name;
  const void* p;
  int64_t bytes, B = 1, T = 1, sb = 0, st = 0;  // strides in bytes
  int64_t low() const { return (sb < 0 ? sb * (B - 1) : 0) + (st < 0 ? st * (T - 1) : 0); }
  int64_t high() const { return (sb > 0 ? sb * (B - 1) : 0) + (st > 0 ? st * (T - 1) : 0) + bytes; }
  bool piece() const { return B == 1 && T == 1; }
};

Extent rows_of(const char* name, const HeadArr& h, int64_t B, int64_t T, int64_t C, int64_t size) {
  return Extent{name, T > 0 ? h.p : nullptr, C * size, B, T, B > 1 ? h.sb * size : 0, T > 1 ? h.st * size : 0};
}

// Whether from + j step lies in (-below, above) for a j of [first, last].
bool lands(int64_t from, int64_t step, int64_t first, int64_t last, int64_t below, int64_t above) {
  int64_t j = first;
  if (step < 0) {
    step = -step;
    j = -last;
    last = -first;
  }
  if (step > 0 && from + j * step <= -below) j += (-below - (from + j * step)) / step + 1;  // the first that is above -below
  return j <= last && from + j * step > -below && from + j * step < above;
}

// Whether two arrays share bytes: exact for a piece, and for rows at the same strides;
// rows at other strides meet where their spans do.
bool meet(const Extent& a, const Extent& b) {
  if (!a.p || !b.p) return false;
  const int64_t from = (int64_t)(reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(a.p));
  if (from + b.low() >= a.high() || from + b.high() <= a.low()) return false;
  if (!a.piece() && !b.piece() && (a.sb != b.sb || a.st != b.st)) return true;
  // one of b's rows begins less than a's bytes after one of a's, or less than b's before it: the shorter axis step by step
  const Extent& r = a.piece() ? b : a;
  const bool by_b = r.B <= r.T;
  for (int64_t i = by_b ? 1 - a.B : 1 - a.T; i < (by_b ? b.B : b.T); ++i)
    if (by_b ? lands(from + i * r.sb, r.st, 1 - a.T, b.T - 1, b.bytes, a.bytes) : lands(from + i * r.st, r.sb, 1 - a.B, b.B - 1, b.bytes, a.bytes)) return true;
  return false;
}

// No result shares bytes with an operand or with another result.  Strides can let rows
// of two arrays lie beside one another, so that their first addresses say little.
int check_apart(const char* who, std::initializer_list<Extent> operands, std::initializer_list<Extent> results) {
  for (auto r = results.begin(); r != results.end(); ++r) {
    for (const Extent& o : operands)
      if (meet(*r, o)) return fail(DIFFOPT_EINVAL, "%s: %s must lie apart from %s", who, r->name, o.name);
    for (auto t = results.begin(); t != r; ++t)
      if (meet(*r, *t)) return fail(DIFFOPT_EINVAL, "%s: %s must lie apart from %s", who, r->name, t->name);
  }
  return DIFFOPT_OK;
}

struct States32 {
  const char* name;
  const float* p;
};

// [B][C] states: aligned; no result over an operand or another result.
int check_states(const char* who, int64_t bytes, std::initializer_list<States32> operands, std::initializer_list<States32> results) {
  for (const auto& list : {operands, results})
    for (const States32& s : list)
      if (!aligned_to(s.p, 4)) return fail(DIFFOPT_EINVAL, "%s: %s is not 4-byte aligned", who, s.name);
  for (auto r = results.begin(); r != results.end(); ++r) {
    for (const States32& o : operands)
      if (overlap(r->p, bytes, o.p, bytes)) return fail(DIFFOPT_EINVAL, "%s: %s must lie apart from %s", who, r->name, o.name);
    for (auto t = results.begin(); t != r; ++t)
      if (overlap(r->p, bytes, t->p, bytes)) return fail(DIFFOPT_EINVAL, "%s: %s must lie apart from %s", who, r->name, t->name);
  }
  return DIFFOPT_OK;
}

int check_call(const char* who, const int32_t* lengths, int64_t B, int64_t T, int64_t C, int32_t dtype) {
  if (B < 0 || T < 0 || C < 0) return fail(DIFFOPT_EINVAL, "%s: sizes must be >= 0", who);
  if (!sizes_ok(B, T, C)) return fail(DIFFOPT_EINVAL, "%s: too many sequences, tokens or channels", who);
  if (!dtype_ok(dtype)) return fail(DIFFOPT_EINVAL, "%s: unknown element type %d", who, (int)dtype);
  if (!aligned_to(lengths, 4)) return fail(DIFFOPT_EINVAL, "%s: lengths is not 4-byte aligned", who);
  return DIFFOPT_OK;
}

int check_workspace(const char* who, int64_t B, int64_t T, int64_t C, int32_t dtype, int mode, const void* workspace, int64_t bytes) {
  const int64_t need = workspace_bytes(B, T, C, dtype, mode);
  if (need > 0 && (!workspace || bytes < need))
    return fail(DIFFOPT_EINVAL, "%s: the workspace has %lld bytes of %lld", who, (long long)(workspace ? bytes : 0), (long long)need);
  if (!aligned_to(workspace, 4)) return fail(DIFFOPT_EINVAL, "%s: the workspace is not 4-byte aligned", who);
  return DIFFOPT_OK;
}

}  // namespace
}  // namespace diffopt

using namespace diffopt;

extern "C" int64_t diffopt_gscan_workspace(int64_t B, int64_t T, int64_t C, int32_t dtype, int32_t order) {
  if (!sizes_ok(B, T, C) || !dtype_ok(dtype) || order < 0 || order > 2) return -1;
  return workspace_bytes(B, T, C, dtype, order);
}

extern "C" int diffopt_gscan_fwd(const diffopt_heads* log_gate, const diffopt_heads* x, const int32_t* lengths, const float* state, int64_t B,
                                 int64_t T, int64_t C, int32_t dtype, const diffopt_heads* h, float* state_out, void* workspace,
                                 int64_t workspace_bytes, void* stream) {
  clear_error();
  static const char* who = "diffopt_gscan_fwd";
  int rc = check_call(who, lengths, B, T, C, dtype);
  if (rc || B == 0 || C == 0) return rc;
  Scan s{};
  if (T > 0) rc = check_arrays(who, dtype, {{"log_gate", log_gate, &s.lg}, {"x", x, &s.x}}, {{"h", h, &s.out[0]}});
  const bool in_place = state && state_out == state;
  if (!rc) rc = check_states(who, 4 * B * C, {{"state", in_place ? nullptr : state}}, {{"state_out", state_out}});
  if (!rc) rc = check_workspace(who, B, T, C, dtype, kFwd, workspace, workspace_bytes);
  const auto rows = [&](const char* name, const HeadArr& h) { return rows_of(name, h, B, T, C, elem_size(dtype)); };
  const Extent ends{"lengths", lengths, 4 * B}, begin{"state", in_place ? nullptr : state, 4 * B * C};
  if (!rc) rc = check_apart(who, {rows("log_gate", s.lg), rows("x", s.x), ends, begin}, {rows("h", s.out[0]), {"state_out", state_out, 4 * B * C}});
  if (rc || (T == 0 && !state_out)) return rc;
  s.lengths = lengths;
  s.state = state;
  s.end = state_out;
  s.parts = static_cast<float*>(workspace);
  s.T = T;
  s.C = C;
  s.S = chunks_of(T, kFwd, dtype);
  return run<kFwd>(who, s, B, dtype, as_stream(stream));
}

extern "C" int diffopt_gscan_bwd(const diffopt_heads* dh, const float* dstate_out, const diffopt_heads* log_gate, const diffopt_heads* x,
                                 const int32_t* lengths, const float* state, int64_t B, int64_t T, int64_t C, int32_t dtype,
                                 const diffopt_heads* dlog_gate, const diffopt_heads* dx, float* dstate, void* workspace,
                                 int64_t workspace_bytes, void* stream) {
  clear_error();
  static const char* who = "diffopt_gscan_bwd";
  int rc = check_call(who, lengths, B, T, C, dtype);
  if (rc || B == 0 || C == 0) return rc;
  Scan s{};
  if (T > 0)
    rc = check_arrays(who, dtype, {{"log_gate", log_gate, &s.lg}, {"x", x, &s.x}, {"dh", dh, &s.dh}},
                      {{"dlog_gate", dlog_gate, &s.out[0], true}, {"dx", dx, &s.out[1], true}});
  if (!rc) rc = check_states(who, 4 * B * C, {{"state", state}, {"dstate_out", dstate_out}}, {{"dstate", dstate}});
  if (!rc) rc = check_workspace(who, B, T, C, dtype, kBwd, workspace, workspace_bytes);
  const auto rows = [&](const char* name, const HeadArr& h) { return rows_of(name, h, B, T, C, elem_size(dtype)); };
  const auto states = [&](const char* name, const float* p) { return Extent{name, p, 4 * B * C}; };
  if (!rc)
    rc = check_apart(who, {rows("log_gate", s.lg), rows("x", s.x), rows("dh", s.dh), {"lengths", lengths, 4 * B}, states("state", state), states("dstate_out", dstate_out)},
                     {rows("dlog_gate", s.out[0]), rows("dx", s.out[1]), states("dstate", dstate)});
  if (rc || ((T == 0 || (!dlog_gate && !dx)) && !dstate)) return rc;
  s.lengths = lengths;
  s.state = state;
  s.dstate_out = dstate_out;
  s.begin = dstate;
  s.parts = static_cast<float*>(workspace);
  s.T = T;
  s.C = C;
  s.S = chunks_of(T, kBwd, dtype);
  return run<kBwd>(who, s, B, dtype, as_stream(stream));
}

extern "C" int diffopt_gscan_bwd_bwd(const diffopt_heads* ddlog_gate, const diffopt_heads* ddx, const float* ddstate, const diffopt_heads* dh,
                                     const float* dstate_out, const diffopt_heads* log_gate, const diffopt_heads* x, const int32_t* lengths,
                                     const float* state, int64_t B, int64_t T, int64_t C, int32_t dtype, const diffopt_heads* out_dh,
                                     float* out_dstate_out, const diffopt_heads* out_log_gate, const diffopt_heads* out_x, float* out_state,
                                     void* workspace, int64_t workspace_bytes, void* stream) {
  clear_error();
  static const char* who = "diffopt_gscan_bwd_bwd";
  int rc = check_call(who, lengths, B, T, C, dtype);
  if (rc || B == 0 || C == 0) return rc;
  Scan s{};
  if (T > 0)
    rc = check_arrays(who, dtype,
                      {{"ddlog_gate", ddlog_gate, &s.r}, {"ddx", ddx, &s.p}, {"dh", dh, &s.dh}, {"log_gate", log_gate, &s.lg}, {"x", x, &s.x}},
                      {{"out_dh", out_dh, &s.out[0]}, {"out_log_gate", out_log_gate, &s.out[1]}, {"out_x", out_x, &s.out[2]}});
  if (!rc)
    rc = check_states(who, 4 * B * C, {{"state", state}, {"dstate_out", dstate_out}, {"ddstate", ddstate}},
                      {{"out_dstate_out", out_dstate_out}, {"out_state", out_state}});
  if (!rc) rc = check_workspace(who, B, T, C, dtype, kSecond, workspace, workspace_bytes);
  const auto rows = [&](const char* name, const HeadArr& h) { return rows_of(name, h, B, T, C, elem_size(dtype)); };
  const auto states = [&](const char* name, const float* p) { return Extent{name, p, 4 * B * C}; };
  if (!rc)
    rc = check_apart(who,
                     {rows("ddlog_gate", s.r), rows("ddx", s.p), rows("dh", s.dh), rows("log_gate", s.lg), rows("x", s.x), {"lengths", lengths, 4 * B},
                      states("state", state), states("dstate_out", dstate_out), states("ddstate", ddstate)},
                     {rows("out_dh", s.out[0]), rows("out_log_gate", s.out[1]), rows("out_x", s.out[2]), states("out_dstate_out", out_dstate_out),
                      states("out_state", out_state)});
  if (rc || (T == 0 && !out_dstate_out && !out_state)) return rc;
  s.lengths = lengths;
  s.state = state;
  s.dstate_out = dstate_out;
  s.ddstate = ddstate;
  s.end = out_dstate_out;
  s.begin = out_state;
  s.parts = static_cast<float*>(workspace);
  s.T = T;
  s.C = C;
  s.S = chunks_of(T, kSecond, dtype);
  return run<kSecond>(who, s, B, dtype, as_stream(stream));
}

extern "C" int diffopt_gscan_step(const diffopt_heads* log_gate, const diffopt_heads* x, int64_t B, int64_t C, int32_t dtype, float* state,
                                  const diffopt_heads* out, void* stream) {
  clear_error();
  static const char* who = "diffopt_gscan_step";
  int rc = check_call(who, nullptr, B, 1, C, dtype);
  if (rc || B == 0 || C == 0) return rc;
  HeadArr lg, xs, o;
  rc = check_arrays(who, dtype, {{"log_gate", log_gate, &lg}, {"x", x, &xs}}, {{"out", out, &o}});
  if (rc) return rc;
  if (!state) return fail(DIFFOPT_EINVAL, "%s: null state", who);
  if (!aligned_to(state, 4)) return fail(DIFFOPT_EINVAL, "%s: state is not 4-byte aligned", who);
  const auto rows = [&](const char* name, const HeadArr& h) { return rows_of(name, h, B, 1, C, elem_size(dtype)); };
  const Extent in_place{"state", state, 4 * B * C};
  for (const Extent& e : {rows("log_gate", lg), rows("x", xs), rows("out", o)})
    if (meet(in_place, e)) return fail(DIFFOPT_EINVAL, "%s: state must lie apart from the operands and out", who);
  rc = check_apart(who, {rows("log_gate", lg), rows("x", xs)}, {rows("out", o)});
  if (rc) return rc;
  const hipStream_t st = as_stream(stream);
  const auto go = [&](auto kernel, int vec) {
    const int64_t cols = C / vec, n = B * cols;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((n + kBlock - 1) / kBlock)), dim3(kBlock), 0, st, lg, xs, o, state, C, cols, n);
    return launch_status(who);
  };
  if (C % 4 == 0) return dtype == DIFFOPT_F32 ? go(gscan_one<float, 4>, 4) : go(gscan_one<bf16, 4>, 4);
  return dtype == DIFFOPT_F32 ? go(gscan_one<float, 1>, 1) : go(gscan_one<bf16, 1>, 1);
}
