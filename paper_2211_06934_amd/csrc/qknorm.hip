// RMS norms of queries and keys for each head with the position rotation in
// the same pass, on gfx950: forward, VJP, and the VJP's own VJP (formulas in
// diffopt.h).
//
// Every direction reads its operands once and writes its results once, so all
// are bound by memory.  A lane holds pairs of elements that the rotation turns
// together (of the rotated part, or two neighbours beyond it with the rotation
// by zero), so nothing crosses lanes but the sums over the head.  Gradients of
// the weights gather in registers over the heads a wave walks, then over the
// workgroup in LDS, then over workgroups in a second small launch: a fixed
// order, no atomics.
// Widths that fall into pairs of 16-byte pieces take qknorm_pieces, others
// qknorm_any, a wave per head with single elements.
#include <algorithm>
#include <initializer_list>

#include "lm_common.hpp"

namespace diffopt {
namespace {

constexpr int kQB = 256;        // threads per workgroup
constexpr int kQWaves = kQB / 64;
constexpr int kMaxBlocks = 2048;  // workgroups per launch (they walk the heads)

struct QkShape {
  int64_t B, T;
  int32_t H, Hk, D, rot, interleaved;
  float inv_d, eps;
  const float *cos, *sin;
  int64_t rows, first;
  const void* positions;
  int32_t position_bytes;
};

// What a direction reads and writes for q (0) and k (1).
struct QkArgs {
  HeadArr x[2], dy[2], a[2], o0[2], o1[2];
  const float *w[2], *b[2];
  float* dw[2];     // results: the weights' gradients (NULL: not wanted)
  float* partial;   // [workgroup][D] of either side, q's workgroups first
};

enum Dir { kFwd, kBwd, kSecond };

template <class E>
__device__ __forceinline__ const E* row_of(const HeadArr& h, int64_t b, int64_t t, int64_t head) {
  return static_cast<const E*>(h.p) + b * h.sb + t * h.st + head * h.sh;
}

__device__ __forceinline__ int64_t position_of(const QkShape& s, int64_t b, int64_t t) {
  if (!s.positions) return s.first + t;
  const int64_t at = b * s.T + t;
  return s.position_bytes == 4 ? (int64_t) static_cast<const int32_t*>(s.positions)[at]
                               : static_cast<const int64_t*>(s.positions)[at];
}

// Any width and few heads: NP pairs per lane, heads of up to 128 NP elements, a wave
// for each.  Element by element, so bound by the number of loads: 16,384 tokens of 40
// heads of 128 in bf16 take 219 us forward and 415 backward, where pieces take 63 and
// 111; one token's 3.0 and 3.4 us are latency.
template <class E, int DIR, int NP>
__global__ __launch_bounds__(kQB) void qknorm_any(QkShape s, QkArgs A, int32_t q_blocks) {
  const int side = (int)blockIdx.x >= q_blocks;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int heads = side ? s.Hk : s.H;
  const int64_t nrow = s.B * s.T * heads;
  const int64_t blk = (int64_t)blockIdx.x - (side ? q_blocks : 0), nblk = side ? (int64_t)gridDim.x - q_blocks : q_blocks;
  const HeadArr X = A.x[side], DY = A.dy[side], AA = A.a[side], O0 = A.o0[side], O1 = A.o1[side];
  const int half = s.rot >> 1, pairs = (s.D + 1) >> 1;

  // where the pairs lie, and what does not change from head to head
  int e0[NP], e1[NP];
  float w0[NP], w1[NP], b0[NP], b1[NP], g0[NP], g1[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int p = lane + 64 * i;
    int u = -1, v = -1;
    if (p < half) {
      u = s.interleaved ? 2 * p : p;
      v = s.interleaved ? 2 * p + 1 : p + half;
    } else if (p < pairs) {
      u = 2 * p;
      v = 2 * p + 1 < s.D ? 2 * p + 1 : -1;
    }
    e0[i] = u;
    e1[i] = v;
    const float* w = A.w[side];
    w0[i] = u >= 0 ? (w ? w[u] : 1.0f) : 0.0f;
    w1[i] = v >= 0 ? (w ? w[v] : 1.0f) : 0.0f;
    const float* b = DIR == kSecond ? A.b[side] : nullptr;
    b0[i] = b && u >= 0 ? b[u] : 0.0f;
    b1[i] = b && v >= 0 ? b[v] : 0.0f;
    g0[i] = g1[i] = 0.0f;
  }

  for (int64_t r = blk * kQWaves + wave; r < nrow; r += nblk * kQWaves) {
    const int64_t h = r % heads, bt = r / heads, b = bt / s.T, t = bt - b * s.T;
    const int64_t pos = position_of(s, b, t);
    const bool known = s.rot == 0 || (pos >= 0 && pos < s.rows);
    const E* x = row_of<E>(X, b, t, h);
    float x0[NP], x1[NP], c[NP], sn[NP];
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int p = lane + 64 * i;
      x0[i] = e0[i] >= 0 ? (float)x[e0[i]] : 0.0f;
      x1[i] = e1[i] >= 0 ? (float)x[e1[i]] : 0.0f;
      ss += x0[i] * x0[i] + x1[i] * x1[i];
      c[i] = 1.0f;
      sn[i] = 0.0f;
      if (p < half) {
        c[i] = known ? s.cos[pos * half + p] : kNan;
        sn[i] = known ? s.sin[pos * half + p] : kNan;
      } else if (!known) {
        c[i] = sn[i] = kNan;
      }
    }
    const float rr = rsqrtf(wave_sum(ss) * s.inv_d + s.eps);
    if (DIR == kFwd) {
      E* y = const_cast<E*>(row_of<E>(O0, b, t, h));
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const float z0 = w0[i] * (x0[i] * rr), z1 = w1[i] * (x1[i] * rr);
        if (e0[i] >= 0) y[e0[i]] = (E)(z0 * c[i] - z1 * sn[i]);
        if (e1[i] >= 0) y[e1[i]] = (E)(z1 * c[i] + z0 * sn[i]);
      }
      continue;
    }
    // xn = x r, dz the cotangent rotated back, u = w dz
    const E* dy = row_of<E>(DY, b, t, h);
    float z0[NP], z1[NP], xu = 0.0f;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      x0[i] *= rr;
      x1[i] *= rr;
      const float y0 = e0[i] >= 0 ? (float)dy[e0[i]] : 0.0f, y1 = e1[i] >= 0 ? (float)dy[e1[i]] : 0.0f;
      z0[i] = y0 * c[i] + y1 * sn[i];
      z1[i] = y1 * c[i] - y0 * sn[i];
      xu += x0[i] * w0[i] * z0[i] + x1[i] * w1[i] * z1[i];
    }
    xu = wave_sum(xu) * s.inv_d;
    if (DIR == kBwd) {
      E* dx = const_cast<E*>(row_of<E>(O0, b, t, h));
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        if (e0[i] >= 0) dx[e0[i]] = (E)(rr * (w0[i] * z0[i] - x0[i] * xu));
        if (e1[i] >= 0) dx[e1[i]] = (E)(rr * (w1[i] * z1[i] - x1[i] * xu));
        g0[i] += z0[i] * x0[i];
        g1[i] += z1[i] * x1[i];
      }
      continue;
    }
    const E* ap = row_of<E>(AA, b, t, h);
    float a0[NP], a1[NP], xa = 0.0f, au = 0.0f, bz = 0.0f;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      a0[i] = AA.p && e0[i] >= 0 ? (float)ap[e0[i]] : 0.0f;
      a1[i] = AA.p && e1[i] >= 0 ? (float)ap[e1[i]] : 0.0f;
      xa += x0[i] * a0[i] + x1[i] * a1[i];
      au += a0[i] * w0[i] * z0[i] + a1[i] * w1[i] * z1[i];
      bz += b0[i] * x0[i] * z0[i] + b1[i] * x1[i] * z1[i];
    }
    xa = wave_sum(xa) * s.inv_d;
    au = wave_sum(au) * s.inv_d;
    bz = wave_sum(bz) * s.inv_d;
    E* oy = const_cast<E*>(row_of<E>(O0, b, t, h));
    E* ox = const_cast<E*>(row_of<E>(O1, b, t, h));
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const float t0 = rr * (a0[i] - x0[i] * xa), t1 = rr * (a1[i] - x1[i] * xa);  // derivative of x r along a
      const float v0 = w0[i] * t0 + b0[i] * x0[i], v1 = w1[i] * t1 + b1[i] * x1[i];
      const float u0 = w0[i] * z0[i], u1 = w1[i] * z1[i];
      const float q0 = rr * (x0[i] * (3.0f * xu * xa - au) - u0 * xa - a0[i] * xu) + b0[i] * z0[i] - x0[i] * bz;
      const float q1 = rr * (x1[i] * (3.0f * xu * xa - au) - u1 * xa - a1[i] * xu) + b1[i] * z1[i] - x1[i] * bz;
      if (e0[i] >= 0) {
        oy[e0[i]] = (E)(v0 * c[i] - v1 * sn[i]);
        ox[e0[i]] = (E)(rr * q0);
      }
      if (e1[i] >= 0) {
        oy[e1[i]] = (E)(v1 * c[i] + v0 * sn[i]);
        ox[e1[i]] = (E)(rr * q1);
      }
      g0[i] += z0[i] * t0;
      g1[i] += z1[i] * t1;
    }
  }
  if (DIR == kFwd || !A.dw[side]) return;
  __shared__ float sum[kQWaves][128 * NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    if (e0[i] >= 0) sum[wave][e0[i]] = g0[i];
    if (e1[i] >= 0) sum[wave][e1[i]] = g1[i];
  }
  __syncthreads();
  for (int d = threadIdx.x; d < s.D; d += kQB) {
    float v = sum[0][d];
    for (int w = 1; w < kQWaves; ++w) v += sum[w][d];
    A.partial[(int64_t)blockIdx.x * s.D + d] = v;
  }
}

// Heads in 16-byte pieces: a lane holds two of them, VN pairs, a head takes L
// lanes of a group of LPG and a wave 64 / LPG heads at a time.  A wave takes a
// token (or one of the `per` parts of its heads, where there are few tokens) and
// walks its heads, so that the rotation's row is read once and the weights stay
// in registers.  The launch covers the card with as many workgroups as
// it holds at once, which walk the tokens (piece_blocks).

template <class E, int DIR, int LPG, bool INTER>
__global__ __launch_bounds__(kQB) void qknorm_pieces(QkShape s, QkArgs A, int32_t per) {
  constexpr int VN = Vec<E>::N, HPW = 64 / LPG;  // pairs of a lane, heads of a wave
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l = lane % LPG, sub = lane / LPG;
  const int turned = s.rot / (2 * VN);  // lanes with rotated pairs
  const bool on = l < s.D / (2 * VN), rotated = l < turned;
  const int half = s.rot >> 1;
  // first elements of the lane's two pieces
  const int u = rotated && !INTER ? VN * l : 2 * VN * l, v = rotated && !INTER ? half + VN * l : u + VN;

  // pairs (a[i], c[i]) of the lane's 2 VN elements
  auto get = [&](const E* p, float* a, float* c) {
    typename Vec<E>::type x{}, y{};
    if (on) {
      x = load_vec(p + u);
      y = load_vec(p + v);
    }
#pragma unroll
    for (int i = 0; i < VN; ++i) {
      a[i] = INTER ? (float)(2 * i < VN ? x[2 * i % VN] : y[2 * i % VN]) : (float)x[i];
      c[i] = INTER ? (float)(2 * i < VN ? x[(2 * i + 1) % VN] : y[(2 * i + 1) % VN]) : (float)y[i];
    }
  };
  auto put = [&](E* p, const float* a, const float* c) {
    float x[VN], y[VN];
#pragma unroll
    for (int i = 0; i < VN; ++i) {
      x[i] = INTER ? (i & 1 ? c[i / 2] : a[i / 2]) : a[i];
      y[i] = INTER ? (i & 1 ? c[(VN + i) / 2] : a[(VN + i) / 2]) : c[i];
    }
    if (on) {
      store_vec(p + u, x);
      store_vec(p + v, y);
    }
  };
  auto get_weights = [&](const float* w, float none, float* a, float* c) {
#pragma unroll
    for (int i = 0; i < VN; ++i) {
      const int first = INTER ? u + 2 * i : u + i, second = INTER ? u + 2 * i + 1 : v + i;
      a[i] = on ? (w ? w[first] : none) : 0.0f;
      c[i] = on ? (w ? w[second] : none) : 0.0f;
    }
  };
  auto group_sum = [](float x) {
#pragma unroll
    for (int o = 1; o < LPG; o <<= 1) x += __shfl_xor(x, o, 64);
    return x;
  };

  float wa[2][VN], wc[2][VN], ba[2][VN], bc[2][VN], ga[2][VN], gc[2][VN];
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    get_weights(A.w[side], 1.0f, wa[side], wc[side]);
    if (DIR == kSecond) get_weights(A.b[side], 0.0f, ba[side], bc[side]);
#pragma unroll
    for (int i = 0; i < VN; ++i) ga[side][i] = gc[side][i] = 0.0f;
  }

  const int64_t items = s.B * s.T * per, step = (int64_t)gridDim.x * kQWaves;
  for (int64_t item = (int64_t)blockIdx.x * kQWaves + wave; item < items; item += step) {
    const uint32_t tok = (uint32_t)item / (uint32_t)per, part = (uint32_t)item - tok * (uint32_t)per;
    const uint32_t b = tok / (uint32_t)s.T, t = tok - b * (uint32_t)s.T;
    const int64_t pos = position_of(s, b, t);
    const bool known = s.rot == 0 || (pos >= 0 && pos < s.rows);
    float cs[VN], sn[VN];
#pragma unroll
    for (int i = 0; i < VN; ++i) {
      cs[i] = known ? 1.0f : kNan;
      sn[i] = known ? 0.0f : kNan;
    }
    if (known && rotated) {
      const float *pc = s.cos + pos * half + VN * l, *psn = s.sin + pos * half + VN * l;
#pragma unroll
      for (int q = 0; q < VN; q += 4) {
        const auto x = load_vec(pc + q), y = load_vec(psn + q);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          cs[q + i] = x[i];
          sn[q + i] = y[i];
        }
      }
    }
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      const int heads = side ? s.Hk : s.H;
      for (int h0 = (int)part * HPW; h0 < heads; h0 += (int)per * HPW) {
        const int h = h0 + sub < heads ? h0 + sub : heads - 1;  // the last groups repeat the last head, and store nothing
        const bool own = h0 + sub < heads;
        const E* x = row_of<E>(A.x[side], b, t, h);
        float xa[VN], xc[VN], ss = 0.0f;
        get(x, xa, xc);
        float ya[VN], yc[VN], aa[VN], ac[VN];
        if (DIR != kFwd) get(row_of<E>(A.dy[side], b, t, h), ya, yc);
        if (DIR == kSecond) {
          if (A.a[side].p) {
            get(row_of<E>(A.a[side], b, t, h), aa, ac);
          } else {
#pragma unroll
            for (int i = 0; i < VN; ++i) aa[i] = ac[i] = 0.0f;
          }
        }
#pragma unroll
        for (int i = 0; i < VN; ++i) ss += xa[i] * xa[i] + xc[i] * xc[i];
        const float rr = rsqrtf(group_sum(ss) * s.inv_d + s.eps);
        if (DIR == kFwd) {
          float oa[VN], oc[VN];
#pragma unroll
          for (int i = 0; i < VN; ++i) {
            const float z0 = wa[side][i] * (xa[i] * rr), z1 = wc[side][i] * (xc[i] * rr);
            oa[i] = z0 * cs[i] - z1 * sn[i];
            oc[i] = z1 * cs[i] + z0 * sn[i];
          }
          if (own) put(const_cast<E*>(row_of<E>(A.o0[side], b, t, h)), oa, oc);
          continue;
        }
        // x r, the cotangent turned back, u = w dz
        float za[VN], zc[VN], xu = 0.0f;
#pragma unroll
        for (int i = 0; i < VN; ++i) {
          xa[i] *= rr;
          xc[i] *= rr;
          za[i] = ya[i] * cs[i] + yc[i] * sn[i];
          zc[i] = yc[i] * cs[i] - ya[i] * sn[i];
          xu += xa[i] * wa[side][i] * za[i] + xc[i] * wc[side][i] * zc[i];
        }
        if (DIR == kBwd) {
          xu = group_sum(xu) * s.inv_d;
          float oa[VN], oc[VN];
#pragma unroll
          for (int i = 0; i < VN; ++i) {
            oa[i] = rr * (wa[side][i] * za[i] - xa[i] * xu);
            oc[i] = rr * (wc[side][i] * zc[i] - xc[i] * xu);
            ga[side][i] += own ? za[i] * xa[i] : 0.0f;
            gc[side][i] += own ? zc[i] * xc[i] : 0.0f;
          }
          if (own) put(const_cast<E*>(row_of<E>(A.o0[side], b, t, h)), oa, oc);
          continue;
        }
        float xa_ = 0.0f, au = 0.0f, bz = 0.0f;
#pragma unroll
        for (int i = 0; i < VN; ++i) {
          xa_ += xa[i] * aa[i] + xc[i] * ac[i];
          au += aa[i] * wa[side][i] * za[i] + ac[i] * wc[side][i] * zc[i];
          bz += ba[side][i] * xa[i] * za[i] + bc[side][i] * xc[i] * zc[i];
        }
        xu = group_sum(xu) * s.inv_d;
        xa_ = group_sum(xa_) * s.inv_d;
        au = group_sum(au) * s.inv_d;
        bz = group_sum(bz) * s.inv_d;
        float oa[VN], oc[VN], pa[VN], pc[VN];
#pragma unroll
        for (int i = 0; i < VN; ++i) {
          const float t0 = rr * (aa[i] - xa[i] * xa_), t1 = rr * (ac[i] - xc[i] * xa_);  // derivative of x r along a
          const float v0 = wa[side][i] * t0 + ba[side][i] * xa[i], v1 = wc[side][i] * t1 + bc[side][i] * xc[i];
          oa[i] = v0 * cs[i] - v1 * sn[i];
          oc[i] = v1 * cs[i] + v0 * sn[i];
          const float k = 3.0f * xu * xa_ - au;
          pa[i] = rr * (rr * (xa[i] * k - wa[side][i] * za[i] * xa_ - aa[i] * xu) + ba[side][i] * za[i] - xa[i] * bz);
          pc[i] = rr * (rr * (xc[i] * k - wc[side][i] * zc[i] * xa_ - ac[i] * xu) + bc[side][i] * zc[i] - xc[i] * bz);
          ga[side][i] += own ? za[i] * t0 : 0.0f;
          gc[side][i] += own ? zc[i] * t1 : 0.0f;
        }
        if (own) {
          put(const_cast<E*>(row_of<E>(A.o0[side], b, t, h)), oa, oc);
          put(const_cast<E*>(row_of<E>(A.o1[side], b, t, h)), pa, pc);
        }
      }
    }
  }
  if (DIR == kFwd || (!A.dw[0] && !A.dw[1])) return;
  __shared__ float sum[kQWaves][2][2 * VN * LPG];
#pragma unroll
  for (int side = 0; side < 2; ++side)
#pragma unroll
    for (int i = 0; i < VN; ++i) {
      float x = ga[side][i], y = gc[side][i];
#pragma unroll
      for (int o = LPG; o < 64; o <<= 1) {
        x += __shfl_xor(x, o, 64);
        y += __shfl_xor(y, o, 64);
      }
      if (sub == 0 && on) {
        sum[wave][side][INTER ? u + 2 * i : u + i] = x;
        sum[wave][side][INTER ? u + 2 * i + 1 : v + i] = y;
      }
    }
  __syncthreads();
  for (int d = threadIdx.x; d < 2 * s.D; d += kQB) {
    const int side = d >= s.D, e = side ? d - s.D : d;
    float x = sum[0][side][e];
#pragma unroll
    for (int w = 1; w < kQWaves; ++w) x += sum[w][side][e];
    A.partial[((int64_t)side * gridDim.x + blockIdx.x) * s.D + e] = x;
  }
}

// dw[d] = the sum of the workgroups' parts: one workgroup per 8 elements of a side,
// 32 rows of parts at a time; bound by latency (768 parts of 128 elements of two
// sides, 0.8 MB: 4.9 us).
constexpr int kRB = 256, kRCols = 8, kRRows = kRB / kRCols;
__global__ __launch_bounds__(kRB) void qknorm_weights(const float* partial, int32_t q_blocks, int32_t k_blocks, int32_t D,
                                                      float* dwq, float* dwk) {
  __shared__ float sum[kRRows][kRCols + 1];
  const int side = blockIdx.y, col = threadIdx.x % kRCols, row = threadIdx.x / kRCols;
  float* dw = side ? dwk : dwq;
  if (!dw) return;
  const int d = blockIdx.x * kRCols + col, n = side ? k_blocks : q_blocks;
  const float* p = partial + (side ? (int64_t)q_blocks * D : 0);
  float v = 0.0f;
  if (d < D) {
#pragma unroll 8
    for (int i = row; i < n; i += kRRows) v += p[(int64_t)i * D + d];
  }
  sum[row][col] = v;
  __syncthreads();
  if (row == 0 && d < D) {
    for (int i = 1; i < kRRows; ++i) v += sum[i][col];
    dw[d] = v;
  }
}

// ---- host -------------------------------------------------------------------

// The workgroups of each side's partial sums.
struct Blocks {
  int32_t q, k;
};

// How a call is launched, by its sizes alone.
struct Plan {
  bool pieces;
  int32_t lpg, per;  // pieces: lanes of a head's group, waves of a token
  int32_t grid;
  Blocks blocks;
};

// Workgroups of a launch in pieces: what the registers of a direction let the card
// hold at once, so that all walk the same share.  Four a compute unit forward (five
// fit and take the same 63 us for 16,384 tokens of 40 heads of 128 in bf16, 5.3
// TB/s); three in the backward (111 us, 4.6 TB/s; four, of which one waits for its
// turn, 123) and in fp32's second one (18.5 us for 4,072 tokens of 16 heads of 64;
// four 21.1); two in bf16's (all three directions of 16,384 tokens of 40 heads of 128:
// 355 us, three 381; of 4,072 tokens of 16 heads of 64 50 and 59).
int64_t piece_blocks(int32_t dtype, Dir dir) { return 256 * (dir == kFwd ? 4 : dir == kSecond && dtype == DIFFOPT_BF16 ? 2 : 3); }

// Widths that fall into pairs of pieces, with up to 32 lanes a head, and counts
// of tokens that 32 bits index.  Calls of few heads take a wave for each instead,
// which starts sooner (40 heads of 128 in bf16, forward and backward: 3.0 and 3.4
// us against 3.6 and 4.5; 64 tokens of them 3.6 and 3.9 against 3.9 and 4.8; but
// 1,024 tokens 14.4 and 18.2 against 6.3 and 8.5).
constexpr double kFewHeads = 4096.0;

Plan plan_of(int64_t B, int64_t T, int64_t H, int64_t Hk, int64_t D, int64_t rot, int32_t dtype, Dir dir) {
  const int64_t most = piece_blocks(dtype, dir);
  Plan p{};
  const int two = dtype == DIFFOPT_F32 ? 8 : 16;  // elements of a lane
  const int64_t lanes = D / two;
  if (D % two == 0 && rot % two == 0 && (double)B * T * (H + Hk) > kFewHeads && lanes <= (dtype == DIFFOPT_F32 ? 32 : 16) && (double)B * T * 256.0 < 2147483648.0 && B * T > 0) {
    p.pieces = true;
    for (p.lpg = 4; p.lpg < lanes;) p.lpg *= 2;
    // a token's heads are split until the card has waves enough
    const int64_t hpw = 64 / p.lpg, parts = std::max((H + hpw - 1) / hpw, (Hk + hpw - 1) / hpw);
    int64_t per = most * kQWaves / (B * T);
    per = per < 1 ? 1 : per > parts ? parts : per;
    if (per > 256) per = 256;
    if (per < 1) per = 1;
    p.per = (int32_t)per;
    const int64_t need = (B * T * per + kQWaves - 1) / kQWaves;
    p.grid = (int32_t)(need < most ? need : most);
    p.blocks = Blocks{p.grid, p.grid};
    return p;
  }
  const double nq = (double)B * T * H, nk = (double)B * T * Hk;
  auto side = [&](double n) -> int32_t {  // a wave per head up to kMaxBlocks workgroups in all
    if (n == 0) return 0;
    double b = std::ceil(n / kQWaves);
    const double share = std::floor(kMaxBlocks * (n / (nq + nk)));
    if (b > share) b = share;
    return b < 1 ? 1 : (int32_t)b;
  };
  p.blocks = Blocks{side(nq), side(nk)};
  p.grid = p.blocks.q + p.blocks.k;
  return p;
}

bool sizes_ok(int64_t B, int64_t T, int64_t H, int64_t Hk, int64_t D) {
  return B >= 0 && T >= 0 && H >= 0 && Hk >= 0 && D >= 1 && D <= 1024 && H <= 65536 && Hk <= 65536;
}

int check_shape(const char* who, const float* cos, const float* sin, int64_t rows, const void* positions,
                int32_t position_bytes, int64_t first, int64_t B, int64_t T, int64_t H, int64_t Hk, int64_t D,
                int64_t rot, int32_t interleaved, int32_t dtype, double eps, QkShape* s) {
  if (!sizes_ok(B, T, H, Hk, D)) return fail(DIFFOPT_EINVAL, "%s: sizes must be >= 0, heads <= 65536, D in [1, 1024]", who);
  if (rot < 0 || rot > D || (rot & 1)) return fail(DIFFOPT_EINVAL, "%s: rot must be even and in [0, D]", who);
  if (!dtype_ok(dtype)) return fail(DIFFOPT_EINVAL, "%s: unknown element type %d", who, (int)dtype);
  if (!(std::isfinite(eps) && eps >= 0.0)) return fail(DIFFOPT_EINVAL, "%s: eps must be finite and >= 0", who);
  if (rot > 0 && (!cos || !sin)) return fail(DIFFOPT_EINVAL, "%s: null cos or sin", who);
  if (rot > 0 && rows < 0) return fail(DIFFOPT_EINVAL, "%s: rows must be >= 0", who);
  if (positions && position_bytes != 4 && position_bytes != 8)
    return fail(DIFFOPT_EINVAL, "%s: position_bytes must be 4 or 8", who);
  if (positions && !aligned_to(positions, position_bytes))
    return fail(DIFFOPT_EINVAL, "%s: positions is not aligned to its elements", who);
  if (!aligned_to(cos, 4) || !aligned_to(sin, 4)) return fail(DIFFOPT_EINVAL, "%s: cos or sin is not 4-byte aligned", who);
  if (!positions && rot > 0 && (first < 0 || T > rows || first > rows - T))
    return fail(DIFFOPT_EINVAL, "%s: positions %lld to %lld are outside the %lld rows of cos and sin", who, (long long)first,
                (long long)(first + T - 1), (long long)rows);
  *s = QkShape{B, T, (int32_t)H, (int32_t)Hk, (int32_t)D, (int32_t)rot, interleaved, (float)(1.0 / (double)D), (float)eps,
               cos, sin, rows, first, positions, position_bytes};
  return DIFFOPT_OK;
}

template <class E, int DIR>
void launch_any(const QkShape& s, const QkArgs& A, const Plan& p, hipStream_t st) {
  const dim3 grid((unsigned)p.grid), block(kQB);
  if (s.D <= 128)
    hipLaunchKernelGGL((qknorm_any<E, DIR, 1>), grid, block, 0, st, s, A, p.blocks.q);
  else if (s.D <= 256)
    hipLaunchKernelGGL((qknorm_any<E, DIR, 2>), grid, block, 0, st, s, A, p.blocks.q);
  else
    hipLaunchKernelGGL((qknorm_any<E, DIR, 8>), grid, block, 0, st, s, A, p.blocks.q);
}

template <class E, int DIR, bool INTER>
void launch_pieces(const QkShape& s, const QkArgs& A, const Plan& p, hipStream_t st) {
  const dim3 grid((unsigned)p.grid), block(kQB);
  if (p.lpg == 4) hipLaunchKernelGGL((qknorm_pieces<E, DIR, 4, INTER>), grid, block, 0, st, s, A, p.per);
  if (p.lpg == 8) hipLaunchKernelGGL((qknorm_pieces<E, DIR, 8, INTER>), grid, block, 0, st, s, A, p.per);
  if (p.lpg == 16) hipLaunchKernelGGL((qknorm_pieces<E, DIR, 16, INTER>), grid, block, 0, st, s, A, p.per);
  if constexpr (sizeof(E) == 4)
    if (p.lpg == 32) hipLaunchKernelGGL((qknorm_pieces<E, DIR, 32, INTER>), grid, block, 0, st, s, A, p.per);
}

template <class E, int DIR>
void launch_dir(const QkShape& s, const QkArgs& A, const Plan& p, hipStream_t st) {
  if (!p.pieces)
    launch_any<E, DIR>(s, A, p, st);
  else if (s.interleaved)
    launch_pieces<E, DIR, true>(s, A, p, st);
  else
    launch_pieces<E, DIR, false>(s, A, p, st);
}

template <int DIR>
int launch(const char* who, const QkShape& s, const QkArgs& A, int32_t dtype, hipStream_t st) {
  const Plan p = plan_of(s.B, s.T, s.H, s.Hk, s.D, s.rot, dtype, (Dir)DIR);
  if (p.grid > 0) {
    if (dtype == DIFFOPT_F32)
      launch_dir<float, DIR>(s, A, p, st);
    else
      launch_dir<bf16, DIR>(s, A, p, st);
    const int rc = launch_status(who);
    if (rc) return rc;
  }
  if (DIR != kFwd && (A.dw[0] || A.dw[1])) {
    hipLaunchKernelGGL(qknorm_weights, dim3((unsigned)((s.D + kRCols - 1) / kRCols), 2), dim3(kRB), 0, st, A.partial, p.blocks.q,
                       p.blocks.k, s.D, A.dw[0], A.dw[1]);
    return launch_status(who);
  }
  return DIFFOPT_OK;
}

// Partial sums of any call of these sizes, whatever its element type.
int64_t workspace_of(int64_t B, int64_t T, int64_t H, int64_t Hk, int64_t D) {
  int64_t most = 0;
  for (int32_t dtype : {DIFFOPT_F32, DIFFOPT_BF16})
    for (int64_t rot : {(int64_t)0, (int64_t)1})  // 1: a rotated part that does not fall into pieces
      for (Dir dir : {kBwd, kSecond}) {
        const Plan p = plan_of(B, T, H, Hk, D, rot, dtype, dir);
        const int64_t n = ((int64_t)p.blocks.q + p.blocks.k) * D * 4;
        most = n > most ? n : most;
      }
  return most;
}

int check_workspace(const char* who, const QkShape& s, QkArgs* A, void* workspace, int64_t bytes) {
  if (!A->dw[0] && !A->dw[1]) return DIFFOPT_OK;
  const int64_t need = workspace_of(s.B, s.T, s.H, s.Hk, s.D);
  if (need > 0 && (!workspace || bytes < need))
    return fail(DIFFOPT_EINVAL, "%s: the workspace has %lld bytes of %lld", who, (long long)(workspace ? bytes : 0), (long long)need);
  if (!aligned_to(workspace, 4)) return fail(DIFFOPT_EINVAL, "%s: the workspace is not 4-byte aligned", who);
  A->partial = static_cast<float*>(workspace);
  return DIFFOPT_OK;
}

// Operands of q and, where there are k heads, of k.
int check_both(const char* who, const char* what, const diffopt_heads* q, const diffopt_heads* k, const QkShape& s, int32_t dtype,
               HeadArr out[2]) {
  int rc = DIFFOPT_OK;
  if (s.H > 0) rc = check_heads(who, what, q, dtype, &out[0]);
  if (!rc && s.Hk > 0) rc = check_heads(who, what, k, dtype, &out[1]);
  return rc;
}

// A head's results may take the place of its operands, which the same lanes have read
// by then: the same tensor of the same side.  Anything else at one address (q's results
// over k's operands, rows another distance apart, two results) would be written while
// other waves read it.
int check_apart(const char* who, const QkShape& s, std::initializer_list<const HeadArr*> results, std::initializer_list<const HeadArr*> operands,
                float* const dw[2]) {
  const int64_t heads[2] = {s.H, s.Hk};
  auto same = [&](const HeadArr& a, const HeadArr& b, int side) {
    return (s.B <= 1 || a.sb == b.sb) && (s.T <= 1 || a.st == b.st) && (heads[side] <= 1 || a.sh == b.sh);
  };
  for (auto r = results.begin(); r != results.end(); ++r)
    for (int i = 0; i < 2; ++i) {
      const HeadArr& x = (*r)[i];
      if (!x.p) continue;
      for (const HeadArr* o : operands)
        for (int j = 0; j < 2; ++j)
          if (x.p == o[j].p && !(i == j && same(x, o[j], i)))
            return fail(DIFFOPT_EINVAL, "%s: a result must not be an operand of other heads or strides", who);
      for (auto t = results.begin(); t <= r; ++t)
        for (int j = 0; j < (t == r ? i : 2); ++j)
          if (x.p == (*t)[j].p) return fail(DIFFOPT_EINVAL, "%s: two results must not be one tensor", who);
    }
  if (overlap(dw[0], s.D * 4, dw[1], s.D * 4)) return fail(DIFFOPT_EINVAL, "%s: two results must not be one tensor", who);
  return DIFFOPT_OK;
}

int check_floats(const char* who, const float* const* p, int n) {
  for (int i = 0; i < n; ++i)
    if (!aligned_to(p[i], 4)) return fail(DIFFOPT_EINVAL, "%s: pointer %p is not 4-byte aligned", who, (const void*)p[i]);
  return DIFFOPT_OK;
}

}  // namespace
}  // namespace diffopt

using namespace diffopt;

extern "C" int64_t diffopt_qknorm_rope_workspace(int64_t B, int64_t T, int64_t H, int64_t Hk, int64_t D) {
  if (!sizes_ok(B, T, H, Hk, D)) return -1;
  return workspace_of(B, T, H, Hk, D);
}

extern "C" int diffopt_qknorm_rope_fwd(const diffopt_heads* q, const diffopt_heads* k, const float* q_weight,
                                       const float* k_weight, const float* cos, const float* sin, int64_t rows,
                                       const void* positions, int32_t position_bytes, int64_t first, int64_t B,
                                       int64_t T, int64_t H, int64_t Hk, int64_t D, int64_t rot, int32_t interleaved,
                                       int32_t dtype, double eps, const diffopt_heads* q_out,
                                       const diffopt_heads* k_out, void* stream) {
  clear_error();
  static const char* who = "diffopt_qknorm_rope_fwd";
  QkShape s;
  int rc = check_shape(who, cos, sin, rows, positions, position_bytes, first, B, T, H, Hk, D, rot, interleaved, dtype, eps, &s);
  if (rc || B == 0 || T == 0) return rc;
  QkArgs A{};
  rc = check_both(who, "q or k", q, k, s, dtype, A.x);
  if (!rc) rc = check_both(who, "q_out or k_out", q_out, k_out, s, dtype, A.o0);
  const float* f[] = {q_weight, k_weight};
  if (!rc) rc = check_floats(who, f, 2);
  if (!rc) rc = check_apart(who, s, {A.o0}, {A.x}, A.dw);
  if (rc) return rc;
  A.w[0] = q_weight;
  A.w[1] = k_weight;
  return launch<kFwd>(who, s, A, dtype, as_stream(stream));
}

extern "C" int diffopt_qknorm_rope_bwd(const diffopt_heads* dq_out, const diffopt_heads* dk_out, const diffopt_heads* q,
                                       const diffopt_heads* k, const float* q_weight, const float* k_weight,
                                       const float* cos, const float* sin, int64_t rows, const void* positions,
                                       int32_t position_bytes, int64_t first, int64_t B, int64_t T, int64_t H,
                                       int64_t Hk, int64_t D, int64_t rot, int32_t interleaved, int32_t dtype,
                                       double eps, const diffopt_heads* dq, const diffopt_heads* dk, float* dq_weight,
                                       float* dk_weight, void* workspace, int64_t workspace_bytes, void* stream) {
  clear_error();
  static const char* who = "diffopt_qknorm_rope_bwd";
  QkShape s;
  int rc = check_shape(who, cos, sin, rows, positions, position_bytes, first, B, T, H, Hk, D, rot, interleaved, dtype, eps, &s);
  if (rc) return rc;
  QkArgs A{};
  A.dw[0] = dq_weight;
  A.dw[1] = dk_weight;
  if (B * T > 0) {
    rc = check_both(who, "q or k", q, k, s, dtype, A.x);
    if (!rc) rc = check_both(who, "dq_out or dk_out", dq_out, dk_out, s, dtype, A.dy);
    if (!rc) rc = check_both(who, "dq or dk", dq, dk, s, dtype, A.o0);
  }
  const float* f[] = {q_weight, k_weight, dq_weight, dk_weight};
  if (!rc) rc = check_floats(who, f, 4);
  if (!rc) rc = check_workspace(who, s, &A, workspace, workspace_bytes);
  if (!rc) rc = check_apart(who, s, {A.o0}, {A.x, A.dy}, A.dw);
  if (rc) return rc;
  A.w[0] = q_weight;
  A.w[1] = k_weight;
  return launch<kBwd>(who, s, A, dtype, as_stream(stream));
}

extern "C" int diffopt_qknorm_rope_bwd_bwd(
    const diffopt_heads* ddq, const diffopt_heads* ddk, const float* ddq_weight, const float* ddk_weight,
    const diffopt_heads* dq_out, const diffopt_heads* dk_out, const diffopt_heads* q, const diffopt_heads* k,
    const float* q_weight, const float* k_weight, const float* cos, const float* sin, int64_t rows,
    const void* positions, int32_t position_bytes, int64_t first, int64_t B, int64_t T, int64_t H, int64_t Hk,
    int64_t D, int64_t rot, int32_t interleaved, int32_t dtype, double eps, const diffopt_heads* out_dq_out,
    const diffopt_heads* out_dk_out, const diffopt_heads* out_q, const diffopt_heads* out_k, float* out_q_weight,
    float* out_k_weight, void* workspace, int64_t workspace_bytes, void* stream) {
  clear_error();
  static const char* who = "diffopt_qknorm_rope_bwd_bwd";
  QkShape s;
  int rc = check_shape(who, cos, sin, rows, positions, position_bytes, first, B, T, H, Hk, D, rot, interleaved, dtype, eps, &s);
  if (rc) return rc;
  QkArgs A{};
  A.dw[0] = out_q_weight;
  A.dw[1] = out_k_weight;
  if (B * T > 0) {
    rc = check_both(who, "q or k", q, k, s, dtype, A.x);
    if (!rc) rc = check_both(who, "dq_out or dk_out", dq_out, dk_out, s, dtype, A.dy);
    if (!rc && ddq) rc = check_heads(who, "ddq", ddq, dtype, &A.a[0]);
    if (!rc && ddk && Hk > 0) rc = check_heads(who, "ddk", ddk, dtype, &A.a[1]);
    if (!rc) rc = check_both(who, "out_dq_out or out_dk_out", out_dq_out, out_dk_out, s, dtype, A.o0);
    if (!rc) rc = check_both(who, "out_q or out_k", out_q, out_k, s, dtype, A.o1);
  }
  const float* f[] = {q_weight, k_weight, ddq_weight, ddk_weight, out_q_weight, out_k_weight};
  if (!rc) rc = check_floats(who, f, 6);
  if (!rc) rc = check_workspace(who, s, &A, workspace, workspace_bytes);
  if (!rc) rc = check_apart(who, s, {A.o0, A.o1}, {A.x, A.dy, A.a}, A.dw);
  if (rc) return rc;
  A.w[0] = q_weight;
  A.w[1] = k_weight;
  A.b[0] = ddq_weight;
  A.b[1] = ddk_weight;
  return launch<kSecond>(who, s, A, dtype, as_stream(stream));
}
