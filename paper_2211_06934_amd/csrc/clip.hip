// The global norm of a gradient, clipping to it, and the VJP of both on gfx950
// (formulas in diffopt.h), over one flat buffer or the leaves of a tree.
//
// Two launches: partial sums in fp64, one a workgroup, in an order that the
// sizes alone decide; then every wave adds the few hundred partial sums while
// its elements are on their way, and scales them (a launch of its own that makes
// them one costs more: 20M elements 40.3 us against 38.7, 354M 754 against 745).
// fp64 holds a square of any fp32 value and its sum to far below an fp32 rounding,
// at no cost: two instructions for an element of four bytes.  Bound by memory, the
// elements being read twice; the second pass goes backwards, so that it begins
// with what the first one left in the Infinity Cache.  A tree of 354M elements: the
// sums read 6.0 TB/s by themselves (236 us), 5.3 (269) where the results of a pass before
// are still on their way to memory; the second pass moves 5.8 (490).
//
// A wave takes one tile of the segment table (512 groups of four elements).  A
// tile inside one leaf reads that leaf's entry with scalar loads; others stage
// their window of the table in the wave's own LDS and search it, so that
// waves never wait for one another (looking a wave's next tile up while this one's
// elements are on their way takes as long or longer: 20M elements in 3,384 leaves 19.1
// and 19.8 us, in 200,000 24.7 and 25.6).  Gradients of up to kAlone elements take one
// launch of one workgroup, which keeps them in registers.
#include <cmath>
#include <initializer_list>
#include <type_traits>

#include "lm_common.hpp"
#include "segtable.hpp"

namespace diffopt {
namespace {

constexpr int kScaleBlock = 256, kScaleWaves = kScaleBlock / 64;
// Waves of a workgroup of sums, and how many workgroups there are at most: one large
// one a compute unit (trees of 354M and of 20M elements, behind other passes' results, 269
// and 20.3 us; 512 workgroups of 8 waves 277 and 18.9, 256 of them 264 and 22.8).
constexpr int kSumWaves = 16, kMostParts = 256;
constexpr int kGroups = (int)(kTileGroups / 64);  // of a lane
constexpr int kAloneBlock = 1024, kAloneEach = 8;
constexpr int64_t kAlone = kAloneBlock * kAloneEach;

// Where the elements are: the table's leaves, or one buffer of n elements.
struct Space {
  const SegEntry* seg;
  const int64_t* tile_first;
  int64_t ntiles, ngroups, n;
  int32_t dense_orig;
};

// Operand trees (device arrays of leaf addresses), or flat buffers.
template <int NA>
struct Operands {
  const void* a[NA];
};

template <int NA>
struct Leaf {
  int64_t goff, numel;
  uint64_t p[NA];
};

template <int NA>
struct Window {
  int64_t goff[kWindowMax], numel[kWindowMax];
  uint64_t p[NA][kWindowMax];
};

__device__ __forceinline__ void wave_sync() {  // LDS written by the wave's lanes is read by its others
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Tile b: a lane's groups of it are counted from the 128-byte line of operand
// PH's leaf (PH < 0: from the leaf), so that stores fill lines.
template <bool FLAT, int NA, int PH>
struct Tile {
  Window<NA>* win;
  Leaf<NA> one;  // of a tile inside one leaf
  int64_t first;
  int W;         // leaves of the window; 0: one leaf
  int mine, lane;  // window place of the leaf that has the lane's eight consecutive groups

  __device__ __forceinline__ Tile(const Space& sp, const Operands<NA>& ops, Window<NA>& window, int64_t b, int lane_)
      : win(&window), one{0, sp.n, {}}, first(b * kTileGroups + lane_), W(0), mine(0), lane(lane_) {
    if constexpr (FLAT) {
#pragma unroll
      for (int q = 0; q < NA; ++q) one.p[q] = reinterpret_cast<uint64_t>(ops.a[q]);
      return;
    }
    const auto tf = caddr<int64_t>(sp.tile_first);
    const int64_t j0 = tf[b];
    W = (int)(tf[b + 1] - j0 + 1);
    if (W == 1) {
      W = 0;
      const auto e = caddr<int64_t>(sp.seg + j0);
      const int64_t at = sp.dense_orig ? j0 : e[3];
      one.goff = e[0];
      one.numel = e[2];
#pragma unroll
      for (int q = 0; q < NA; ++q) one.p[q] = caddr<uint64_t>(ops.a[q])[at];
      return;
    }
    const auto stage = [&](int t, auto dense) {  // with dense the addresses do not wait for the entries
      const SegEntry e = sp.seg[j0 + t];
      uint64_t v[NA];
#pragma unroll
      for (int q = 0; q < NA; ++q) v[q] = static_cast<const uint64_t*>(ops.a[q])[decltype(dense)::value ? j0 + t : e.orig];
      win->goff[t] = e.goff;
      win->numel[t] = e.numel;
#pragma unroll
      for (int q = 0; q < NA; ++q) win->p[q][t] = v[q];
    };
    for (int t = lane; t < W; t += 64)
      if (sp.dense_orig) stage(t, std::true_type{});
      else stage(t, std::false_type{});
    wave_sync();
    // Leaves begin at multiples of kLeafGroupAlign groups: a lane searches for one such run of the tile, the others ask it.
    static_assert(kTileGroups == 64 * kLeafGroupAlign, "a lane has one run of groups that share a leaf");
    const int64_t g = b * kTileGroups + lane * kLeafGroupAlign;
    int hi = W - 1;  // goff[0] <= g
    while (mine < hi) {
      const int mid = (mine + hi + 1) >> 1;
      if (win->goff[mid] <= g) mine = mid;
      else hi = mid - 1;
    }
  }

  __device__ __forceinline__ Leaf<NA> find(int u) const {
    if (FLAT || W == 0) return one;
    const int lo = __shfl(mine, u * (64 / (int)kLeafGroupAlign) + lane / (int)kLeafGroupAlign, 64);
    Leaf<NA> leaf{win->goff[lo], win->numel[lo], {}};
#pragma unroll
    for (int q = 0; q < NA; ++q) leaf.p[q] = win->p[q][lo];
    return leaf;
  }

  // f(leaf, w, own) for a lane's group u: the bits of own are those of the leaf's
  // elements [w, w + 4) that the group has (none past the table's last leaf).
  template <class F>
  __device__ __forceinline__ void group(int u, F f) const {
    const int64_t g = first + u * 64;
    const Leaf<NA> leaf = find(u);
    int64_t e0 = 4 * (g - leaf.goff);
    if constexpr (PH >= 0) e0 -= (int64_t)(leaf.p[PH] >> 2 & 31u);
    int64_t w = e0 + 4 <= leaf.numel ? e0 : leaf.numel - 4;
    if (w < 0) w = 0;
    int own = 0;
    if (e0 + 4 > 0 && e0 < leaf.numel) {
      const int d = (int)(e0 - w);  // -3..3
      own = d < 0 ? 15 >> -d : (15 << d) & 15;
      if (leaf.numel < 4) own &= (1 << (int)leaf.numel) - 1;
    }
    f(leaf, w, own);
  }

  // f(u, leaf, w, own) for each group, own 0 for those of leaves of fewer than
  // four elements; whether the lane has any such.
  template <class F>
  __device__ __forceinline__ bool groups(F f) const {
    bool few = false;
#pragma unroll
    for (int u = 0; u < kGroups; ++u)
      group(u, [&](const Leaf<NA>& leaf, int64_t w, int own) {
        const bool small = leaf.numel < 4;
        few |= small && own;
        f(u, leaf, w, small ? 0 : own);
      });
    return few;
  }
  // f(leaf, element) for the elements of leaves of fewer than four.
  template <class F>
  __device__ __forceinline__ void few(F f) const {
#pragma unroll 1
    for (int u = 0; u < kGroups; ++u)
      group(u, [&](const Leaf<NA>& leaf, int64_t w, int own) {
        if (leaf.numel < 4)
          for (int i = 0; i < 3; ++i)
            if (own >> i & 1) f(leaf, w + i);
      });
  }
};

__device__ __forceinline__ f32x4 load4(uint64_t leaf, int64_t i) {
  typedef f32x4 loose __attribute__((aligned(4)));
  return *(gptr<const loose>)(leaf + 4 * (uint64_t)i);
}
__device__ __forceinline__ void store4(uint64_t leaf, int64_t i, const f32x4& x) {
  typedef f32x4 loose __attribute__((aligned(4)));
  *(gptr<loose>)(leaf + 4 * (uint64_t)i) = x;
}

// Those of four elements whose bits are set.
__device__ __forceinline__ void store_own(uint64_t to, uint32_t own, const f32x4& y) {
  if (own == 15u) {
    store4(to, 0, y);
  } else if (own) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (own >> i & 1u) gaddr<float>(to)[i] = y[i];
  }
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}

// Partial sums of a b over the operands' elements (b = a with one operand).
// With two, nothing is read where stats says that the gradient was not clipped:
// the sum has no weight then.
template <bool FLAT, int NA>
__global__ __launch_bounds__(64 * kSumWaves, 4) void clip_sums(Space sp, Operands<NA> ops, const float* stats, double* parts) {
  __shared__ std::conditional_t<FLAT, char, Window<NA>> windows[kSumWaves];
  __shared__ double sums[kSumWaves];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  double acc[2] = {0.0, 0.0};
  static_assert(kGroups * 4 == 32, "a lane's elements are the bits of a word");
  const bool skip = NA == 2 && stats[1] >= 1.0f;
  using T = Tile<FLAT, NA, -1>;  // groups counted from the first element: an order that goes by no address
  // wave after wave takes a tile, workgroup after workgroup: neighbouring tiles are read together
  if (!skip)
    for (int64_t b = (int64_t)wave * gridDim.x + blockIdx.x; b < sp.ntiles; b += (int64_t)gridDim.x * kSumWaves) {
      const T tile(sp, ops, reinterpret_cast<Window<NA>&>(windows[FLAT ? 0 : wave]), b, lane);
      f32x4 v[NA][kGroups];
      uint32_t own = 0;  // four bits a group
      const uint64_t dummy = FLAT ? reinterpret_cast<uint64_t>(ops.a[0]) : reinterpret_cast<uint64_t>(sp.seg);  // 16 bytes that are there
      const bool few = tile.groups([&](int u, const Leaf<NA>& leaf, int64_t w, int o) {
        own |= (uint32_t)o << (4 * u);
#pragma unroll
        for (int q = 0; q < NA; ++q) v[q][u] = load4(o ? leaf.p[q] : dummy, o ? w : 0);
      });
      if (!__all(own == ~0u)) {
#pragma unroll
        for (int u = 0; u < kGroups; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!(own >> (4 * u + i) & 1u))
#pragma unroll
              for (int q = 0; q < NA; ++q) v[q][u][i] = 0.0f;
      }
#pragma unroll
      for (int u = 0; u < kGroups; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i & 1] = __builtin_fma((double)v[0][u][i], (double)v[NA - 1][u][i], acc[i & 1]);
      if (__any(few))
        tile.few([&](const Leaf<NA>& leaf, int64_t i) {
          const double x = gaddr<const float>(leaf.p[0])[i], y = gaddr<const float>(leaf.p[NA - 1])[i];
          acc[0] += x * y;
        });
      if constexpr (!FLAT) wave_sync();  // the next tile's window takes this one's place
    }
  const double sum = wave_sum(acc[0] + acc[1]);
  if (lane == 0) sums[wave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    double all = 0.0;
    for (int w = 0; w < kSumWaves; ++w) all += sums[w];
    parts[blockIdx.x] = all;
  }
}

// The sum of n partial sums, the same in every lane of every wave.
struct Parts {
  double v[kMostParts / 64];
  __device__ __forceinline__ Parts(const double* p, int n, int lane) {
#pragma unroll
    for (int i = 0; i < kMostParts / 64; ++i) v[i] = lane + 64 * i < n ? p[lane + 64 * i] : 0.0;
  }
  __device__ __forceinline__ double sum() const {
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < kMostParts / 64; ++i) s += v[i];
    return wave_sum(s);
  }
};

// c = min(1, max_norm / (norm + eps)), rounded once to fp32; NaN for a NaN.
__device__ __forceinline__ float scale_of(double norm, double max_norm, double eps) {
  return norm + eps <= max_norm ? 1.0f : (float)(max_norm / (norm + eps));
}

// The factor of the gradient in its own gradient: d norm / d g = g / norm, d c / d
// norm = -c / (norm + eps) where c < 1.  A norm below 3e-39 has a factor above any fp32
// number, a large one may have one below, though the product is an ordinary number: the
// factor is rounded to 24 bits and keeps its power of two apart, which goes to the
// element before the product where it is large and after it where it is small.
struct Factor {
  float part;
  int32_t before, after;
  __device__ __forceinline__ explicit Factor(double x) : part((float)x), before(0), after(0) {
    if (x == 0.0 || !__builtin_isfinite(x)) return;
    const int32_t e = __builtin_amdgcn_frexp_exp(x);
    part = (float)__builtin_amdgcn_frexp_mant(x);  // in [1/2, 1]
    if (e > 0) {
      part *= 2.0f;
      before = e - 1;
    } else {
      after = e;
    }
  }
  __device__ __forceinline__ float times(float g) const { return __builtin_ldexpf(__builtin_ldexpf(g, before) * part, after); }
};

__device__ __forceinline__ Factor slope_of(double dot, const float* dnorm, float norm, float c, double eps) {
  if (norm == 0.0f) return Factor(0.0);
  double x = dnorm ? (double)*dnorm : 0.0;
  if (!(c >= 1.0f)) x -= (double)c * dot / ((double)norm + eps);
  return Factor(x / (double)norm);
}

// out = c grad (operands 0 grad, 1 out); workgroup 0 writes the norm and c.
template <bool FLAT>
__global__ __launch_bounds__(kScaleBlock) void clip_scale(Space sp, Operands<2> ops, const double* part, int32_t nparts, double max_norm, double eps, float* stats) {
  __shared__ std::conditional_t<FLAT, char, Window<2>> windows[kScaleWaves];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t b = sp.ntiles - 1 - ((int64_t)blockIdx.x * kScaleWaves + wave);
  const Parts parts(part, nparts, lane);
  const auto finish = [&] {
    const double norm = sqrt(parts.sum());
    const float c = scale_of(norm, max_norm, eps);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
      stats[0] = (float)norm;
      stats[1] = c;
    }
    return c;
  };
  if (b < 0 || !ops.a[1]) {
    if (blockIdx.x == 0) finish();
    return;
  }
  const Tile<FLAT, 2, 1> tile(sp, ops, reinterpret_cast<Window<2>&>(windows[FLAT ? 0 : wave]), b, lane);
  f32x4 v[kGroups];
  uint64_t to[kGroups];
  uint32_t own = 0;  // four bits a group
  const uint64_t dummy = FLAT ? reinterpret_cast<uint64_t>(ops.a[0]) : reinterpret_cast<uint64_t>(sp.seg);
  const bool few = tile.groups([&](int u, const Leaf<2>& leaf, int64_t w, int o) {
    own |= (uint32_t)o << (4 * u);
    to[u] = leaf.p[1] + 4 * (uint64_t)w;
    v[u] = load4(o ? leaf.p[0] : dummy, o ? w : 0);
  });
  const float c = finish();
  if (c == 1.0f && ops.a[0] == ops.a[1]) return;  // in place and not clipped
#pragma unroll
  for (int u = 0; u < kGroups; ++u) {
    const f32x4 y = v[u] * c;
    store_own(to[u], own >> (4 * u) & 15u, y);
  }
  if (__any(few)) tile.few([&](const Leaf<2>& leaf, int64_t i) { gaddr<float>(leaf.p[1])[i] = c * gaddr<const float>(leaf.p[0])[i]; });
}

// dgrad = c dout + slope grad (operands 0 grad, 1 dgrad, 2 dout or none).
template <bool FLAT, bool DOUT>
__global__ __launch_bounds__(kScaleBlock) void clip_gradient(Space sp, Operands<DOUT ? 3 : 2> ops, const double* part, int32_t nparts,
                                                             const float* dnorm, const float* stats, double eps) {
  constexpr int NA = DOUT ? 3 : 2;
  __shared__ std::conditional_t<FLAT, char, Window<NA>> windows[kScaleWaves];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t b = sp.ntiles - 1 - ((int64_t)blockIdx.x * kScaleWaves + wave);
  if (b < 0) return;
  const Parts parts(part, nparts, lane);
  const float norm = stats[0], c = stats[1];
  const Tile<FLAT, NA, 1> tile(sp, ops, reinterpret_cast<Window<NA>&>(windows[FLAT ? 0 : wave]), b, lane);
  f32x4 v[kGroups], d[DOUT ? kGroups : 1];
  uint64_t to[kGroups];
  uint32_t own = 0;  // four bits a group
  const uint64_t dummy = FLAT ? reinterpret_cast<uint64_t>(ops.a[0]) : reinterpret_cast<uint64_t>(sp.seg);
  const bool few = tile.groups([&](int u, const Leaf<NA>& leaf, int64_t w, int o) {
    own |= (uint32_t)o << (4 * u);
    to[u] = leaf.p[1] + 4 * (uint64_t)w;
    v[u] = load4(o ? leaf.p[0] : dummy, o ? w : 0);
    if constexpr (DOUT) d[u] = load4(o ? leaf.p[NA - 1] : dummy, o ? w : 0);
  });
  const Factor slope = slope_of(parts.sum(), dnorm, norm, c, eps);
  const auto value = [&](float g, float dy) { return DOUT ? __builtin_fmaf(c, dy, slope.times(g)) : slope.times(g); };
#pragma unroll
  for (int u = 0; u < kGroups; ++u) {
    f32x4 y;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = value(v[u][i], DOUT ? d[DOUT ? u : 0][i] : 0.0f);
    store_own(to[u], own >> (4 * u) & 15u, y);
  }
  if (__any(few))
    tile.few([&](const Leaf<NA>& leaf, int64_t i) {
      gaddr<float>(leaf.p[1])[i] = value(gaddr<const float>(leaf.p[0])[i], DOUT ? gaddr<const float>(leaf.p[NA - 1])[i] : 0.0f);
    });
}

// ---- few elements: one workgroup --------------------------------------------

// Where element j of a small tree or buffer lies in operand q: an address, 0
// where there is none.
template <bool FLAT>
__device__ __forceinline__ bool small_slot(const TinyTable& tt, int64_t n, int64_t j, int& leaf, int64_t& i) {
  if (FLAT) {
    leaf = 0;
    i = j;
    return j < n;
  }
  return tiny_slot(tt, j, leaf, i);
}

template <bool FLAT>
__device__ __forceinline__ gptr<float> small_at(const void* arr, int leaf, int64_t i) {
  return gaddr<float>(FLAT ? reinterpret_cast<uint64_t>(arr) : static_cast<const uint64_t*>(arr)[leaf]) + i;
}

__device__ __forceinline__ double alone_sum(double x) {
  __shared__ double sums[kAloneBlock / 64];
  x = wave_sum(x);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = x;
  __syncthreads();
  double all = 0.0;
  for (int w = 0; w < kAloneBlock / 64; ++w) all += sums[w];
  return all;
}

template <bool FLAT>
__global__ __launch_bounds__(kAloneBlock) void clip_alone(TinyTable tt, int64_t n, Operands<2> ops, double max_norm, double eps, float* stats) {
  float v[kAloneEach];
  gptr<float> to[kAloneEach];
  double acc = 0.0;
#pragma unroll
  for (int k = 0; k < kAloneEach; ++k) {
    v[k] = 0.0f;
    to[k] = nullptr;
    if (k * kAloneBlock < n) {
      int leaf;
      int64_t i;
      if (small_slot<FLAT>(tt, n, k * kAloneBlock + threadIdx.x, leaf, i)) {
        v[k] = *small_at<FLAT>(ops.a[0], leaf, i);
        if (ops.a[1]) to[k] = small_at<FLAT>(ops.a[1], leaf, i);
      }
    }
  }
#pragma unroll
  for (int k = 0; k < kAloneEach; ++k) acc = __builtin_fma((double)v[k], (double)v[k], acc);
  const double norm = sqrt(alone_sum(acc));
  const float c = scale_of(norm, max_norm, eps);
  if (threadIdx.x == 0) {
    stats[0] = (float)norm;
    stats[1] = c;
  }
#pragma unroll
  for (int k = 0; k < kAloneEach; ++k)
    if (to[k]) *to[k] = c * v[k];
}

template <bool FLAT, bool DOUT>
__global__ __launch_bounds__(kAloneBlock) void clip_gradient_alone(TinyTable tt, int64_t n, Operands<DOUT ? 3 : 2> ops, const float* dnorm,
                                                                   const float* stats, double eps) {
  float v[kAloneEach], d[kAloneEach];
  gptr<float> to[kAloneEach];
  double acc = 0.0;
  const float norm = stats[0], c = stats[1];
#pragma unroll
  for (int k = 0; k < kAloneEach; ++k) {
    v[k] = d[k] = 0.0f;
    to[k] = nullptr;
    if (k * kAloneBlock < n) {
      int leaf;
      int64_t i;
      if (small_slot<FLAT>(tt, n, k * kAloneBlock + threadIdx.x, leaf, i)) {
        v[k] = *small_at<FLAT>(ops.a[0], leaf, i);
        if constexpr (DOUT) d[k] = *small_at<FLAT>(ops.a[DOUT ? 2 : 0], leaf, i);
        to[k] = small_at<FLAT>(ops.a[1], leaf, i);
      }
    }
  }
#pragma unroll
  for (int k = 0; k < kAloneEach; ++k) acc = __builtin_fma((double)v[k], (double)d[k], acc);
  const Factor slope = slope_of(DOUT ? alone_sum(acc) : 0.0, dnorm, norm, c, eps);
#pragma unroll
  for (int k = 0; k < kAloneEach; ++k)
    if (to[k]) *to[k] = DOUT ? __builtin_fmaf(c, d[k], slope.times(v[k])) : slope.times(v[k]);
}

// ---- host -------------------------------------------------------------------

constexpr int64_t kMostElements = int64_t(1) << 36;

// A call's elements: a table's, or n of a buffer.
struct Elements {
  const diffopt_segtable* table;
  int64_t n;
  bool flat() const { return !table; }
  int64_t count() const { return table ? table->elems : n; }
  int64_t tiles() const { return table ? table->ntiles : ((n + 3) / 4 + 8 + kTileGroups - 1) / kTileGroups; }
  bool alone() const { return count() <= kAlone && (!table || table->tiny); }
  int32_t parts() const {
    const int64_t blocks = (tiles() + kSumWaves - 1) / kSumWaves;
    return (int32_t)(blocks < kMostParts ? blocks : kMostParts);
  }
  int64_t workspace() const { return count() == 0 || alone() ? 0 : (int64_t)parts() * 8; }
  Space space() const {
    return table ? Space{table->d_seg, table->d_tile_first, table->ntiles, table->ngroups, 0, table->dense_orig}
                 : Space{nullptr, nullptr, tiles(), tiles() * kTileGroups, n, 0};
  }
  int64_t scale_blocks() const { return (tiles() + kScaleWaves - 1) / kScaleWaves; }
  // what a call takes: a launch has fewer than 2^32 threads (a tree's leaves begin tiles of their own)
  bool fits() const { return count() >= 0 && count() < kMostElements && scale_blocks() < (int64_t(1) << 32) / kScaleBlock; }
};

#define DIFFOPT_LAUNCH(kernel, grid, block, ...) hipLaunchKernelGGL((kernel), dim3((unsigned)(grid)), dim3(block), 0, st, __VA_ARGS__)

template <bool FLAT>
int fwd(const char* who, const Elements& e, const void* grad, double max_norm, double eps, const void* out, float* stats, void* workspace, hipStream_t st) {
  const Operands<2> ops{{grad, out}};
  if (e.alone()) {
    DIFFOPT_LAUNCH((clip_alone<FLAT>), 1, kAloneBlock, FLAT ? TinyTable{} : e.table->small, e.count(), ops, max_norm, eps, stats);
    return launch_status(who);
  }
  const Space sp = e.space();
  double* parts = static_cast<double*>(workspace);
  const Operands<1> one{{grad}};
  const float* none = nullptr;
  DIFFOPT_LAUNCH((clip_sums<FLAT, 1>), e.parts(), 64 * kSumWaves, sp, one, none, parts);
  DIFFOPT_LAUNCH((clip_scale<FLAT>), out ? e.scale_blocks() : 1, kScaleBlock, sp, ops, parts, e.parts(), max_norm, eps, stats);
  return launch_status(who);
}

template <bool FLAT>
int bwd(const char* who, const Elements& e, const void* dout, const float* dnorm, const void* grad, const float* stats, double eps, const void* dgrad,
        void* workspace, hipStream_t st) {
  const Operands<3> three{{grad, dgrad, dout}};
  const Operands<2> two{{grad, dgrad}};
  if (e.alone()) {
    const TinyTable small = FLAT ? TinyTable{} : e.table->small;
    if (dout) DIFFOPT_LAUNCH((clip_gradient_alone<FLAT, true>), 1, kAloneBlock, small, e.count(), three, dnorm, stats, eps);
    else DIFFOPT_LAUNCH((clip_gradient_alone<FLAT, false>), 1, kAloneBlock, small, e.count(), two, dnorm, stats, eps);
    return launch_status(who);
  }
  const Space sp = e.space();
  if (dout) {
    double* parts = static_cast<double*>(workspace);
    const Operands<2> product{{grad, dout}};
    DIFFOPT_LAUNCH((clip_sums<FLAT, 2>), e.parts(), 64 * kSumWaves, sp, product, stats, parts);
    DIFFOPT_LAUNCH((clip_gradient<FLAT, true>), e.scale_blocks(), kScaleBlock, sp, three, parts, e.parts(), dnorm, stats, eps);
  } else {
    DIFFOPT_LAUNCH((clip_gradient<FLAT, false>), e.scale_blocks(), kScaleBlock, sp, two, nullptr, 0, dnorm, stats, eps);
  }
  return launch_status(who);
}

int check_numbers(const char* who, double max_norm, double eps) {
  if (!(max_norm >= 0.0)) return fail(DIFFOPT_EINVAL, "%s: max_norm must be >= 0", who);
  if (!(eps >= 0.0 && std::isfinite(eps))) return fail(DIFFOPT_EINVAL, "%s: eps must be finite and >= 0", who);
  return DIFFOPT_OK;
}

int check_elements(const char* who, const Elements& e, void* workspace, int64_t bytes) {
  if (!e.fits()) return fail(DIFFOPT_EINVAL, "%s: too many elements", who);
  const int64_t need = e.workspace();
  if (need > 0 && (!workspace || bytes < need))
    return fail(DIFFOPT_EINVAL, "%s: the workspace has %lld bytes of %lld", who, (long long)(workspace ? bytes : 0), (long long)need);
  if (!aligned_to(workspace, 8)) return fail(DIFFOPT_EINVAL, "%s: the workspace is not 8-byte aligned", who);
  return DIFFOPT_OK;
}

int check_table(const char* who, const diffopt_segtable* t) {
  if (!t) return fail(DIFFOPT_EINVAL, "%s: table is NULL", who);
  if (t->elem_bytes != 4) return fail(DIFFOPT_EINVAL, "%s: the table must describe fp32 leaves (elem_bytes 4)", who);
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev != t->device)
    return fail(DIFFOPT_EINVAL, "%s: the table lives on device %d, the current device is %d", who, t->device, dev);
  return DIFFOPT_OK;
}

int check_floats(const char* who, std::initializer_list<const void*> floats) {
  for (const void* p : floats)
    if (!aligned_to(p, 4)) return fail(DIFFOPT_EINVAL, "%s: pointer %p is not 4-byte aligned", who, p);
  return DIFFOPT_OK;
}

// Flat buffers: whole or apart.
int check_buffers(const char* who, const char* what, const float* result, std::initializer_list<const float*> operands, int64_t n) {
  for (const float* o : operands)
    if (o != result && overlap(result, 4 * n, o, 4 * n)) return fail(DIFFOPT_EINVAL, "%s: %s must be an operand or lie apart from it", who, what);
  return DIFFOPT_OK;
}

}  // namespace
}  // namespace diffopt

using namespace diffopt;

extern "C" int64_t diffopt_clip_norm_workspace(int64_t n) {
  const Elements e{nullptr, n};
  return e.fits() ? e.workspace() : -1;
}

extern "C" int64_t diffopt_clip_norm_workspace_tree(const diffopt_segtable* table) {
  const Elements e{table, 0};
  return table && e.fits() ? e.workspace() : -1;
}

extern "C" int diffopt_clip_norm_fwd(const float* grad, int64_t n, double max_norm, double eps, float* out, float* stats, void* workspace,
                                     int64_t workspace_bytes, void* stream) {
  clear_error();
  static const char* who = "diffopt_clip_norm_fwd";
  if (n < 0) return fail(DIFFOPT_EINVAL, "%s: n must be >= 0", who);
  int rc = check_numbers(who, max_norm, eps);
  if (rc) return rc;
  if (!stats || (n > 0 && !grad)) return fail(DIFFOPT_EINVAL, "%s: null grad or stats", who);
  rc = check_floats(who, {grad, out, stats});
  const Elements e{nullptr, n};
  if (!rc) rc = check_elements(who, e, workspace, workspace_bytes);
  if (!rc) rc = check_buffers(who, "out", out, {grad}, n);
  if (!rc && (overlap(stats, 8, grad, 4 * n) || overlap(stats, 8, out, 4 * n))) rc = fail(DIFFOPT_EINVAL, "%s: stats must lie apart", who);
  if (rc) return rc;
  return fwd<true>(who, e, grad, max_norm, eps, out, stats, workspace, as_stream(stream));
}

extern "C" int diffopt_clip_norm_fwd_tree(const diffopt_segtable* table, const uint64_t* grad, double max_norm, double eps, const uint64_t* out,
                                          float* stats, void* workspace, int64_t workspace_bytes, void* stream) {
  clear_error();
  static const char* who = "diffopt_clip_norm_fwd_tree";
  int rc = check_table(who, table);
  if (!rc) rc = check_numbers(who, max_norm, eps);
  if (rc) return rc;
  const Elements e{table, 0};
  if (!stats || (e.count() > 0 && !grad)) return fail(DIFFOPT_EINVAL, "%s: null grad or stats", who);
  rc = check_floats(who, {stats});
  if (!rc) rc = check_elements(who, e, workspace, workspace_bytes);
  if (rc) return rc;
  return e.count() == 0 ? fwd<true>(who, Elements{nullptr, 0}, nullptr, max_norm, eps, nullptr, stats, workspace, as_stream(stream))
                        : fwd<false>(who, e, grad, max_norm, eps, out, stats, workspace, as_stream(stream));
}

extern "C" int diffopt_clip_norm_bwd(const float* dout, const float* dnorm, const float* grad, const float* stats, int64_t n, double eps, float* dgrad,
                                     void* workspace, int64_t workspace_bytes, void* stream) {
  clear_error();
  static const char* who = "diffopt_clip_norm_bwd";
  if (n < 0) return fail(DIFFOPT_EINVAL, "%s: n must be >= 0", who);
  int rc = check_numbers(who, 0.0, eps);
  if (rc || n == 0) return rc;
  if (!grad || !stats || !dgrad) return fail(DIFFOPT_EINVAL, "%s: null grad, stats or dgrad", who);
  rc = check_floats(who, {dout, dnorm, grad, stats, dgrad});
  const Elements e{nullptr, n};
  if (!rc) rc = check_elements(who, e, workspace, workspace_bytes);
  if (!rc) rc = check_buffers(who, "dgrad", dgrad, {dout, grad}, n);
  if (!rc && (overlap(stats, 8, dgrad, 4 * n) || overlap(dnorm, 4, dgrad, 4 * n))) rc = fail(DIFFOPT_EINVAL, "%s: dgrad must lie apart from stats and dnorm", who);
  if (rc) return rc;
  return bwd<true>(who, e, dout, dnorm, grad, stats, eps, dgrad, workspace, as_stream(stream));
}

extern "C" int diffopt_clip_norm_bwd_tree(const diffopt_segtable* table, const uint64_t* dout, const float* dnorm, const uint64_t* grad, const float* stats,
                                          double eps, const uint64_t* dgrad, void* workspace, int64_t workspace_bytes, void* stream) {
  clear_error();
  static const char* who = "diffopt_clip_norm_bwd_tree";
  int rc = check_table(who, table);
  if (!rc) rc = check_numbers(who, 0.0, eps);
  const Elements e{table, 0};
  if (rc || e.count() == 0) return rc;
  if (!grad || !stats || !dgrad) return fail(DIFFOPT_EINVAL, "%s: null grad, stats or dgrad", who);
  rc = check_floats(who, {dnorm, stats});
  if (!rc) rc = check_elements(who, e, workspace, workspace_bytes);
  if (rc) return rc;
  return bwd<false>(who, e, dout, dnorm, grad, stats, eps, dgrad, workspace, as_stream(stream));
}
