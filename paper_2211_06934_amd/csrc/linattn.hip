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

// One scan: state head j of sequence b reads query heads j nq .. + nq and k/v
// heads j nk .. + nk (one of nq, nk is 1).
struct Scan {
  HeadArr q, k, v, o;
  const float* s0;  // initial state or NULL: [Dk][Dv] blocks, or [Dv][Dk] ones with flip
  float* s1;        // final state or NULL: [Dk][Dv] blocks
  int32_t flip, flip_seg;  // whether s0 / the segments' states are [Dv][Dk]
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

// One token of any width and alignment (the others: linattn_one).  A workgroup holds
// 64 columns of one state, a lane R rows by 4 columns of them, read and written
// element by element.  Bound by the state's memory, in pieces of 4 bytes: 256 sequences
// of 16 heads of 128 whose states lie 4 bytes off a piece take 282 us in bf16 and 247 in
// fp32 (1.9 and 2.2 TB/s), where linattn_one takes 120 for aligned ones.
constexpr int kAnyB = 256, kAnyCols = 64;

template <class E, int R>
__global__ __launch_bounds__(kAnyB) void linattn_one_any(Shape s, Scan a, int32_t col_tiles) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int rg = lane >> 2;
  const int64_t state = blockIdx.x / (uint32_t)col_tiles, b = state / s.Hs;
  const int j = (int)(state - b * s.Hs);
  const int c0 = (int)(blockIdx.x % (uint32_t)col_tiles) * kAnyCols + wave * 16 + (lane & 3) * 4;
  // the decay to 48 bits: one rounding of it would grow with every token
  const double gd = exp((double)s.log_decay[j]);
  const float g = (float)gd, g_lo = (float)(gd - (double)g);
  const int64_t block = state * a.Dk * a.Dv;
  float S[R][4], vv[4];
  // all loads before the first store: they may be the same memory
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int r = rg + 16 * i;
      S[i][c] = r < a.Dk && c0 + c < a.Dv ? a.s0[block + r * a.Dv + c0 + c] : 0.0f;
    }
  const E *k = at<E>(a.k, b, 0, j), *v = at<E>(a.v, b, 0, j);
#pragma unroll
  for (int c = 0; c < 4; ++c) vv[c] = c0 + c < a.Dv ? (float)v[c0 + c] : 0.0f;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int r = rg + 16 * i;
    const float kk = r < a.Dk ? (float)k[r] : 0.0f;
#pragma unroll
    for (int c = 0; c < 4; ++c) S[i][c] = fmaf(kk, vv[c], fmaf(S[i][c], g, S[i][c] * g_lo));
  }
  for (int h = 0; h < a.nq; ++h) {
    const E* q = at<E>(a.q, b, 0, (int64_t)j * a.nq + h);
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
      E* out = at<E>(a.o, b, 0, (int64_t)j * a.nq + h);
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (c0 + c < a.Dv) out[c0 + c] = (E)(o[c] * a.qs);
    }
  }
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int r = rg + 16 * i;
      if (r < a.Dk && c0 + c < a.Dv) a.s1[block + r * a.Dv + c0 + c] = S[i][c];
    }
}

// One token: the state is read and written once, which is nearly all there is
// to move, in 16-byte pieces.  A workgroup takes 4 CG columns of one state and
// all its rows; a lane holds 4 columns of R rows, so that every load of a call
// is in flight at once and the product with q is joined over lanes and waves.
// Few columns a workgroup (32) put a single sequence's states on many compute
// units; whole lines of 128 bytes a row are enough for the memory as well.  Heads
// of 128, 16 a sequence: one sequence 3.9 us, bound by latency; 256 of them (537
// MB) 101 us repeated in a graph, 120 us on fresh states (4.5 TB/s), bound by
// memory (64 columns a workgroup 127 us, 128 columns 133, and one sequence 6.1;
// stores that pass the caches by 125).
constexpr int kStepB = 256, kStepCG = 8, kStepGroup = 8;

template <class E, int R>
__global__ __launch_bounds__(kStepB) void linattn_one(Shape s, Scan a, int32_t col_tiles) {
  constexpr int RG = kStepB / kStepCG;  // row groups of a workgroup
  __shared__ float part[kStepB / 64][kStepGroup][4 * kStepCG];
  const int cg = threadIdx.x % kStepCG, rg = threadIdx.x / kStepCG, wave = threadIdx.x >> 6;
  const int64_t state = blockIdx.x / (uint32_t)col_tiles;
  const int64_t b = state / s.Hs;
  const int j = (int)(state - b * s.Hs), c0 = ((int)(blockIdx.x % (uint32_t)col_tiles) * kStepCG + cg) * 4;
  const bool in = c0 < a.Dv;
  const float* s0 = a.s0 + state * a.Dk * a.Dv + c0;
  f32x4 S[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int r = rg + i * RG;
    S[i] = in && r < a.Dk ? *reinterpret_cast<const f32x4*>(s0 + r * a.Dv) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  const E *k = at<E>(a.k, b, 0, j), *v = at<E>(a.v, b, 0, j);
  float kk[R];
  f32x4 vv;
#pragma unroll
  for (int i = 0; i < R; ++i) kk[i] = rg + i * RG < a.Dk ? (float)k[rg + i * RG] : 0.0f;
#pragma unroll
  for (int c = 0; c < 4; ++c) vv[c] = in ? (float)v[c0 + c] : 0.0f;
  // the decay to 48 bits: one rounding of it would grow with every token
  const double gd = exp((double)s.log_decay[j]);
  const float g = (float)gd, g_lo = (float)(gd - (double)g);
  float* s1 = a.s1 + state * a.Dk * a.Dv + c0;
#pragma unroll
  for (int i = 0; i < R; ++i) {
#pragma unroll
    for (int c = 0; c < 4; ++c) S[i][c] = fmaf(S[i][c], g, fmaf(S[i][c], g_lo, kk[i] * vv[c]));
    const int r = rg + i * RG;
    if (in && r < a.Dk) *reinterpret_cast<f32x4*>(s1 + r * a.Dv) = S[i];
  }
  for (int h0 = 0; h0 < a.nq; h0 += kStepGroup) {
    const int n = a.nq - h0 < kStepGroup ? a.nq - h0 : kStepGroup;
    for (int h = 0; h < n; ++h) {
      const E* q = at<E>(a.q, b, 0, (int64_t)j * a.nq + h0 + h);
      f32x4 o{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const float qq = rg + i * RG < a.Dk ? (float)q[rg + i * RG] : 0.0f;
#pragma unroll
        for (int c = 0; c < 4; ++c) o[c] = fmaf(qq, S[i][c], o[c]);
      }
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int m = kStepCG; m < 64; m <<= 1) o[c] += __shfl_xor(o[c], m, 64);
      if ((threadIdx.x & 63) < kStepCG)
#pragma unroll
        for (int c = 0; c < 4; ++c) part[wave][h][4 * cg + c] = o[c];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n * 4 * kStepCG; i += kStepB) {
      const int h = i / (4 * kStepCG), c = i % (4 * kStepCG), col = c0 - 4 * cg + c;
      float o = part[0][h][c];
#pragma unroll
      for (int w = 1; w < kStepB / 64; ++w) o += part[w][h][c];
      if (col < a.Dv) at<E>(a.o, b, 0, (int64_t)j * a.nq + h0 + h)[col] = (E)(o * a.qs);
    }
    __syncthreads();
  }
}

// ---- chunks -----------------------------------------------------------------
// C tokens at a time, all as matrix products.  With t, s counted inside a chunk
// of L <= C tokens and S the state before it,
//   O = W_q (Q S) + (P o M) V,  P = Q K^T,  M_ts = g^(t-s) for s <= t
//   S = g^L S + K^T (W_k V)
// where W_q, W_k are diagonal: g^(t+1), g^(L-1-s) forward and g^t, g^(L-s) back
// in time (no power is ever negative).  A workgroup of four waves walks the
// chunks of one segment of a sequence; wave w owns 16 NCT columns of the state,
// all DK rows of them, in registers for the whole walk.
//
// Fragments: v_mfma 16x16 takes row (or column) lane % 16 and, of a block of 32
// along the contraction, 8 elements per 16-lane group g = lane / 16; it returns
// column lane % 16, rows 4 g .. + 4.  Two results are an operand as they lie in
// the registers, P^T as computed for P V and the state for Q S: a block of 32
// tokens is numbered 4 g .. + 4 and 16 + 4 g .. + 4; of 32 rows of the state one
// tile takes 8 g .. + 4, the other 8 g + 4 .. + 4, so that Q is read in whole
// pieces.  V and K^T come out of LDS transposed, four tokens at a time
// (ds_read_b64_tr_b16).  The products are computed transposed, so that a lane
// holds 4 neighbouring elements of one token's output.
//
// In bf16 three operands of the products are not of the type, and are taken in parts
// of bf16, each the rounding of what the ones before leave out.  The scores and the
// fp32 state meet the values and the queries in two, exact to 2^-16; the state's update
// takes W_k V in SPLIT, exact to 2^-8 SPLIT: two where only outputs follow, three where
// a state is handed out (three everywhere cost 11% of a training step, for a part that
// the outputs' own rounding hides).  So results lie 1.66e-3 from 64-bit ones, which
// is the rounding of the outputs alone.  With one part of the scores they lie at 1.75e-3
// and training takes 362 us instead of 373, a prompt 132 instead of 133; with one of the
// state too 2.35e-3, 331 and 121.  fp32 runs on the fp32 matrix instructions.
//
// What bounds it is the walk: a chunk's products need one another (scores, barrier,
// outputs, state), and a compute unit holds two workgroups of 128 columns (76 KiB of
// LDS, 256 registers, 10 of them spilled) to fill each other's waits.  The matrix unit
// is busy 31% of the outputs' cycles forward and 35% backward, 24 to 35% of the states'
// (counters).  bf16, 16 heads of 128:
//   16,384 tokens: 77 us for the outputs (3.9 TB/s of q, k, v, o and states), 43 for
//   the segments' states, 17 for their join; the bytes alone would take 43
//   2 x 8,192 tokens backward: 218 us for dq, dk, dv (805 MB, 3.7 TB/s), 74 states
// Before the operands had parts, eight waves of 16 columns on two buffers, one
// workgroup a compute unit, took 530 us for both ways of the latter where two
// workgroups of four waves took 442; chunks through registers instead of straight to
// LDS 710.  For dq, dk, dv the operands are read three times: one walk of all three
// would need three states in registers.

template <class E>
struct Frag;
template <>
struct Frag<bf16> {
  typedef bf16x8 type;
};
template <>
struct Frag<float> {
  typedef float type __attribute__((ext_vector_type(8)));
};

__device__ __forceinline__ f32x4 mfma32(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma32(Frag<float>::type a, Frag<float>::type b, f32x4 c) {
#pragma unroll
  for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
  return c;
}

// A matrix of rows of W elements in LDS, as loads that go there directly write it:
// a wave's 64 pieces of 16 bytes follow one another in the order of its lanes.
// Within its row a piece lies at its number xor mix(row), so that 16 rows at one
// piece, and the rows that a transposing read takes together, fall on different
// banks.
template <class E, int W>
struct Tile {
  static constexpr int VN = 16 / (int)sizeof(E), NP = W / VN, RB = 64 / NP, BLOCK = 64 * VN;
  static_assert(NP >= 4 && NP <= 64 && RB * NP == 64, "rows of 64 bytes to 1 KiB");
  static constexpr int elements(int rows) { return rows * W; }
  typedef typename Frag<E>::type frag;

  // xor of parts that depend on (r & 3), (r & 12) and so on alone
  static __device__ __forceinline__ constexpr int mix(int r) {
    if (sizeof(E) == 4) return NP >= 16 ? r & 15 : NP == 8 ? (r >> 1) & 7 : (r >> 2) & 3;
    return NP >= 16 ? ((r & 3) << 2) | ((r >> 1) & 2) | ((r >> 3) & 1) : NP == 8 ? (r & 6) | ((r >> 3) & 1) : ((r >> 1) & 2) | ((r >> 3) & 1);
  }

  // Addresses, in bytes: a part of the lane, xor a constant in the bits of a row's
  // pieces, plus a constant of whole rows (16 of them leave mix as it is).
  static constexpr int kRow = W * (int)sizeof(E);
  static __device__ __forceinline__ const char* to(const E* base, int lane, int piece, int rows) {
    return reinterpret_cast<const char*>(base) + (lane ^ (piece * 16)) + rows * kRow;
  }

  // elements 32 b + 8 g .. + 8 of row r + m (r a multiple of 16)
  static __device__ __forceinline__ int row_lane(int g, int m) { return m * kRow + ((sizeof(E) == 2 ? g : 2 * g) ^ mix(m)) * 16; }
  static __device__ __forceinline__ frag row(const E* base, int lane, int r, int b) {
    if constexpr (sizeof(E) == 2) {
      return *reinterpret_cast<const frag*>(to(base, lane, 4 * b, r));
    } else {
      const f32x4 lo = *reinterpret_cast<const f32x4*>(to(base, lane, 8 * b, r)), hi = *reinterpret_cast<const f32x4*>(to(base, lane, 8 * b + 1, r));
      return frag{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    }
  }
  // element col + m, m = lane % 16, of rows 32 b + 4 g .. + 4 and 16 further (col a
  // multiple of 16)
  static __device__ __forceinline__ int column_lane(int g, int m) {
    if (sizeof(E) == 2) {
      const int r = 4 * g + (m >> 2);
      return r * kRow + (((m & 3) >> 1) ^ mix(r)) * 16 + (m & 1) * 8;
    }
    return 4 * g * kRow + ((m >> 2) ^ mix(4 * g)) * 16 + (m & 3) * 4;
  }
  static __device__ __forceinline__ frag column(const E* base, int lane, int b, int col) { return columns(base, lane, b, col / VN, 0); }
  // the same of element 32 kb + 8 (m / 4) + 4 u + m % 4
  static __device__ __forceinline__ int spread_lane(int g, int m) {
    if (sizeof(E) == 2) {
      const int r = 4 * g + (m >> 2);
      return r * kRow + ((m & 3) ^ mix(r)) * 16;
    }
    return 4 * g * kRow + ((2 * (m >> 2)) ^ mix(4 * g)) * 16 + (m & 3) * 4;
  }
  static __device__ __forceinline__ frag spread(const E* base, int lane, int b, int kb, int u) {
    return sizeof(E) == 2 ? columns(base, lane, b, 4 * kb, u) : columns(base, lane, b, 8 * kb + u, 0);
  }
  static __device__ __forceinline__ frag columns(const E* base, int lane, int b, int piece, int half) {
    if constexpr (sizeof(E) == 2) {
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      typedef short s16x8 __attribute__((ext_vector_type(8)));
      typedef __attribute__((address_space(3))) s16x4 lds4;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(to(base, lane, piece, 32 * b) + 8 * half));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(to(base, lane, piece, 32 * b + 16) + 8 * half));
      return __builtin_bit_cast(frag, (s16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      frag f;
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = *reinterpret_cast<const float*>(to(base, lane, piece ^ mix(j & 3), 32 * b + (j >> 2) * 16 + (j & 3)));
      return f;
    }
  }
};

// All of the wave's loads from memory, those to LDS among them.
__device__ __forceinline__ void wait_for_loads() {
  asm volatile("" : : : "memory");
  __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
  asm volatile("" : : : "memory");
}

// The address of a shared object in LDS.
template <class E>
__device__ __forceinline__ uint32_t lds_address(E* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) E*)p;
}

__device__ __forceinline__ bf16x8 pack(f32x4 a, f32x4 b, bf16) {
  return bf16x8{(bf16)a[0], (bf16)a[1], (bf16)a[2], (bf16)a[3], (bf16)b[0], (bf16)b[1], (bf16)b[2], (bf16)b[3]};
}
__device__ __forceinline__ Frag<float>::type pack(f32x4 a, f32x4 b, float) {
  return Frag<float>::type{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}

// A fragment in fp32, from its registers (the compiler would convert each element
// again on its own).
__device__ __forceinline__ Frag<float>::type widened(bf16x8 f) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  u32x4 u = __builtin_bit_cast(u32x4, f);
  asm volatile("" : "+v"(u));
  Frag<float>::type y;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[2 * i] = __builtin_bit_cast(float, u[i] << 16);
    y[2 * i + 1] = __builtin_bit_cast(float, u[i] & 0xffff0000u);
  }
  return y;
}
__device__ __forceinline__ Frag<float>::type widened(Frag<float>::type f) { return f; }

// g^n for n >= 0; lg2 = log2 g may be -inf (g = 0, g^0 = 1).
__device__ __forceinline__ float power(float lg2, int n) { return n == 0 ? 1.0f : __builtin_amdgcn_exp2f((float)n * lg2); }

// A value that all lanes hold, in a scalar register.
__device__ __forceinline__ float uniform(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x)));
}
__device__ __forceinline__ int64_t uniform(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}
template <class E>
__device__ __forceinline__ E* uniform(E* p) { return reinterpret_cast<E*>(uniform(reinterpret_cast<int64_t>(p))); }

// 16 bytes a lane from memory, `offset` bytes from `from` on, to LDS: the lanes'
// pieces follow one another from LDS address `to` + OFFSET (both the same in every
// lane) on.  Counted with the wave's other loads; the caller waits for all of them
// before the workgroup's barrier.  (Of the builtin the compiler takes every
// transposing read to depend, and waits for the next chunk before this one is used.
// The instruction has no result register, and nothing else here uses m0, which it
// takes its address from.  The wait covers a pointer that a vector instruction wrote
// just before.)
template <int OFFSET>
__device__ __forceinline__ void load_to_lds(const void* from, uint32_t offset, uint32_t to) {
  asm volatile("s_add_i32 m0, %0, %3\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(to), "v"(offset), "s"(uniform(from)), "i"(OFFSET) : "memory", "scc");
}

// What a launch runs: up to three scans of one shape, each cut into segments of
// whole chunks; seg[i] holds the segments' states ([state][segment][Dk][Dv]).
struct Jobs {
  Scan scan[3];
  float* seg[3];
  int32_t nseg;
  int64_t seg_tokens;  // whole chunks
};

// Tokens of a chunk.
template <class E, int DK>
struct ChunkOf {
  static constexpr int C = sizeof(E) == 2 && DK <= 128 ? 64 : 32;
};

constexpr int kWaves = 4, kChunkB = 64 * kWaves;
constexpr int kRescale = 8;  // powers of two between a state's rescalings (linattn_chunks)

// Rows of a chunk in memory: row r lies r `st` elements from row 0 (st < 0: back in
// time).  Addresses are a pointer that all lanes share, to the row that comes first in
// memory, and a 32-bit offset in bytes (the host sees to it that it holds).
struct Rows {
  int64_t st;
  __device__ __forceinline__ uint32_t offset(int r, int rows, int bytes) const {
    return (uint32_t)(st < 0 ? rows - 1 - r : r) * (uint32_t)((st < 0 ? -st : st) * bytes);
  }
  template <class E>
  __device__ __forceinline__ E* base(E* row0, int rows) const { return st < 0 ? row0 + (rows - 1) * st : row0; }
};

// One matrix of a chunk on its way to LDS, to elements AT .. of what begins at `lds`
// (this wave's first block of it at LDS address `address`), by a workgroup of four
// waves: C rows of W columns, whole blocks of pieces a wave.
template <class E, int W, int C, int AT>
struct Stage {
  typedef Tile<E, W> T;
  typedef E whole __attribute__((ext_vector_type(16 / sizeof(E))));
  static constexpr int N = C / T::RB / kWaves, STEP = kWaves * T::RB;  // blocks of a wave, rows between them
  static_assert(N * STEP == C, "whole blocks for every wave");

  static __device__ __forceinline__ int row_of(int i, int lane, int wave) { return i * STEP + wave * T::RB + lane / T::NP; }
  static __device__ __forceinline__ int column_of(int i, int lane, int wave) { return ((lane % T::NP) ^ T::mix(row_of(i, lane, wave))) * T::VN; }
  // a lane's place in memory: its first block's
  static __device__ __forceinline__ uint32_t offset(Rows m, int lane, int wave) {
    return m.offset(row_of(0, lane, wave), C, sizeof(E)) + column_of(0, lane, wave) * (int)sizeof(E);
  }

  // From row 0 at `row0` (its first column here) on.  WHOLE: all rows and columns are
  // there; else rows from L and columns from `width` on become zero.
  template <bool WHOLE, int I = 0>
  static __device__ __forceinline__ void pieces(E* lds, uint32_t address, const E* base, Rows m, uint32_t offset, int L, int width, int lane, int wave) {
    if constexpr (I < N) {
      constexpr int to = (AT + I * kWaves * T::BLOCK) * (int)sizeof(E);
      uint32_t at = offset;
      if constexpr (STEP % 16 != 0) at += (column_of(I, lane, wave) - column_of(0, lane, wave)) * (int)sizeof(E);
      if (WHOLE) {
        load_to_lds<to>(base, at, address);
      } else if (row_of(I, lane, wave) < L && column_of(I, lane, wave) < width) {
        load_to_lds<to>(base, at, address);
      } else {
        *reinterpret_cast<whole*>(lds + AT + (wave + kWaves * I) * T::BLOCK + lane * T::VN) = whole{};
      }
      pieces<WHOLE, I + 1>(lds, address, base + STEP * m.st, m, offset, L, width, lane, wave);
    }
  }
  // any width and alignment: through registers, element by element
  static __device__ __forceinline__ void elements(E* lds, const E* row0, Rows m, int L, int width, int lane, int wave) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = row_of(i, lane, wave), c = column_of(i, lane, wave);
      whole x{};
      if (r < L) {
#pragma unroll
        for (int e = 0; e < T::VN; ++e)
          if (c + e < width) x[e] = row0[r * m.st + c + e];
      }
      *reinterpret_cast<whole*>(lds + AT + (wave + kWaves * i) * T::BLOCK + lane * T::VN) = x;
    }
  }
};

// What a chunk kernel keeps in LDS: K of two chunks, V and Q of one, the scores'
// operands and the outputs, which take the place of a K that is done with where they
// fit there; where only states are wanted, K and V of two chunks.
template <class E, int DK, int NCT, bool OUT>
struct ChunkLds {
  static constexpr int C = ChunkOf<E, DK>::C, NT = C / 16, NB = C / 32, CT = 64 * NCT;
  static constexpr int kq = Tile<E, DK>::elements(C), kv = Tile<E, CT>::elements(C);
  static constexpr int turn = OUT ? 2 * kq + kv : kq + kv;  // elements from one K to the other
  static constexpr int all = (OUT ? 3 : 2) * kq + (OUT ? 1 : 2) * kv;
  static constexpr bool over = OUT && DK >= CT;
  E in[all];
  static constexpr int PARTS = sizeof(E) == 2 ? 2 : 1;  // of the state and the scores in a product
  // the scores of 16 queries and 32 keys, as far as the diagonal goes, by parts
  static constexpr int scores = NT + 2 * (NB - 1);
  static __device__ __forceinline__ constexpr int score(int t, int nb) { return (t + 2 * nb) * 64; }
  typename Frag<E>::type P[OUT ? PARTS * scores * 64 : 1];
  E out[OUT && !over ? kv : 1];
};

template <class E, int DK, int NCT, int SPLIT, bool OUT, bool PIECES>
__global__ __launch_bounds__(kChunkB, (sizeof(ChunkLds<E, DK, NCT, OUT>) > 80 * 1024 ? 1 : 2)) void linattn_chunks(Shape sh, Jobs jobs,
                                                                                                               int32_t col_tiles) {
  typedef ChunkLds<E, DK, NCT, OUT> Lds;
  constexpr int C = Lds::C, NT = Lds::NT, NB = Lds::NB, KB = DK / 32, CT = Lds::CT, B = kChunkB;
  typedef typename Frag<E>::type frag;
  typedef Tile<E, DK> KTile;
  typedef Tile<E, CT> VTile;
  constexpr int PARTS = Lds::PARTS;
  constexpr int AHEAD = DK <= 128 ? 1 : 0;  // LDS is read a step ahead; a state of 256 rows leaves no registers for it
  __shared__ __attribute__((aligned(16))) Lds lds;

  const Scan a = jobs.scan[blockIdx.y];
  const int nq = OUT ? a.nq : 1;
  uint32_t x = blockIdx.x;
  const int ct0 = (int)(x % (uint32_t)col_tiles) * CT;
  x /= (uint32_t)col_tiles;
  const int seg = (int)(x % (uint32_t)jobs.nseg);
  x /= (uint32_t)jobs.nseg;
  const int qh = (int)(x % (uint32_t)nq);
  const int64_t state = x / (uint32_t)nq, b = (uint32_t)state / (uint32_t)sh.Hs;
  if (b >= sh.B) return;  // the launch's scans differ in heads
  if (!OUT && !a.s1 && seg == jobs.nseg - 1) return;  // nothing follows the last segment
  const int j = (int)(state - b * sh.Hs);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g_ = lane >> 4, m_ = lane & 15;
  const int64_t len = uniform(length_of(sh, b));
  const double lgd = (double)sh.log_decay[j];
  const float lg2 = (float)(lgd * 1.4426950408889634074);
  const int back = a.back;
  const int64_t first = seg * (jobs.seg_tokens / C);
  int64_t last = first + jobs.seg_tokens / C;
  const int64_t chunks = (sh.T + C - 1) / C;
  if (last > chunks) last = chunks;
  const int64_t live = (len + C - 1) / C;  // chunks with tokens
  const int64_t end = last < live ? last : live;

  const int wcol = 16 * NCT * wave;
  const bool all_columns = a.Dk == DK && a.Dv - ct0 >= CT;

  const int dir = back ? -1 : 1;
  const Rows mq{dir * a.q.st}, mk{dir * a.k.st}, mv{dir * a.v.st}, mo{dir * a.o.st};
  const int64_t t0 = back ? len - 1 - first * C : first * C;  // the walk's first token
  const int qhead = j * a.nq + qh, khead = j * a.nk;
  typedef Stage<E, DK, C, 0> StageK;
  typedef Stage<E, CT, C, Lds::kq> StageV;
  typedef Stage<E, DK, C, OUT ? Lds::kq + Lds::kv : 0> StageQ;
  const uint32_t off_k = StageK::offset(mk, lane, wave), off_v = StageV::offset(mv, lane, wave), off_q = OUT ? StageQ::offset(mq, lane, wave) : 0;

  // a finished chunk's outputs, from LDS in whole pieces of a token's row
  constexpr int OSTEP = B / VTile::NP;
  const int orow0 = threadIdx.x / VTile::NP, ocol = threadIdx.x % VTile::NP;
  const uint32_t off_o = mo.offset(orow0, C, sizeof(E)) + ocol * 16;
  typedef E whole __attribute__((ext_vector_type(16 / sizeof(E))));
  whole done[C / OSTEP];
  auto read_outputs = [&](const E* out) {
#pragma unroll
    for (int i = 0; i < C / OSTEP; ++i) {
      const int r = orow0 + i * OSTEP;
      done[i] = *reinterpret_cast<const whole*>(out + r * CT + (ocol ^ VTile::mix(r)) * VTile::VN);
    }
  };
  auto store_outputs = [&](E* row0, int L) {
    typedef __attribute__((address_space(1))) typename Vec<E>::type global;
    int64_t p = reinterpret_cast<int64_t>(mo.base(row0, C));
    const bool all = all_columns && L == C;
#pragma unroll
    for (int i = 0; i < C / OSTEP; ++i, p += OSTEP * mo.st * (int)sizeof(E)) {
      asm volatile("" : "+s"(p));  // a pointer that all lanes share
      if (all || (orow0 + i * OSTEP < L && ct0 + ocol * VTile::VN < a.Dv)) *(global*)(p + off_o) = done[i];
    }
  };

  const E* sQ = lds.in + (OUT ? Lds::kq + Lds::kv : 0);
  frag* sP = lds.P;
  const uint32_t address = __builtin_amdgcn_readfirstlane(lds_address(lds.in) + wave * 1024);
  auto stage = [&](auto how, const E* row0, Rows m, uint32_t offset, int L, int width, int at) {
    typedef decltype(how) How;
    const uint32_t to = address + at * (int)sizeof(E);
    if (!PIECES)
      How::elements(lds.in + at, row0, m, L, width, lane, wave);
    else if (all_columns && L == C)
      How::template pieces<true>(lds.in + at, to, m.base(row0, C), m, offset, L, width, lane, wave);
    else
      How::template pieces<false>(lds.in + at, to, m.base(row0, C), m, offset, L, width, lane, wave);
  };
  auto stage_k = [&](const E* row0, int L, int at = 0) { stage(StageK(), row0, mk, off_k, L, a.Dk, at); };
  auto stage_v = [&](const E* row0, int L, int at = 0) { stage(StageV(), row0, mv, off_v, L, a.Dv - ct0, at); };
  auto stage_q = [&](const E* row0, int L) { stage(StageQ(), row0, mq, off_q, L, a.Dk, 0); };

  // item n of the walk: k/v head n % nk of chunk first + n / nk.  K, V and Q of the
  // next item are on their way from the second barrier of this one on; the other
  // workgroup of the compute unit works meanwhile.  Where only states are wanted,
  // the next item arrives in the other buffer.
  int count = first < end ? (int)(end - first) : 0;  // chunks left
  int64_t left = len - first * C;                    // tokens left
  const E *pq = uniform(OUT ? at<E>(a.q, b, t0, qhead) : nullptr), *pk = uniform(at<E>(a.k, b, t0, khead)), *pv = uniform(at<E>(a.v, b, t0, khead) + ct0);
  E* po = uniform(OUT && a.o.p ? at<E>(a.o, b, t0, qhead) + ct0 : nullptr);
  E* pending = nullptr;  // row 0 of outputs that wait in LDS
  int pending_rows = 0;
  f32x4 O[NT][NCT];
  if (count > 0) {
    const int L = left < C ? (int)left : C;
    stage_v(pv, L);
    if (OUT) stage_q(pq, L);
    stage_k(pk, L);
  }

  // What the registers hold is the state over `scale`: the product of the decays since
  // the beginning (kept to 48 bits, as its roundings would add up over the chunks),
  // times a power of two that keeps it between 1 and 2^(kRescale + 1).  So the registers
  // never hold more than the state itself, and 1 / scale, which rides on the weights of
  // the values, is never above 1: no state overflows that the recurrence's would not
  // (states below 2^-117 lose their last bits).  scale rides on the outputs' weights.
  const double gcd = exp(lgd * C);
  const float gc = uniform((float)gcd), gc_lo = uniform((float)(gcd - (double)(float)gcd));
  const double gld = len % C ? exp(lgd * (double)(len % C)) : 1.0;  // of the last chunk, where it is not whole
  const float gl = uniform((float)gld), gl_lo = uniform((float)(gld - (double)(float)gld));
  float scale = 1.0f, scale_lo = 0.0f;

  // The powers of a chunk's tokens are products of one per lane and some that all
  // lanes share (scalar registers): g^(16 t) and g, g^2, g^3.
  const float ps = a.qs * a.ks;
  const float qw = a.qs * power(lg2, m_ + 1 - back), kw = a.ks * power(lg2, 12 - 4 * g_ + back);
  float tiles[NT], step[4];
#pragma unroll
  for (int t = 0; t < NT; ++t) tiles[t] = uniform(power(lg2, 16 * t));
#pragma unroll
  for (int e = 0; e < 4; ++e) step[e] = uniform(power(lg2, e));

  // the state: tile (kb, u), column tile ct; a lane holds column 16 (NCT wave + ct)
  // + m, rows 32 kb + 8 g + 4 u + i
  const bool cut = jobs.nseg > 1;
  float* segments = cut ? jobs.seg[blockIdx.y] + (state * jobs.nseg + seg) * a.Dk * a.Dv : nullptr;
  f32x4 S[KB][2][NCT];
  {
    const float* s0 = cut ? (OUT ? segments : nullptr) : a.s0 ? a.s0 + state * a.Dk * a.Dv : nullptr;
    const bool flip = cut ? a.flip_seg : a.flip;
    typedef f32x4 four __attribute__((aligned(4)));
    if (!s0) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int ct = 0; ct < NCT; ++ct) S[kb][u][ct] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    } else if (all_columns && flip) {
      const float* p = s0 + (ct0 + wcol + m_) * DK + 8 * g_;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int ct = 0; ct < NCT; ++ct) S[kb][u][ct] = *reinterpret_cast<const four*>(p + 16 * ct * DK + 32 * kb + 4 * u);
    } else if (all_columns) {
      const int own = 8 * g_ * a.Dv + ct0 + wcol + m_;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int ct = 0; ct < NCT; ++ct) S[kb][u][ct][i] = s0[own + (32 * kb + 4 * u + i) * a.Dv + 16 * ct];
    } else {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int r = 32 * kb + 8 * g_ + 4 * u + i, c = ct0 + wcol + 16 * ct + m_;
              S[kb][u][ct][i] = r < a.Dk && c < a.Dv ? s0[flip ? c * a.Dk + r : r * a.Dv + c] : 0.0f;
            }
    }
  }

  wait_for_loads();  // the state's, which the compiler would count in the walk
  int h = 0, turn = 0;
  while (count > 0) {
    const int L = left < C ? (int)left : C;
    const bool last_head = h + 1 == a.nk;
    const int h_next = last_head ? 0 : h + 1;
    const int64_t left_next = last_head ? left - C : left;
    const int L_next = left_next < C ? (int)left_next : C;
    const bool more = !last_head || count > 1;
    const int64_t to_chunk = last_head ? C : 0, to_head = last_head ? h : -1;
    pk += to_chunk * mk.st - to_head * a.k.sh;
    pv += to_chunk * mv.st - to_head * a.v.sh;
    if (OUT) pq += to_chunk * mq.st;
    wait_for_loads();
    __syncthreads();
    E *sK = lds.in + turn, *other = lds.in + (turn ^= Lds::turn);
    const E* sV = OUT ? lds.in + Lds::kq : sK + Lds::kq;
    if (!OUT && more) {
      stage_k(pk, L_next, turn);
      stage_v(pv, L_next, turn);
    }
    if (OUT && PIECES && AHEAD && pending) read_outputs(Lds::over ? other : lds.out);
    // what follows from these is made anew in every chunk: kept over the walk, it
    // would cost the registers of a second workgroup
    int m = m_, g = g_;
    float kwc = kw, qwc = qw * scale;
    asm volatile("" : "+v"(m), "+v"(g), "+v"(kwc), "+v"(qwc));
    const int gap0 = m - 4 * g, at_row = KTile::row_lane(g, m);
    if (OUT) {
      // P^T by tiles of 16 queries and 16 keys, masked and decayed, as operands of
      // P V.  Of 64 tokens a wave takes the first two of a row of four and one of the
      // others, so that none waits for another; those past the diagonal are zero.
      constexpr int TILES = NT == 4 ? 3 : 1;
      f32x4 P[TILES];
      int tq[TILES], tk[TILES];
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
        tq[i] = NT == 2 ? wave >> 1 : i < 2 ? 3 - wave : wave & 1 ? 2 : 3;
        tk[i] = NT == 2 ? wave & 1 : i < 2 ? i : 2 + (wave >> 1);
        P[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      }
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        frag q;
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
          if (i != 1) q = KTile::row(sQ + KTile::elements(16) * tq[i], at_row, 0, kb);
          P[i] = mfma32(KTile::row(sK + KTile::elements(16) * tk[i], at_row, 0, kb), q, P[i]);
        }
      }
      // decays of a tile on the diagonal, and of one before it
      float near[4], off[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        near[e] = ps * power(lg2, gap0 > e ? gap0 - e : 0);
        off[e] = ps * __builtin_amdgcn_exp2f((float)(gap0 + 16 - e) * lg2);  // a power of at least one
      }
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
        const int apart = tq[i] - tk[i];
        float far = 0.0f;
#pragma unroll
        for (int t = 1; t < NT; ++t) far = apart == t ? tiles[t - 1] : far;
#pragma unroll
        for (int e = 0; e < 4; ++e) P[i][e] = gap0 + 16 * apart >= e ? P[i][e] * (apart == 0 ? near[e] : off[e] * far) : 0.0f;
      }
      typedef E four __attribute__((ext_vector_type(4)));
      constexpr int one = TILES - 1;
#pragma unroll
      for (int p = 0; p < PARTS; ++p) {
        frag* to = sP + p * Lds::scores * 64 + lane;
        if (TILES == 3) to[Lds::score(tq[0], 0)] = pack(P[0], P[1], E());
        reinterpret_cast<four*>(to + Lds::score(tq[one], tk[one] >> 1))[tk[one] & 1] = __builtin_convertvector(P[one], four);
        if (p + 1 < PARTS)
#pragma unroll
          for (int i = 0; i < TILES; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) P[i][e] -= (float)(E)P[i][e];
      }
    }

    if (OUT && PIECES && pending) {
      if (!AHEAD) read_outputs(Lds::over ? other : lds.out);
      store_outputs(pending, pending_rows);
      pending = nullptr;
    }
    asm volatile("" : "+v"(m), "+v"(g));
    const int at_q = KTile::row_lane(g, m), at_v = VTile::column_lane(g, m) ^ (wcol / VTile::VN * 16);
    frag V[NB][NCT];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct) V[nb][ct] = VTile::column(sV, at_v, nb, 16 * ct);

    bool odd = false;
    if (OUT) {
      // zeros times the values: zero unless one is infinite or NaN
      f32x4 z{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct) {
          if constexpr (sizeof(E) == 2) {
            z = mfma32(V[nb][ct], frag{}, z);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e & 3] = fmaf(V[nb][ct][e], 0.0f, z[e & 3]);
          }
        }
      odd = !__all(z[0] + z[1] + z[2] + z[3] == 0.0f);
      if (h == 0) {
        frag q[2][NT];
        if (AHEAD) {
#pragma unroll
          for (int t = 0; t < NT; ++t) q[0][t] = KTile::row(sQ, at_q, 16 * t, 0);
        }
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
          frag s[PARTS][NCT];
#pragma unroll
          for (int ct = 0; ct < NCT; ++ct) {
            s[0][ct] = pack(S[kb][0][ct], S[kb][1][ct], E());
            if constexpr (PARTS == 2) s[1][ct] = __builtin_convertvector(pack(S[kb][0][ct], S[kb][1][ct], float()) - widened(s[0][ct]), frag);
          }
          if (kb + AHEAD < KB) {
#pragma unroll
            for (int t = 0; t < NT; ++t) q[(kb + AHEAD) & 1][t] = KTile::row(sQ, at_q, 16 * t, kb + AHEAD);
          }
          __builtin_amdgcn_sched_barrier(0);  // reads stay ahead of the products
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int ct = 0; ct < NCT; ++ct) {
              O[t][ct] = mfma32(s[0][ct], q[kb & 1][t], kb ? O[t][ct] : f32x4{0.0f, 0.0f, 0.0f, 0.0f});
              if constexpr (PARTS == 2) O[t][ct] = mfma32(s[1][ct], q[kb & 1][t], O[t][ct]);
            }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int ct = 0; ct < NCT; ++ct) O[t][ct] *= qwc * tiles[t];
      }
    }
    if (OUT) {
      __syncthreads();
      frag p[NT][NB];
      auto read_scores = [&] {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int nb = 0; nb <= t / 2; ++nb) p[t][nb] = sP[Lds::score(t, nb) + lane];
      };
      if (AHEAD) read_scores();
      if (more) stage_k(pk, L_next, turn);
      if (!odd) {
        if (!AHEAD) read_scores();
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int t = 2 * nb; t < NT; ++t)
#pragma unroll
            for (int ct = 0; ct < NCT; ++ct) O[t][ct] = mfma32(V[nb][ct], p[t][nb], O[t][ct]);
        if constexpr (PARTS == 2) {
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int t = 2 * nb; t < NT; ++t) {
              const frag low = sP[Lds::scores * 64 + Lds::score(t, nb) + lane];
#pragma unroll
              for (int ct = 0; ct < NCT; ++ct) O[t][ct] = mfma32(V[nb][ct], low, O[t][ct]);
            }
        }
      } else {
        // a product with the zeros of the mask would carry an infinity or NaN to
        // earlier tokens, so the sum stops at the token
        asm volatile("" : "+v"(m), "+v"(g));
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll 1
          for (int n = 0; n < 32; ++n) {  // token 32 nb + 16 (n / 16) + 4 sg + n % 4 of the block, element e of the lanes of group sg
            const int sg = (n >> 2) & 3, e = ((n >> 4) << 2) | (n & 3), late = 32 * nb + n - m;  // from query 16 t + m >= s on
            float p[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              p[t] = 0.0f;
#pragma unroll
              for (int part = 0; part < PARTS; ++part)
                p[t] += late <= 16 * t ? (float)reinterpret_cast<const E*>(&sP[part * Lds::scores * 64 + Lds::score(t, nb) + sg * 16 + m])[e] : 0.0f;
            }
#pragma unroll
            for (int ct = 0; ct < NCT; ++ct) {
              float own = 0.0f;
#pragma unroll
              for (int k = 0; k < 8; ++k) own = e == k ? (float)V[nb][ct][k] : own;
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float v = __shfl(own, sg * 16 + 4 * g + i, 64);
#pragma unroll
                for (int t = 0; t < NT; ++t) O[t][ct][i] = fmaf(p[t], late <= 16 * t ? v : 0.0f, O[t][ct][i]);
              }
            }
          }
      }
      if (more) stage_v(pv, L_next);
      if (!PIECES && last_head && po) {
        const int col = wcol + 4 * g;
        E* p = po + m * mo.st + col;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
          for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (16 * t + m < L && ct0 + col + 16 * ct + i < a.Dv) p[16 * ct + i] = (E)O[t][ct][i];
          p += 16 * mo.st;
        }
        po += C * mo.st;
      }
    }

    asm volatile("" : "+v"(m), "+v"(g));
    const int at_k = KTile::spread_lane(g, m);
    if (h == 0) {
      const float d = L < C ? gl : gc, d_lo = L < C ? gl_lo : gc_lo;
      const float x = scale * d, y = fmaf(scale, d, -x) + fmaf(scale, d_lo, scale_lo * d);
      scale = uniform(x + y);
      scale_lo = uniform(y - (scale - x));
      if (!(scale >= 1.0f)) {
        const bool far = !(scale > 0x1p-60f);  // hardly anything is left, or nothing at all
        const uint32_t bits = __builtin_bit_cast(uint32_t, scale) & 0x7f800000u, one = 127u << 23, top = (uint32_t)kRescale << 23;
        const float down = far ? scale : __builtin_bit_cast(float, bits - top), up = __builtin_bit_cast(float, 2 * one - bits + top);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int ct = 0; ct < NCT; ++ct) S[kb][u][ct] *= down;
        scale = far ? 1.0f : scale * up;
        scale_lo = far ? 0.0f : scale_lo * up;
      }
    }
    const float back_to = uniform(1.0f / scale);
    kwc *= back_to;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      float w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        w[e] = kwc * tiles[NT - 1 - 2 * nb - (e >> 2)];
        if ((e & 3) < 3) w[e] *= step[3 - (e & 3)];
      }
      if (L < C) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int n = L - 1 + back - 4 * g - (32 * nb + (e >> 2) * 16 + (e & 3));
          w[e] = n >= back ? a.ks * back_to * power(lg2, n) : 0.0f;
        }
      }
      // the weighted values in SPLIT parts, each the rounding of what is left
      frag part[SPLIT][NCT];
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct) {
        typename Frag<float>::type y;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = (float)V[nb][ct][e] * w[e];
#pragma unroll
        for (int p = 0; p < SPLIT; ++p) {
          part[p][ct] = __builtin_convertvector(y, frag);
          if (p + 1 < SPLIT) y -= widened(part[p][ct]);
        }
      }
      frag k[2][2];
      if (AHEAD) {
#pragma unroll
        for (int u = 0; u < 2; ++u) k[0][u] = KTile::spread(sK, at_k, nb, 0, u);
      }
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        if (kb + AHEAD < KB) {
#pragma unroll
          for (int u = 0; u < 2; ++u) k[(kb + AHEAD) & 1][u] = KTile::spread(sK, at_k, nb, kb + AHEAD, u);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int p = 0; p < SPLIT; ++p)
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int ct = 0; ct < NCT; ++ct) S[kb][u][ct] = mfma32(k[kb & 1][u], part[p][ct], S[kb][u][ct]);
      }
      if (OUT && nb == 0 && more && last_head) stage_q(pq, L_next);
    }
    if (OUT && PIECES && last_head && po) {
      if (Lds::over) __syncthreads();  // K is done with
      typedef E four __attribute__((ext_vector_type(4)));
      E* out = (Lds::over ? sK : lds.out) + m * CT;
      asm volatile("" : "+v"(m), "+v"(g));
      constexpr int per = VTile::VN / 4;  // fours of a piece
      const int piece = (wcol / VTile::VN + g / per) ^ VTile::mix(m);
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct)
          *reinterpret_cast<four*>(out + 16 * t * CT + (piece ^ (16 * ct / VTile::VN)) * VTile::VN + g % per * 4) = __builtin_convertvector(O[t][ct], four);
      pending = po;
      pending_rows = L;
      po += C * mo.st;
    }
    count -= last_head ? 1 : 0;
    left = left_next;
    h = h_next;
  }

  if (OUT && PIECES && pending) {
    __syncthreads();
    read_outputs(Lds::over ? lds.in + (turn ^ Lds::turn) : lds.out);
    store_outputs(pending, pending_rows);
  }

  if (OUT && a.o.p) {  // tokens past the sequence's length
    E* o = at<E>(a.o, b, 0, qhead);
    const int64_t from = len > first * C ? len : first * C, to = last * C < sh.T ? last * C : sh.T;
    for (int64_t t = from + wave; t < to; t += kWaves)
      for (int col = ct0 + lane; col < ct0 + CT && col < a.Dv; col += 64) o[t * a.o.st + col] = (E)0.0f;
  }
  float* s1 = cut ? (OUT ? nullptr : segments) : a.s1 && qh == 0 ? a.s1 + state * a.Dk * a.Dv : nullptr;
  if (s1) {
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));  // addresses anew: those of the initial state are not kept over the walk
    const int r0 = 8 * ((tid & 63) >> 4), c0 = ct0 + 16 * NCT * (tid >> 6) + (tid & 15), own = r0 * a.Dv + c0;
    if (all_columns) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int ct = 0; ct < NCT; ++ct)
              s1[own + (32 * kb + 4 * u + i) * a.Dv + 16 * ct] = fmaf(S[kb][u][ct][i], scale, S[kb][u][ct][i] * scale_lo);
      return;
    }
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int r = r0 + 32 * kb + 4 * u + i, col = c0 + 16 * ct;
            if (r < a.Dk && col < a.Dv) s1[r * a.Dv + col] = fmaf(S[kb][u][ct][i], scale, S[kb][u][ct][i] * scale_lo);
          }
  }
}

// The segments' own states to the states before them, in place, and the last:
//   before_0 = s0, before_{i+1} = g^(tokens of i) before_i + own_i
// One element a lane, eight segments in flight; bound by memory (32 segments of 16
// heads of 128, 67 MB: 16 us, 4.1 TB/s).
constexpr int kJoinB = 256, kJoinAhead = 8;
__global__ __launch_bounds__(kJoinB) void linattn_join(Shape sh, Jobs jobs) {
  const Scan& a = jobs.scan[blockIdx.y];
  const int n = a.Dk * a.Dv, blocks = (n + kJoinB - 1) / kJoinB;
  const int64_t state = blockIdx.x / blocks, b = state / sh.Hs;
  const int e = (int)(blockIdx.x % blocks) * kJoinB + threadIdx.x;
  if (b >= sh.B || e >= n) return;
  const int64_t len = length_of(sh, b), per = jobs.seg_tokens;
  const double lgd = (double)sh.log_decay[state - b * sh.Hs];
  const float whole = (float)exp(lgd * (double)per);
  float* buf = jobs.seg[blockIdx.y] + state * jobs.nseg * n + e;
  float S = a.s0 ? a.s0[state * n + (a.flip ? e % a.Dv * a.Dk + e / a.Dv : e)] : 0.0f;
  for (int i0 = 0; i0 < jobs.nseg; i0 += kJoinAhead) {
    float own[kJoinAhead];
#pragma unroll
    for (int i = 0; i < kJoinAhead; ++i) own[i] = i0 + i < jobs.nseg - (a.s1 ? 0 : 1) ? buf[(int64_t)(i0 + i) * n] : 0.0f;
#pragma unroll
    for (int i = 0; i < kJoinAhead; ++i)
      if (i0 + i < jobs.nseg) {
        const int64_t left = len - (i0 + i) * per;
        buf[(int64_t)(i0 + i) * n] = S;
        if (left >= per) S = fmaf(S, whole, own[i]);
        else if (left > 0) S = fmaf(S, (float)exp(lgd * (double)left), own[i]);
      }
  }
  if (a.s1) a.s1[state * n + e] = S;
}

// ---- host -------------------------------------------------------------------

constexpr int kMaxWidth = 256;
constexpr int kUnit = 64;  // tokens in whole chunks of every kernel

template <class E>
void launch_any(const Shape& s, const Scan& a, hipStream_t st) {
  const int tiles = (a.Dv + kAnyCols - 1) / kAnyCols;
  const dim3 grid((unsigned)(s.B * s.Hs * tiles)), block(kAnyB);
  if (a.Dk <= 64)
    hipLaunchKernelGGL((linattn_one_any<E, 4>), grid, block, 0, st, s, a, tiles);
  else if (a.Dk <= 128)
    hipLaunchKernelGGL((linattn_one_any<E, 8>), grid, block, 0, st, s, a, tiles);
  else
    hipLaunchKernelGGL((linattn_one_any<E, 16>), grid, block, 0, st, s, a, tiles);
}

template <class E>
void launch_one(const Shape& s, const Scan& a, hipStream_t st) {
  const int tiles = (a.Dv + 4 * kStepCG - 1) / (4 * kStepCG);
  const dim3 grid((unsigned)(s.B * s.Hs * tiles)), block(kStepB);
  if (a.Dk <= 32)
    hipLaunchKernelGGL((linattn_one<E, 1>), grid, block, 0, st, s, a, tiles);
  else if (a.Dk <= 64)
    hipLaunchKernelGGL((linattn_one<E, 2>), grid, block, 0, st, s, a, tiles);
  else if (a.Dk <= 128)
    hipLaunchKernelGGL((linattn_one<E, 4>), grid, block, 0, st, s, a, tiles);
  else
    hipLaunchKernelGGL((linattn_one<E, 8>), grid, block, 0, st, s, a, tiles);
}

// A chunk's rows lie within 32-bit offsets.
bool near_rows(const HeadArr& h, int32_t dtype) { return (h.st < 0 ? -h.st : h.st) <= (int64_t(1) << 31) / kUnit / elem_size(dtype); }

// Loads that go to LDS take addresses of whole 4 bytes.
bool loads_in_pieces(const HeadArr& h, int32_t dtype) {
  const int per = 4 / (int)elem_size(dtype);
  return aligned_to(h.p, 4) && h.sb % per == 0 && h.st % per == 0 && h.sh % per == 0 && near_rows(h, dtype);
}

// Which chunk kernel a scan takes: key rows, column tiles of a wave.
struct Class {
  int dk, nct;
  bool pieces;
};

Class class_of(const Scan& a, int32_t dtype) {
  Class c;
  c.dk = a.Dk <= 32 ? 32 : a.Dk <= 64 ? 64 : a.Dk <= 128 ? 128 : 256;
  c.nct = c.dk == 128 || (c.dk == 256 && dtype == DIFFOPT_BF16) ? 2 : 1;
  const int vn = dtype == DIFFOPT_F32 ? 4 : 8;
  c.pieces = a.Dk % vn == 0 && a.Dv % vn == 0 && loads_in_pieces(a.q, dtype) && loads_in_pieces(a.k, dtype) && loads_in_pieces(a.v, dtype) &&
             near_rows(a.o, dtype);
  return c;
}

// Segments of a call's scans.  A workgroup walks its chunks one after another,
// so with few heads a sequence is cut until the workgroups fill the card: two of
// them share a compute unit, three or more where the state has at most 64 rows
// (six ragged sequences of up to 1,021 tokens, heads of 64, both ways: 86 us for
// four, 86 for three, 105 for two; a prompt of 16,384 tokens with heads of 128: 134 for
// two, 164 for four).  A cut costs one more read of k and v and the segments' states,
// so there is none from half of that on, and no segment is shorter than kMinUnits (with
// 8 the ragged ones take 114 us, with 2 they take 83, and the states of wide heads cost
// as much as their tokens).
constexpr int kFill = 512, kFillNarrow = 1024, kMinUnits = 4;

struct Plan {
  int32_t nseg;
  int64_t seg_tokens;  // a multiple of kUnit
};

Plan plan_of(int64_t workgroups, int64_t T, int64_t fill) {
  const int64_t units = (T + kUnit - 1) / kUnit;
  int64_t n = workgroups > 0 ? fill / workgroups : 1;
  if (n > units / kMinUnits) n = units / kMinUnits;
  if (n < 1) n = 1;
  const int64_t per = units > 0 ? (units + n - 1) / n : 1;
  n = (units + per - 1) / per;
  return Plan{(int32_t)(n > 1 ? n : 1), per * kUnit};
}

int64_t col_tiles(const Scan& a, int32_t dtype) {
  const int ct = 64 * class_of(a, dtype).nct;
  return (a.Dv + ct - 1) / ct;
}

int64_t main_groups(const Shape& s, const Scan& a, int32_t dtype) { return s.B * s.Hs * a.nq * col_tiles(a, dtype); }

int64_t segment_bytes(const Shape& s, const Scan& a, const Plan& p) {
  return p.nseg > 1 ? (s.B * s.Hs * p.nseg * a.Dk * a.Dv * 4 + 255) / 256 * 256 : 0;
}

Plan plan_of(const Shape& s, const Scan* a, int n, int32_t dtype) {
  int64_t w = 0, fill = kFillNarrow;
  for (int i = 0; i < n; ++i) {
    w += main_groups(s, a[i], dtype);
    if (a[i].Dk > 64) fill = kFill;
  }
  return plan_of(w, s.T, fill);
}

// The scans of a call, as the sizes alone make them.
int forward_scans(int64_t H, int64_t Hk, int64_t Dk, int64_t Dv, Scan* a) {
  a[0] = Scan{};
  a[0].nq = (int32_t)(H / Hk);
  a[0].nk = 1;
  a[0].Dk = (int32_t)Dk;
  a[0].Dv = (int32_t)Dv;
  return 1;
}

// dq, dk, dv
int backward_scans(int64_t H, int64_t Hk, int64_t Dk, int64_t Dv, Scan* a) {
  for (int i = 0; i < 3; ++i) {
    a[i] = Scan{};
    a[i].nq = i == 0 ? (int32_t)(H / Hk) : 1;
    a[i].nk = i == 0 ? 1 : (int32_t)(H / Hk);
    a[i].Dk = (int32_t)(i == 2 ? Dk : Dv);
    a[i].Dv = (int32_t)(i == 2 ? Dv : Dk);
    a[i].back = i > 0;
    a[i].flip = i < 2;
    a[i].flip_seg = i == 1;  // dk's states are dv's transposed: it reads those
  }
  return 3;
}

int64_t workspace_of(const Shape& s, const Scan* a, int n, int32_t dtype) {
  const Plan p = plan_of(s, a, n, dtype);
  int64_t bytes = 0;
  for (int i = 0; i < n; ++i) bytes += a[i].flip_seg ? 0 : segment_bytes(s, a[i], p);
  return bytes;
}

template <class E, int DK, int NCT, bool PIECES>
void launch_class(const Shape& s, const Jobs& jobs, int n, bool states, bool keep, hipStream_t st) {
  constexpr int MOST = sizeof(E) == 2 ? 3 : 1, SPLIT = sizeof(E) == 2 && PIECES ? 2 : MOST;
  int64_t tiles = 0, main = 0, own = 0;
  for (int i = 0; i < n; ++i) {
    const int64_t c = col_tiles(jobs.scan[i], sizeof(E) == 4 ? DIFFOPT_F32 : DIFFOPT_BF16);
    tiles = c > tiles ? c : tiles;
    keep |= jobs.scan[i].s1 != nullptr && (states || jobs.nseg == 1);  // a state is handed out
  }
  for (int i = 0; i < n; ++i) {
    const int64_t w = s.B * s.Hs * jobs.nseg * tiles;
    own = w > own ? w : own;
    main = w * jobs.scan[i].nq > main ? w * jobs.scan[i].nq : main;
  }
  const dim3 grid((unsigned)(states ? own : main), n), block(kChunkB);
  if (states && keep)
    hipLaunchKernelGGL((linattn_chunks<E, DK, NCT, MOST, false, PIECES>), grid, block, 0, st, s, jobs, (int32_t)tiles);
  else if (states)
    hipLaunchKernelGGL((linattn_chunks<E, DK, NCT, SPLIT, false, PIECES>), grid, block, 0, st, s, jobs, (int32_t)tiles);
  else if (keep)
    hipLaunchKernelGGL((linattn_chunks<E, DK, NCT, MOST, true, PIECES>), grid, block, 0, st, s, jobs, (int32_t)tiles);
  else
    hipLaunchKernelGGL((linattn_chunks<E, DK, NCT, SPLIT, true, PIECES>), grid, block, 0, st, s, jobs, (int32_t)tiles);
}

// `keep`: the values' parts as where a state is handed out, also if none is.
template <class E>
void launch_chunks(const Shape& s, const Jobs& jobs, int n, bool states, bool keep, hipStream_t st) {
  // scans of one class share a launch
  bool done[3] = {false, false, false};
  const int32_t dtype = sizeof(E) == 4 ? DIFFOPT_F32 : DIFFOPT_BF16;
  for (int i = 0; i < n; ++i) {
    if (done[i]) continue;
    const Class c = class_of(jobs.scan[i], dtype);
    Jobs part = jobs;
    int k = 0;
    for (int l = i; l < n; ++l) {
      const Class d = class_of(jobs.scan[l], dtype);
      if (done[l] || d.dk != c.dk || d.pieces != c.pieces || col_tiles(jobs.scan[l], dtype) != col_tiles(jobs.scan[i], dtype)) continue;
      done[l] = true;
      part.scan[k] = jobs.scan[l];
      part.seg[k++] = jobs.seg[l];
    }
#define DIFFOPT_CLASS(DK, NCT)                                        \
  if (c.dk == DK && c.pieces) launch_class<E, DK, NCT, true>(s, part, k, states, keep, st); \
  if (c.dk == DK && !c.pieces) launch_class<E, DK, NCT, false>(s, part, k, states, keep, st);
    DIFFOPT_CLASS(32, 1)
    DIFFOPT_CLASS(64, 1)
    DIFFOPT_CLASS(128, 2)
    if constexpr (sizeof(E) == 2) {
      DIFFOPT_CLASS(256, 2)
    } else {
      DIFFOPT_CLASS(256, 1)
    }
#undef DIFFOPT_CLASS
  }
}

// Workgroups write results while others still read operands, in no order: a result
// at the address of an operand or of another result is refused.  (Other overlaps, of
// views that are cut differently, are the caller's to avoid.)
int check_apart(const char* who, std::initializer_list<const void*> results, std::initializer_list<const void*> operands) {
  for (auto r = results.begin(); r != results.end(); ++r) {
    if (!*r) continue;
    for (const void* p : operands)
      if (*r == p) return fail(DIFFOPT_EINVAL, "%s: a result must not be an operand", who);
    for (auto t = results.begin(); t != r; ++t)
      if (*r == *t) return fail(DIFFOPT_EINVAL, "%s: two results must not be one tensor", who);
  }
  return DIFFOPT_OK;
}

// A call's workspace against what its scans need.
int check_workspace(const char* who, const Shape& s, const Scan* a, int n, int32_t dtype, void* workspace, int64_t bytes) {
  const int64_t need = workspace_of(s, a, n, dtype);
  if (need > 0 && (!workspace || bytes < need))
    return fail(DIFFOPT_EINVAL, "%s: the workspace has %lld bytes of %lld", who, (long long)(workspace ? bytes : 0), (long long)need);
  if (!aligned_to(workspace, 16)) return fail(DIFFOPT_EINVAL, "%s: the workspace is not 16-byte aligned", who);
  return DIFFOPT_OK;
}

// Runs the scans whose `run` is set; `a` holds all the call's scans, by which
// the plan goes.
int run_scans(const char* who, const Shape& s, const Scan* a, const bool* run, int n, int32_t dtype, void* workspace, hipStream_t st) {
  const Plan p = plan_of(s, a, n, dtype);
  // `walk`: the scans whose outputs are wanted; `own`: those that have states of
  // their own to find first (dk takes dv's)
  Jobs walk{}, own{};
  walk.nseg = own.nseg = p.nseg;
  walk.seg_tokens = own.seg_tokens = p.seg_tokens;
  float* at = static_cast<float*>(workspace);
  int nwalk = 0, nown = 0;
  for (int i = 0; i < n; ++i) {
    const bool shared = i + 1 < n && a[i].flip_seg;
    if (run[i]) {
      walk.scan[nwalk] = a[i];
      walk.seg[nwalk++] = at;
    }
    if (!shared) {
      if (run[i] || (i > 0 && a[i - 1].flip_seg && run[i - 1])) {
        own.scan[nown] = a[i];
        own.seg[nown++] = at;
      }
      at += segment_bytes(s, a[i], p) / 4;
    }
  }
  if (nwalk == 0) return DIFFOPT_OK;
  const bool f32 = dtype == DIFFOPT_F32;
  if (p.nseg > 1) {
    f32 ? launch_chunks<float>(s, own, nown, true, false, st) : launch_chunks<bf16>(s, own, nown, true, false, st);
    const int64_t groups = s.B * s.Hs * ((own.scan[0].Dk * own.scan[0].Dv + kJoinB - 1) / kJoinB);
    hipLaunchKernelGGL(linattn_join, dim3((unsigned)groups, nown), dim3(kJoinB), 0, st, s, own);
  }
  // A state in place, in one segment, that several workgroups begin from (one for each
  // query head): no order holds between one's last store and another's loads, so the
  // outputs come first and the state in a launch of its own, a workgroup for each.
  Scan& only = walk.scan[0];
  const bool after = p.nseg == 1 && nwalk == 1 && only.nq > 1 && only.s1 && only.s1 == only.s0;
  const Jobs state = walk;
  if (after) only.s1 = nullptr;
  f32 ? launch_chunks<float>(s, walk, nwalk, false, after, st) : launch_chunks<bf16>(s, walk, nwalk, false, after, st);
  if (after) f32 ? launch_chunks<float>(s, state, 1, true, true, st) : launch_chunks<bf16>(s, state, 1, true, true, st);
  return launch_status(who);
}

const char* sizes_wrong(int64_t B, int64_t T, int64_t H, int64_t Hk, int64_t Dk, int64_t Dv, int32_t dtype) {
  if (B < 0 || T < 0 || H < 0 || Hk < 0) return "B, T, H and Hk must be >= 0";
  if ((H == 0) != (Hk == 0) || (Hk > 0 && H % Hk)) return "H must be a multiple of Hk";
  if (Dk < 1 || Dk > kMaxWidth || Dv < 1 || Dv > kMaxWidth) return "Dk and Dv must be in [1, 256]";
  if (!dtype_ok(dtype)) return "unknown element type";
  // a launch has fewer than 2^32 threads, a workgroup of 256 for each head and 32
  // columns at most
  constexpr int64_t kMost = int64_t(1) << 24;
  if (H > 65536 || B >= kMost || B * H * (((Dk > Dv ? Dk : Dv) + 31) / 32) >= kMost || T > (int64_t(1) << 35))
    return "too many heads, sequences or tokens";
  return nullptr;
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
  if (sizes_wrong(B, T, H, Hk, Dk, Dv, dtype)) return -1;
  if (B == 0 || Hk == 0 || T == 0) return 0;
  Scan a[3];
  const int n = backward ? backward_scans(H, Hk, Dk, Dv, a) : forward_scans(H, Hk, Dk, Dv, a);
  return workspace_of(Shape{B, T, (int32_t)Hk, nullptr, nullptr}, a, n, dtype);
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
  Scan a[1];
  forward_scans(H, Hk, Dk, Dv, a);
  if (T > 0) {
    rc = check_heads(who, "q", q, dtype, &a[0].q);
    if (!rc) rc = check_heads(who, "k", k, dtype, &a[0].k);
    if (!rc) rc = check_heads(who, "v", v, dtype, &a[0].v);
    if (!rc) rc = check_heads(who, "out", out, dtype, &a[0].o);
    if (rc) return rc;
  } else if (!state_out) {
    return DIFFOPT_OK;
  }
  a[0].s0 = state;
  a[0].s1 = state_out;
  a[0].qs = (float)scale;
  a[0].ks = 1.0f;
  const bool run[1] = {true};
  const Shape s{B, T, (int32_t)Hk, log_decay, lengths};
  rc = check_workspace(who, s, a, 1, dtype, workspace, workspace_bytes);
  if (!rc) rc = check_apart(who, {a[0].o.p}, {a[0].q.p, a[0].k.p, a[0].v.p});
  if (!rc && state != state_out && overlap(state, B * Hk * Dk * Dv * 4, state_out, B * Hk * Dk * Dv * 4))
    rc = fail(DIFFOPT_EINVAL, "%s: state_out must be state or lie apart from it", who);
  return rc ? rc : run_scans(who, s, a, run, 1, dtype, workspace, as_stream(stream));
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
  const int64_t state_bytes = B * Hk * Dk * Dv * 4;
  if (overlap(dstate, state_bytes, dstate_out, state_bytes) || overlap(dstate, state_bytes, state, state_bytes))
    return fail(DIFFOPT_EINVAL, "%s: dstate must be neither dstate_out nor state", who);
  HeadArr Q{}, K{}, V{}, DO{};
  Scan a[3];
  backward_scans(H, Hk, Dk, Dv, a);
  if (T > 0) {
    rc = check_heads(who, "q", q, dtype, &Q);
    if (!rc) rc = check_heads(who, "k", k, dtype, &K);
    if (!rc) rc = check_heads(who, "v", v, dtype, &V);
    if (!rc) rc = check_heads(who, "dout", dout, dtype, &DO);
    if (!rc && dq) rc = check_heads(who, "dq", dq, dtype, &a[0].o);
    if (!rc && dk) rc = check_heads(who, "dk", dk, dtype, &a[1].o);
    if (!rc && dv) rc = check_heads(who, "dv", dv, dtype, &a[2].o);
    if (rc) return rc;
  }
  const HeadArr in[3][3] = {{DO, V, K}, {V, DO, Q}, {K, Q, DO}};
  for (int i = 0; i < 3; ++i) {
    a[i].q = in[i][0];
    a[i].k = in[i][1];
    a[i].v = in[i][2];
    a[i].s0 = i == 0 ? state : dstate_out;
    a[i].qs = i == 0 ? (float)scale : 1.0f;
    a[i].ks = i == 0 ? 1.0f : (float)scale;
  }
  a[2].s1 = dstate;
  const bool run[3] = {a[0].o.p != nullptr, a[1].o.p != nullptr, a[2].o.p != nullptr || dstate != nullptr};
  const Shape s{B, T, (int32_t)Hk, log_decay, lengths};
  rc = check_workspace(who, s, a, 3, dtype, workspace, workspace_bytes);
  if (!rc) rc = check_apart(who, {a[0].o.p, a[1].o.p, a[2].o.p}, {DO.p, Q.p, K.p, V.p});
  return rc ? rc : run_scans(who, s, a, run, 3, dtype, workspace, as_stream(stream));
}

extern "C" int diffopt_linattn_step(const diffopt_heads* q, const diffopt_heads* k, const diffopt_heads* v,
                                    const float* log_decay, int64_t B, int64_t H, int64_t Hk, int64_t Dk, int64_t Dv,
                                    int32_t dtype, double scale, float* state, const diffopt_heads* out, void* stream) {
  clear_error();
  static const char* who = "diffopt_linattn_step";
  int rc = check_call(who, B, 1, H, Hk, Dk, Dv, dtype, scale, log_decay, nullptr, {state});
  if (rc || B == 0 || Hk == 0) return rc;
  if (!state) return fail(DIFFOPT_EINVAL, "%s: null state", who);
  Scan a[1];
  forward_scans(H, Hk, Dk, Dv, a);
  rc = check_heads(who, "q", q, dtype, &a[0].q);
  if (!rc) rc = check_heads(who, "k", k, dtype, &a[0].k);
  if (!rc) rc = check_heads(who, "v", v, dtype, &a[0].v);
  if (!rc) rc = check_heads(who, "out", out, dtype, &a[0].o);
  if (!rc) rc = check_apart(who, {a[0].o.p}, {a[0].q.p, a[0].k.p, a[0].v.p});
  if (rc) return rc;
  a[0].s0 = state;
  a[0].s1 = state;
  a[0].qs = (float)scale;
  a[0].ks = 1.0f;
  const Shape s{B, 1, (int32_t)Hk, log_decay, nullptr};
  hipStream_t st = as_stream(stream);
  const bool pieces = Dv % 4 == 0 && aligned_to(state, 16);  // rows of whole 16-byte pieces
  if (dtype == DIFFOPT_F32)
    pieces ? launch_one<float>(s, a[0], st) : launch_any<float>(s, a[0], st);
  else
    pieces ? launch_one<bf16>(s, a[0], st) : launch_any<bf16>(s, a[0], st);
  return launch_status(who);
}
