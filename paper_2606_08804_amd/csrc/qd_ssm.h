// Shared pieces of the selective state space scan's kernels.
//
// MFMA operands here are "quads": a step covers 32 values of k as two blocks
// of 16, and lane l holds k = 4 (l / 16) .. + 3 of either block.  That is the
// order in which a 16 x 16 accumulator holds its rows, so an accumulator pair
// is an operand as it stands (its rows become k), without a trip through LDS.
// bf16 takes one 16x16x32 instruction a step, fp32 eight 16x16x4 ones.
//
// A fp32 value enters a bf16 product as a sum of bf16 values ("planes"):
// x = hi + lo is off by 2^-16 at most, x = hi + mid + lo is exact.  Two planes
// where the result is rounded to bf16, three where it is fp32.
#pragma once

#include "qd_mixer.h"

namespace qd {

constexpr int PT = 64;             // rows of the state (components of x) a workgroup owns

typedef float f8 __attribute__((ext_vector_type(8)));

template <typename E> struct Fr;
template <> struct Fr<__bf16> { bf8 v; };
template <> struct Fr<float> { f4 a, b; };

__device__ inline f4 mma(const Fr<__bf16>& x, const Fr<__bf16>& y, f4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.v, y.v, c, 0, 0, 0);
}
__device__ inline f4 mma(const Fr<float>& x, const Fr<float>& y, f4 c) {
#pragma unroll
  for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x.a[j], y.a[j], c, 0, 0, 0);
#pragma unroll
  for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x.b[j], y.b[j], c, 0, 0, 0);
  return c;
}

// The planes of two quads of fp32 values (fp32 products take them as they are).
template <typename E, int PL> struct Planes {
  static constexpr int N = sizeof(E) == 2 ? PL : 1;
  Fr<E> p[N];
};
template <typename E, int PL>
__device__ inline Planes<E, PL> planes(f4 x, f4 y) {
  Planes<E, PL> r;
  if constexpr (sizeof(E) == 2) {
    f8 v = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
    for (int i = 0; i < PL; ++i) {
      r.p[i].v = __builtin_convertvector(v, bf8);
      if (i + 1 < PL) v -= __builtin_convertvector(r.p[i].v, f8);
    }
  } else {
    r.p[0].a = x;
    r.p[0].b = y;
  }
  return r;
}
template <typename E, int PL>
__device__ inline f4 mma(const Planes<E, PL>& x, const Fr<E>& y, f4 c) {
#pragma unroll
  for (int i = Planes<E, PL>::N - 1; i >= 0; --i) c = mma(x.p[i], y, c);
  return c;
}
template <typename E, int PL>
__device__ inline f4 mma(const Fr<E>& x, const Planes<E, PL>& y, f4 c) {
#pragma unroll
  for (int i = Planes<E, PL>::N - 1; i >= 0; --i) c = mma(x, y.p[i], c);
  return c;
}

// Four consecutive values.
template <typename E> struct Q4;
template <> struct Q4<__bf16> { typedef bf4 t; };
template <> struct Q4<float> { typedef f4 t; };
template <typename E>
__device__ inline f4 widen(typename Q4<E>::t q) {
  if constexpr (sizeof(E) == 2) return __builtin_convertvector(q, f4);
  else return q;
}
template <typename E>
__device__ inline typename Q4<E>::t narrow(f4 q) {
  if constexpr (sizeof(E) == 2) return __builtin_convertvector(q, bf4);
  else return q;
}

// LDS row length in elements: 16 bytes of padding spread rows over the banks.
template <typename E> constexpr int lds_ld(int cols) { return cols + 16 / (int)sizeof(E); }

// Operand with i = row0 + l % 16 and k along the row, from k0.
template <typename E>
__device__ inline Fr<E> row_frag(const E* t, int ld, int row0, int k0, int lane) {
  typedef typename Q4<E>::t q4;
  const E* p = t + (row0 + (lane & 15)) * ld + k0 + 4 * (lane >> 4);
  const q4 a = *(const q4*)p, b = *(const q4*)(p + 16);
  Fr<E> r;
  if constexpr (sizeof(E) == 2) {
    r.v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  } else {
    r.a = a;
    r.b = b;
  }
  return r;
}
// Operand with i = column j0 + l % 16 and k down the rows, from row k0: the LDS
// transpose read for bf16 (a group of 16 lanes names the 8-byte pieces of a 4 x
// 16 block, lane L gets its column L).
template <typename E>
__device__ inline Fr<E> col_frag(const E* t, int ld, int k0, int j0, int lane) {
  Fr<E> r;
  if constexpr (sizeof(E) == 2) {
    typedef __attribute__((address_space(3))) bf4* lp;
    const int L = lane & 15;
    const E* p = t + (k0 + 4 * (lane >> 4) + (L >> 2)) * ld + j0 + 4 * (L & 3);
    const bf4 a = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lp)(uintptr_t)(uint32_t)(uintptr_t)p);
    const bf4 b = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lp)(uintptr_t)(uint32_t)(uintptr_t)(p + 16 * ld));
    r.v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  } else {
    const E* p = t + (k0 + 4 * (lane >> 4)) * ld + j0 + (lane & 15);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      r.a[j] = p[j * ld];
      r.b[j] = p[(16 + j) * ld];
    }
  }
  return r;
}
// The two quads of an operand in fp32, and scaled by w (one value per k).
template <typename E>
__device__ inline void quads(const Fr<E>& r, f4& a, f4& b) {
  if constexpr (sizeof(E) == 2) {
    const f8 v = __builtin_convertvector(r.v, f8);
    a = __builtin_shufflevector(v, v, 0, 1, 2, 3);
    b = __builtin_shufflevector(v, v, 4, 5, 6, 7);
  } else {
    a = r.a;
    b = r.b;
  }
}

struct ScanArgs {
  Seqs q;
  int H, G, P, N;                  // heads, groups of B and C, components of x a head, state size
  int softplus;
  long ldx, ldb, ldc;              // elements from one token to the next of x, B and C
  const void *x, *B, *C;
  const float *dt, *A, *D, *bias;  // dt [tokens][H]; A, D, bias [H], D and bias optional
  const float* S0;                 // [N][H][P][N], optional
  void* y;
  float* Sf;
  // backward
  const void* dy;
  const float* dSf;
  void *dx, *dB, *dC;
  float *ddt, *dA, *dD, *dbias, *dS0;
  // Walks over segments: slots of `seg` tokens (a multiple of C).  Entry and
  // total of each, [slot][H][P][N], and the decay of each, [slot][H].
  int seg;
  float *entry[2], *total[2], *decay;
  // backward: state at every chunk's start and state gradient at its end,
  // [chunk slot][H][tile of P] in the walk's register order
  float *states, *grads;
  int splits;                      // workgroups that share a chunk's heads
  float *partB, *partC;            // [split][tokens][G][N] where splits > 1
  float* sums;                     // [chunk slot][H][4]: dA, dD, dbias
  float* gates;                    // [chunk slot][H] Gates
};

__host__ __device__ inline int p_tiles(int P) { return (P + PT - 1) / PT; }

// Work item of a workgroup: XCD x (workgroup number mod 8) takes a contiguous
// eighth of the items, so that neighbouring heads, which read the same B and C,
// meet in one L2.  False past the end.
__device__ inline bool xcd_item(long n, long& item) {
  const long per = (n + 7) / 8;
  const long j = blockIdx.x >> 3;
  item = (blockIdx.x & 7) * per + j;
  return j < per && item < n;
}
inline unsigned xcd_grid(long n) { return (unsigned)((n + 7) / 8 * 8); }

// A tile of 64 rows x COLS staged through registers: loads first, LDS later.
// Rows from `rows` and columns from `cols` on are zeros.
template <typename E, int COLS, int NT>
struct Stage {
  static constexpr int V = 16 / (int)sizeof(E), PIECES = 64 * COLS / V, K = PIECES / NT;
  static_assert(PIECES % NT == 0, "pieces split evenly");
  u32x4 r[K];
  __device__ inline void load(const E* src, long ld, int rows, int cols, bool vec, int t) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int i = k * NT + t, row = i / (COLS / V), c = i % (COLS / V) * V;
      r[k] = u32x4{0, 0, 0, 0};
      if (row >= rows || c >= cols) continue;
      const E* p = src + row * ld + c;
      if (vec) {
        r[k] = *(const u32x4*)p;
      } else {
        E e[V];
#pragma unroll
        for (int j = 0; j < V; ++j) e[j] = c + j < cols ? p[j] : fromf<E>(0.f);
        r[k] = __builtin_bit_cast(u32x4, e);
      }
    }
  }
  __device__ inline void put(E* dst, int ld, int t) const {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int i = k * NT + t, row = i / (COLS / V), c = i % (COLS / V) * V;
      *(u32x4*)(dst + row * ld + c) = r[k];
    }
  }
};

// Whether rows of `cols` values, `ld` apart from p on, are whole aligned 16-byte pieces.
template <typename E>
__device__ inline bool vec_rows(const void* p, long ld, int cols) {
  constexpr int V = 16 / (int)sizeof(E);
  return ((uintptr_t)p & 15) == 0 && ld % V == 0 && cols % V == 0;
}

template <int CTRL, int ROWS, bool BOUND>
__device__ inline double dpp_src64(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, ROWS, 0xF, BOUND);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, ROWS, 0xF, BOUND);
  return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
__device__ inline double wave_incl_scan64(double x) {
  x += dpp_src64<0x111, 0xF, true>(x);
  x += dpp_src64<0x112, 0xF, true>(x);
  x += dpp_src64<0x114, 0xF, true>(x);
  x += dpp_src64<0x118, 0xF, true>(x);
  x += dpp_src64<0x142, 0xA, false>(x);
  x += dpp_src64<0x143, 0xC, false>(x);
  return x;
}

// Time steps and prefix sums b of dt A of a chunk, formed once for all kernels
// of a call ([chunk slot][H] of them).  b is kept as two floats: what counts
// are differences b_r - b_i, and a token that wipes the state (dt A = -10^4)
// would leave a single float's differences after it off by 6e-4.  Tokens past
// the chunk's end have dt = 0, so that b stays where it is.
struct Gates {
  float dt[C], bh[C], bl[C];
};
constexpr int GATES = 3 * C;
__device__ inline float step_size(float z, int softplus) {
  return softplus ? fmaxf(z, 0.f) + log1pf(expf(-fabsf(z))) : z;
}
// exp(b_r - b_i); exp(b_r) with zeros for b_i.
__device__ inline float decay(float hr, float lr, float hi, float li) { return fast_exp((hr - hi) + (lr - li)); }

hipError_t launch_scan_gates(const ScanArgs& a, hipStream_t st);
hipError_t launch_scan_fwd(const ScanArgs& a, int dtype, hipStream_t st);
hipError_t launch_scan_bwd(const ScanArgs& a, int dtype, hipStream_t st);
hipError_t launch_scan_step(const ScanArgs& a, int dtype, hipStream_t st);
// Walks of the states alone, in direction `dirs` (1: states, 2: gradients, 3: both).
hipError_t launch_scan_walks(const ScanArgs& a, int dtype, int dirs, bool chunks, hipStream_t st);
// From the segments' totals and decays to their entries (direction as above), and the ends.
hipError_t launch_scan_compose(const ScanArgs& a, int dirs, hipStream_t st);
// Tokens of a segment for a walk of `dirs` directions; 0: whole sequences.
int scan_segment(const Seqs& q, int H, int P, int dirs);
int scan_splits(const Seqs& q, int H, int G);

}  // namespace qd
