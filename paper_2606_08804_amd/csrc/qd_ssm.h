// Shared pieces of the selective state space scan's kernels.
//
// MFMA operands here are "quads": a step covers 32 values of k as two blocks
// of 16, and lane l holds k = 4 (l / 16) .. + 3 of either block.  That is the
// order in which a 16 x 16 accumulator holds its rows, so an accumulator pair
// is an operand as it stands (its rows become k), without a trip through LDS.
// bf16 takes one 16x16x32 instruction a step, fp32 eight 16x16x4 ones.
//
// A fp32 value enters a bf16 product as a sum of three bf16 values ("planes"),
// x = hi + mid + lo, which is exact.  Two of them are off by up to 2^-16: results
// that are rounded to bf16 afterwards then differ from those of fp32 products in
// one of 500 (dB, dC) to 1500 values (y), and cost a tenth less (4 x 4096 tokens, 64
// heads, training 1012 us instead of 1098; a prompt of 65536, 16 heads, 594 and 664).
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
// Two fp32 values as bf16 in one register (one instruction: without the line
// that hides where the register comes from, taking the values apart again makes
// the compiler convert each by itself and join them).
__device__ inline uint32_t pack2(float x, float y) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  uint32_t r = __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{x, y}, b2));
  asm("" : "+v"(r));
  return r;
}
// A quad as bf16; plane4 also leaves in v what that rounds off.
__device__ inline uint2 pack4(const f4& v) { return make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3])); }
__device__ inline uint2 plane4(f4& v) {
  const uint2 r = pack4(v);
  v[0] -= __builtin_bit_cast(float, r.x << 16);
  v[1] -= __builtin_bit_cast(float, r.x & 0xffff0000u);
  v[2] -= __builtin_bit_cast(float, r.y << 16);
  v[3] -= __builtin_bit_cast(float, r.y & 0xffff0000u);
  return r;
}
template <typename E, int PL>
__device__ inline Planes<E, PL> planes(f4 x, f4 y) {
  Planes<E, PL> r;
  if constexpr (sizeof(E) == 2) {
#pragma unroll
    for (int i = 0; i < PL; ++i) {
      const uint2 p = i + 1 < PL ? plane4(x) : pack4(x), q = i + 1 < PL ? plane4(y) : pack4(y);
      r.p[i].v = __builtin_bit_cast(bf8, u32x4{p.x, p.y, q.x, q.y});
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

// A quad's planes one after the other to p, p + step (fp32: the quad itself).
template <typename E, int PL>
__device__ inline void put_planes(E* p, int step, f4 x) {
#pragma unroll
  for (int i = 0; i < PL; ++i) {
    if constexpr (sizeof(E) == 2) {
      *(uint2*)(p + i * step) = i + 1 < PL ? plane4(x) : pack4(x);
    } else {
      *(f4*)p = x;
    }
  }
}

// LDS tiles are row-major, rows `lds_ld` elements apart.  In bf16 tiles the two
// 16-byte halves of every 16 columns change places in rows 8 to 15 of 16
// (`flip`): rows then lie 8 banks apart, and the three ways they are accessed
// (16-byte pieces of a row, quads of 16 rows at one column, transpose reads of
// four rows by 16 columns) each meet every bank once.
template <typename E> constexpr int lds_ld(int cols) { return cols + (sizeof(E) == 2 ? 16 : 4); }
template <typename E> __device__ inline int flip(int row, int c) { return sizeof(E) == 2 ? c ^ (row & 8) : c; }

// Tiles that are read along rows alone ("steps") hold a row's columns in groups
// of 32 in the order in which a step takes them, the quad 16 blk + 4 g of a group
// at 8 g + 4 blk: a lane's two quads are then one 16-byte read.  (Transpose reads
// of this order would meet half of the banks twice.)
template <typename E> constexpr int steps_ld(int cols) { return cols + 16 / (int)sizeof(E); }
template <typename E> __device__ constexpr int step_at(int c) {
  return sizeof(E) == 2 ? (c & ~31) + ((c >> 2) & 3) * 8 + ((c >> 4) & 1) * 4 : c;
}
template <typename E>
__device__ inline Fr<E> step_frag(const E* t, int ld, int row0, int k0, int lane) {
  Fr<E> f;
  if constexpr (sizeof(E) == 2) {
    f.v = *(const bf8*)(t + (row0 + (lane & 15)) * ld + k0 + 8 * (lane >> 4));
  } else {
    const E* p = t + (row0 + (lane & 15)) * ld + k0 + 4 * (lane >> 4);
    f.a = *(const f4*)p;
    f.b = *(const f4*)(p + 16);
  }
  return f;
}

// Operand with i = row0 + l % 16 and k along the row, from k0.  The two reads
// are kept from being joined into one instruction, which takes 16 lanes at a
// time and so meets half of the banks twice (three times the conflicts of the
// backward's tiles).
template <typename E>
__device__ inline Fr<E> row_frag(const E* t, int ld, int row0, int k0, int lane) {
  typedef typename Q4<E>::t q4;
  const int r = lane & 15;
  const E* p = t + (row0 + r) * ld + k0 + flip<E>(r, 4 * (lane >> 4));
  const q4 a = *(const q4*)p;
  __builtin_amdgcn_sched_barrier(0);
  const q4 b = *(const q4*)(p + 16);
  __builtin_amdgcn_sched_barrier(0);
  Fr<E> f;
  if constexpr (sizeof(E) == 2) {
    f.v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  } else {
    f.a = a;
    f.b = b;
  }
  return f;
}
// Operand with i = column j0 + l % 16 and k down the rows, from row k0: the LDS
// transpose read for bf16 (a group of 16 lanes names the 8-byte pieces of a 4 x
// 16 block, lane L gets its column L).
template <typename E>
__device__ inline Fr<E> col_frag(const E* t, int ld, int k0, int j0, int lane) {
  Fr<E> r;
  if constexpr (sizeof(E) == 2) {
    typedef __attribute__((address_space(3))) bf4* lp;
    const int L = lane & 15, row = 4 * (lane >> 4) + (L >> 2);
    const E* p = t + (k0 + row) * ld + j0 + flip<E>(row, 4 * (L & 3));
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
  double* sums;                    // [chunk slot][H][4]: dA, dD, dbias
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

// Two waves a SIMD are what these kernels' LDS allows: their registers are theirs to use.
#define QD_TWO_WAVES __attribute__((amdgpu_waves_per_eu(2, 2)))
// A line that the scheduler moves nothing across.  Operands are read in batches
// before it and multiplied after it: left alone, the compiler reads each right
// before its product, which then waits out the LDS's latency.
__device__ inline void phase() { __builtin_amdgcn_sched_barrier(0); }

// The lane number as a value the compiler cannot trace: what is formed from it
// (LDS addresses, masks of the triangles) is formed again every turn of a loop
// instead of being kept in registers, which are all taken (hoisted, 130 such
// values went to scratch memory and back).  Counted from the hardware's lane
// mask, it takes no register between turns either.
__device__ inline int fresh_lane() {
  uint32_t zero = 0;
  asm volatile("" : "+s"(zero));
  return (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, zero));
}

// A tile of 64 rows x COLS staged through registers: loads first, LDS later.
// Rows from `rows` and columns from `cols` on are zeros: a row past the last
// lies past the end of the buffer that the load names, which reads as zero, and
// so do the lanes of columns past the last.  A load then is one instruction, with
// a lane offset formed once (as masked 64-bit addresses the ten loads of a
// chunk took their wave 2500 cycles).
__device__ inline __amdgpu_buffer_rsrc_t buffer(const void* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00020000);
}
// Four consecutive values per lane to a tile of rows: lanes whose offset lies
// past the buffer's end (rows past the last, by the buffer's size; columns past
// the last, by an offset of 2^31) write nothing.
template <typename E>
__device__ inline void store_quad(__amdgpu_buffer_rsrc_t b, uint32_t off, f4 v) {
  if constexpr (sizeof(E) == 2) {
    typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
    __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, narrow<E>(v)), b, off, 0, 0);
  } else {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), b, off, 0, 0);
  }
}
template <typename E, int COLS, int NT>
struct Stage {
  static constexpr int V = 16 / (int)sizeof(E), PIECES = 64 * COLS / V, K = PIECES / NT, STEP = NT / (COLS / V);
  static_assert(PIECES % NT == 0 && NT % (COLS / V) == 0, "pieces split evenly, by whole rows");
  u32x4 r[K];
  // Byte offset of a thread's first piece, and from one of its pieces to the next.
  static __device__ inline uint32_t offset(long ld, int cols, int t) {
    const int c = t % (COLS / V) * V;
    return c < cols ? (uint32_t)((t / (COLS / V)) * ld + c) * (uint32_t)sizeof(E) : 0x80000000u;
  }
  // Nothing is loaded where rows are not whole pieces: `put` then reads them, a
  // piece from any element on (4 x 1024 tokens, 32 heads, state 64 x 100, training
  // in bf16: 275 us, whole pieces of 64 x 128 196; value by value it took 533 where
  // these were 279 and 214).
  __device__ inline void load(const E* src, long ld, int rows, bool vec, uint32_t off) {
    const __amdgpu_buffer_rsrc_t b = buffer(uniform_ptr(src), vec ? (uint32_t)(rows * ld) * (uint32_t)sizeof(E) : 0u);
#pragma unroll
    for (int k = 0; k < K; ++k)
      r[k] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(b, off + (uint32_t)(k * STEP * ld) * (uint32_t)sizeof(E), 0, 0));
  }
  template <bool STEPS>
  static __device__ inline void place(E* dst, int ldd, int t, int k, u32x4 v) {
    const int row = t / (COLS / V) + k * STEP, c = t % (COLS / V) * V;
    if constexpr (STEPS && sizeof(E) == 2) {   // two quads of one block
      typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
      E* d = dst + row * ldd + step_at<E>(c);
      *(u32x2*)d = u32x2{v[0], v[1]};
      *(u32x2*)(d + 8) = u32x2{v[2], v[3]};
    } else {
      *(u32x4*)(dst + row * ldd + flip<E>(row, c)) = v;
    }
  }
  // src, ld, rows and cols as of the load.
  template <bool STEPS = false>
  __device__ inline void put(E* dst, int ldd, const E* src, long ld, int rows, int cols, bool vec, int t) const {
    if (vec) {
#pragma unroll
      for (int k = 0; k < K; ++k) place<STEPS>(dst, ldd, t, k, r[k]);
    } else {
      typedef typename Vec<E, V, false>::any_t any_t;
#pragma unroll 1
      for (int k = 0; k < K; ++k) {
        const int row = t / (COLS / V) + k * STEP, c = t % (COLS / V) * V, last = row < rows ? cols : 0;
        u32x4 v = {};
        if (c + V <= last) v = *(const any_t*)(src + row * ld + c);
        place<STEPS>(dst, ldd, t, k, v);
        if (c + V > last)
#pragma unroll 1
          for (int i = c; i < last; ++i) dst[row * ldd + (STEPS ? step_at<E>(i & ~3) + (i & 3) : flip<E>(row, i))] = src[row * ld + i];
      }
    }
  }
};

// Whether quads of rows of `cols` values, `ld` apart, are whole and aligned
// (and 64 rows lie within a store's offsets).
template <typename E>
__device__ inline bool quad_rows(const void* p, long ld, int cols) {
  return ((uintptr_t)p & (4 * sizeof(E) - 1)) == 0 && ld % 4 == 0 && cols % 4 == 0 && ld < (1L << 24) / (int)sizeof(E);
}
// Whether rows of `cols` values, `ld` apart from p on, are whole aligned
// 16-byte pieces (and 64 of them lie within a load's offsets).
template <typename E>
__device__ inline bool vec_rows(const void* p, long ld, int cols) {
  constexpr int V = 16 / (int)sizeof(E);
  return ((uintptr_t)p & 15) == 0 && ld % V == 0 && cols % V == 0 && ld < (1L << 24) / (int)sizeof(E);
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
  float dt[C], bh[C], bl[C];         // dt, b
  float head[C], tail[C];            // e^{b_r}, e^{b_C - b_i}
  float head16[C], tail16[C];        // the same from the end of the 16 tokens before and to the end of its own 16
};
constexpr int GATES = 7 * C;
// One of the values of a chunk's gates (threads past them get zero).
__device__ inline float load_gate(const float* gates, int t) {
  return __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(
      __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(uniform_ptr(gates)), 0, GATES * 4, 0x00020000), 4 * t, 0, 0));
}
__device__ inline float step_size(float z, int softplus) {
  return softplus ? fmaxf(z, 0.f) + log1pf(expf(-fabsf(z))) : z;
}
// exp(b_r - b_i).
template <typename E> __device__ inline float decay(float hr, float lr, float hi, float li) { return exp_of<E>((hr - hi) + (lr - li)); }

// exp of b's step from the end of block i to the end of the block before r's
// (i < r, blocks of 16): what head16 and tail16 leave out of exp(b_r - b_i).
template <typename E> __device__ inline float between(const Gates& g, int r, int i) {
  const int e = 16 * r - 1, f = 16 * i + 15;
  return decay<E>(g.bh[e], g.bl[e], g.bh[f], g.bl[f]);
}

hipError_t launch_scan_gates(const ScanArgs& a, hipStream_t st);
hipError_t launch_scan_fwd(const ScanArgs& a, int dtype, hipStream_t st);
hipError_t launch_scan_bwd(const ScanArgs& a, int dtype, hipStream_t st);
hipError_t launch_scan_step(const ScanArgs& a, int dtype, hipStream_t st);
// Walks of the states alone, in direction `dirs` (1: states, 2: gradients, 3: both).
hipError_t launch_scan_walks(const ScanArgs& a, int dtype, int dirs, bool chunks, hipStream_t st);
// From the segments' totals and decays to their entries (direction as above), and the ends.
hipError_t launch_scan_compose(const ScanArgs& a, int dirs, hipStream_t st);
// Tokens of a segment for a walk of `dirs` directions; 0: whole sequences.
int scan_segment(const Seqs& q, int H, int P, int dirs, bool f32);
int scan_splits(const Seqs& q, int H, int G);

}  // namespace qd
