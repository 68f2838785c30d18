// Shared pieces of the operators around the recurrence (convolution, row
// normalisation, state space scan): row vectors, sequence tiles, column sums.
#pragma once

#include <type_traits>

#include "qd_common.h"

namespace qd {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// V consecutive activations of a row, widened to fp32.  V is 16 or 8 bytes'
// worth, or 1 where rows are not whole aligned 16-byte pieces.
template <typename E, int V>
struct Vec {
  static_assert(V == 1 || V * sizeof(E) == 16 || V * sizeof(E) == 8, "pieces of 16 or 8 bytes");
  typedef unsigned int words __attribute__((ext_vector_type(V * sizeof(E) == 16 ? 4 : 2)));
  typedef std::conditional_t<V == 1, E, words> raw_t;    // as it lies in memory
  float v[V];
  __device__ inline void take(const raw_t& raw) {
    const E* e = (const E*)&raw;
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = tof(e[i]);
  }
  __device__ inline void load(const E* p) { take(*(const raw_t*)p); }
  __device__ inline void store(E* p) const {
    raw_t raw;
    E* e = (E*)&raw;
#pragma unroll
    for (int i = 0; i < V; ++i) e[i] = fromf<E>(v[i]);
    *(raw_t*)p = raw;
  }
  __device__ inline void zero() {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = 0.f;
  }
};

// sigmoid and x sigmoid(x) from the hardware's exponential and reciprocal
// (one unit in the last place each): relative error below 2^-20 for |x| < 16,
// and 0 or 1 where the exponential leaves the range of fp32.
__device__ inline float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }
__device__ inline float fast_sigmoid(float x) { return __builtin_amdgcn_rcpf(1.f + fast_exp(-x)); }

// Sequences of a call: dense (cu == nullptr: N sequences of T tokens) or
// packed (T tokens in all, cu[N + 1] on the device).  Tiles of L consecutive
// tokens restart at every sequence; a packed batch has T / L + N tile slots,
// of which sequence n's start at cu[n] / L + n.
struct Seqs {
  int T, N;
  const int* cu;
  __host__ __device__ inline long slots(int L) const {
    return cu ? (N > 0 ? (long)(T / L) + N : 0) : (long)N * ((T + L - 1) / L);
  }
  // First token and length of sequence n; false (and no tokens) where cu is malformed there.
  __device__ inline bool range(int n, long& s, int& len) const {
    if (!cu) {
      s = (long)n * T;
      len = T;
      return true;
    }
    const int a = cu[n], b = cu[n + 1];
    s = a;
    len = b - a;
    if (a >= 0 && a <= b && b <= T) return true;
    s = 0;
    len = 0;
    return false;
  }
  // Tile slot g -> sequence n (its range s, len) and the tile's first position in it; false for a slot without tokens.
  __device__ inline bool locate(long g, int L, int& n, long& s, int& len, int& pos) const {
    if (!cu) {
      const int per = (T + L - 1) / L;
      n = (int)(g / per);
      pos = (int)(g - (long)n * per) * L;
      range(n, s, len);
      return n < N && pos < len;
    }
    int lo = 0, hi = N - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      const int c = cu[mid];
      if ((long)(c >= 0 ? c / L : 0) + mid <= g) lo = mid; else hi = mid - 1;
    }
    n = lo;
    if (!range(n, s, len)) return false;
    const long k = g - (s / L + n);
    pos = (int)k * L;
    return k >= 0 && k * L < len;
  }
};

// out_w[d * J + j] = sum over the n partial rows [J (+ 1)][D] of part, and
// out_b[d] that of row J (out_b may be nullptr; then part has J rows or one
// more that is not read: `rows` of them), in a fixed order.
hipError_t launch_colsum(const float* part, int n, int rows, int J, int D, int dtype, void* out_w, void* out_b,
                         hipStream_t st);

// ------------------------------------------------------------ convolution
struct ConvArgs {
  Seqs q;
  int D, W, silu;
  long ldx;                       // elements from one token's row of x to the next
  const void *x, *w, *b, *s0;
  void *y, *sf;                   // forward
  const void *dy, *dsf;           // backward
  void *dx, *dw, *db, *ds0;
  float* part;
};
long conv_bwd_slots(const Seqs& q);
hipError_t launch_conv_fwd(const ConvArgs& a, int dtype, hipStream_t st);
hipError_t launch_conv_bwd(const ConvArgs& a, int dtype, hipStream_t st);
// One token of N sequences: state s0 -> sf (which may be the same).
hipError_t launch_conv_step(const ConvArgs& a, int dtype, hipStream_t st);

// ------------------------------------------------------------ row normalisation
struct RowNormArgs {
  long rows;
  int D, rms;
  float eps;
  long ldx, ldg;
  const void *x, *w, *b, *g;
  void* y;
  float* stats;                   // [rows][2]: mean, 1 / deviation
  const void* dy;
  void *dx, *dw, *db, *dg;
  float* part;
};
int norm_bwd_blocks(long rows, int D);
hipError_t launch_norm_fwd(const RowNormArgs& a, int dtype, hipStream_t st);
hipError_t launch_norm_bwd(const RowNormArgs& a, int dtype, hipStream_t st);

}  // namespace qd
