// Shared pieces of the operators around the recurrence (convolution, row
// normalisation, state space scan): row vectors, sequence tiles, column sums.
#pragma once

#include "qd_common.h"

namespace qd {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// V consecutive activations of a row, widened to fp32.  V is 16 or 8 bytes'
// worth.  Where rows are not WHOLE aligned 16-byte pieces, the last piece of a
// row has n < V values, the others being zero, and a piece starts at any element:
// the hardware takes such loads and stores as they are (single values in
// their place: norm of 16384 x 2049 in bf16, forward and backward, 486 us instead
// of 131, convolution of 4 x 4096 tokens, 6145 channels, 373 instead of 348).
template <typename E, int V, bool WHOLE>
struct Vec {
  static_assert(V * sizeof(E) == 16 || V * sizeof(E) == 8, "pieces of 16 or 8 bytes");
  typedef unsigned int raw_t __attribute__((ext_vector_type(V * sizeof(E) == 16 ? 4 : 2)));   // as it lies in memory
  typedef raw_t any_t __attribute__((aligned(sizeof(E))));
  float v[V];
  // n: values from p to the row's end.
  static __device__ inline raw_t fetch(const E* p, int n) {
    if constexpr (WHOLE) return *(const raw_t*)p;
    if (n >= V) return *(const any_t*)p;
    raw_t raw = {};
    E* e = (E*)&raw;
#pragma unroll
    for (int i = 0; i < V - 1; ++i)
      if (i < n) e[i] = p[i];
    return raw;
  }
  __device__ inline void take(const raw_t& raw) {
    const E* e = (const E*)&raw;
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = tof(e[i]);
  }
  __device__ inline void load(const E* p, int n) { take(fetch(p, n)); }
  __device__ inline void store(E* p, int n) const {
    raw_t raw;
    E* e = (E*)&raw;
#pragma unroll
    for (int i = 0; i < V; ++i) e[i] = fromf<E>(v[i]);
    if constexpr (WHOLE) {
      *(raw_t*)p = raw;
    } else if (n >= V) {
      *(any_t*)p = raw;
    } else {
#pragma unroll
      for (int i = 0; i < V - 1; ++i)
        if (i < n) p[i] = e[i];
    }
  }
  __device__ inline void zero() {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = 0.f;
  }
};

// exp, and the sigmoid from it and the hardware's reciprocal (one unit in the last
// place; 0 or 1 where the exponential leaves the range of fp32).  With bf16
// activations exp is the hardware's 2^t of the rounded t = x log2(e), off by
// |x| 2^-23 relative: below 2^-18 for every decay or sigmoid above e^-32, in sums
// whose bf16 operands are themselves rounded by 2^-8.  With fp32 activations, and for
// decays of the fp32 state in either type, it is the library's, good to the last
// place at every x (65536 gated rows of 1024 in fp32, forward: 141.3 -> 142.5 us;
// the scan of 4 x 4096 tokens, 16 heads, 64 x 64 in fp32: 143 -> 150).
__device__ inline float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }
template <typename E> __device__ inline float exp_of(float x) {
  if constexpr (sizeof(E) == 2) return fast_exp(x);
  else return expf(x);
}
// exp(hi + lo) for lo within hi's last place: exp(hi) alone is off by the lo that
// its argument has lost, |hi| 2^-24.  (An infinite hi or e leaves no such product.)
__device__ inline float exp_sum(float hi, float lo) {
  const float e = expf(hi), f = fmaf(e, lo, e);
  return f == f ? f : e;
}
__device__ inline float exp_of64(double x) { return exp_sum((float)x, (float)(x - (double)(float)x)); }
template <typename E> __device__ inline float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.f + exp_of<E>(-x)); }

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
// Backward: tiles of `tile` tokens a wave, `turns` of them one after the other,
// and the workgroups (four waves) that gives for a group of channels: the
// partial rows of the weight's gradient.
struct ConvBwdPlan {
  int tile, turns;
  long groups;
};
ConvBwdPlan conv_bwd_plan(const Seqs& q, int D);
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
