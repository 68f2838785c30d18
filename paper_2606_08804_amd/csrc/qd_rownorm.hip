// Row normalisation with weight, bias and a SiLU gate, forward and backward,
// and the sum of partial columns that this file's and the convolution's weight
// gradients end with.
//
//   xh = (x - mean) r,  r = 1 / sqrt(var + eps)      ("rms": mean = 0, var = mean of x^2)
//   y  = (xh w + b) s,  s = g sigmoid(g)             (s = 1 without a gate)
//   backward, d = dy s w:  dx = r (d - mean(d) - xh mean(d xh))  ("rms": without mean(d))
//             dw = sum dy s xh,  db = sum dy s,  dg = dy (xh w + b) sigmoid(g) (1 + g (1 - sigmoid(g)))
//
// Both directions are bound by HBM: a row is read once into registers (LANES
// lanes with K pieces of V elements each) and everything that needs its sums is
// formed from there.  16384 rows of 2048 in bf16: forward 26 us (134 MB, 5.1
// TB/s), backward 44 us (201 MB, 4.5 TB/s); 262144 gated rows of 128: 33 and 60
// us (201 MB, 6.1 TB/s, and 336 MB, 5.6 TB/s, some of it from the last level
// cache).  Gated rows of 1025 to 2048 and of 4097 to 8192 values in bf16 take all
// registers in the backward, one wave a SIMD and no row read ahead: on the same
// tensors again and again, 16384 x 2048 forward 34 us (6.0 TB/s), backward 94 (3.6
// TB/s), 4096 x 8192 33 and 94.
// The backward's row groups walk rows with the weight's
// gradient in registers, sum it over the workgroup in LDS and write one partial
// row per workgroup; no atomics, so results do not change from run to run.
#include "qd_mixer.h"

namespace qd {

namespace {

// Sum over the LANES lanes of a row, the same value in each of them.
template <int LANES>
__device__ inline float row_sum(float x, float* red) {
  if constexpr (LANES == 8) {
#pragma unroll
    for (int off = 1; off < 8; off *= 2) x += __shfl_xor(x, off, 64);
  } else {
    x = sum16(x);
  }
  if constexpr (LANES >= 32) x += __shfl_xor(x, 16, 64);
  if constexpr (LANES >= 64) x += __shfl_xor(x, 32, 64);
  if constexpr (LANES == 256) {
    const int w = threadIdx.x >> 6;
    __syncthreads();                       // the last sum has been read
    if ((threadIdx.x & 63) == 0) red[w] = x;
    __syncthreads();
    x = (red[0] + red[1]) + (red[2] + red[3]);
  }
  return x;
}

template <typename E, int V, bool WHOLE, int LANES, int K>
__global__ __launch_bounds__(NTHREADS) void k_norm_fwd(RowNormArgs a) {
  __shared__ float red[4];
  constexpr int RPB = NTHREADS / LANES;
  const long row = ((long)blockIdx.y * gridDim.x + blockIdx.x) * RPB + threadIdx.x / LANES;
  const int lane = threadIdx.x % LANES;
  if (row >= a.rows) return;               // whole lane groups leave together, a workgroup that is one as a whole
  const E* x = (const E*)a.x + row * a.ldx;
  Vec<E, V, WHOLE> v[K];
  float s = 0.f;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int c = (k * LANES + lane) * V;
    if (c < a.D) v[k].load(x + c, a.D - c); else v[k].zero();
#pragma unroll
    for (int i = 0; i < V; ++i) s += v[k].v[i];
  }
  const float inv = 1.f / (float)a.D;
  const float mean = a.rms ? 0.f : row_sum<LANES>(s, red) * inv;
  float ss = 0.f;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int c = (k * LANES + lane) * V;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      v[k].v[i] -= mean;
      ss += c + (WHOLE ? 0 : i) < a.D ? v[k].v[i] * v[k].v[i] : 0.f;
    }
  }
  const float r = 1.f / sqrtf(row_sum<LANES>(ss, red) * inv + a.eps);
  E* y = (E*)a.y + row * a.D;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int c = (k * LANES + lane) * V;
    if (c >= a.D) break;
    Vec<E, V, WHOLE> w, b, g;
    if (a.w) w.load((const E*)a.w + c, a.D - c);
    if (a.b) b.load((const E*)a.b + c, a.D - c);
    if (a.g) g.load((const E*)a.g + row * a.ldg + c, a.D - c);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float o = v[k].v[i] * r;
      if (a.w) o *= w.v[i];
      if (a.b) o += b.v[i];
      if (a.g) o *= g.v[i] * sigmoid<E>(g.v[i]);
      v[k].v[i] = o;
    }
    v[k].store(y + c, a.D - c);
  }
  if (a.stats && lane == 0) {
    a.stats[2 * row] = mean;
    a.stats[2 * row + 1] = r;
  }
}

template <typename E, int V, bool WHOLE, int LANES, int K, bool GATE>
__global__ __launch_bounds__(NTHREADS) void k_norm_bwd(RowNormArgs a) {
  __shared__ float red[4];
  extern __shared__ float cols[];          // [2][LANES * K * V] where the workgroup has more than one row
  constexpr int RPB = NTHREADS / LANES;
  const int lane = threadIdx.x % LANES;
  const float inv = 1.f / (float)a.D;
  float dw[K * V] = {}, db[K * V] = {};
  // The pieces of a row, and where registers allow it those of the next one read
  // while this one is worked on (16384 x 2048 in bf16: 49 -> 44 us).
  constexpr bool AHEAD = K * V <= (GATE ? 16 : 32) && K <= 4;
  typedef Vec<E, V, WHOLE> Piece;
  typedef typename Piece::raw_t raw_t;
  raw_t xn[K], dn[K], gn[GATE ? K : 1];
  float mean_n = 0.f, r_n = 0.f;
  auto fetch = [&](long row) {
    mean_n = a.stats[2 * row];
    r_n = a.stats[2 * row + 1];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * LANES + lane) * V;
      xn[k] = dn[k] = raw_t{};
      if constexpr (GATE) gn[k] = raw_t{};
      if (c < a.D) {
        xn[k] = Piece::fetch((const E*)a.x + row * a.ldx + c, a.D - c);
        dn[k] = Piece::fetch((const E*)a.dy + row * a.D + c, a.D - c);
        if constexpr (GATE) gn[k] = Piece::fetch((const E*)a.g + row * a.ldg + c, a.D - c);
      }
    }
  };
  const long row0 = (long)blockIdx.x * RPB + threadIdx.x / LANES;
  if (AHEAD && row0 < a.rows) fetch(row0);
  // LANES == 256: row is uniform over the workgroup, so its barriers are met by all
  for (long row = row0; row < a.rows; row += (long)gridDim.x * RPB) {
    Vec<E, V, WHOLE> xh[K], d[K], g[GATE ? K : 1];
    if constexpr (!AHEAD) fetch(row);
    const float mean = mean_n, r = r_n;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      xh[k].take(xn[k]);
      d[k].take(dn[k]);
      if constexpr (GATE) g[k].take(gn[k]);
    }
    if constexpr (AHEAD) {
      fetch(min(row + (long)gridDim.x * RPB, a.rows - 1));
      __builtin_amdgcn_sched_barrier(0);
    }
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * LANES + lane) * V;
      const bool in = c < a.D;
      Vec<E, V, WHOLE> w, b, o;
      if (in && a.w) w.load((const E*)a.w + c, a.D - c);
      if (GATE && in && a.b) b.load((const E*)a.b + c, a.D - c);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float h = (xh[k].v[i] - mean) * r;
        float e = d[k].v[i];
        if constexpr (GATE) {
          const float gv = g[k].v[i], sg = sigmoid<E>(gv);
          float lin = h;
          if (a.w) lin *= w.v[i];
          if (a.b) lin += b.v[i];
          o.v[i] = e * lin * (sg * (1.f + gv * (1.f - sg)));
          e *= gv * sg;
        }
        if (in) {
          dw[k * V + i] += e * h;
          db[k * V + i] += e;
        }
        if (a.w) e *= w.v[i];
        xh[k].v[i] = h;
        d[k].v[i] = e;
        if (in) {
          s1 += e;
          s2 += e * h;
        }
      }
      if constexpr (GATE)
        if (in) o.store((E*)a.dg + row * a.D + c, a.D - c);
    }
    s1 = a.rms ? 0.f : row_sum<LANES>(s1, red) * inv;
    s2 = row_sum<LANES>(s2, red) * inv;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * LANES + lane) * V;
      if (c >= a.D) break;
#pragma unroll
      for (int i = 0; i < V; ++i) d[k].v[i] = r * (d[k].v[i] - s1 - xh[k].v[i] * s2);
      d[k].store((E*)a.dx + row * a.D + c, a.D - c);
    }
  }
  if (!a.part) return;
  // one partial row [2][D] per workgroup: over the rows of a wave by lane moves, over the waves in order
#pragma unroll
  for (int off = LANES; off < 64; off *= 2)
#pragma unroll
    for (int i = 0; i < K * V; ++i) {
      dw[i] += __shfl_xor(dw[i], off, 64);
      db[i] += __shfl_xor(db[i], off, 64);
    }
  float* out = a.part + (long)blockIdx.x * 2 * a.D;
  if constexpr (LANES < 256) {
    constexpr int N = LANES * K * V;
    const int w = threadIdx.x >> 6;
    for (int turn = 0; turn < 4; ++turn) {
      if (w == turn && (threadIdx.x & 63) < LANES) {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const int c = (k * LANES + lane) * V + i;
            cols[c] = (turn ? cols[c] : 0.f) + dw[k * V + i];
            cols[N + c] = (turn ? cols[N + c] : 0.f) + db[k * V + i];
          }
      }
      __syncthreads();
    }
    for (int c = threadIdx.x; c < a.D; c += NTHREADS) {
      out[c] = cols[c];
      out[a.D + c] = cols[N + c];
    }
  } else {
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int c = (k * LANES + lane) * V + i;
        if (c < a.D) {
          out[c] = dw[k * V + i];
          out[a.D + c] = db[k * V + i];
        }
      }
  }
}

// 64 columns by 16 row groups a workgroup.
constexpr int CS_COLS = 64, CS_ROWS = 16;
template <typename E>
__global__ __launch_bounds__(CS_COLS* CS_ROWS) void k_colsum(const float* __restrict__ part, int n, int rows, int J,
                                                             int D, E* __restrict__ w, E* __restrict__ b) {
  __shared__ float red[CS_ROWS][CS_COLS];
  const int c = threadIdx.x % CS_COLS, g = threadIdx.x / CS_COLS;
  const long col = (long)blockIdx.x * CS_COLS + c;      // j * D + d
  const long cols = (long)rows * D;
  const int j = (int)(col / D);
  const bool want = col < cols && (j < J ? w != nullptr : b != nullptr);
  float s = 0.f;
  if (want)
#pragma unroll 8
    for (int i = g; i < n; i += CS_ROWS) s += part[(long)i * cols + col];
  red[g][c] = s;
  __syncthreads();
  if (g || !want) return;
  for (int i = 1; i < CS_ROWS; ++i) s += red[i][c];
  const int d = (int)(col - (long)j * D);
  if (j < J) w[(long)d * J + j] = fromf<E>(s);
  else b[d] = fromf<E>(s);
}

template <typename E, int V, bool WHOLE, int LANES, int K>
hipError_t fwd(const RowNormArgs& a, hipStream_t st) {
  constexpr int RPB = NTHREADS / LANES;
  const long blocks = (a.rows + RPB - 1) / RPB, wide = 1L << 23;     // a launch's dimension has less than 2^32 threads
  const dim3 grid((unsigned)(blocks < wide ? blocks : wide), (unsigned)((blocks + wide - 1) / wide));
  hipLaunchKernelGGL((k_norm_fwd<E, V, WHOLE, LANES, K>), grid, dim3(NTHREADS), 0, st, a);
  return hipGetLastError();
}

template <typename E, int V, bool WHOLE, int LANES, int K>
hipError_t bwd(const RowNormArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)norm_bwd_blocks(a.rows, a.D));
  const size_t lds = LANES < 256 ? 2 * sizeof(float) * LANES * K * V : 0;
  if (a.g) hipLaunchKernelGGL((k_norm_bwd<E, V, WHOLE, LANES, K, true>), grid, dim3(NTHREADS), lds, st, a);
  else hipLaunchKernelGGL((k_norm_bwd<E, V, WHOLE, LANES, K, false>), grid, dim3(NTHREADS), lds, st, a);
  return hipGetLastError();
}

// Lanes a row by its pieces: the fewest of 8 to 64 that hold one each, a wave
// with two or four, else the workgroup (rows of 256 pieces by the workgroup, one
// each: backward 56 us instead of 49, its sums meet barriers).  A variant twice as
// wide as the row runs half of its lanes or registers for nothing (forward and
// backward in bf16, next wider and its own: 524288 gated rows of 64 152 and 104
// us, 131072 of 200 150 and 92, 16384 rows of 1024 59 and 49, of 4096 227 and 196).
#define QD_ROWNORM(FN)                                             \
  const int nv = (a.D + V - 1) / V;                                \
  if (nv <= 8) return FN<E, V, WHOLE, 8, 1>(a, st);                \
  if (nv <= 16) return FN<E, V, WHOLE, 16, 1>(a, st);              \
  if (nv <= 32) return FN<E, V, WHOLE, 32, 1>(a, st);              \
  if (nv <= 64) return FN<E, V, WHOLE, 64, 1>(a, st);              \
  if (nv <= 128) return FN<E, V, WHOLE, 64, 2>(a, st);             \
  if (nv <= 256) return FN<E, V, WHOLE, 64, 4>(a, st);             \
  if (nv <= 512) return FN<E, V, WHOLE, 256, 2>(a, st);            \
  if (nv <= 1024) return FN<E, V, WHOLE, 256, 4>(a, st);           \
  if constexpr (V == 4)                                            \
    if (nv <= 2048) return FN<E, V, WHOLE, 256, 8>(a, st);         \
  return hipErrorInvalidValue

template <typename E, int V, bool WHOLE>
hipError_t by_size_fwd(const RowNormArgs& a, hipStream_t st) { QD_ROWNORM(fwd); }
template <typename E, int V, bool WHOLE>
hipError_t by_size_bwd(const RowNormArgs& a, hipStream_t st) { QD_ROWNORM(bwd); }
#undef QD_ROWNORM

// Whether every row of every tensor of the call is whole aligned 16-byte pieces.
bool whole(const RowNormArgs& a, int esz) {
  const int v = 16 / esz;
  uintptr_t p = 0;
  for (const void* q : {a.x, a.w, a.b, a.g, (const void*)a.y, a.dy, (const void*)a.dx, (const void*)a.dg})
    p |= (uintptr_t)q;
  return a.D % v == 0 && a.ldx % v == 0 && (!a.g || a.ldg % v == 0) && (p & 15) == 0;
}

}  // namespace

// Workgroups of the backward: enough to fill the chip, few enough that the partial
// rows (2 D floats each) of large calls stay small beside their tensors (forward
// and backward repeated on the same tensors with 256, 512 and 1024: 16384 x 2048 in
// bf16 78, 71, 82 us; 262144 gated rows of 128 with 512, 1024 and 2048: 106, 95, 99).
// Counted by rows, not by the rows a workgroup takes: calls of fewer rows than these
// workgroups take have some without any, which write zeros (777 x 1003 in fp32: 582 of
// 777; backward and column sum 15 us of a call's 30).
int norm_bwd_blocks(long rows, int D) {
  long n = (1L << 20) / D;
  n = n < 256 ? 256 : n > 1024 ? 1024 : n;
  return (int)(rows < n ? (rows < 1 ? 1 : rows) : n);
}

hipError_t launch_norm_fwd(const RowNormArgs& a, int dtype, hipStream_t st) {
  if (dtype == 1) return whole(a, 2) ? by_size_fwd<__bf16, 8, true>(a, st) : by_size_fwd<__bf16, 8, false>(a, st);
  return whole(a, 4) ? by_size_fwd<float, 4, true>(a, st) : by_size_fwd<float, 4, false>(a, st);
}

hipError_t launch_norm_bwd(const RowNormArgs& a, int dtype, hipStream_t st) {
  hipError_t e;
  if (dtype == 1) e = whole(a, 2) ? by_size_bwd<__bf16, 8, true>(a, st) : by_size_bwd<__bf16, 8, false>(a, st);
  else e = whole(a, 4) ? by_size_bwd<float, 4, true>(a, st) : by_size_bwd<float, 4, false>(a, st);
  if (e != hipSuccess || !a.part) return e;
  return launch_colsum(a.part, norm_bwd_blocks(a.rows, a.D), 2, 1, a.D, dtype, a.dw, a.db, st);
}

hipError_t launch_colsum(const float* part, int n, int rows, int J, int D, int dtype, void* w, void* b,
                         hipStream_t st) {
  const dim3 grid((unsigned)(((long)rows * D + CS_COLS - 1) / CS_COLS)), thr(CS_COLS * CS_ROWS);
  if (dtype == 1)
    hipLaunchKernelGGL((k_colsum<__bf16>), grid, thr, 0, st, part, n, rows, J, D, (__bf16*)w, (__bf16*)b);
  else
    hipLaunchKernelGGL((k_colsum<float>), grid, thr, 0, st, part, n, rows, J, D, (float*)w, (float*)b);
  return hipGetLastError();
}

}  // namespace qd
