// Short causal depthwise convolution along the tokens of each sequence, with
// bias and SiLU: prompts (dense or packed), their backward, and single tokens.
//
//   u_t = b + sum_j w[:, j] x_{t - W + 1 + j},   y = u  or  u sigmoid(u)
//   backward, du = dy (SiLU'(u)):  dx_t = sum_j w[:, j] du_{t + W - 1 - j},
//             dw[:, j] = sum_t du_t x_{t - W + 1 + j},  db = sum_t du_t
//
// x before a sequence's first token are the rows of its state [W - 1][D], the
// oldest first, or zero.  A thread owns V channels and walks a tile of tokens
// with the last W - 1 rows in registers, so a row is read once and the W - 1
// rows before a tile (after it, in the backward, which forms u again) twice.
// The weight's gradient is summed in registers over a wave's tile, over the
// workgroup's four tiles in LDS and over the workgroups by a second launch,
// each in a fixed order.
//
// HBM bounds the forward: 4 x 4096 tokens of 6144 channels in bf16, W = 4, take
// 84 us (403 MB, 4.8 TB/s; pieces of 8 bytes instead of 16: 97 us).  The
// backward moves 604 MB in 136 us (4.4 TB/s) and runs its vector instructions
// for 83 us of them; what it needs is loads in flight.  Pieces of 8 bytes keep
// four of its waves on a SIMD in place of two (190 -> 158 us), and the rows of
// the next turn are read while this one's are used (158 -> 136 us).
#include "qd_mixer.h"

namespace qd {

namespace {

// Row `pos` of a sequence (negative: the state's, or zero without one).
template <typename E, int V, bool WHOLE, int W>
__device__ inline void load_row(Vec<E, V, WHOLE>& r, const ConvArgs& a, int n, long s, int pos, int c) {
  if (pos >= 0) r.load((const E*)a.x + (s + pos) * a.ldx + c, a.D - c);
  else if (a.s0) r.load((const E*)a.s0 + ((long)n * (W - 1) + W - 1 + pos) * a.D + c, a.D - c);
  else r.zero();
}

template <typename E, int V, bool WHOLE, int W>
__device__ inline void load_weights(float (&w)[W][V], float (&b)[V], const ConvArgs& a, int c) {
  const E* p = (const E*)a.w + (long)c * W;
#pragma unroll
  for (int k = 0; k < W; ++k) {    // the V channels' taps are W pieces
    Vec<E, V, WHOLE> t;
    if (WHOLE || (a.D - c) * W > k * V) t.load(p + k * V, (a.D - c) * W - k * V);
    else t.zero();
#pragma unroll
    for (int i = 0; i < V; ++i) w[(k * V + i) % W][(k * V + i) / W] = t.v[i];
  }
  Vec<E, V, WHOLE> t;
  if (a.b) t.load((const E*)a.b + c, a.D - c);
  else t.zero();
#pragma unroll
  for (int i = 0; i < V; ++i) b[i] = t.v[i];
}

// Tiles of L tokens by flat thread index, then the final states by further threads.
template <typename E, int V, bool WHOLE, int W>
__global__ __launch_bounds__(NTHREADS) void k_conv_fwd(ConvArgs a, int L, long tile_threads) {
  constexpr int U = 8;             // tokens whose loads are in flight together
  const int nv = (a.D + V - 1) / V;
  long i = (long)blockIdx.x * NTHREADS + threadIdx.x;
  int n, len, pos;
  long s;
  if (i >= tile_threads) {         // one piece of a final state row
    i -= tile_threads;
    if (!a.sf || i >= (long)a.q.N * (W - 1) * nv) return;
    const int c = (int)(i % nv) * V, j = (int)(i / nv % (W - 1));
    n = (int)(i / nv / (W - 1));
    if (!a.q.range(n, s, len)) return;
    Vec<E, V, WHOLE> r;
    load_row<E, V, WHOLE, W>(r, a, n, s, len - (W - 1) + j, c);
    r.store((E*)a.sf + ((long)n * (W - 1) + j) * a.D + c, a.D - c);
    return;
  }
  const long slot = i / nv;
  const int c = (int)(i - slot * nv) * V;
  if (slot >= a.q.slots(L) || !a.q.locate(slot, L, n, s, len, pos)) return;
  const int end = min(pos + L, len);
  float w[W][V], b[V];
  load_weights<E, V, WHOLE, W>(w, b, a, c);
  Vec<E, V, WHOLE> x[W - 1 + U];
#pragma unroll
  for (int j = 0; j < W - 1; ++j) load_row<E, V, WHOLE, W>(x[j], a, n, s, pos - (W - 1) + j, c);
  E* y = (E*)a.y + s * a.D + c;
  const E* xp = (const E*)a.x + s * a.ldx + c;
  for (; pos < end; pos += U) {
#pragma unroll
    for (int k = 0; k < U; ++k)
      if (pos + k < end) x[W - 1 + k].load(xp + (long)(pos + k) * a.ldx, a.D - c);
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (pos + k >= end) break;
      Vec<E, V, WHOLE> o;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        float u = b[e];
#pragma unroll
        for (int j = 0; j < W; ++j) u += w[j][e] * x[k + j].v[e];
        o.v[e] = a.silu ? u * sigmoid<E>(u) : u;
      }
      o.store(y + (long)(pos + k) * a.D, a.D - c);
    }
#pragma unroll
    for (int j = 0; j < W - 1; ++j) x[j] = x[U + j];
  }
}

// du from u and dy.
template <typename E>
__device__ inline float act_grad(float u, float dy, int silu) {
  if (!silu) return dy;
  const float sg = sigmoid<E>(u);
  return dy * (sg * (1.f + u * (1.f - sg)));
}

// Gradient of the initial state, piece k: row i of it is x at position i - (W - 1).
template <typename E, int V, bool WHOLE, int W>
__device__ inline void initial_grad(const ConvArgs& a, long k) {
  const int nv = (a.D + V - 1) / V;
  if (k >= (long)a.q.N * (W - 1) * nv) return;
  const int c = (int)(k % nv) * V, i = (int)(k / nv % (W - 1)), n = (int)(k / nv / (W - 1));
  int len;
  long s;
  if (!a.q.range(n, s, len)) return;
  float w[W][V], b[V];
  load_weights<E, V, WHOLE, W>(w, b, a, c);
  Vec<E, V, WHOLE> o;
  if (a.dsf && i >= len) o.load((const E*)a.dsf + ((long)n * (W - 1) + i - len) * a.D + c, a.D - c);   // that row is still in the final state
  else o.zero();
  // token t reads the row with tap i - t
  Vec<E, V, WHOLE> x[2 * W - 2];
#pragma unroll
  for (int j = 0; j < 2 * W - 2; ++j) {
    if (j < W - 1 + min(len, W - 1)) load_row<E, V, WHOLE, W>(x[j], a, n, s, j - (W - 1), c);
    else x[j].zero();
  }
#pragma unroll
  for (int t = 0; t < W - 1; ++t) {
    if (t >= len || t > i) continue;
    Vec<E, V, WHOLE> g;
    g.load((const E*)a.dy + (s + t) * a.D + c, a.D - c);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      float u = b[e], tap = 0.f;
#pragma unroll
      for (int j = 0; j < W; ++j) {
        u += w[j][e] * x[t + j].v[e];
        if (j == i - t) tap = w[j][e];
      }
      o.v[e] += tap * act_grad<E>(u, g.v[e], a.silu);
    }
  }
  o.store((E*)a.ds0 + ((long)n * (W - 1) + i) * a.D + c, a.D - c);
}

// Workgroup: 64 pieces of channels (one a lane) by four successive tiles (one a
// wave), `turns` times; grid: groups of 4 x turns tiles by groups of 64 pieces,
// then the initial states' gradients by flat thread index.
template <typename E, int V, bool WHOLE, int W>
__global__ __launch_bounds__(NTHREADS) void k_conv_bwd(ConvArgs a, int cgroups, ConvBwdPlan plan) {
  constexpr int U = 4, R = W + 1;
  __shared__ float sum[R][64 * V];
  const long group = blockIdx.x / cgroups;
  if (group >= plan.groups) return initial_grad<E, V, WHOLE, W>(a, (blockIdx.x - plan.groups * cgroups) * NTHREADS + threadIdx.x);
  const int cg = (int)(blockIdx.x - group * cgroups), lane = threadIdx.x & 63, wave = wave_id(threadIdx.x);
  const int c = (cg * 64 + lane) * V;
  const bool mine = c < a.D;
  float dw[R][V] = {};             // W taps, then the bias
  float w[W][V], b[V];
  if (mine) load_weights<E, V, WHOLE, W>(w, b, a, c);
  for (int turn = 0; turn < plan.turns; ++turn) {
    int n, len, pos;
    long s;
    if (!a.q.locate((group * plan.turns + turn) * 4 + wave, plan.tile, n, s, len, pos) || !mine) continue;
    const int end = min(pos + plan.tile, len), stop = min(end + W - 1, len);
    Vec<E, V, WHOLE> x[W - 1 + U];
    float du[W - 1 + U][V];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
      load_row<E, V, WHOLE, W>(x[j], a, n, s, pos - (W - 1) + j, c);
#pragma unroll
      for (int e = 0; e < V; ++e) du[j][e] = 0.f;       // read for rows before the tile only, which are not written
    }
    const E* xp = (const E*)a.x + s * a.ldx + c;
    const E* gp = (const E*)a.dy + s * a.D + c;
    E* dx = (E*)a.dx + s * a.D + c;
    // the rows of the next turn are read while this one's are used; rows from `stop` on are read as the last one, and not used
    typedef typename Vec<E, V, WHOLE>::raw_t raw_t;
    raw_t xn[U], gn[U];
    auto fetch = [&](int t0) {
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int t = min(t0 + k, stop - 1);
        xn[k] = Vec<E, V, WHOLE>::fetch(xp + (long)t * a.ldx, a.D - c);
        gn[k] = Vec<E, V, WHOLE>::fetch(gp + (long)t * a.D, a.D - c);
      }
    };
    fetch(pos);
    for (int t0 = pos; t0 < end + W - 1; t0 += U) {
      raw_t xr[U], gr[U];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        xr[k] = xn[k];
        gr[k] = gn[k];
      }
      fetch(t0 + U);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int t = t0 + k;                            // du_t, then the row t - (W - 1) of dx
        Vec<E, V, WHOLE> g;
        g.take(gr[k]);
        x[W - 1 + k].take(xr[k]);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          float u = b[e];
#pragma unroll
          for (int j = 0; j < W; ++j) u += w[j][e] * x[k + j].v[e];
          const float d = t < stop ? act_grad<E>(u, g.v[e], a.silu) : 0.f;
          du[W - 1 + k][e] = d;
          if (t < end) {
#pragma unroll
            for (int j = 0; j < W; ++j) dw[j][e] += d * x[k + j].v[e];
            dw[W][e] += d;
          }
        }
        const int p = t - (W - 1);
        if (p < pos || p >= end) continue;
        Vec<E, V, WHOLE> o;
        if (a.dsf && p >= len - (W - 1)) o.load((const E*)a.dsf + ((long)n * (W - 1) + p - (len - (W - 1))) * a.D + c, a.D - c);
        else o.zero();
#pragma unroll
        for (int e = 0; e < V; ++e)
#pragma unroll
          for (int j = 0; j < W; ++j) o.v[e] += w[j][e] * du[W - 1 + k - j][e];
        o.store(dx + (long)p * a.D, a.D - c);
      }
#pragma unroll
      for (int j = 0; j < W - 1; ++j) {
        x[j] = x[U + j];
#pragma unroll
        for (int e = 0; e < V; ++e) du[j][e] = du[U + j][e];
      }
    }
  }
  for (int turn = 0; turn < 4; ++turn) {
    if (wave == turn)
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < V; ++e) sum[r][lane * V + e] = (turn ? sum[r][lane * V + e] : 0.f) + dw[r][e];
    __syncthreads();
  }
  for (int k = threadIdx.x; k < R * 64 * V; k += NTHREADS) {
    const int r = k / (64 * V), d = cg * 64 * V + k % (64 * V);
    if (d < a.D) a.part[(group * R + r) * a.D + d] = sum[r][k % (64 * V)];
  }
}

// One token: a thread owns V channels of one sequence and reads all of its rows before it writes.
template <typename E, int V, bool WHOLE, int W>
__global__ __launch_bounds__(64) void k_conv_step(ConvArgs a) {
  const int nv = (a.D + V - 1) / V;
  const long k = (long)blockIdx.x * 64 + threadIdx.x;
  if (k >= (long)a.q.N * nv) return;
  const int n = (int)(k / nv), c = (int)(k - (long)n * nv) * V;
  Vec<E, V, WHOLE> x[W], o;
#pragma unroll
  for (int j = 0; j < W - 1; ++j) x[j].load((const E*)a.s0 + ((long)n * (W - 1) + j) * a.D + c, a.D - c);
  x[W - 1].load((const E*)a.x + n * a.ldx + c, a.D - c);
  float w[W][V], b[V];
  load_weights<E, V, WHOLE, W>(w, b, a, c);
#pragma unroll
  for (int e = 0; e < V; ++e) {
    float u = b[e];
#pragma unroll
    for (int j = 0; j < W; ++j) u += w[j][e] * x[j].v[e];
    o.v[e] = a.silu ? u * sigmoid<E>(u) : u;
  }
  o.store((E*)a.y + (long)n * a.D + c, a.D - c);
#pragma unroll
  for (int j = 0; j < W - 1; ++j) x[j + 1].store((E*)a.sf + ((long)n * (W - 1) + j) * a.D + c, a.D - c);
}

template <typename E, int V, bool WHOLE, int W>
hipError_t fwd(const ConvArgs& a, hipStream_t st) {
  const int nv = (a.D + V - 1) / V;
  const long tokens = a.q.cu ? a.q.T : (long)a.q.N * a.q.T;
  // The longest tiles that give every CU eight waves: few rows are read twice
  // then, but short prompts need the threads more (6144 channels, forward and
  // backward with tiles of 8, 16, 32, 64: 4 x 4096 tokens 241, 229, 224, 219 us,
  // 4096 tokens 59, 56, 58, 70, 1024 tokens 35, 37, 44, 59).
  int L = 64;
  while (L > 8 && tokens / L * nv < 1 << 17) L /= 2;
  const long tiles = a.q.slots(L) * nv, states = a.sf ? (long)a.q.N * (W - 1) * nv : 0;
  if (tiles + states == 0) return hipSuccess;
  const dim3 grid((unsigned)((tiles + states + NTHREADS - 1) / NTHREADS));
  hipLaunchKernelGGL((k_conv_fwd<E, V, WHOLE, W>), grid, dim3(NTHREADS), 0, st, a, L, tiles);
  return hipGetLastError();
}

template <typename E, int V, bool WHOLE, int W>
hipError_t bwd(const ConvArgs& a, hipStream_t st) {
  const int nv = (a.D + V - 1) / V, cgroups = (nv + 63) / 64;
  const ConvBwdPlan plan = conv_bwd_plan(a.q, a.D);
  const long states = a.ds0 ? (long)a.q.N * (W - 1) * nv : 0;
  const long blocks = plan.groups * cgroups + (states + NTHREADS - 1) / NTHREADS;
  if (blocks > 0)
    hipLaunchKernelGGL((k_conv_bwd<E, V, WHOLE, W>), dim3((unsigned)blocks), dim3(NTHREADS), 0, st, a, cgroups, plan);
  return hipGetLastError();
}

template <typename E, int V, bool WHOLE, int W>
hipError_t step(const ConvArgs& a, hipStream_t st) {
  const long n = (long)a.q.N * ((a.D + V - 1) / V);
  if (n > 0) hipLaunchKernelGGL((k_conv_step<E, V, WHOLE, W>), dim3((unsigned)((n + 63) / 64)), dim3(64), 0, st, a);
  return hipGetLastError();
}

bool whole(const ConvArgs& a, int esz) {
  const int v = 16 / esz;
  uintptr_t p = 0;
  for (const void* q : {a.x, a.w, a.b, a.s0, (const void*)a.y, (const void*)a.sf, a.dy, a.dsf, (const void*)a.dx, (const void*)a.ds0})
    p |= (uintptr_t)q;
  return a.D % v == 0 && a.ldx % v == 0 && (p & 15) == 0;
}

// VB: channels of a thread for bf16 (see above); for fp32, 16 bytes of them.
#define QD_CONV(FN, VB)                                                                                                \
  template <typename E, int V, bool WHOLE>                                                                             \
  hipError_t FN##_w(const ConvArgs& a, hipStream_t st) {                                                               \
    if (a.W == 2) return FN<E, V, WHOLE, 2>(a, st);                                                                    \
    if (a.W == 3) return FN<E, V, WHOLE, 3>(a, st);                                                                    \
    return a.W == 4 ? FN<E, V, WHOLE, 4>(a, st) : hipErrorInvalidValue;                                                \
  }                                                                                                                    \
  hipError_t FN##_e(const ConvArgs& a, int dtype, hipStream_t st) {                                                    \
    if (dtype == 1) return whole(a, 2) ? FN##_w<__bf16, VB, true>(a, st) : FN##_w<__bf16, VB, false>(a, st);           \
    return whole(a, 4) ? FN##_w<float, 4, true>(a, st) : FN##_w<float, 4, false>(a, st);                               \
  }
QD_CONV(fwd, 8)
QD_CONV(bwd, 4)
QD_CONV(step, 8)
#undef QD_CONV

}  // namespace

// The longest tiles of 8 to 32 tokens that give every SIMD two waves (4 channels
// a lane in either type; training steps in bf16 with 8, 16, 32: 4 x 4096 tokens
// of 6144 channels 239, 224, 217 us, 4096 tokens 64, 60, 56, 2003 tokens of 1001
// channels 36, 36, 47).  Beyond what fills the chip tiles are taken in turns, so
// that the partial rows (W + 1 times D floats each) stay few and a wave reads
// the weights once (4096 sequences of 4 tokens, 4096 channels: 1068 -> 574 us).
ConvBwdPlan conv_bwd_plan(const Seqs& q, int D) {
  const long cgroups = (D + 255) / 256, most = D < 512 ? 2048 : (1L << 20) / D < 64 ? 64 : (1L << 20) / D;
  ConvBwdPlan p;
  p.tile = 32;
  while (p.tile > 8 && q.slots(p.tile) * cgroups < 2048) p.tile /= 2;
  const long groups = (q.slots(p.tile) + 3) / 4;
  p.turns = (int)((groups + most - 1) / most);
  if (p.turns < 1) p.turns = 1;
  p.groups = (groups + p.turns - 1) / p.turns;
  return p;
}

hipError_t launch_conv_fwd(const ConvArgs& a, int dtype, hipStream_t st) { return fwd_e(a, dtype, st); }

hipError_t launch_conv_bwd(const ConvArgs& a, int dtype, hipStream_t st) {
  const hipError_t e = bwd_e(a, dtype, st);
  if (e != hipSuccess || (!a.dw && !a.db)) return e;
  return launch_colsum(a.part, (int)conv_bwd_plan(a.q, a.D).groups, a.W + 1, a.W, a.D, dtype, a.dw, a.db, st);
}

hipError_t launch_conv_step(const ConvArgs& a, int dtype, hipStream_t st) { return step_e(a, dtype, st); }

}  // namespace qd
