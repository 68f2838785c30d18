// Selective state space scan, backward.
//
// Per chunk of 64 tokens with entry state S, exit gradient G = dL/dS', b the
// prefix sums of dt A, W_ri = exp(b_r - b_i) for i <= r, K = C B^T, E = dY X^T:
//
//   dx_i = dt_i u_i + D dy_i,   u_i = sum_r W_ri K_ri dy_r + e^{b_C - b_i} G B_i
//   dC_r = e^{b_r} S^T dy_r + sum_i W_ri dt_i E_ri B_i          (over the group's heads)
//   dB_i = dt_i (sum_r W_ri E_ri C_r + e^{b_C - b_i} G^T x_i)   (over the group's heads)
//   x_i . u_i = sum_r W_ri K_ri E_ri + e^{b_C - b_i} x_i . G B_i
//
// and for l = dt A, whose gradient is dl_t = e^{l_t} <G_t, S_{t-1}>: with
// M_ri = W_ri K_ri E_ri dt_i (i < r), it is the sum of M over r >= t > i, of
// e^{b_r} dy_r . S C_r over r >= t, of dt_i e^{b_C - b_i} x_i . G B_i over i < t,
// and e^{b_C} <G, S>.  The first is formed from the pairs that straddle t alone
// (differences of row and column sums would leave the rounding of all other
// pairs, which is what remains where a token wipes the state).
// Then ddt_t = x_t . u_t + A dl_t, dA = sum dt dl, dD = sum_r E_rr.
//
// The states S and gradients G of all chunks come from two walks (one launch);
// then chunks are independent.  A workgroup takes a chunk and loops over the
// heads of a group (or a share of them: `splits`, whose dB and dC are then
// summed in order), with K and the group's dB and dC in registers.  Waves 0 to
// 3 form dC (S, E^T) and G B^T, waves 4 to 7 dB and dX (G, E); of each four
//   wave w, tokens 16 w ..      the products over the chunk's tokens, from
//                               E and E^T as they stand in the accumulators;
//   wave w, a quarter of n      the products with S and G, whose operands are
//                               read straight from the walks' register order;
//   wave w, rows 16 w .. of p   G B^T, with G through LDS.
#include "qd_ssm.h"

namespace qd {

namespace {

template <typename E, int NP>
struct BwdLds {
  static constexpr int LDN = lds_ld<E>(NP), LDP = lds_ld<E>(PT), PL = sizeof(E) == 2 ? 2 : 1;
  static constexpr int LDS_ = lds_ld<float>(NP), LDT = lds_ld<float>(PT);
  E B[C * LDN], Cm[C * LDN], X[C * LDP], dY[C * LDP];
  union {
    E G[PL][NP * LDP];               // G^T: [n][p], planes
    float sum[C * LDS_];             // the end: one half of dC, of dB
  };
  float dX[C * LDT];                 // [i][p]: the part of dX with G
  Gates g;
  float cs[3][C], fd[C];             // M: sums over r in block w > 0 by i < 16 w; pairs with r in t's own block
  float mcol[C], diag[C], err[C], srow[4][C], gcol[4][C], sg[4];
};

// Keeps the scheduler from drawing the loads of one phase of a turn into the
// phase before, where all registers are taken.
__device__ inline void phase() { __builtin_amdgcn_sched_barrier(0); }

// The lane number as a value the compiler cannot trace: what is formed from it
// (LDS addresses, masks of the triangles) is formed again every turn of the
// loop over heads instead of being kept in registers, which are all taken
// (hoisted, 130 such values went to scratch memory and back).
__device__ inline int fresh(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Sum over the four lane groups (the rows of an accumulator's columns).
__device__ inline float groups_sum(float x) {
  x += __shfl_xor(x, 16, 64);
  return x + __shfl_xor(x, 32, 64);
}

// Sum over the lanes before this one: the inclusive sum of the lane below, so
// that nothing is taken away again.
__device__ inline float before_lane(float x, int lane) {
  const float s = lane_from(wave_incl_scan_dpp(x), lane - 1);
  return lane ? s : 0.f;
}

template <typename E, int NP>
__global__ __launch_bounds__(2 * NTHREADS, 1) void k_ssm_bwd(ScanArgs a, long items) {
  typedef BwdLds<E, NP> L;
  typedef typename Q4<E>::t q4;
  __shared__ __attribute__((aligned(16))) L s;
  constexpr int NB = NP / 16, KN = NP / 32, NQ = NB / 4, PL = L::PL, NT = 2 * NTHREADS;
  long item;
  if (!xcd_item(items, item)) return;
  const int per = a.G * a.splits, grp = (int)(item % per) / a.splits, split = (int)(item % a.splits);
  const long slot = item / per;
  int n, len, pos;
  long s0;
  if (!a.q.locate(slot, C, n, s0, len, pos)) return;
  const int rows = min(C, len - pos), t = threadIdx.x, lane0 = t & 63, lane = lane0, wave = wave_id(t), w = wave & 3;
  const int g4 = 4 * (lane >> 4), col = lane & 15, own = 16 * w + col;     // this lane's token in the products over tokens
  const long t0 = s0 + pos;
  const int pts = p_tiles(a.P), hg = a.H / a.G;
  const int h0 = grp * hg + hg * split / a.splits, h1 = grp * hg + hg * (split + 1) / a.splits;
  const int turns = (h1 - h0) * pts;

  {
    Stage<E, NP, NT> rb, rc;
    const E* B = (const E*)a.B + t0 * a.ldb + (long)grp * a.N;
    const E* Cm = (const E*)a.C + t0 * a.ldc + (long)grp * a.N;
    rb.load(B, a.ldb, rows, a.N, vec_rows<E>(B, a.ldb, a.N), t);
    rc.load(Cm, a.ldc, rows, a.N, vec_rows<E>(Cm, a.ldc, a.N), t);
    rb.put(s.B, L::LDN, t);
    rc.put(s.Cm, L::LDN, t);
  }
  Stage<E, PT, NT> rx, ry;
  float rg = 0.f;
  auto fetch = [&](int turn) {
    const int h = h0 + turn / pts, pt = turn % pts, cols = min(PT, a.P - pt * PT);
    const E* x = (const E*)a.x + t0 * a.ldx + (long)h * a.P + pt * PT;
    const E* dy = (const E*)a.dy + (t0 * a.H + h) * a.P + pt * PT;
    rx.load(x, a.ldx, rows, cols, vec_rows<E>(x, a.ldx, cols), t);
    ry.load(dy, (long)a.H * a.P, rows, cols, vec_rows<E>(dy, (long)a.H * a.P, cols), t);
    if (t < GATES) rg = a.gates[(slot * a.H + h) * GATES + t];
  };
  auto put = [&]() {
    rx.put(s.X, L::LDP, t);
    ry.put(s.dY, L::LDP, t);
    if (t < GATES) ((float*)&s.g)[t] = rg;
  };
  // this wave's quarter of a state or gradient: f4 [pb][nq] holds rows p = 16 pb + g4 + j of column n
  auto quarter = [&](f4(&v)[4][NQ], const float* from, int turn, int lane) {
    const float* src = from + (slot * a.H * pts + (long)h0 * pts + turn) * (long)(PT * NP);
#pragma unroll
    for (int pb = 0; pb < 4; ++pb)
#pragma unroll
      for (int q = 0; q < NQ; ++q) v[pb][q] = *(const f4*)(src + ((pb * NB + w * NQ + q) * 64 + lane) * 4);
  };
  // dB or dC of the chunk: [n][token] accumulators of this lane's token over all n, and of all tokens over a quarter of n
  const long gn = (long)a.G * a.N;
  auto half = [&](const f4(&v)[NQ][4]) {
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
      for (int b = 0; b < 4; ++b) *(f4*)(s.sum + (16 * b + col) * L::LDS_ + 16 * (w * NQ + q) + g4) = v[q][b];
  };
  auto write = [&](const f4(&v)[NB], void* whole, float* part) {
    if (own >= rows) return;
    const bool vq = a.N % 4 == 0 && ((uintptr_t)whole & (4 * sizeof(E) - 1)) == 0;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int nn = 16 * b + g4;
      const f4 x = v[b] + *(const f4*)(s.sum + own * L::LDS_ + nn);
      const long at = (t0 + own) * gn + (long)grp * a.N + nn;
      if (a.splits > 1) {
        const long tokens = a.q.cu ? a.q.T : (long)a.q.N * a.q.T;
        float* out = part + split * tokens * gn + at;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (nn + j < a.N) out[j] = x[j];
      } else if (vq) {
        if (nn < a.N) *(q4*)((E*)whole + at) = narrow<E>(x);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (nn + j < a.N) ((E*)whole)[at + j] = fromf<E>(x[j]);
      }
    }
  };
  fetch(0);

  if (wave < 4) {
    f4 S[4][NQ], kr[4], dct[NB], dcn[NQ][4];
    quarter(S, a.states, 0, lane);
#pragma unroll
    for (int b = 0; b < NB; ++b) dct[b] = zero4();
#pragma unroll
    for (int b = 0; b < NQ; ++b)
#pragma unroll
      for (int k = 0; k < 4; ++k) dcn[b][k] = zero4();
    __syncthreads();
    // K of rows r = own: accumulator rows are i
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      kr[b] = zero4();
      if (b <= w)
#pragma unroll
        for (int k = 0; k < KN; ++k)
          kr[b] = mma(row_frag<E>(s.B, L::LDN, 16 * b, 32 * k, lane), row_frag<E>(s.Cm, L::LDN, 16 * w, 32 * k, lane), kr[b]);
    }
    for (int turn = 0; turn < turns; ++turn) {
      const bool first = turn % pts == 0;
      const int lane = fresh(lane0), g4 = 4 * (lane >> 4), col = lane & 15, own = 16 * w + col;
      put();
      __syncthreads();
      if (turn + 1 < turns) fetch(turn + 1);
      const float he = s.g.bh[C - 1], le = s.g.bl[C - 1];
      // e^{b_r} S^T dy_r over this wave's quarter of n
      {
        float sr[4] = {};
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          const int n0 = 16 * (w * NQ + q) + g4;
          f4 u[4];
#pragma unroll
          for (int b = 0; b < 4; ++b) u[b] = zero4();
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const Planes<E, 3> sp = planes<E, 3>(S[2 * k][q], S[2 * k + 1][q]);
#pragma unroll
            for (int b = 0; b < 4; ++b) u[b] = mma(sp, row_frag<E>(s.dY, L::LDP, 16 * b, 32 * k, lane), u[b]);
          }
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            const int r = 16 * b + col;
            u[b] *= decay(s.g.bh[r], s.g.bl[r], 0.f, 0.f);
            const f4 c = widen<E>(*(const q4*)(s.Cm + r * L::LDN + n0));
#pragma unroll
            for (int j = 0; j < 4; ++j) sr[b] += c[j] * u[b][j];
            dcn[q][b] += u[b];
          }
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          sr[b] = groups_sum(sr[b]);
          if (g4 == 0) s.srow[w][16 * b + col] = (first ? 0.f : s.srow[w][16 * b + col]) + sr[b];
        }
      }
      phase();
      if (turn + 1 < turns) quarter(S, a.states, turn + 1, lane);
      phase();
      // W E diag(dt) of rows r = own: accumulator rows are i
      f4 e[4], md = zero4();
      {
        const float hr = s.g.bh[own], lr = s.g.bl[own];
        float before = 0.f;                // sum of M_ri over the blocks i < 16 w
        Fr<E> yf[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) yf[k] = row_frag<E>(s.dY, L::LDP, 16 * w, 32 * k, lane);
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          e[b] = zero4();
          if (b > w) continue;
#pragma unroll
          for (int k = 0; k < 2; ++k) e[b] = mma(row_frag<E>(s.X, L::LDP, 16 * b, 32 * k, lane), yf[k], e[b]);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int i = 16 * b + g4 + j;
            const float f = i <= own ? e[b][j] * decay(hr, lr, s.g.bh[i], s.g.bl[i]) * s.g.dt[i] : 0.f;
            e[b][j] = f;
            const float m = i < own ? f * kr[b][j] : 0.f;
            if (b == w) {
              md[j] = m;
            } else {
              before += m;
              const float c = sum16(m);
              if (col == 0) s.cs[w - 1][i] = (first ? 0.f : s.cs[w - 1][i]) + c;
            }
          }
          phase();
        }
        // sum over r >= t in this block and all i < t, t = own: (M V)_rt with V_it = [i < t] as a product, the
        // blocks before as one more column, then the rows r >= t
        before = groups_sum(before);
        f4 v = __builtin_amdgcn_mfma_f32_16x16x4f32(g4 == 0 ? before : 0.f, 1.f, zero4(), 0, 0, 0);
#pragma unroll
        for (int j = 0; j < 4; ++j) v = __builtin_amdgcn_mfma_f32_16x16x4f32(md[j], g4 + j < col ? 1.f : 0.f, v, 0, 0, 0);
        float f = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) f += g4 + j >= col ? v[j] : 0.f;
        f = groups_sum(f);
        if (g4 == 0) s.fd[own] = (first ? 0.f : s.fd[own]) + f;
      }
      phase();
      // rows p = 16 w .. of G B^T for all tokens, to the waves that own them
      {
        f4 v[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) v[b] = zero4();
#pragma unroll
        for (int k = 0; k < KN; ++k) {
          Fr<E> gp[PL];
#pragma unroll
          for (int pl = 0; pl < PL; ++pl) gp[pl] = col_frag<E>(s.G[pl], L::LDP, 32 * k, 16 * w, lane);
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            const Fr<E> bf = row_frag<E>(s.B, L::LDN, 16 * b, 32 * k, lane);
#pragma unroll
            for (int pl = PL - 1; pl >= 0; --pl) v[b] = mma(gp[pl], bf, v[b]);
          }
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const int i = 16 * b + col;
          *(f4*)(s.dX + i * L::LDT + 16 * w + g4) = v[b] * decay(he, le, s.g.bh[i], s.g.bl[i]);
        }
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if (2 * k > w) break;
        const Planes<E, 2> ep = planes<E, 2>(e[2 * k], e[2 * k + 1]);
#pragma unroll
        for (int b = 0; b < NB; ++b) dct[b] = mma(col_frag<E>(s.B, L::LDN, 32 * k, 16 * b, lane), ep, dct[b]);
      }
      __syncthreads();
    }
    half(dcn);
    __syncthreads();
    write(dct, a.dC, a.partC);
    __syncthreads();
    __syncthreads();
    return;
  }

  f4 G[4][NQ], kc[4], dbt[NB], dbn[NQ][4];
  quarter(G, a.grads, 0, lane);
#pragma unroll
  for (int b = 0; b < NB; ++b) dbt[b] = zero4();
#pragma unroll
  for (int b = 0; b < NQ; ++b)
#pragma unroll
    for (int k = 0; k < 4; ++k) dbn[b][k] = zero4();
  __syncthreads();
  // K of columns i = own: accumulator rows are r
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    kc[b] = zero4();
    if (b >= w)
#pragma unroll
      for (int k = 0; k < KN; ++k)
        kc[b] = mma(row_frag<E>(s.Cm, L::LDN, 16 * b, 32 * k, lane), row_frag<E>(s.B, L::LDN, 16 * w, 32 * k, lane), kc[b]);
  }
  for (int turn = 0; turn < turns; ++turn) {
    const bool first = turn % pts == 0;
    const int h = h0 + turn / pts, pt = turn % pts;
    const int lane = fresh(lane0), g4 = 4 * (lane >> 4), col = lane & 15, own = 16 * w + col;
    put();
    float sg = 0.f;
    {
      const float* S = a.states + (slot * a.H * pts + (long)h0 * pts + turn) * (long)(PT * NP);
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        const int nn = 16 * (w * NQ + q) + col;
#pragma unroll
        for (int pb = 0; pb < 4; ++pb) {
          f4 v = G[pb][q];
          const f4 sv = *(const f4*)(S + ((pb * NB + w * NQ + q) * 64 + lane) * 4);
#pragma unroll
          for (int j = 0; j < 4; ++j) sg += v[j] * sv[j];
#pragma unroll
          for (int pl = 0; pl < PL; ++pl) {
            const q4 x = narrow<E>(v);
            *(q4*)(s.G[pl] + nn * L::LDP + 16 * pb + g4) = x;
            if (pl + 1 < PL) v -= widen<E>(x);
          }
        }
        phase();
      }
    }
    sg = groups_sum(sum16(sg));
    if (lane == 0) s.sg[w] = (first ? 0.f : s.sg[w]) + sg;
    __syncthreads();
    if (turn + 1 < turns) fetch(turn + 1);
    const float he = s.g.bh[C - 1], le = s.g.bl[C - 1];
    // e^{b_C - b_i} G^T x_i over this wave's quarter of n
    {
      float gc[4] = {};
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        const int n0 = 16 * (w * NQ + q) + g4;
        f4 v[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) v[b] = zero4();
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const Planes<E, 3> gp = planes<E, 3>(G[2 * k][q], G[2 * k + 1][q]);
#pragma unroll
          for (int b = 0; b < 4; ++b) v[b] = mma(gp, row_frag<E>(s.X, L::LDP, 16 * b, 32 * k, lane), v[b]);
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const int i = 16 * b + col;
          v[b] *= decay(he, le, s.g.bh[i], s.g.bl[i]);
          const f4 bb = widen<E>(*(const q4*)(s.B + i * L::LDN + n0));
#pragma unroll
          for (int j = 0; j < 4; ++j) gc[b] += bb[j] * v[b][j];
          dbn[q][b] += s.g.dt[i] * v[b];
        }
      }
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        gc[b] = groups_sum(gc[b]);
        if (g4 == 0) s.gcol[w][16 * b + col] = (first ? 0.f : s.gcol[w][16 * b + col]) + gc[b];
      }
    }
    phase();
    if (turn + 1 < turns) quarter(G, a.grads, turn + 1, lane);
    phase();
    // W E and W K of columns i = own: accumulator rows are r
    f4 xacc[4];
    const float dt = s.g.dt[own];
    {
      const float hi = s.g.bh[own], li = s.g.bl[own];
      float mcol = 0.f, diag = 0.f, err = 0.f;
      f4 e[4], wk[4];
      Fr<E> xf[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) xf[k] = row_frag<E>(s.X, L::LDP, 16 * w, 32 * k, lane);
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        e[b] = wk[b] = zero4();
        if (b < w) continue;
#pragma unroll
        for (int k = 0; k < 2; ++k) e[b] = mma(row_frag<E>(s.dY, L::LDP, 16 * b, 32 * k, lane), xf[k], e[b]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int r = 16 * b + g4 + j;
          const float wt = r >= own ? decay(s.g.bh[r], s.g.bl[r], hi, li) : 0.f;
          const float ev = r >= own ? e[b][j] : 0.f, f = ev * wt;
          mcol += r > own ? f * kc[b][j] : 0.f;
          diag += r == own ? ev * kc[b][j] : 0.f;
          err += r == own ? ev : 0.f;
          e[b][j] = f * dt;
          wk[b][j] = r >= own ? wt * kc[b][j] : 0.f;
        }
        phase();
      }
      mcol = groups_sum(mcol);
      diag = groups_sum(diag);
      err = groups_sum(err);
      if (g4 == 0) {
        s.mcol[own] = (first ? 0.f : s.mcol[own]) + mcol;
        s.diag[own] = (first ? 0.f : s.diag[own]) + diag;
        s.err[own] = (first ? 0.f : s.err[own]) + err;
      }
      phase();
#pragma unroll
      for (int b = 0; b < 4; ++b) xacc[b] = zero4();
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if (2 * k + 1 < w) continue;
        const Planes<E, 2> ep = planes<E, 2>(e[2 * k], e[2 * k + 1]);
#pragma unroll
        for (int b = 0; b < NB; ++b) dbt[b] = mma(col_frag<E>(s.Cm, L::LDN, 32 * k, 16 * b, lane), ep, dbt[b]);
        const Planes<E, 2> wp = planes<E, 2>(wk[2 * k], wk[2 * k + 1]);
#pragma unroll
        for (int b = 0; b < 4; ++b) xacc[b] = mma(col_frag<E>(s.dY, L::LDP, 32 * k, 16 * b, lane), wp, xacc[b]);
      }
    }
    __syncthreads();
    {
      const int cols = min(PT, a.P - pt * PT);
      const float D = a.D ? a.D[h] : 0.f;
      E* out = (E*)a.dx + ((t0 + own) * a.H + h) * (long)a.P + pt * PT;
      const bool vo = a.P % 4 == 0 && ((uintptr_t)a.dx & (4 * sizeof(E) - 1)) == 0;
      if (own < rows)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const int p = 16 * b + g4;
          f4 v = dt * (xacc[b] + *(const f4*)(s.dX + own * L::LDT + p));
          if (a.D) v += D * widen<E>(*(const q4*)(s.dY + own * L::LDP + p));
          if (vo) {
            if (p < cols) *(q4*)(out + p) = narrow<E>(v);
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (p + j < cols) out[p + j] = fromf<E>(v[j]);
          }
        }
    }
    // the time step's gradient and the head's sums, a token a lane, on the wave with the fewest products
    if (pt == pts - 1 && w == 3) {
      const int r = lane;
      const float step = s.g.dt[r], A = a.A[h];
      const float srow = (s.srow[0][r] + s.srow[1][r]) + (s.srow[2][r] + s.srow[3][r]);
      const float gcol = (s.gcol[0][r] + s.gcol[1][r]) + (s.gcol[2][r] + s.gcol[3][r]);
      float dl = ((s.sg[0] + s.sg[1]) + (s.sg[2] + s.sg[3])) * decay(he, le, 0.f, 0.f);
      dl += lane_from(wave_incl_scan_dpp(lane_from(srow, 63 - lane)), 63 - lane);          // over r >= t
      dl += before_lane(step * gcol, lane) + s.fd[r];                                      // over i < t
#pragma unroll
      for (int b = 1; b < 4; ++b) {
        const float c = before_lane(r < 16 * b ? s.cs[b - 1][r] : 0.f, lane);
        dl += r < 16 * b ? c : 0.f;
      }
      float raw = s.mcol[r] + s.diag[r] + gcol + A * dl;
      const bool in = r < rows;
      if (a.softplus) raw *= -expm1f(-step);             // sigmoid of the raw step, from its softplus
      if (in) a.ddt[(t0 + r) * a.H + h] = raw;
      float sa = in ? step * dl : 0.f, sd = in ? s.err[r] : 0.f, sb = in ? raw : 0.f;
      sa = groups_sum(sum16(sa));
      sd = groups_sum(sum16(sd));
      sb = groups_sum(sum16(sb));
      if (lane == 0) *(f4*)(a.sums + (slot * a.H + h) * 4) = f4{sa, sd, sb, 0.f};
    }
    __syncthreads();
  }
  __syncthreads();
  __syncthreads();
  half(dbn);
  __syncthreads();
  write(dbt, a.dB, a.partB);
}

// dB and dC from the shares of the splits, in order.
template <typename E>
__global__ __launch_bounds__(NTHREADS) void k_ssm_join(ScanArgs a, long n) {
  const float* part = blockIdx.y ? a.partB : a.partC;
  E* out = (E*)(blockIdx.y ? a.dB : a.dC);
  for (long i = (long)blockIdx.x * NTHREADS + threadIdx.x; i < n; i += (long)gridDim.x * NTHREADS) {
    float v = part[i];
    for (int k = 1; k < a.splits; ++k) v += part[k * n + i];
    out[i] = fromf<E>(v);
  }
}

// dA, dD and the bias's gradient of a head: its chunks' sums, in a fixed order.
__global__ __launch_bounds__(NTHREADS) void k_ssm_heads(ScanArgs a, long slots) {
  __shared__ f4 red[NTHREADS];
  const int h = blockIdx.x, t = threadIdx.x;
  f4 v = zero4();
  for (long k = t; k < slots; k += NTHREADS) {
    int n, len, pos;
    long s0;
    if (a.q.cu && !a.q.locate(k, C, n, s0, len, pos)) continue;
    v += *(const f4*)(a.sums + (k * a.H + h) * 4);
  }
  red[t] = v;
  __syncthreads();
#pragma unroll
  for (int off = NTHREADS / 2; off >= 1; off >>= 1) {
    if (t < off) red[t] += red[t + off];
    __syncthreads();
  }
  if (t) return;
  a.dA[h] = red[0][0];
  if (a.dD) a.dD[h] = red[0][1];
  if (a.dbias) a.dbias[h] = red[0][2];
}

template <typename E, int NP>
hipError_t chunks(const ScanArgs& a, hipStream_t st) {
  const long items = a.q.slots(C) * a.G * a.splits;
  if (items == 0) return hipSuccess;
  hipLaunchKernelGGL((k_ssm_bwd<E, NP>), dim3(xcd_grid(items)), dim3(2 * NTHREADS), 0, st, a, items);
  return hipGetLastError();
}

}  // namespace

// Workgroups that share the heads of a chunk: as many as give every CU one.
int scan_splits(const Seqs& q, int H, int G) {
  const long units = q.slots(C) * G, cus = device_cu_count();
  if (units <= 0) return 1;
  const long s = (cus + units - 1) / units;
  return (int)(s < 1 ? 1 : s > H / G ? H / G : s);
}

hipError_t launch_scan_bwd(const ScanArgs& a, int dtype, hipStream_t st) {
  hipError_t e = launch_scan_gates(a, st);
  if (e == hipSuccess && a.seg) {
    e = launch_scan_walks(a, dtype, 3, false, st);
    if (e == hipSuccess) e = launch_scan_compose(a, 3, st);
  }
  if (e == hipSuccess) e = launch_scan_walks(a, dtype, 3, true, st);
  if (e != hipSuccess) return e;
  if (dtype == 1) e = a.N <= 64 ? chunks<__bf16, 64>(a, st) : chunks<__bf16, 128>(a, st);
  else e = a.N <= 64 ? chunks<float, 64>(a, st) : chunks<float, 128>(a, st);
  if (e != hipSuccess) return e;
  const long n = (a.q.cu ? a.q.T : (long)a.q.N * a.q.T) * a.G * a.N;
  if (a.splits > 1 && n > 0) {
    const long blocks = (n + NTHREADS - 1) / NTHREADS;
    const dim3 grid((unsigned)(blocks > 4096 ? 4096 : blocks), 2);
    if (dtype == 1) hipLaunchKernelGGL((k_ssm_join<__bf16>), grid, dim3(NTHREADS), 0, st, a, n);
    else hipLaunchKernelGGL((k_ssm_join<float>), grid, dim3(NTHREADS), 0, st, a, n);
  }
  hipLaunchKernelGGL(k_ssm_heads, dim3(a.H), dim3(NTHREADS), 0, st, a, a.q.slots(C));
  return hipGetLastError();
}

}  // namespace qd
