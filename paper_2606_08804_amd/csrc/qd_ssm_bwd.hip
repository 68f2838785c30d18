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
// 3 form dC (S, E^T) and G B^T, waves 4 to 7 dB and dx (G, E); of each four
//   wave w, tokens 16 w ..      the products over the chunk's tokens, from
//                               E and E^T as they stand in the accumulators;
//   wave w, a quarter of n      the products with S and G, whose operands are
//                               read straight from the walks' register order;
//   wave w, rows 16 w .. of p   G B^T, with G through LDS.
// A spilled register costs more than its own bytes: its reload waits for every
// prefetch issued before it.  Within the loop over heads, waves 0 to 3 reload one
// quad of K a turn in bf16 with N > 64 (none with N <= 64); fp32 with N > 64, where the
// operands of a product take twice the registers, stores five quads a turn and
// reloads up to nine.
//
// 4 x 4096 tokens, 64 heads of one group, state 64 x 128, bf16: 541 us, 8.5 us a
// chunk and head.  States and gradients are 1.08 of the 1.61 GB it moves (3.0
// TB/s); vector instructions take 48% of the cycles and matrix products 21%,
// on two waves a SIMD, which the registers (256 each) and LDS allow.
#include "qd_ssm.h"

namespace qd {

namespace {

template <typename E, int NP>
struct BwdLds {
  static constexpr int LDN = lds_ld<E>(NP), LDP = lds_ld<E>(PT), LDX = steps_ld<E>(PT), PL = Planes<E, 3>::N;
  static constexpr int LDS_ = lds_ld<float>(NP), LDT = sizeof(E) == 4 && NP == 128 ? PT : lds_ld<float>(PT);   // (no room for padding there)
  E B[C * LDN], Cm[C * LDN], dY[C * LDP];
  E X[C * LDX];                      // steps
  union {
    E G[PL][NP * LDP];               // G^T: [n][p], planes
    float sum[C * LDS_];             // the end: one half of dC, of dB
  };
  float dX[C * LDT];                 // [i][p]: the part of dX with G
  Gates g;
  struct Sums {                      // of a head, over its tiles
    float cs[3][C], fd[C];           // M: sums over r in block w > 0 by i < 16 w; pairs with r in t's own block
    float mcol[C], diag[C], err[C], srow[4][C], gcol[4][C], sg[4], dt[C], total;
  };
  Sums sums[2];                      // this head's and the one's before
};

// Sum over the four lane groups (the rows of an accumulator's columns).
// (The lane number formed here: what __shfl_xor forms of it would be kept over the
// loops, in scratch memory.)
__device__ inline float groups_sum(float x) {
  const int lane = fresh_lane();
  x += lane_from(x, lane ^ 16);
  return x + lane_from(x, lane ^ 32);
}

// Sum over the lanes before this one: the inclusive sum of the lane below, so
// that nothing is taken away again.
__device__ inline float before_lane(float x, int lane) {
  const float s = lane_from(wave_incl_scan_dpp(x), lane - 1);
  return lane ? s : 0.f;
}

// WHOLE: all rows of x, dy, B and C are whole aligned pieces; without the other
// way of reading them in the loops a training step of the size above takes 1058
// us instead of 1062, repeated on the same tensors.
template <typename E, int NP, bool WHOLE>
__global__ __launch_bounds__(2 * NTHREADS, 1) QD_TWO_WAVES void k_ssm_bwd(ScanArgs a, long items) {
  typedef BwdLds<E, NP> L;
  typedef typename Q4<E>::t q4;
  __shared__ __attribute__((aligned(16))) L s;
  constexpr int NB = NP / 16, KN = NP / 32, NQ = NB / 4, PL = L::PL, NT = NTHREADS;
  long item;
  if (!xcd_item(items, item)) return;
  const int per = a.G * a.splits, grp = (int)(item % per) / a.splits, split = (int)(item % a.splits);
  const long slot = item / per;
  int n, len, pos;
  long s0;
  if (!a.q.locate(slot, C, n, s0, len, pos)) return;
  const int rows = min(C, len - pos), tid = threadIdx.x, wave = wave_id(tid), w = wave & 3;
  const long t0 = s0 + pos;
  const int pts = p_tiles(a.P), hg = a.H / a.G;
  const int h0 = grp * hg + hg * split / a.splits, h1 = grp * hg + hg * (split + 1) / a.splits;
  const int turns = (h1 - h0) * pts;
  const long ldy = (long)a.H * a.P;

  // Staging: the first half of the threads loads B, then every turn's x; the
  // second C, then dy.  Both read rows of one matrix.
  const int half = wave >> 2, st = tid & (NT - 1);
  {
    Stage<E, NP, NT> r;
    const long ld = half ? a.ldc : a.ldb;
    const E* m = (const E*)(half ? a.C : a.B) + t0 * ld + (long)grp * a.N;
    const bool vec = WHOLE || vec_rows<E>(m, ld, a.N);
    r.load(m, ld, rows, vec, r.offset(ld, a.N, st));
    r.put(half ? s.Cm : s.B, L::LDN, m, ld, rows, a.N, vec, st);
  }
  Stage<E, PT, NT> rt;
  float rg = 0.f;
  const long ldt = half ? ldy : a.ldx;
  const E* tile0 = (half ? (const E*)a.dy : (const E*)a.x) + t0 * ldt + (long)h0 * a.P;
  // whole pieces in one tile of a head are whole pieces in all of them
  const bool vt = WHOLE || (a.P % (16 / (int)sizeof(E)) == 0 && vec_rows<E>(tile0, ldt, a.P));
  auto fetch = [&](int turn) {
    const int p0 = turn % pts * PT, st = (wave & 3) * 64 + fresh_lane();
    rt.load(tile0 + (long)(turn / pts) * a.P + p0, ldt, rows, vt, rt.offset(ldt, min(PT, a.P - p0), st));
    rg = load_gate(a.gates + (slot * a.H + h0 + turn / pts) * GATES, half * NT + st);
  };
  auto put = [&](int turn) {
    const int p0 = turn % pts * PT, st = (wave & 3) * 64 + fresh_lane();
    const E* src = tile0 + (long)(turn / pts) * a.P + p0;
    if (half) rt.put(s.dY, L::LDP, src, ldt, rows, min(PT, a.P - p0), vt, st);
    else rt.template put<true>(s.X, L::LDX, src, ldt, rows, min(PT, a.P - p0), vt, st);
    if (half * NT + st < GATES) ((float*)&s.g)[half * NT + st] = rg;
  };
  // 16 columns q of a wave's quarter of a state or gradient: f4 [pb] holds rows p = 16 pb + g4 + j of column n
  auto columns = [&](f4(&v)[4], const float* from, int turn, int q) {
    const float* src = from + (slot * a.H * pts + (long)h0 * pts + turn) * (long)(PT * NP);
    const int lane = fresh_lane();
#pragma unroll
    for (int pb = 0; pb < 4; ++pb) v[pb] = *(const f4*)(src + ((pb * NB + w * NQ + q) * 64 + lane) * 4);
  };
  // dB or dC of the chunk: [n][token] accumulators, of a wave's 16 tokens over all n (written to global memory), and
  // of all tokens over its quarter of n (added through LDS)
  const long gn = (long)a.G * a.N;
  auto add = [&](const f4(&v)[NQ][4]) {
    const int lane = fresh_lane(), g4 = 4 * (lane >> 4), col = lane & 15;
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
      for (int b = 0; b < 4; ++b) *(f4*)(s.sum + (16 * b + col) * L::LDS_ + 16 * (w * NQ + q) + g4) = v[q][b];
  };
  auto write = [&](const f4(&v)[NB], void* whole, float* part) {
    const int lane = fresh_lane(), g4 = 4 * (lane >> 4), own = 16 * w + (lane & 15);
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

  // Every turn: the tile and its gates into LDS (and G), barrier, the products,
  // barrier, dx and the head's sums by waves 4 to 7, which read what they still
  // need of the tile before the second barrier.
  f4 acc[NB], accn[NQ][4];               // dC^T or dB^T [n][token]: of this wave's tokens, and over its quarter of n
#pragma unroll
  for (int b = 0; b < NB; ++b) acc[b] = zero4();
#pragma unroll
  for (int q = 0; q < NQ; ++q)
#pragma unroll
    for (int b = 0; b < 4; ++b) accn[q][b] = zero4();

  // The time steps' gradients and the sums of head h, a token a lane, by the
  // wave with the fewest products while the next head's are formed.
  auto finish = [&](int h) {
    const typename L::Sums& f = s.sums[(h - h0) & 1];
    const int lane = fresh_lane(), r = lane;
    const float A = a.A[h], step = f.dt[r];
    const float srow = (f.srow[0][r] + f.srow[1][r]) + (f.srow[2][r] + f.srow[3][r]);
    const float gcol = (f.gcol[0][r] + f.gcol[1][r]) + (f.gcol[2][r] + f.gcol[3][r]);
    float dl = ((f.sg[0] + f.sg[1]) + (f.sg[2] + f.sg[3])) * f.total;
    dl += lane_from(wave_incl_scan_dpp(lane_from(srow, 63 - lane)), 63 - lane);            // over r >= t
    dl += before_lane(step * gcol, lane) + f.fd[r];                                        // over i < t
#pragma unroll
    for (int b = 1; b < 4; ++b) {
      const float c = before_lane(r < 16 * b ? f.cs[b - 1][r] : 0.f, lane);
      dl += r < 16 * b ? c : 0.f;
    }
    float raw = f.mcol[r] + f.diag[r] + gcol + A * dl;
    const bool in = r < rows;
    if (a.softplus) raw *= -expm1f(-step);               // sigmoid of the raw step, from its softplus
    if (in) a.ddt[(t0 + r) * a.H + h] = raw;
    // in 64 bits: these sums cancel over the tokens (dA is 1% of its terms' absolute sum at 16384 tokens)
    const double sa = wave_incl_scan64(in ? (double)step * (double)dl : 0.0), sd = wave_incl_scan64(in ? (double)f.err[r] : 0.0),
                 sb = wave_incl_scan64(in ? (double)raw : 0.0);
    if (lane == 63) {
      double* out = a.sums + (slot * a.H + h) * 4;
      out[0] = sa;
      out[1] = sd;
      out[2] = sb;
    }
  };

  if (wave < 4) {
    f4 S[NQ][4], G[NQ][4], kr[4];
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      columns(S[q], a.states, 0, q);
      columns(G[q], a.grads, 0, q);
    }
    block_sync_lds();
    {
      const int lane = fresh_lane();
      // K of rows r = own: accumulator rows are i
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        kr[b] = zero4();
        if (b <= w)
#pragma unroll
          for (int k = 0; k < KN; ++k)
            kr[b] = mma(row_frag<E>(s.B, L::LDN, 16 * b, 32 * k, lane), row_frag<E>(s.Cm, L::LDN, 16 * w, 32 * k, lane), kr[b]);
      }
    }
    for (int turn = 0; turn < turns; ++turn) {
      const bool first = turn % pts == 0;
      const int next = min(turn + 1, turns - 1);      // the last turn loads itself again: no branch around the loads
      put(turn);
      block_sync_lds();
      const int lane = fresh_lane(), g4 = 4 * (lane >> 4), col = lane & 15, own = 16 * w + col;
      typename L::Sums& f = s.sums[turn / pts & 1];
      if (wave == 0) {
        f.dt[lane] = s.g.dt[lane];
        if (lane == 0) f.total = s.g.head[C - 1];
      }
      // <G, S>, then e^{b_r} S^T dy_r over this wave's quarter of n
      {
        float sg = 0.f;
#pragma unroll
        for (int q = 0; q < NQ; ++q)
#pragma unroll
          for (int pb = 0; pb < 4; ++pb)
#pragma unroll
            for (int j = 0; j < 4; ++j) sg += G[q][pb][j] * S[q][pb][j];
        sg = groups_sum(sum16(sg));
        if (lane == 0) f.sg[w] = (first ? 0.f : f.sg[w]) + sg;
        phase();
      }
      float sr[4] = {};
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        // every second 16 columns with the sign turned, so that the products' one-sided rounding cancels in sr
        const float sign = NQ > 1 ? (q & 1 ? -1.f : 1.f) : (w & 1 ? -1.f : 1.f);
        Planes<E, 3> sp[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) sp[k] = planes<E, 3>(sign * S[q][2 * k], sign * S[q][2 * k + 1]);
        phase();
        columns(S[q], a.states, next, q);
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          Fr<E> yf[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) yf[k] = row_frag<E>(s.dY, L::LDP, 16 * b, 32 * k, lane);
          const q4 c = *(const q4*)(s.Cm + (16 * b + col) * L::LDN + flip<E>(col, 16 * (w * NQ + q) + g4));
          const float er = s.g.head[16 * b + col];
          f4 u = zero4();
#pragma unroll
          for (int k = 0; k < 2; ++k) u = mma(sp[k], yf[k], u);
          u *= sign * er;
          accn[q][b] += u;
#pragma unroll
          for (int j = 0; j < 4; ++j) sr[b] += tof(c[j]) * u[j];
        }
        phase();
      }
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        sr[b] = groups_sum(sr[b]);
        if (g4 == 0) f.srow[w][16 * b + col] = (first ? 0.f : f.srow[w][16 * b + col]) + sr[b];
      }
      phase();
      fetch(next);
      // rows p = 16 w .. of G B^T for all tokens, to the waves that own them
      {
        f4 v[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) v[b] = zero4();
#pragma unroll
        for (int k = 0; k < KN; ++k) {
          Fr<E> gp[PL], bf[4];
#pragma unroll
          for (int pl = 0; pl < PL; ++pl) gp[pl] = col_frag<E>(s.G[pl], L::LDP, 32 * k, 16 * w, lane);
#pragma unroll
          for (int b = 0; b < 4; ++b) bf[b] = row_frag<E>(s.B, L::LDN, 16 * b, 32 * k, lane);
          phase();
#pragma unroll
          for (int pl = PL - 1; pl >= 0; --pl)
#pragma unroll
            for (int b = 0; b < 4; ++b) v[b] = mma(gp[pl], bf[b], v[b]);
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const int i = 16 * b + col;
          *(f4*)(s.dX + i * L::LDT + 16 * w + g4) = v[b] * s.g.tail[i];
        }
      }
      phase();
      // W E diag(dt) of rows r = own: accumulator rows are i
      f4 md = zero4();
      float before = 0.f;                // sum of M_ri over the blocks i < 16 w
      Fr<E> yf[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) yf[k] = row_frag<E>(s.dY, L::LDP, 16 * w, 32 * k, lane);
      const float h16 = s.g.head16[own];
#pragma unroll
      for (int pair = 0; pair < 2; ++pair) {
        if (2 * pair > w) break;
        f4 e[2];
#pragma unroll
        for (int b2 = 0; b2 < 2; ++b2) {
          const int b = 2 * pair + b2;
          e[b2] = zero4();
          if (b > w) continue;
          Fr<E> xf[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) xf[k] = step_frag<E>(s.X, L::LDX, 16 * b, 32 * k, lane);
          f4 wt;
          if (b < w) {
            wt = (h16 * between<E>(s.g, w, b)) * *(const f4*)(s.g.tail16 + 16 * b + g4);
          } else {
            const f4 hi = *(const f4*)(s.g.bh + 16 * b + g4), li = *(const f4*)(s.g.bl + 16 * b + g4);
            const float hr = s.g.bh[own], lr = s.g.bl[own];
#pragma unroll
            for (int j = 0; j < 4; ++j) wt[j] = g4 + j <= col ? decay<E>(hr, lr, hi[j], li[j]) : 0.f;
          }
          wt *= *(const f4*)(s.g.dt + 16 * b + g4);
#pragma unroll
          for (int k = 0; k < 2; ++k) e[b2] = mma(xf[k], yf[k], e[b2]);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int i = 16 * b + g4 + j;
            e[b2][j] = b < w || i <= own ? e[b2][j] * wt[j] : 0.f;
            const float m = b < w || i < own ? e[b2][j] * kr[b][j] : 0.f;
            if (b == w) {
              md[j] = m;
            } else {
              before += m;
              const float c = sum16(m);
              if (col == 0) f.cs[w - 1][i] = (first ? 0.f : f.cs[w - 1][i]) + c;
            }
          }
        }
        const Planes<E, 3> ep = planes<E, 3>(e[0], e[1]);
#pragma unroll
        for (int b4 = 0; b4 < NB; b4 += 4) {
          Fr<E> bt[4];
#pragma unroll
          for (int b = 0; b < 4; ++b) bt[b] = col_frag<E>(s.B, L::LDN, 32 * pair, 16 * (b4 + b), lane);
          phase();
#pragma unroll
          for (int pl = Planes<E, 3>::N - 1; pl >= 0; --pl)
#pragma unroll
            for (int b = 0; b < 4; ++b) acc[b4 + b] = mma(bt[b], ep.p[pl], acc[b4 + b]);
        }
        phase();
      }
      // sum over r >= t in this block and all i < t, t = own: (M V)_rt with V_it = [i < t] as a product, the blocks
      // before as one more column, then the rows r >= t
      before = groups_sum(before);
      f4 v = __builtin_amdgcn_mfma_f32_16x16x4f32(g4 == 0 ? before : 0.f, 1.f, zero4(), 0, 0, 0);
#pragma unroll
      for (int j = 0; j < 4; ++j) v = __builtin_amdgcn_mfma_f32_16x16x4f32(md[j], g4 + j < col ? 1.f : 0.f, v, 0, 0, 0);
      float m = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) m += g4 + j >= col ? v[j] : 0.f;
      m = groups_sum(m);
      if (g4 == 0) f.fd[own] = (first ? 0.f : f.fd[own]) + m;
      phase();
#pragma unroll
      for (int q = 0; q < NQ; ++q) columns(G[q], a.grads, next, q);
      if (wave == 0 && first && turn > 0) finish(h0 + turn / pts - 1);
      block_sync_lds();
    }
    if (wave == 0) finish(h1 - 1);
    add(accn);
    block_sync_lds();
    write(acc, a.dC, a.partC);
    block_sync_lds();
    block_sync_lds();
    return;
  }

  f4 G[NQ][4], kc[4];
#pragma unroll
  for (int q = 0; q < NQ; ++q) columns(G[q], a.grads, 0, q);
  block_sync_lds();
  {
    const int lane = fresh_lane();
    // K of columns i = own: accumulator rows are r
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      kc[b] = zero4();
      if (b >= w)
#pragma unroll
        for (int k = 0; k < KN; ++k)
          kc[b] = mma(row_frag<E>(s.Cm, L::LDN, 16 * b, 32 * k, lane), row_frag<E>(s.B, L::LDN, 16 * w, 32 * k, lane), kc[b]);
    }
  }
  for (int turn = 0; turn < turns; ++turn) {
    const bool first = turn % pts == 0;
    const int next = min(turn + 1, turns - 1);      // the last turn loads itself again: no branch around the loads
    const int h = h0 + turn / pts, pt = turn % pts;
    put(turn);
    const int lane = fresh_lane(), g4 = 4 * (lane >> 4), col = lane & 15, own = 16 * w + col;
    typename L::Sums& f = s.sums[turn / pts & 1];
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const int nn = 16 * (w * NQ + q) + col;
#pragma unroll
      for (int pb = 0; pb < 4; ++pb) put_planes<E, PL>(s.G[0] + nn * L::LDP + flip<E>(nn, 16 * pb + g4), NP * L::LDP, G[q][pb]);
    }
    block_sync_lds();
    // e^{b_C - b_i} G^T x_i over this wave's quarter of n
    float gc[4] = {};
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      // as above, for gc
      const float sign = NQ > 1 ? (q & 1 ? -1.f : 1.f) : (w & 1 ? -1.f : 1.f);
      Planes<E, 3> gp[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) gp[k] = planes<E, 3>(sign * G[q][2 * k], sign * G[q][2 * k + 1]);
      phase();
      columns(G[q], a.grads, next, q);
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        Fr<E> xf[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) xf[k] = step_frag<E>(s.X, L::LDX, 16 * b, 32 * k, lane);
        const q4 c = *(const q4*)(s.B + (16 * b + col) * L::LDN + flip<E>(col, 16 * (w * NQ + q) + g4));
        const float ei = s.g.tail[16 * b + col], dt = s.g.dt[16 * b + col];
        f4 u = zero4();
#pragma unroll
        for (int k = 0; k < 2; ++k) u = mma(gp[k], xf[k], u);
        u *= sign * ei;
        accn[q][b] += dt * u;
#pragma unroll
        for (int j = 0; j < 4; ++j) gc[b] += tof(c[j]) * u[j];
      }
      phase();
    }
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      gc[b] = groups_sum(gc[b]);
      if (g4 == 0) f.gcol[w][16 * b + col] = (first ? 0.f : f.gcol[w][16 * b + col]) + gc[b];
    }
    phase();
    fetch(next);
    // W E and W K of columns i = own: accumulator rows are r
    f4 xacc[4];
    float mcol = 0.f, diag = 0.f, err = 0.f;
    const float dt = s.g.dt[own], t16 = s.g.tail16[own];
    Fr<E> xf[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) xf[k] = step_frag<E>(s.X, L::LDX, 16 * w, 32 * k, lane);
#pragma unroll
    for (int b = 0; b < 4; ++b) xacc[b] = zero4();
#pragma unroll
    for (int pair = 0; pair < 2; ++pair) {
      if (2 * pair + 1 < w) continue;
      f4 e[2], wk[2];
#pragma unroll
      for (int b2 = 0; b2 < 2; ++b2) {
        const int b = 2 * pair + b2;
        e[b2] = wk[b2] = zero4();
        if (b < w) continue;
        Fr<E> yf[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) yf[k] = row_frag<E>(s.dY, L::LDP, 16 * b, 32 * k, lane);
        f4 wt;
        if (b > w) {
          wt = (t16 * between<E>(s.g, b, w)) * *(const f4*)(s.g.head16 + 16 * b + g4);
        } else {
          const f4 hr = *(const f4*)(s.g.bh + 16 * b + g4), lr = *(const f4*)(s.g.bl + 16 * b + g4);
          const float hi = s.g.bh[own], li = s.g.bl[own];
#pragma unroll
          for (int j = 0; j < 4; ++j) wt[j] = g4 + j >= col ? decay<E>(hr[j], lr[j], hi, li) : 0.f;
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) e[b2] = mma(yf[k], xf[k], e[b2]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int r = 16 * b + g4 + j;
          const bool in = b > w || r >= own;
          const float ev = in ? e[b2][j] : 0.f, we = ev * wt[j];
          if (b > w) {
            mcol += we * kc[b][j];
          } else {
            mcol += r > own ? we * kc[b][j] : 0.f;
            diag += r == own ? ev * kc[b][j] : 0.f;
            err += r == own ? ev : 0.f;
          }
          e[b2][j] = we * dt;
          wk[b2][j] = in ? wt[j] * kc[b][j] : 0.f;
        }
      }
      {
        const Planes<E, 3> wp = planes<E, 3>(wk[0], wk[1]);
        Fr<E> yt[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) yt[b] = col_frag<E>(s.dY, L::LDP, 32 * pair, 16 * b, lane);
        phase();
#pragma unroll
        for (int pl = Planes<E, 3>::N - 1; pl >= 0; --pl)
#pragma unroll
          for (int b = 0; b < 4; ++b) xacc[b] = mma(yt[b], wp.p[pl], xacc[b]);
      }
      const Planes<E, 3> ep = planes<E, 3>(e[0], e[1]);
#pragma unroll
      for (int b4 = 0; b4 < NB; b4 += 4) {
        Fr<E> ct[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) ct[b] = col_frag<E>(s.Cm, L::LDN, 32 * pair, 16 * (b4 + b), lane);
        phase();
#pragma unroll
        for (int pl = Planes<E, 3>::N - 1; pl >= 0; --pl)
#pragma unroll
          for (int b = 0; b < 4; ++b) acc[b4 + b] = mma(ct[b], ep.p[pl], acc[b4 + b]);
      }
      phase();
    }
    mcol = groups_sum(mcol);
    diag = groups_sum(diag);
    err = groups_sum(err);
    if (g4 == 0) {
      f.mcol[own] = (first ? 0.f : f.mcol[own]) + mcol;
      f.diag[own] = (first ? 0.f : f.diag[own]) + diag;
      f.err[own] = (first ? 0.f : f.err[own]) + err;
    }
    q4 dq[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) dq[b] = *(const q4*)(s.dY + own * L::LDP + flip<E>(col, 16 * b + g4));
    block_sync_lds();
    {
      const int cols = min(PT, a.P - pt * PT);
      const float D = a.D ? a.D[h] : 0.f;
      E* out = (E*)a.dx + t0 * ldy + (long)h * a.P + pt * PT;
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        xacc[b] = dt * (xacc[b] + *(const f4*)(s.dX + own * L::LDT + 16 * b + g4));
        if (a.D) xacc[b] += D * widen<E>(dq[b]);
      }
      if (__builtin_expect(quad_rows<E>(out, ldy, cols), 1)) {
        const __amdgpu_buffer_rsrc_t buf = buffer(uniform_ptr(out), (uint32_t)(rows * ldy) * (uint32_t)sizeof(E));
#pragma unroll
        for (int b = 0; b < 4; ++b)
          store_quad<E>(buf, 16 * b + g4 < cols ? (uint32_t)(own * ldy + 16 * b + g4) * (uint32_t)sizeof(E) : 0x80000000u, xacc[b]);
      } else {
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (own < rows && 16 * b + g4 + j < cols) out[own * ldy + 16 * b + g4 + j] = fromf<E>(xacc[b][j]);
      }
    }
  }
  block_sync_lds();
  block_sync_lds();
  add(accn);
  block_sync_lds();
  write(acc, a.dB, a.partB);
}

// dB and dC from the shares of the splits, in order.
template <typename E>
__global__ __launch_bounds__(NTHREADS) void k_ssm_join(ScanArgs a, long n) {
  const float* part = blockIdx.y ? a.partB : a.partC;
  E* out = (E*)(blockIdx.y ? a.dB : a.dC);
  long n_end = n;
  if (a.q.cu) n_end = min(n_end, (long)max(a.q.cu[a.q.N], 0) * a.G * a.N);   // rows from the last sequence's end on stay as they are
  for (long i = (long)blockIdx.x * NTHREADS + threadIdx.x; i < n_end; i += (long)gridDim.x * NTHREADS) {
    float v = part[i];
    for (int k = 1; k < a.splits; ++k) v += part[k * n + i];
    out[i] = fromf<E>(v);
  }
}

// dA, dD and the bias's gradient of a head: its chunks' sums, in a fixed order.
__global__ __launch_bounds__(NTHREADS) void k_ssm_heads(ScanArgs a, long slots) {
  __shared__ double red[3][NTHREADS];
  const int h = blockIdx.x, t = threadIdx.x;
  double v[3] = {};
  for (long k = t; k < slots; k += NTHREADS) {
    int n, len, pos;
    long s0;
    if (a.q.cu && !a.q.locate(k, C, n, s0, len, pos)) continue;
#pragma unroll
    for (int i = 0; i < 3; ++i) v[i] += a.sums[(k * a.H + h) * 4 + i];
  }
#pragma unroll
  for (int i = 0; i < 3; ++i) red[i][t] = v[i];
  __syncthreads();
#pragma unroll
  for (int off = NTHREADS / 2; off >= 1; off >>= 1) {
    if (t < off)
#pragma unroll
      for (int i = 0; i < 3; ++i) red[i][t] += red[i][t + off];
    __syncthreads();
  }
  if (t) return;
  a.dA[h] = (float)red[0][0];
  if (a.dD) a.dD[h] = (float)red[1][0];
  if (a.dbias) a.dbias[h] = (float)red[2][0];
}

template <typename E, int NP>
hipError_t chunks(const ScanArgs& a, hipStream_t st) {
  const long items = a.q.slots(C) * a.G * a.splits;
  if (items == 0) return hipSuccess;
  constexpr int V = 16 / (int)sizeof(E);
  const uintptr_t bases = (uintptr_t)a.x | (uintptr_t)a.dy | (uintptr_t)a.B | (uintptr_t)a.C;
  const long lds = a.ldx | a.ldb | a.ldc, far = (1L << 24) / (int)sizeof(E), ldy = (long)a.H * a.P;
  const bool whole = (bases & 15) == 0 && lds % V == 0 && a.P % V == 0 && a.N % V == 0 && a.ldx < far && a.ldb < far &&
                     a.ldc < far && ldy < far;
  if (whole) hipLaunchKernelGGL((k_ssm_bwd<E, NP, true>), dim3(xcd_grid(items)), dim3(2 * NTHREADS), 0, st, a, items);
  else hipLaunchKernelGGL((k_ssm_bwd<E, NP, false>), dim3(xcd_grid(items)), dim3(2 * NTHREADS), 0, st, a, items);
  return hipGetLastError();
}

}  // namespace

// Workgroups that share the heads of a chunk: as many as give every CU one, and
// no more than the largest share needs (1 x 4096 tokens of 64 heads, training
// step with 1, 2, 4, 8 and 16: 718, 494, 399, 413, 450 us; the rule takes 4).
int scan_splits(const Seqs& q, int H, int G) {
  const long units = q.slots(C) * G, cus = device_cu_count(), heads = H / G;
  if (units <= 0) return 1;
  const long s = (cus + units - 1) / units;
  if (s >= heads) return (int)heads;
  const long share = (heads + s - 1) / s;
  return (int)((heads + share - 1) / share);
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
