// Selective state space scan, forward: prompts (dense or packed) and single tokens.
//
//   dt = softplus(raw + bias) or raw;  S_t = exp(dt A) S_{t-1} + dt x_t B_t^T;  y_t = S_t C_t + D x_t
//
// per head, S [P][N]; B and C are shared by the H / G heads of a group.  Per
// chunk of 64 tokens with entry state S, b the prefix sums of dt A,
// W_ri = exp(b_r - b_i) for i <= r:
//
//   Y  = diag(e^b) C S^T + (W o C B^T) diag(dt) X + D X
//   S' = e^{b_C} S + sum_i e^{b_C - b_i} dt_i x_i B_i^T
//
// A workgroup walks the chunks of one (sequence, head, 64 rows of the state)
// with the state in registers: wave w owns 16 of the rows, as accumulators
// [n][p], which are operands of the products with C as they stand.  C B^T is
// formed by rows (wave w: tokens 16 w .. of the chunk) and goes to the other
// waves through LDS.
//
// Few sequences and heads leave most of the chip idle in such a walk.  Then it
// is cut into segments: a walk without outputs forms each segment's own
// contribution, these are put together along the sequence, and the walk with
// outputs starts every segment from its entry.
#include "qd_ssm.h"

namespace qd {

namespace {

// Gates of a chunk slot's 16 heads a workgroup: the raw steps are read along
// the heads, transposed in LDS, then a token is a lane.
// 16384 tokens of 64 heads: 13 us, 29 MB written.
__global__ __launch_bounds__(NTHREADS) void k_ssm_gates(ScanArgs a) {
  __shared__ float raw[16][C + 1];
  const int hb = (a.H + 15) / 16, h0 = (int)(blockIdx.x % hb) * 16, t = threadIdx.x, lane = t & 63, w = wave_id(t);
  const long slot = blockIdx.x / hb;
  int n, len, pos;
  long s0;
  if (!a.q.locate(slot, C, n, s0, len, pos)) return;
  const int rows = min(C, len - pos), heads = min(16, a.H - h0);
  for (int i = t; i < 16 * C; i += NTHREADS) {
    const int r = i >> 4, h = i & 15;
    if (r < rows && h < heads) raw[h][r] = a.dt[(s0 + pos + r) * a.H + h0 + h];
  }
  __syncthreads();
  for (int k = w; k < heads; k += NWAVES) {
    const int h = h0 + k;
    const float dt = lane < rows ? step_size(raw[k][lane] + (a.bias ? a.bias[h] : 0.f), a.softplus) : 0.f;
    const double b = wave_incl_scan64((double)dt * (double)a.A[h]);
    float* g = a.gates + (slot * a.H + h) * GATES + lane;
    g[0] = dt;
    g[C] = (float)b;
    g[2 * C] = (float)(b - (double)(float)b);
    // each from a difference formed in 64 bits
    const double before = __shfl(b, max(lane & ~15, 1) - 1, 64);
    g[3 * C] = exp_of64(b);
    g[4 * C] = exp_of64(__shfl(b, C - 1, 64) - b);
    g[5 * C] = exp_of64(lane < 16 ? b : b - before);
    g[6 * C] = exp_of64(__shfl(b, lane | 15, 64) - b);
  }
}

// Whether any of a piece's values is infinite or NaN: all ones in the exponent.
template <typename E>
__device__ inline bool not_finite(u32x4 v) {
  constexpr uint32_t exps = sizeof(E) == 2 ? 0x7f807f80u : 0x7f800000u, one = sizeof(E) == 2 ? 0x00800080u : 0x00800000u;
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) any |= (v[i] & exps) + one;
  return (any & (sizeof(E) == 2 ? 0x80008000u : 0x80000000u)) != 0;
}

// Operands of a chunk in LDS; rows and columns outside the matrices are zeros.
template <typename E, int NP>
struct OutLds {
  static constexpr int LDN = lds_ld<E>(NP), LDP = lds_ld<E>(PT), LDM = steps_ld<E>(NP), LDC = steps_ld<E>(C),
                       PL = Planes<E, 3>::N;
  struct Buf {
    E B[C * LDN], X[C * LDP];
    E Cm[C * LDM];                     // steps
    E W[PL][C * LDC];                  // W o C B^T diag(dt), [r][i], planes; steps
    Gates g;
  };
  static constexpr int NBUF = 2 * sizeof(Buf) + 64 <= 163840 ? 2 : 1;
  Buf buf[NBUF];
  int bad[2];                          // chunk + 1 whose x has an infinity or a NaN
};

// Waves 4 to 7 produce: they load the next chunk's operands into LDS and form
// its W o C B^T diag(dt) (wave 4 + w: tokens 16 w .. of it), which needs no
// state; waves 0 to 3 consume: outputs, then the state.  Per chunk two
// barriers, after the operands are in LDS and at the end.  fp32 with N > 64
// has room for one chunk in LDS only: there the two halves take turns.
//
// 4 x 4096 tokens, 64 heads, state 64 x 128, bf16: 261 us, one walk a CU, 4.1 us
// a chunk (270 MB, 1.0 TB/s; 65536 tokens, 16 heads, 128 x 128: 513 us).  The
// chain of a chunk bounds it: two barriers, vector instructions 38% of the
// cycles (planes of the state and of the weighted x), matrix products 21%.
// Producers and consumers on the same SIMDs fill each other's waits; all eight
// waves doing both took 350 us where this form took 236 (two planes a product).
template <typename E, int NP>
__global__ __launch_bounds__(2 * NTHREADS, 1) QD_TWO_WAVES void k_ssm_out(ScanArgs a, long items) {
  typedef OutLds<E, NP> L;
  typedef typename Q4<E>::t q4;
  __shared__ __attribute__((aligned(16))) L s;
  constexpr int NB = NP / 16, KN = NP / 32, PL = L::PL, NBUF = L::NBUF;
  long item;
  if (!xcd_item(items, item)) return;
  const int pts = p_tiles(a.P), hp = (int)(item % (a.H * pts)), h = hp / pts, p0 = hp % pts * PT;
  const long slot = item / (a.H * pts);
  int n, len, pos;
  long s0;
  const bool whole = a.seg == 0;       // one walk a sequence, empty ones included: they hand their state on
  if (whole) {
    n = (int)slot;
    pos = 0;
    if (!a.q.range(n, s0, len)) return;
  } else if (!a.q.locate(slot, a.seg, n, s0, len, pos)) {
    return;
  }
  const int end = whole ? len : min(pos + a.seg, len), chunks = (end - pos + C - 1) / C;
  const int t_ = threadIdx.x & (NTHREADS - 1), t = t_, wave = wave_id(threadIdx.x), w = wave & 3;
  const int cols = min(PT, a.P - p0), grp = h / (a.H / a.G);

  if (wave >= 4) {
    const E* x = (const E*)a.x + (s0 + pos) * a.ldx + (long)h * a.P + p0;
    const E* B = (const E*)a.B + (s0 + pos) * a.ldb + (long)grp * a.N;
    const E* Cm = (const E*)a.C + (s0 + pos) * a.ldc + (long)grp * a.N;
    const bool vx = vec_rows<E>(x, a.ldx, cols), vb = vec_rows<E>(B, a.ldb, a.N), vc = vec_rows<E>(Cm, a.ldc, a.N);
    const long cslot = (a.q.cu ? s0 / C + n : (long)n * ((a.q.T + C - 1) / C)) + pos / C;
    Stage<E, PT, NTHREADS> rx;
    Stage<E, NP, NTHREADS> rb, rc;
    float rg[2];
    const uint32_t ox = rx.offset(a.ldx, cols, t), ob = rb.offset(a.ldb, a.N, t), oc = rc.offset(a.ldc, a.N, t);
    auto fetch = [&](int c) {
      const int rows = min(C, end - pos - c * C);
      rx.load(x + (long)c * C * a.ldx, a.ldx, rows, vx, ox);
      rb.load(B + (long)c * C * a.ldb, a.ldb, rows, vb, ob);
      rc.load(Cm + (long)c * C * a.ldc, a.ldc, rows, vc, oc);
      rg[0] = load_gate(a.gates + ((cslot + c) * a.H + h) * GATES, t);
      rg[1] = load_gate(a.gates + ((cslot + c) * a.H + h) * GATES, NTHREADS + t);
    };
    auto put = [&](int c) {
      typename L::Buf& u = s.buf[c % NBUF];
      const int t = w * 64 + fresh_lane(), rows = min(C, end - pos - c * C);
      rx.put(u.X, L::LDP, x + (long)c * C * a.ldx, a.ldx, rows, cols, vx, t);
      rb.put(u.B, L::LDN, B + (long)c * C * a.ldb, a.ldb, rows, a.N, vb, t);
      rc.template put<true>(u.Cm, L::LDM, Cm + (long)c * C * a.ldc, a.ldc, rows, a.N, vc, t);
      ((float*)&u.g)[t] = rg[0];
      if (t < GATES - NTHREADS) ((float*)&u.g)[NTHREADS + t] = rg[1];
      bool bad = !vx;                    // not looked at: the consumers do
#pragma unroll
      for (int k = 0; k < rx.K; ++k) bad |= not_finite<E>(rx.r[k]);
      if (bad) s.bad[c & 1] = c + 1;
    };
    // rows r = 16 w + col, formed as their transposes: accumulator rows are i
    auto scores = [&](int c) {
      typename L::Buf& u = s.buf[c % NBUF];
      const int lane = fresh_lane(), g4 = 4 * (lane >> 4), col = lane & 15;
      Fr<E> cf[KN];
#pragma unroll
      for (int k = 0; k < KN; ++k) cf[k] = step_frag<E>(u.Cm, L::LDM, 16 * w, 32 * k, lane);
      const int r = 16 * w + col;
      const float hr = u.g.bh[r], lr = u.g.bl[r];
#pragma unroll
      for (int pair = 0; pair < 2; ++pair) {       // products take blocks of i in pairs
        if (2 * pair > w) break;
        Fr<E> bf[2][KN];
        f4 hi[2], li[2], dt[2], v[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const int i0 = 32 * pair + 16 * b;
#pragma unroll
          for (int k = 0; k < KN; ++k) bf[b][k] = row_frag<E>(u.B, L::LDN, i0, 32 * k, lane);
          hi[b] = *(const f4*)(u.g.bh + i0 + g4);
          li[b] = *(const f4*)(u.g.bl + i0 + g4);
          dt[b] = *(const f4*)(u.g.dt + i0 + g4);
          v[b] = zero4();
        }
        phase();
#pragma unroll
        for (int k = 0; k < KN; ++k)
#pragma unroll
          for (int b = 0; b < 2; ++b) v[b] = mma(bf[b][k], cf[k], v[b]);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const int i0 = 32 * pair + 16 * b;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            v[b][j] = i0 + g4 + j <= r ? v[b][j] * (decay<E>(hr, lr, hi[b][j], li[b][j]) * dt[b][j]) : 0.f;
          put_planes<E, PL>(u.W[0] + r * L::LDC + step_at<E>(i0 + g4), C * L::LDC, v[b]);
        }
      }
    };
    if (t < 2) s.bad[t] = 0;
    if (chunks > 0) fetch(0);
    block_sync_lds();
    if (chunks > 0) put(0);
    if (chunks > 1) fetch(1);
    block_sync_lds();
    if (chunks > 0) scores(0);
    block_sync_lds();
    for (int c = 0; c < chunks; ++c) {
      if (NBUF == 1) block_sync_lds();    // the consumers have read this chunk
      const bool more = c + 1 < chunks;
      if (more) put(c + 1);
      block_sync_lds();
      if (c + 2 < chunks) fetch(c + 2);
      if (more) scores(c + 1);
      block_sync_lds();
    }
    return;
  }

  const long ldy = (long)a.H * a.P;
  E* y = (E*)a.y + ((s0 + pos) * a.H + h) * (long)a.P + p0;
  const bool vy = quad_rows<E>(y, ldy, cols);
  const float D = a.D ? a.D[h] : 0.f;
  // state: f4 S[nb] holds n = 16 nb + g4 + j of row p = p0 + 16 w + col
  const int p = p0 + 16 * w + (t & 15), g4_ = 4 * ((t & 63) >> 4);
  const float* in = whole ? (a.S0 ? a.S0 + ((long)n * a.H + h) * a.P * a.N : nullptr)
                          : a.entry[0] + (slot * a.H + h) * (long)a.P * a.N;
  f4 S[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int nn = 16 * nb + g4_ + j;
      S[nb][j] = in && p < a.P && nn < a.N ? in[(long)p * a.N + nn] : 0.f;
    }
  block_sync_lds();
  block_sync_lds();
  block_sync_lds();
  // operands with C, read a chunk ahead where there is room
  constexpr bool AHEAD = NBUF == 2 && sizeof(E) == 2;
  Fr<E> cf[AHEAD ? KN : 1][4];
  auto read_c = [&](int c, int lane) {
#pragma unroll
    for (int k = 0; k < KN; ++k)
#pragma unroll
      for (int b = 0; b < 4; ++b) cf[AHEAD ? k : 0][b] = step_frag<E>(s.buf[c % NBUF].Cm, L::LDM, 16 * b, 32 * k, lane);
  };
  if (AHEAD && chunks > 0) read_c(0, t & 63);
  for (int c = 0; c < chunks; ++c) {
    const typename L::Buf& u = s.buf[c % NBUF];
    const int rows = min(C, end - pos - c * C);
    const int lane = fresh_lane(), g4 = 4 * (lane >> 4), col = lane & 15;
    Fr<E> xt[2];                         // x^T: row p, k = i
#pragma unroll
    for (int k = 0; k < 2; ++k) xt[k] = col_frag<E>(u.X, L::LDP, 32 * k, 16 * w, lane);
    // An infinity or a NaN in x must not meet the zero weights of the tokens
    // before it: it is taken out, and what it enters becomes NaN.
    int first = C;                       // token of row p's first one
    if (__builtin_expect(s.bad[c & 1] == c + 1, 0)) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        f4 v[2];
        quads<E>(xt[k], v[0], v[1]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const bool fine = fabsf(v[i / 4][i % 4]) < __builtin_inff();
          if (!fine) {
            first = min(first, 32 * k + 16 * (i / 4) + g4 + i % 4);
            v[i / 4][i % 4] = 0.f;
          }
        }
        xt[k] = planes<E, 1>(v[0], v[1]).p[0];
      }
      first = min(first, __shfl_xor(first, 16, 64));
      first = min(first, __shfl_xor(first, 32, 64));
    }
    // Y^T: rows p, columns r
    f4 o[4];
    float er[4];
    Fr<E> wf[2][4][PL];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int b = 2 * k; b < 4; ++b)
#pragma unroll
        for (int pl = 0; pl < PL; ++pl) wf[k][b][pl] = step_frag<E>(u.W[pl], L::LDC, 16 * b, 32 * k, lane);
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      o[b] = zero4();
      er[b] = u.g.head[16 * b + col];
    }
    q4 xd[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) xd[b] = *(const q4*)(u.X + (16 * b + col) * L::LDP + flip<E>(col, 16 * w + g4));
    phase();
#pragma unroll
    for (int k = 0; k < KN; ++k) {
      if (!AHEAD) {
#pragma unroll
        for (int b = 0; b < 4; ++b) cf[0][b] = step_frag<E>(u.Cm, L::LDM, 16 * b, 32 * k, lane);
        phase();
      }
      const Planes<E, 3> sp = planes<E, 3>(S[2 * k], S[2 * k + 1]);
#pragma unroll
      for (int pl = Planes<E, 3>::N - 1; pl >= 0; --pl)
#pragma unroll
        for (int b = 0; b < 4; ++b) o[b] = mma(sp.p[pl], cf[AHEAD ? k : 0][b], o[b]);
    }
#pragma unroll
    for (int b = 0; b < 4; ++b) o[b] *= er[b];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int pl = PL - 1; pl >= 0; --pl)
#pragma unroll
        for (int b = 2 * k; b < 4; ++b) o[b] = mma(xt[k], wf[k][b][pl], o[b]);
    phase();
    if (NBUF == 2) block_sync_lds();
    // operands of the state's update, in flight over the outputs
    Fr<E> bt[2][NB];
    auto read_b = [&](int k) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) bt[k][nb] = col_frag<E>(u.B, L::LDN, 32 * k, 16 * nb, lane);
    };
    read_b(0);
    if (sizeof(E) == 2) read_b(1);
    f4 ws[2][2];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        ws[k][i] = *(const f4*)(u.g.dt + 32 * k + 16 * i + g4) * *(const f4*)(u.g.tail + 32 * k + 16 * i + g4);
    const float total = u.g.head[C - 1];
    phase();
    if (a.D)
#pragma unroll
      for (int b = 0; b < 4; ++b) o[b] += D * widen<E>(xd[b]);
    if (__builtin_expect(s.bad[c & 1] == c + 1, 0))
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (16 * b + col >= __shfl(first, g4 + j, 64)) o[b][j] = __builtin_nanf("");
    {
      const int pc = 16 * w + g4;
      E* out = y + (long)c * C * ldy;
      if (__builtin_expect(vy, 1)) {
        const __amdgpu_buffer_rsrc_t buf = buffer(uniform_ptr(out), (uint32_t)(rows * ldy) * (uint32_t)sizeof(E));
        const uint32_t off = pc < cols ? (uint32_t)(col * ldy + pc) * (uint32_t)sizeof(E) : 0x80000000u;
#pragma unroll
        for (int b = 0; b < 4; ++b) store_quad<E>(buf, off + (uint32_t)(16 * b * ldy) * (uint32_t)sizeof(E), o[b]);
      } else {
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (16 * b + col < rows && pc + j < cols) out[(16 * b + col) * ldy + pc + j] = fromf<E>(o[b][j]);
      }
    }
    // S': rows n, columns p
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) S[nb] *= total;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (sizeof(E) != 2 && k) {
        read_b(1);
        phase();
      }
      f4 v[2];
      quads<E>(xt[k], v[0], v[1]);
      const Planes<E, 3> xw = planes<E, 3>(v[0] * ws[k][0], v[1] * ws[k][1]);
#pragma unroll
      for (int pl = Planes<E, 3>::N - 1; pl >= 0; --pl)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) S[nb] = mma(bt[k][nb], xw.p[pl], S[nb]);
    }
    if (AHEAD && c + 1 < chunks) read_c(c + 1, lane);
    if (first < C)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) S[nb] = zero4() + __builtin_nanf("");
    if (NBUF == 1) {
      block_sync_lds();
      block_sync_lds();
    }
    block_sync_lds();
  }
  if (whole && a.Sf && p < a.P) {
    float* out = a.Sf + (((long)n * a.H + h) * a.P + p) * a.N;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (16 * nb + g4_ + j < a.N) out[16 * nb + g4_ + j] = S[nb][j];
  }
}

// Walk of the state alone (dir 0: S, over x and B from the front), or of its
// gradient (dir 1: G = dL/dS, over dy and C from the back,
// G <- e^{b_C} G + sum_r e^{b_r} dy_r C_r^T), over a segment or a whole
// sequence.  Accumulators [p][n]: f4 S[nb] holds rows p = 16 w + g4 + j of
// column n = 16 nb + col, which is also the order in `states` and `grads`: a
// wave's stores are whole and the backward's loads are operands as they come.
// Both directions in one launch, 4 x 4096 tokens, 64 heads, state 64 x 128: 280
// us for 1.08 GB written and 0.37 read (5.1 TB/s): bound by HBM.
template <typename E, int NP>
struct WalkLds {
  static constexpr int LDN = lds_ld<E>(NP), LDP = lds_ld<E>(PT);
  E B[C * LDN], X[C * LDP];
  Gates g;
};

template <typename E, int NP>
__global__ __launch_bounds__(NTHREADS, 2) QD_TWO_WAVES void k_ssm_walk(ScanArgs a, long items, int dir0, int keep) {
  typedef WalkLds<E, NP> L;
  __shared__ __attribute__((aligned(16))) L s;
  constexpr int NB = NP / 16;
  long item;
  if (!xcd_item(items, item)) return;
  const int dir = dir0 + (int)blockIdx.y;
  const int pts = p_tiles(a.P), hp = (int)(item % (a.H * pts)), h = hp / pts, p0 = hp % pts * PT;
  const long slot = item / (a.H * pts);
  int n, len, pos;
  long s0;
  const bool whole = a.seg == 0;
  if (whole) {
    n = (int)slot;
    pos = 0;
    if (!a.q.range(n, s0, len)) return;
  } else if (!a.q.locate(slot, a.seg, n, s0, len, pos)) {
    return;
  }
  const int end = whole ? len : min(pos + a.seg, len);
  const int t = threadIdx.x, lane = t & 63, w = wave_id(t), g4 = 4 * (lane >> 4), col = lane & 15;
  const int cols = min(PT, a.P - p0), grp = h / (a.H / a.G);
  const long ldx = dir ? (long)a.H * a.P : a.ldx, ldb = dir ? a.ldc : a.ldb;
  const E* x = (const E*)(dir ? a.dy : a.x) + (s0 + pos) * ldx + (long)h * a.P + p0;
  const E* B = (const E*)(dir ? a.C : a.B) + (s0 + pos) * ldb + (long)grp * a.N;
  const bool vx = vec_rows<E>(x, ldx, cols), vb = vec_rows<E>(B, ldb, a.N);

  // Every second wave holds its rows with the sign turned.  The matrix
  // instructions' sums lean to one side by a fraction of a last place a step;
  // that would add up over the chunks and, as <G, S> sums every entry, over P x N
  // as well.  Rows of both signs cancel it (dA's error 1.0e-6 -> 1.0e-7 of its
  // largest entry, 4 x 4096 tokens, 64 heads, with the same in the backward).
  const float sign = w & 1 ? -1.f : 1.f;
  // Without `keep` this is a segment's own contribution, from zero; with it the
  // walk starts from the segment's entry, or the sequence's.
  const float* ends = dir ? a.dSf : a.S0;
  const float* in = whole ? (ends ? ends + ((long)n * a.H + h) * a.P * a.N : nullptr)
                          : keep ? a.entry[dir] + (slot * a.H + h) * (long)a.P * a.N : nullptr;
  f4 S[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int p = p0 + 16 * w + g4 + j, nn = 16 * nb + col;
      S[nb][j] = in && p < a.P && nn < a.N ? sign * in[(long)p * a.N + nn] : 0.f;
    }
  double run = 0.0;                      // sum of dt A over the segment
  const int chunks = (end - pos + C - 1) / C;
  const long cslot = (a.q.cu ? s0 / C + n : (long)n * ((a.q.T + C - 1) / C)) + pos / C;

  Stage<E, PT, NTHREADS> rx;
  Stage<E, NP, NTHREADS> rb;
  float rg[2];
  const uint32_t ox = rx.offset(ldx, cols, t), ob = rb.offset(ldb, a.N, t);
  auto fetch = [&](int c) {
    const int rows = min(C, end - pos - c * C);
    rx.load(x + (long)c * C * ldx, ldx, rows, vx, ox);
    rb.load(B + (long)c * C * ldb, ldb, rows, vb, ob);
    rg[0] = load_gate(a.gates + ((cslot + c) * a.H + h) * GATES, t);
    rg[1] = load_gate(a.gates + ((cslot + c) * a.H + h) * GATES, NTHREADS + t);
  };
  if (chunks > 0) fetch(dir ? chunks - 1 : 0);
  for (int k0 = 0; k0 < chunks; ++k0) {
    const int c = dir ? chunks - 1 - k0 : k0;
    if (keep) {
      float* out = (dir ? a.grads : a.states) + ((cslot + c) * a.H * pts + hp) * (long)(PT * NP);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) *(f4*)(out + ((w * NB + nb) * 64 + lane) * 4) = sign * S[nb];
    }
    {
      const int rows = min(C, end - pos - c * C);
      rx.put(s.X, L::LDP, x + (long)c * C * ldx, ldx, rows, cols, vx, t);
      rb.put(s.B, L::LDN, B + (long)c * C * ldb, ldb, rows, a.N, vb, t);
    }
    ((float*)&s.g)[t] = rg[0];
    if (t < GATES - NTHREADS) ((float*)&s.g)[NTHREADS + t] = rg[1];
    block_sync_lds();
    if (k0 + 1 < chunks) fetch(dir ? c - 1 : c + 1);
    const float total = s.g.head[C - 1];
    run += (double)s.g.bh[C - 1] + (double)s.g.bl[C - 1];
    Fr<E> xt[2], bt[2][NB];
    f4 ws[2][2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      xt[k] = col_frag<E>(s.X, L::LDP, 32 * k, 16 * w, lane);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int at = 32 * k + 16 * i + g4;
        ws[k][i] = (dir ? *(const f4*)(s.g.head + at) : *(const f4*)(s.g.dt + at) * *(const f4*)(s.g.tail + at)) * sign;
      }
    }
#pragma unroll
    for (int k = 0; k < (sizeof(E) == 2 ? 2 : 1); ++k)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) bt[k][nb] = col_frag<E>(s.B, L::LDN, 32 * k, 16 * nb, lane);
    phase();
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) S[nb] *= total;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      f4 v[2];
      quads<E>(xt[k], v[0], v[1]);
      const Planes<E, 3> xw = planes<E, 3>(v[0] * ws[k][0], v[1] * ws[k][1]);
      if (sizeof(E) != 2 && k) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) bt[k][nb] = col_frag<E>(s.B, L::LDN, 32 * k, 16 * nb, lane);
        phase();
      }
#pragma unroll
      for (int pl = Planes<E, 3>::N - 1; pl >= 0; --pl)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) S[nb] = mma(xw.p[pl], bt[k][nb], S[nb]);
    }
    block_sync_lds();
  }
  float* out = whole ? (dir ? a.dS0 : nullptr) : keep ? nullptr : a.total[dir];
  if (whole && out) out += ((long)n * a.H + h) * a.P * a.N;
  else if (out) out += (slot * a.H + h) * (long)a.P * a.N;
  if (out)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int p = p0 + 16 * w + g4 + j, nn = 16 * nb + col;
        if (p < a.P && nn < a.N) out[(long)p * a.N + nn] = sign * S[nb][j];
      }
  if (!whole && !keep && dir == dir0 && p0 == 0 && t == 0) a.decay[slot * a.H + h] = exp_of64(run);
}

// Entries of the segments of each sequence from their own contributions and
// decays, dir 0 from the front (S0, to Sf), dir 1 from the back (dSf, to dS0).
__global__ __launch_bounds__(NTHREADS) void k_ssm_compose(ScanArgs a, int dir0) {
  const int dir = dir0 + (int)blockIdx.z;
  const long per = (long)a.P * a.N, i = (long)blockIdx.x * NTHREADS + threadIdx.x;
  const int n = blockIdx.y / a.H, h = blockIdx.y % a.H;
  int len;
  long s0;
  if (i >= per || !a.q.range(n, s0, len)) return;
  const long base = a.q.cu ? s0 / a.seg + n : (long)n * ((a.q.T + a.seg - 1) / a.seg), at = ((long)n * a.H + h) * per + i;
  const int k = (len + a.seg - 1) / a.seg;
  const float* ends = dir ? a.dSf : a.S0;
  float S = ends ? ends[at] : 0.f;
  for (int j = 0; j < k; ++j) {
    const long slot = base + (dir ? k - 1 - j : j), u = slot * a.H + h;
    a.entry[dir][u * per + i] = S;
    S = a.decay[u] * S + a.total[dir][u * per + i];
  }
  float* out = dir ? a.dS0 : a.Sf;
  if (out) out[at] = S;
}

// One token of N sequences.  A wave owns rows of one head's state, R lanes a
// row with four consecutive n a lane and piece; the row's sum over n is formed
// by lane moves.  Bound by the state's bytes, read and written once: 64 sequences
// of 64 heads of 64 x 128 in 43 us (270 MB, 6.3 TB/s with the last level cache).
template <typename E>
__global__ __launch_bounds__(NTHREADS) void k_ssm_step(ScanArgs a) {
  constexpr int RPW = 4;                 // rows a wave handles at once: 16 lanes each
  const int per = (a.P + 4 * RPW - 1) / (4 * RPW);
  const long unit = blockIdx.x / per;    // (sequence, head)
  const int n = (int)(unit / a.H), h = (int)(unit % a.H), lane = threadIdx.x & 63, w = wave_id(threadIdx.x);
  const int p = (int)(blockIdx.x % per) * 4 * RPW + w * RPW + (lane >> 4), l = lane & 15;
  const int grp = h / (a.H / a.G);
  const float z = a.dt[unit] + (a.bias ? a.bias[h] : 0.f);
  const float dt = step_size(z, a.softplus), da = dt * a.A[h], al = exp_sum(da, fmaf(dt, a.A[h], -da));
  if (p >= a.P) return;
  const float x = tof(((const E*)a.x)[n * a.ldx + (long)h * a.P + p]), dx = dt * x;
  const E* B = (const E*)a.B + n * a.ldb + (long)grp * a.N;
  const E* Cm = (const E*)a.C + n * a.ldc + (long)grp * a.N;
  const float* in = a.S0 + (unit * a.P + p) * a.N;
  float* out = a.Sf + (unit * a.P + p) * a.N;
  float y = 0.f;
  if (a.N % 4 == 0 && (((uintptr_t)a.S0 | (uintptr_t)a.Sf) & 15) == 0) {
    for (int k = 4 * l; k < a.N; k += 64) {
      f4 S = *(const f4*)(in + k);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        S[j] = al * S[j] + dx * tof(B[k + j]);
        y += S[j] * tof(Cm[k + j]);
      }
      *(f4*)(out + k) = S;
    }
  } else {
    for (int k = l; k < a.N; k += 16) {
      const float S = al * in[k] + dx * tof(B[k]);
      y += S * tof(Cm[k]);
      out[k] = S;
    }
  }
  y = sum16(y);
  if (l == 0) ((E*)a.y)[unit * a.P + p] = fromf<E>(a.D ? y + a.D[h] * x : y);
}

long walk_slots(const ScanArgs& a) { return a.seg ? a.q.slots(a.seg) : a.q.N; }

template <typename E, int NP>
hipError_t out_walk(const ScanArgs& a, hipStream_t st) {
  const long items = walk_slots(a) * a.H * p_tiles(a.P);
  if (items == 0) return hipSuccess;
  hipLaunchKernelGGL((k_ssm_out<E, NP>), dim3(xcd_grid(items)), dim3(2 * NTHREADS), 0, st, a, items);
  return hipGetLastError();
}

template <typename E, int NP>
hipError_t walks(const ScanArgs& a, int dirs, bool chunks, hipStream_t st) {
  const long items = walk_slots(a) * a.H * p_tiles(a.P);
  if (items == 0) return hipSuccess;
  hipLaunchKernelGGL((k_ssm_walk<E, NP>), dim3(xcd_grid(items), dirs == 3 ? 2 : 1), dim3(NTHREADS), 0, st, a, items,
                     dirs == 2 ? 1 : 0, chunks ? 1 : 0);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_scan_walks(const ScanArgs& a, int dtype, int dirs, bool chunks, hipStream_t st) {
  if (dtype == 1) return a.N <= 64 ? walks<__bf16, 64>(a, dirs, chunks, st) : walks<__bf16, 128>(a, dirs, chunks, st);
  return a.N <= 64 ? walks<float, 64>(a, dirs, chunks, st) : walks<float, 128>(a, dirs, chunks, st);
}

hipError_t launch_scan_compose(const ScanArgs& a, int dirs, hipStream_t st) {
  const long per = (long)a.P * a.N;
  if (a.q.N == 0) return hipSuccess;
  hipLaunchKernelGGL(k_ssm_compose, dim3((unsigned)((per + NTHREADS - 1) / NTHREADS), (unsigned)(a.q.N * a.H), dirs == 3 ? 2 : 1),
                     dim3(NTHREADS), 0, st, a, dirs == 2 ? 1 : 0);
  return hipGetLastError();
}

// Walks are serial over their chunks, so a call of few heads is cut into
// segments until two of them run on every CU (16 heads of 128 x 128, bf16
// prompts, segments for one, two and four a CU: 65536 tokens 685, 638, 653 us,
// 16384 tokens 181, 176, 197; uncut 3754 and 890).  A segment costs a second
// walk without outputs and its state, so it has eight chunks at least in bf16
// (4096 tokens, four and eight chunks: 77 and 70 us) and two in fp32, where a
// chunk takes longer (3001 packed tokens of 8 heads of 64 x 64, forward and
// backward, two, four and eight: 116, 139 and 168 us).
int scan_segment(const Seqs& q, int H, int P, int dirs, bool f32) {
  const long tokens = q.cu ? q.T : (long)q.N * q.T, want = 2L * device_cu_count();
  const long units = (long)q.N * H * p_tiles(P) * dirs;
  if (units <= 0 || units >= want / 2) return 0;
  const long slots = want / ((long)H * p_tiles(P) * dirs);       // segments to have in all
  long chunks = (tokens / (slots > 0 ? slots : 1) + C - 1) / C;
  const long least = f32 ? 2 : 8;
  if (chunks < least) chunks = least;
  return q.T <= chunks * C ? 0 : (int)(chunks * C);
}

hipError_t launch_scan_gates(const ScanArgs& a, hipStream_t st) {
  const long blocks = a.q.slots(C) * ((a.H + 15) / 16);
  if (blocks == 0) return hipSuccess;
  hipLaunchKernelGGL(k_ssm_gates, dim3((unsigned)blocks), dim3(NTHREADS), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_scan_fwd(const ScanArgs& a, int dtype, hipStream_t st) {
  hipError_t e = launch_scan_gates(a, st);
  if (e != hipSuccess) return e;
  if (a.seg) {
    e = launch_scan_walks(a, dtype, 1, false, st);
    if (e == hipSuccess) e = launch_scan_compose(a, 1, st);
    if (e != hipSuccess) return e;
  }
  if (dtype == 1) return a.N <= 64 ? out_walk<__bf16, 64>(a, st) : out_walk<__bf16, 128>(a, st);
  return a.N <= 64 ? out_walk<float, 64>(a, st) : out_walk<float, 128>(a, st);
}

hipError_t launch_scan_step(const ScanArgs& a, int dtype, hipStream_t st) {
  const long blocks = (long)a.q.N * a.H * ((a.P + 15) / 16);
  if (blocks == 0) return hipSuccess;
  if (dtype == 1) hipLaunchKernelGGL((k_ssm_step<__bf16>), dim3((unsigned)blocks), dim3(NTHREADS), 0, st, a);
  else hipLaunchKernelGGL((k_ssm_step<float>), dim3((unsigned)blocks), dim3(NTHREADS), 0, st, a);
  return hipGetLastError();
}

}  // namespace qd
