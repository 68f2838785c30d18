// C ABI of the operators around the recurrence (declared in
// include/qdelta_mixer.h): argument validation, workspace layout, launches.
#include <stddef.h>
#include <stdint.h>

#include "qd_ssm.h"
#include "qdelta_mixer.h"

namespace {

// A pointer to elements of `size` bytes: required, or optional.
bool ok_ptr(const void* p, int size) { return p != nullptr && (reinterpret_cast<uintptr_t>(p) & (size - 1)) == 0; }
bool ok_opt(const void* p, int size) { return p == nullptr || ok_ptr(p, size); }

int elem_size(int32_t dtype) { return dtype == QDELTA_BF16 ? 2 : 4; }
int status(hipError_t e) { return e == hipSuccess ? QDELTA_OK : QDELTA_EHIP; }

// Tokens of a sequence (of the whole call where packed).  Positions are counted in
// 32 bits, and a tile of the convolution (64 tokens at most) that starts before
// token T ends before T + 64.  (The scan's launches end at 2^29 tokens.)
constexpr int64_t kMaxLength = (int64_t(1) << 31) - 64;

int check_seqs(int32_t N, int32_t T, const int32_t* cu, qd::Seqs& q) {
  if (N < 0 || T < 0 || !ok_opt(cu, 4)) return QDELTA_EINVAL;
  if (cu && N == 0 && T > 0) return QDELTA_EINVAL;
  q.N = N;
  q.T = T;
  q.cu = cu;
  // row numbers stay within 32 bits
  if (T > kMaxLength) return QDELTA_EUNSUPPORTED;
  if ((cu ? (int64_t)T : (int64_t)N * T) >= (int64_t(1) << 31)) return QDELTA_EUNSUPPORTED;
  return QDELTA_OK;
}

int64_t n_tokens(const qd::Seqs& q) { return q.cu ? (int64_t)q.T : (int64_t)q.N * q.T; }

// A launch has less than 2^32 threads.
constexpr int64_t kMaxThreads = int64_t(1) << 32;

int check_conv(const qd::Seqs& q, int32_t D, int32_t W, int32_t dtype, int64_t ldx) {
  if (D <= 0 || W <= 0 || ldx < D) return QDELTA_EINVAL;
  if (dtype != QDELTA_F32 && dtype != QDELTA_BF16) return QDELTA_EINVAL;
  if (W < 2 || W > 4) return QDELTA_EUNSUPPORTED;
  if ((int64_t)D * W >= (int64_t(1) << 31)) return QDELTA_EUNSUPPORTED;   // the taps are counted in 32 bits
  // threads of the forward and the step in single channels; tiles shorter than
  // 64 tokens are taken up to 2^17 threads of tiles of 64
  if ((q.slots(64) + 3 * (int64_t)q.N) * D + (int64_t(1) << 20) >= kMaxThreads) return QDELTA_EUNSUPPORTED;
  return QDELTA_OK;
}

int check_norm(int64_t rows, int32_t D, int32_t dtype, int64_t ldx, const void* gate, int64_t ldg) {
  if (rows < 0 || D <= 0 || ldx < D || (gate && ldg < D)) return QDELTA_EINVAL;
  if (dtype != QDELTA_F32 && dtype != QDELTA_BF16) return QDELTA_EINVAL;
  if (D > 8192 || rows >= (int64_t(1) << 31)) return QDELTA_EUNSUPPORTED;
  return QDELTA_OK;
}

int check_scan(const qd::Seqs& q, int32_t H, int32_t G, int32_t P, int32_t Ns, int32_t dtype, int64_t ldx, int64_t ldb,
               int64_t ldc) {
  if (H <= 0 || G <= 0 || P <= 0 || Ns <= 0 || H % G != 0) return QDELTA_EINVAL;
  if (dtype != QDELTA_F32 && dtype != QDELTA_BF16) return QDELTA_EINVAL;
  if (P > 256 || Ns > 128) return QDELTA_EUNSUPPORTED;
  if (ldx < (int64_t)H * P || ldb < (int64_t)G * Ns || ldc < (int64_t)G * Ns) return QDELTA_EINVAL;
  // (token, head) numbers stay within 32 bits, and launches of 512 threads a
  // walk or (chunk, group) and of 256 for 16 heads of a chunk within theirs
  if ((n_tokens(q) + 64 * (int64_t)q.N) * H >= (int64_t(1) << 31)) return QDELTA_EUNSUPPORTED;
  const int64_t walks = (int64_t)(q.N > 0 ? q.N : 1) * H * qd::p_tiles(P), chunks = q.slots(qd::C);
  if ((walks + 8) * 512 >= kMaxThreads || (chunks * G + 8) * 512 >= kMaxThreads || chunks * ((H + 15) / 16) * 256 >= kMaxThreads)
    return QDELTA_EUNSUPPORTED;
  return QDELTA_OK;
}

// Workspace of a scan: the chunks' gates; segments (contributions and entries a direction, and
// decays), and for the backward the chunks' states and gradients, the heads'
// sums and the splits' shares of dB and dC.
struct ScanWs {
  int seg = 0, splits = 1;
  size_t entry[2] = {0, 0}, total[2] = {0, 0}, decay = 0, states = 0, grads = 0, partB = 0, partC = 0, sums = 0, gates = 0, bytes = 0;
};
ScanWs scan_ws(const qd::Seqs& q, int H, int G, int P, int Ns, bool bwd, bool f32) {
  ScanWs w;
  auto take = [&](size_t n) {
    const size_t at = w.bytes;
    w.bytes += (n + 255) & ~size_t(255);
    return at;
  };
  w.gates = take((size_t)q.slots(qd::C) * H * qd::GATES * 4);
  w.seg = qd::scan_segment(q, H, P, bwd ? 2 : 1, f32);
  if (w.seg) {
    const size_t heads = (size_t)q.slots(w.seg) * H;
    for (int d = 0; d < (bwd ? 2 : 1); ++d) {
      w.entry[d] = take(heads * P * Ns * 4);
      w.total[d] = take(heads * P * Ns * 4);
    }
    w.decay = take(heads * 4);
  }
  if (bwd) {
    const size_t slots = (size_t)q.slots(qd::C), tile = (size_t)qd::PT * (Ns <= 64 ? 64 : 128) * 4;
    w.states = take(slots * H * qd::p_tiles(P) * tile);
    w.grads = take(slots * H * qd::p_tiles(P) * tile);
    w.sums = take(slots * H * 32);
    w.splits = qd::scan_splits(q, H, G);
    if (w.splits > 1) {
      w.partB = take((size_t)w.splits * n_tokens(q) * G * Ns * 4);
      w.partC = take((size_t)w.splits * n_tokens(q) * G * Ns * 4);
    }
  }
  return w;
}
void bind_ws(qd::ScanArgs& a, const ScanWs& w, void* ws) {
  char* p = static_cast<char*>(ws);
  auto at = [&](size_t off) { return reinterpret_cast<float*>(p + off); };
  a.seg = w.seg;
  a.splits = w.splits;
  for (int d = 0; d < 2; ++d) {
    a.entry[d] = at(w.entry[d]);
    a.total[d] = at(w.total[d]);
  }
  a.decay = at(w.decay);
  a.states = at(w.states);
  a.grads = at(w.grads);
  a.partB = at(w.partB);
  a.partC = at(w.partC);
  a.sums = reinterpret_cast<double*>(p + w.sums);
  a.gates = at(w.gates);
}

// Fills the arguments that all scan entry points share and checks them.
int scan_args(qd::ScanArgs& a, int32_t N, int32_t T, const int32_t* cu, int32_t H, int32_t G, int32_t P, int32_t Ns,
              int32_t dtype, int32_t softplus, const void* x, int64_t ldx, const float* dt, const float* A,
              const void* B, int64_t ldb, const void* C, int64_t ldc, const float* D, const float* dt_bias,
              const float* S0) {
  int rc = check_seqs(N, T, cu, a.q);
  if (rc) return rc;
  if ((rc = check_scan(a.q, H, G, P, Ns, dtype, ldx, ldb, ldc))) return rc;
  const int e = elem_size(dtype);
  if (n_tokens(a.q) > 0)
    if (!(ok_ptr(x, e) && ok_ptr(B, e) && ok_ptr(C, e) && ok_ptr(dt, 4))) return QDELTA_EINVAL;
  if (N > 0 && !ok_ptr(A, 4)) return QDELTA_EINVAL;
  if (!ok_opt(D, 4) || !ok_opt(dt_bias, 4) || !ok_opt(S0, 4)) return QDELTA_EINVAL;
  a.H = H; a.G = G; a.P = P; a.N = Ns;
  a.softplus = softplus != 0;
  a.x = x; a.ldx = ldx; a.dt = dt; a.A = A; a.B = B; a.ldb = ldb; a.C = C; a.ldc = ldc;
  a.D = D; a.bias = dt_bias; a.S0 = S0;
  return QDELTA_OK;
}

}  // namespace

extern "C" {

size_t qdelta_scan_workspace_bytes(int32_t N, int32_t T, int32_t packed, int32_t H, int32_t G, int32_t P, int32_t Ns,
                                   int32_t is_bwd) {
  static const int32_t any = 0;
  qd::Seqs q;
  if (check_seqs(N, T, packed ? &any : nullptr, q) ||
      check_scan(q, H, G, P, Ns, QDELTA_F32, INT64_MAX, INT64_MAX, INT64_MAX))
    return 0;
  return scan_ws(q, H, G, P, Ns, is_bwd != 0, true).bytes;   // of either type: fp32 has the shorter segments
}

int qdelta_scan_fwd(int32_t N, int32_t T, const int32_t* cu_seqlens, int32_t H, int32_t G, int32_t P, int32_t Ns,
                    int32_t dtype, int32_t softplus, const void* x, int64_t ldx, const float* dt, const float* A,
                    const void* B, int64_t ldb, const void* C, int64_t ldc, const float* D, const float* dt_bias,
                    const float* initial_state, void* y, float* final_state, void* ws, size_t ws_bytes,
                    hipStream_t stream) {
  qd::ScanArgs a{};
  const int rc = scan_args(a, N, T, cu_seqlens, H, G, P, Ns, dtype, softplus, x, ldx, dt, A, B, ldb, C, ldc, D, dt_bias,
                           initial_state);
  if (rc) return rc;
  if (n_tokens(a.q) > 0 && !ok_ptr(y, elem_size(dtype))) return QDELTA_EINVAL;
  if (!ok_opt(final_state, 4)) return QDELTA_EINVAL;
  const size_t need = scan_ws(a.q, H, G, P, Ns, false, true).bytes;
  if (need > 0 && !ok_ptr(ws, 16)) return QDELTA_EINVAL;
  if (ws_bytes < need) return QDELTA_ENOWORKSPACE;
  const ScanWs w = scan_ws(a.q, H, G, P, Ns, false, dtype == QDELTA_F32);
  if (N == 0) return QDELTA_OK;
  a.y = y;
  a.Sf = final_state;
  bind_ws(a, w, ws);
  return status(qd::launch_scan_fwd(a, dtype, stream));
}

int qdelta_scan_bwd(int32_t N, int32_t T, const int32_t* cu_seqlens, int32_t H, int32_t G, int32_t P, int32_t Ns,
                    int32_t dtype, int32_t softplus, const void* x, int64_t ldx, const float* dt, const float* A,
                    const void* B, int64_t ldb, const void* C, int64_t ldc, const float* D, const float* dt_bias,
                    const float* initial_state, const void* dy, const float* d_final_state, void* dx, float* ddt,
                    float* dA, void* dB, void* dC, float* dD, float* ddt_bias, float* d_initial_state, void* ws,
                    size_t ws_bytes, hipStream_t stream) {
  qd::ScanArgs a{};
  const int rc = scan_args(a, N, T, cu_seqlens, H, G, P, Ns, dtype, softplus, x, ldx, dt, A, B, ldb, C, ldc, D, dt_bias,
                           initial_state);
  if (rc) return rc;
  const int e = elem_size(dtype);
  if (n_tokens(a.q) > 0) {
    for (const void* p : {dy, (const void*)dx, (const void*)dB, (const void*)dC})
      if (!ok_ptr(p, e)) return QDELTA_EINVAL;
    if (!ok_ptr(ddt, 4)) return QDELTA_EINVAL;
  }
  if (!ok_ptr(dA, 4) || !ok_opt(dD, 4) || !ok_opt(ddt_bias, 4) || !ok_opt(d_initial_state, 4) || !ok_opt(d_final_state, 4))
    return QDELTA_EINVAL;
  const size_t need = scan_ws(a.q, H, G, P, Ns, true, true).bytes;
  if (need > 0 && !ok_ptr(ws, 16)) return QDELTA_EINVAL;
  if (ws_bytes < need) return QDELTA_ENOWORKSPACE;
  const ScanWs w = scan_ws(a.q, H, G, P, Ns, true, dtype == QDELTA_F32);
  a.dy = dy; a.dSf = d_final_state;
  a.dx = dx; a.ddt = ddt; a.dA = dA; a.dB = dB; a.dC = dC; a.dD = dD; a.dbias = ddt_bias; a.dS0 = d_initial_state;
  bind_ws(a, w, ws);
  return status(qd::launch_scan_bwd(a, dtype, stream));   // no sequences: the heads' gradients are still written (zero)
}

int qdelta_scan_step(int32_t N, int32_t H, int32_t G, int32_t P, int32_t Ns, int32_t dtype, int32_t softplus,
                     const void* x, int64_t ldx, const float* dt, const float* A, const void* B, int64_t ldb,
                     const void* C, int64_t ldc, const float* D, const float* dt_bias, const float* state,
                     float* state_out, void* y, hipStream_t stream) {
  qd::ScanArgs a{};
  const int rc = scan_args(a, N, 1, nullptr, H, G, P, Ns, dtype, softplus, x, ldx, dt, A, B, ldb, C, ldc, D, dt_bias, state);
  if (rc) return rc;
  if (N > 0 && !(ok_ptr(state, 4) && ok_ptr(state_out, 4) && ok_ptr(y, elem_size(dtype)))) return QDELTA_EINVAL;
  if ((int64_t)N * H * ((P + 15) / 16) * 256 >= kMaxThreads) return QDELTA_EUNSUPPORTED;
  a.y = y;
  a.Sf = state_out;
  return status(qd::launch_scan_step(a, dtype, stream));
}

int qdelta_conv_fwd(int32_t N, int32_t T, const int32_t* cu_seqlens, int32_t D, int32_t W, int32_t dtype, int32_t silu,
                    const void* x, int64_t ldx, const void* weight, const void* bias, const void* initial_state,
                    void* y, void* final_state, hipStream_t stream) {
  qd::ConvArgs a{};
  int rc = check_seqs(N, T, cu_seqlens, a.q);
  if (rc) return rc;
  if ((rc = check_conv(a.q, D, W, dtype, ldx))) return rc;
  const int e = elem_size(dtype);
  if (n_tokens(a.q) > 0 && !(ok_ptr(x, e) && ok_ptr(y, e))) return QDELTA_EINVAL;
  if (N > 0 && !ok_ptr(weight, e)) return QDELTA_EINVAL;
  if (!ok_opt(bias, e) || !ok_opt(initial_state, e) || !ok_opt(final_state, e)) return QDELTA_EINVAL;
  if (N == 0) return QDELTA_OK;
  a.D = D; a.W = W; a.silu = silu != 0; a.ldx = ldx;
  a.x = x; a.w = weight; a.b = bias; a.s0 = initial_state;
  a.y = y; a.sf = final_state;
  return status(qd::launch_conv_fwd(a, dtype, stream));
}

size_t qdelta_conv_workspace_bytes(int32_t N, int32_t T, int32_t packed, int32_t D, int32_t W) {
  static const int32_t any = 0;
  qd::Seqs q;
  if (check_seqs(N, T, packed ? &any : nullptr, q) || check_conv(q, D, W, QDELTA_F32, INT64_MAX)) return 0;
  return (size_t)qd::conv_bwd_plan(q, D).groups * (W + 1) * D * sizeof(float);
}

int qdelta_conv_bwd(int32_t N, int32_t T, const int32_t* cu_seqlens, int32_t D, int32_t W, int32_t dtype, int32_t silu,
                    const void* x, int64_t ldx, const void* weight, const void* bias, const void* initial_state,
                    const void* dy, const void* d_final_state, void* dx, void* dweight, void* dbias,
                    void* d_initial_state, void* ws, size_t ws_bytes, hipStream_t stream) {
  qd::ConvArgs a{};
  int rc = check_seqs(N, T, cu_seqlens, a.q);
  if (rc) return rc;
  if ((rc = check_conv(a.q, D, W, dtype, ldx))) return rc;
  const int e = elem_size(dtype);
  if (n_tokens(a.q) > 0 && !(ok_ptr(x, e) && ok_ptr(dy, e) && ok_ptr(dx, e))) return QDELTA_EINVAL;
  if (N > 0 && !ok_ptr(weight, e)) return QDELTA_EINVAL;
  for (const void* p : {bias, initial_state, d_final_state, (const void*)dweight, (const void*)dbias,
                        (const void*)d_initial_state})
    if (!ok_opt(p, e)) return QDELTA_EINVAL;
  const size_t need = (size_t)qd::conv_bwd_plan(a.q, D).groups * (W + 1) * D * sizeof(float);
  if (need > 0 && !ok_ptr(ws, 16)) return QDELTA_EINVAL;
  if (ws_bytes < need) return QDELTA_ENOWORKSPACE;
  if ((int64_t)qd::conv_bwd_plan(a.q, D).groups * (D + 255) + 3 * (int64_t)N * D + 256 >= kMaxThreads) return QDELTA_EUNSUPPORTED;
  // 16 threads a column of the sum over the workgroups
  if ((dweight || dbias) && 16 * ((int64_t)(W + 1) * D + 63) >= kMaxThreads) return QDELTA_EUNSUPPORTED;
  a.D = D; a.W = W; a.silu = silu != 0; a.ldx = ldx;
  a.x = x; a.w = weight; a.b = bias; a.s0 = initial_state;
  a.dy = dy; a.dsf = d_final_state;
  a.dx = dx; a.dw = dweight; a.db = dbias; a.ds0 = d_initial_state;
  a.part = static_cast<float*>(ws);
  return status(qd::launch_conv_bwd(a, dtype, stream));   // no sequences: the weight's gradients are still written (zero)
}

int qdelta_conv_step(int32_t N, int32_t D, int32_t W, int32_t dtype, int32_t silu, const void* x, int64_t ldx,
                     const void* weight, const void* bias, const void* state, void* state_out, void* y,
                     hipStream_t stream) {
  qd::ConvArgs a{};
  int rc = check_seqs(N, 1, nullptr, a.q);
  if (rc) return rc;
  if ((rc = check_conv(a.q, D, W, dtype, ldx))) return rc;
  const int e = elem_size(dtype);
  if (N > 0)
    for (const void* p : {x, weight, state, (const void*)state_out, (const void*)y})
      if (!ok_ptr(p, e)) return QDELTA_EINVAL;
  if (!ok_opt(bias, e)) return QDELTA_EINVAL;
  a.D = D; a.W = W; a.silu = silu != 0; a.ldx = ldx;
  a.x = x; a.w = weight; a.b = bias; a.s0 = state; a.sf = state_out; a.y = y;
  return status(qd::launch_conv_step(a, dtype, stream));
}

int qdelta_norm_fwd(int64_t rows, int32_t D, int32_t dtype, int32_t rms, float eps, const void* x, int64_t ldx,
                    const void* weight, const void* bias, const void* gate, int64_t ldg, void* y, float* stats,
                    hipStream_t stream) {
  const int rc = check_norm(rows, D, dtype, ldx, gate, ldg);
  if (rc) return rc;
  const int e = elem_size(dtype);
  if (rows > 0 && !(ok_ptr(x, e) && ok_ptr(y, e))) return QDELTA_EINVAL;
  if (!ok_opt(weight, e) || !ok_opt(bias, e) || !ok_opt(gate, e) || !ok_opt(stats, 4)) return QDELTA_EINVAL;
  if (!(eps >= 0.f)) return QDELTA_EINVAL;
  if (rows == 0) return QDELTA_OK;
  qd::RowNormArgs a{};
  a.rows = rows; a.D = D; a.rms = rms != 0; a.eps = eps; a.ldx = ldx; a.ldg = ldg;
  a.x = x; a.w = weight; a.b = bias; a.g = gate; a.y = y; a.stats = stats;
  return status(qd::launch_norm_fwd(a, dtype, stream));
}

size_t qdelta_norm_workspace_bytes(int64_t rows, int32_t D) {
  if (rows < 0 || D <= 0 || D > 8192) return 0;
  return (size_t)qd::norm_bwd_blocks(rows, D) * 2 * D * sizeof(float);
}

int qdelta_norm_bwd(int64_t rows, int32_t D, int32_t dtype, int32_t rms, const void* x, int64_t ldx,
                    const void* weight, const void* bias, const void* gate, int64_t ldg, const float* stats,
                    const void* dy, void* dx, void* dweight, void* dbias, void* dgate, void* ws, size_t ws_bytes,
                    hipStream_t stream) {
  const int rc = check_norm(rows, D, dtype, ldx, gate, ldg);
  if (rc) return rc;
  const int e = elem_size(dtype);
  if (rows > 0 && !(ok_ptr(x, e) && ok_ptr(dy, e) && ok_ptr(dx, e) && ok_ptr(stats, 4))) return QDELTA_EINVAL;
  for (const void* p : {weight, bias, gate, (const void*)dweight, (const void*)dbias, (const void*)dgate})
    if (!ok_opt(p, e)) return QDELTA_EINVAL;
  if (rows > 0 && gate && !dgate) return QDELTA_EINVAL;
  const bool sums = dweight || dbias;
  if (sums && !ok_ptr(ws, 16)) return QDELTA_EINVAL;
  if (sums && ws_bytes < qdelta_norm_workspace_bytes(rows, D)) return QDELTA_ENOWORKSPACE;
  if (rows == 0 && !sums) return QDELTA_OK;
  qd::RowNormArgs a{};
  a.rows = rows; a.D = D; a.rms = rms != 0; a.ldx = ldx; a.ldg = ldg;
  a.x = x; a.w = weight; a.b = bias; a.g = gate; a.stats = const_cast<float*>(stats);
  a.dy = dy; a.dx = dx; a.dw = dweight; a.db = dbias; a.dg = dgate;
  a.part = sums ? static_cast<float*>(ws) : nullptr;
  return status(qd::launch_norm_bwd(a, dtype, stream));   // no rows: one workgroup writes sums of zero
}

}  // extern "C"
