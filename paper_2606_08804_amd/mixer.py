"""Operators that stand around the recurrence in a block, on the kernels of
libqdelta.so (``include/qdelta_mixer.h``).  Argument marshalling only, as in
``qdelta``: there is no fallback, and without the built library every call raises.

conv_fwd(x, weight, bias=None, initial_state=None, cu_seqlens=None, activation=None)
          -> (y, final_state)                    short causal convolution per channel
conv_bwd(x, weight, bias, initial_state, d_y, d_final_state=None, cu_seqlens=None, activation=None)
          -> dict of gradients
conv_step(x, weight, bias, state, activation=None) -> y       (one token; state updated in place)
norm_fwd(x, weight=None, bias=None, gate=None, eps=1e-5, kind="layer") -> (y, stats)
norm_bwd(x, weight, bias, gate, stats, d_y, kind="layer") -> dict of gradients
scan_fwd(x, dt, A, B, C, D=None, dt_bias=None, initial_state=None, cu_seqlens=None, softplus=False)
          -> (y, final_state)                    selective state space scan, one decay per head
scan_bwd(x, dt, A, B, C, D, dt_bias, initial_state, d_y, d_final_state=None, cu_seqlens=None, softplus=False)
          -> dict of gradients
scan_step(x, dt, A, B, C, state, D=None, dt_bias=None, softplus=False) -> y   (one token; state updated in place)

x, B and C of the convolution and the scan and x and gate of the norm may be
views with evenly spaced rows (slices of a fused projection); other tensors
are contiguous.  cu_seqlens ends at T: padding behind the last sequence is a
sequence of its own (rows of new outputs past cu_seqlens[-1] are not written).
All tensors of a call live on one device, whose current
stream the call runs on.  Differentiable forms are in ``layer``.
"""
import ctypes
import math

import torch

from . import qdelta as _q

EXPORTS = (
    "qdelta_conv_fwd", "qdelta_conv_workspace_bytes", "qdelta_conv_bwd", "qdelta_conv_step",
    "qdelta_norm_fwd", "qdelta_norm_workspace_bytes", "qdelta_norm_bwd",
    "qdelta_scan_workspace_bytes", "qdelta_scan_fwd", "qdelta_scan_bwd", "qdelta_scan_step",
)

_lib = None
_p, _need, _opt, _dt = _q._p, _q._need, _q._opt, _q._dt


def lib():
    """libqdelta.so with the signatures of these entry points."""
    global _lib
    if _lib is None:
        L = _q.lib()
        i32, i64, sz, f32, P = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float, ctypes.c_void_p
        # N, T, cu, D, W, dtype, silu, x, ldx, weight, bias, ...
        L.qdelta_conv_fwd.argtypes = [i32, i32, P] + [i32] * 4 + [P, i64] + [P] * 6
        L.qdelta_conv_workspace_bytes.argtypes = [i32] * 5
        L.qdelta_conv_workspace_bytes.restype = sz
        L.qdelta_conv_bwd.argtypes = [i32, i32, P] + [i32] * 4 + [P, i64] + [P] * 10 + [sz, P]
        L.qdelta_conv_step.argtypes = [i32] * 5 + [P, i64] + [P] * 6
        # rows, D, dtype, rms, eps, x, ldx, weight, bias, gate, ldg, y, stats
        L.qdelta_norm_fwd.argtypes = [i64] + [i32] * 3 + [f32, P, i64, P, P, P, i64, P, P, P]
        L.qdelta_norm_workspace_bytes.argtypes = [i64, i32]
        L.qdelta_norm_workspace_bytes.restype = sz
        L.qdelta_norm_bwd.argtypes = [i64] + [i32] * 3 + [P, i64, P, P, P, i64] + [P] * 7 + [sz, P]
        L.qdelta_scan_workspace_bytes.argtypes = [i32] * 8
        L.qdelta_scan_workspace_bytes.restype = sz
        # H, G, P, Ns, dtype, softplus, x, ldx, dt, A, B, ldb, C, ldc, D, dt_bias, state, ...
        scan = [i32] * 6 + [P, i64, P, P, P, i64, P, i64, P, P, P]
        L.qdelta_scan_fwd.argtypes = [i32, i32, P] + scan + [P] * 3 + [sz, P]
        L.qdelta_scan_bwd.argtypes = [i32, i32, P] + scan + [P] * 11 + [sz, P]
        L.qdelta_scan_step.argtypes = [i32] + scan + [P] * 3
        _lib = L
    return _lib


def _call(fn, device, *args):
    """The entry point on the device's current stream; the device is made the current one for the launch."""
    f = getattr(lib(), fn)
    if device.index == torch.cuda.current_device():
        rc = f(*args, _q._stream())
    else:
        with torch.cuda.device(device):
            rc = f(*args, torch.cuda.current_stream().cuda_stream)
    if rc:
        raise _q.QDeltaError(fn, rc)


def _one_device(first, *others):
    index = first.get_device()
    for t in others:
        if t is not None and t.get_device() != index:
            raise ValueError(f"tensors on {first.device} and {t.device}: all of a call's live on one device")
    return first.device


def _workspace(nbytes, device, workspace):
    return _q._workspace(nbytes, device, _opt(workspace, "workspace"))


def _rows(t, name, dtype, lead, size):
    """Elements from one row of t [*lead, *size] to the next; t may be a view whose rows are evenly spaced and whose
    last len(size) dimensions are contiguous within a row."""
    if isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.is_contiguous() and t.shape == lead + size:
        return math.prod(size)
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} is required")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != lead + size:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {lead + size}")
    width = math.prod(size)
    if t.numel() == 0:
        return width
    k, inner, strides = len(lead), 1, t.stride()
    for i in range(t.dim() - 1, k - 1, -1):
        if t.shape[i] > 1 and strides[i] != inner:
            raise ValueError(f"{name} must be contiguous within a row")
        inner *= t.shape[i]
    ld, step = None, None
    for i in range(k - 1, -1, -1):
        if t.shape[i] > 1:
            if ld is None:
                ld, step = strides[i], strides[i]
            elif strides[i] != step:
                raise ValueError(f"{name} must have evenly spaced rows")
        if step is not None:
            step *= t.shape[i]
    if ld is None:
        return width
    if ld < width:
        raise ValueError(f"{name} must have evenly spaced rows that do not overlap")
    return ld


def _sequences(lead, cu_seqlens, name="x"):
    """(N, T) of a call's leading dimensions [B, T]."""
    if len(lead) != 2:
        raise ValueError(f"{name} must have leading dimensions [B, T]")
    if cu_seqlens is None:
        return lead
    if lead[0] != 1:
        raise ValueError("a packed batch has leading dimension 1")
    _need(cu_seqlens, "cu_seqlens", torch.int32)
    if cu_seqlens.dim() != 1 or cu_seqlens.numel() < 1:
        raise ValueError("cu_seqlens must hold the N + 1 boundaries of N sequences")
    return cu_seqlens.numel() - 1, lead[1]


def _silu(activation):
    if activation not in (None, "silu"):
        raise ValueError(f"activation must be None or 'silu', got {activation!r}")
    return int(activation == "silu")


def _conv_args(x, weight, bias, lead):
    _dt(x)
    if weight is None or weight.dim() != 2:
        raise ValueError("weight must be [D, W]")
    D, W = weight.shape
    ld = _rows(x, "x", x.dtype, lead, (D,))
    _need(weight, "weight", x.dtype)
    _opt(bias, "bias", x.dtype, (D,))
    return D, W, ld


def conv_fwd(x, weight, bias=None, initial_state=None, cu_seqlens=None, activation=None, output_final_state=True):
    """Causal convolution of width W in {2, 3, 4}, one filter per channel:
    u_t = bias + sum_j weight[:, j] x_{t-W+1+j}, y = u or (activation "silu") u sigmoid(u).
    x [B,T,D] (B = 1 with cu_seqlens), weight [D,W], bias [D], initial_state
    [N,W-1,D]: the rows before each sequence, the oldest first (None: zeros).
    Returns (y [B,T,D], final_state [N,W-1,D] or None)."""
    lead = tuple(x.shape[:-1])
    N, T = _sequences(lead, cu_seqlens)
    D, W, ld = _conv_args(x, weight, bias, lead)
    _opt(initial_state, "initial_state", x.dtype, (N, W - 1, D))
    dev = _one_device(x, weight, bias, initial_state, cu_seqlens)
    y = torch.empty(lead + (D,), dtype=x.dtype, device=dev)
    sf = torch.empty((N, max(W - 1, 0), D), dtype=x.dtype, device=dev) if output_final_state else None
    _call("qdelta_conv_fwd", dev, N, T, _p(cu_seqlens), D, W, _dt(x), _silu(activation), _p(x), ld, _p(weight), _p(bias),
          _p(initial_state), _p(y), _p(sf))
    return y, sf


def conv_workspace_bytes(N, T, D, W, packed=False):
    return int(lib().qdelta_conv_workspace_bytes(N, T, int(packed), D, W))


def conv_bwd(x, weight, bias, initial_state, d_y, d_final_state=None, cu_seqlens=None, activation=None,
             need_d_initial_state=True, workspace=None):
    """Backward of conv_fwd.  Returns a dict: dx, dweight, dbias (None without
    a bias), d_initial_state (None if not requested)."""
    lead = tuple(x.shape[:-1])
    N, T = _sequences(lead, cu_seqlens)
    D, W, ld = _conv_args(x, weight, bias, lead)
    _opt(initial_state, "initial_state", x.dtype, (N, W - 1, D))
    _need(d_y, "d_y", x.dtype, lead + (D,))
    _opt(d_final_state, "d_final_state", x.dtype, (N, W - 1, D))
    dev = _one_device(x, weight, bias, initial_state, cu_seqlens, d_y, d_final_state, workspace)
    dx = torch.empty(lead + (D,), dtype=x.dtype, device=dev)
    dw = torch.empty_like(weight)
    db = None if bias is None else torch.empty_like(bias)
    ds0 = torch.empty((N, max(W - 1, 0), D), dtype=x.dtype, device=dev) if need_d_initial_state else None
    nbytes = conv_workspace_bytes(N, T, D, W, cu_seqlens is not None)
    ws = _workspace(nbytes, dev, workspace)
    _call("qdelta_conv_bwd", dev, N, T, _p(cu_seqlens), D, W, _dt(x), _silu(activation), _p(x), ld, _p(weight), _p(bias),
          _p(initial_state), _p(d_y), _p(d_final_state), _p(dx), _p(dw), _p(db), _p(ds0), _p(ws), nbytes)
    return dict(dx=dx, dweight=dw, dbias=db, d_initial_state=ds0)


def conv_step(x, weight, bias, state, activation=None, out=None, state_out=None):
    """One token of conv_fwd for N sequences: x [N,D], state [N,W-1,D], updated
    in place unless state_out takes the new one.  Returns y [N,D]."""
    lead = tuple(x.shape[:-1])
    if len(lead) != 1:
        raise ValueError("x must be [N, D]")
    D, W, ld = _conv_args(x, weight, bias, lead)
    _need(state, "state", x.dtype, lead + (W - 1, D))
    new = state if state_out is None else _need(state_out, "state_out", x.dtype, lead + (W - 1, D))
    y = torch.empty(lead + (D,), dtype=x.dtype, device=x.device) if out is None else \
        _need(out, "out", x.dtype, lead + (D,))
    dev = _one_device(x, weight, bias, state, new, y)
    _call("qdelta_conv_step", dev, lead[0], D, W, _dt(x), _silu(activation), _p(x), ld, _p(weight), _p(bias), _p(state),
          _p(new), _p(y))
    return y


def _norm_args(x, weight, bias, gate, kind):
    if kind not in ("layer", "rms"):
        raise ValueError(f"kind must be 'layer' or 'rms', got {kind!r}")
    _dt(x)
    if x.dim() < 1:
        raise ValueError("x must have at least one dimension")
    lead, D = tuple(x.shape[:-1]), x.shape[-1]
    ldx = _rows(x, "x", x.dtype, lead, (D,))
    _opt(weight, "weight", x.dtype, (D,))
    _opt(bias, "bias", x.dtype, (D,))
    ldg = D if gate is None else _rows(gate, "gate", x.dtype, lead, (D,))
    return lead, math.prod(lead), D, ldx, ldg


def norm_fwd(x, weight=None, bias=None, gate=None, eps=1e-5, kind="layer"):
    """Normalisation of the rows of x [..., D] (D <= 8192): xh = (x - mean) rstd,
    y = (xh weight + bias) gate sigmoid(gate); kind "rms" has mean 0 and rstd
    from mean(x^2).  weight, bias [D] and gate [..., D] may be None.
    Returns (y, stats): stats [..., 2] fp32, mean and rstd, for the backward."""
    lead, rows, D, ldx, ldg = _norm_args(x, weight, bias, gate, kind)
    dev = _one_device(x, weight, bias, gate)
    y = torch.empty(lead + (D,), dtype=x.dtype, device=dev)
    stats = torch.empty(lead + (2,), dtype=torch.float32, device=dev)
    _call("qdelta_norm_fwd", dev, rows, D, _dt(x), int(kind == "rms"), eps, _p(x), ldx, _p(weight), _p(bias), _p(gate), ldg,
          _p(y), _p(stats))
    return y, stats


def norm_workspace_bytes(rows, D):
    return int(lib().qdelta_norm_workspace_bytes(rows, D))


def norm_bwd(x, weight, bias, gate, stats, d_y, kind="layer", workspace=None):
    """Backward of norm_fwd.  Returns a dict: dx, dweight, dbias, dgate (None where the input is None)."""
    lead, rows, D, ldx, ldg = _norm_args(x, weight, bias, gate, kind)
    _need(stats, "stats", torch.float32, lead + (2,))
    _need(d_y, "d_y", x.dtype, lead + (D,))
    dev = _one_device(x, weight, bias, gate, stats, d_y, workspace)
    dx = torch.empty(lead + (D,), dtype=x.dtype, device=dev)
    dw = None if weight is None else torch.empty_like(weight)
    db = None if bias is None else torch.empty_like(bias)
    dg = None if gate is None else torch.empty_like(dx)
    nbytes = norm_workspace_bytes(rows, D) if dw is not None or db is not None else 0
    ws = _workspace(nbytes, dev, workspace)
    _call("qdelta_norm_bwd", dev, rows, D, _dt(x), int(kind == "rms"), _p(x), ldx, _p(weight), _p(bias), _p(gate), ldg,
          _p(stats), _p(d_y), _p(dx), _p(dw), _p(db), _p(dg), _p(ws), nbytes)
    return dict(dx=dx, dweight=dw, dbias=db, dgate=dg)


def _scan_args(x, dt, A, B, C, D, dt_bias, lead):
    """Checked sizes and strides of a scan's inputs: (H, G, P, Ns), (ldx, ldb, ldc)."""
    _dt(x)
    if x.dim() != len(lead) + 2:
        raise ValueError(f"x must be [{'B, T' if len(lead) == 2 else 'N'}, H, P]")
    H, P = x.shape[-2:]
    if B is None or B.dim() != x.dim():
        raise ValueError("B must have as many dimensions as x: [..., G, Ns]")
    G, Ns = B.shape[-2:]
    if G == 0 or H % G:
        raise ValueError(f"{H} heads cannot share {G} groups of B and C")
    ld = (_rows(x, "x", x.dtype, lead, (H, P)), _rows(B, "B", x.dtype, lead, (G, Ns)),
          _rows(C, "C", x.dtype, lead, (G, Ns)))
    _need(dt, "dt", torch.float32, lead + (H,))
    _need(A, "A", torch.float32, (H,))
    _opt(D, "D", torch.float32, (H,))
    _opt(dt_bias, "dt_bias", torch.float32, (H,))
    return (H, G, P, Ns), ld


def _scan_pointers(x, dt, A, B, C, D, dt_bias, state, ld):
    return (_p(x), ld[0], _p(dt), _p(A), _p(B), ld[1], _p(C), ld[2], _p(D), _p(dt_bias), _p(state))


def scan_workspace_bytes(N, T, H, G, P, Ns, packed=False, is_bwd=False):
    return int(lib().qdelta_scan_workspace_bytes(N, T, int(packed), H, G, P, Ns, int(is_bwd)))


def scan_fwd(x, dt, A, B, C, D=None, dt_bias=None, initial_state=None, cu_seqlens=None, softplus=False,
             output_final_state=True, workspace=None):
    """Selective state space scan, per sequence and head with a state S [P, Ns]:
    S_t = exp(dt A) S_{t-1} + dt x_t B_t^T, y_t = S_t C_t + D x_t, where dt is
    raw + dt_bias or (softplus) log(1 + exp(raw + dt_bias)).
    x [B,T,H,P] (P <= 256), B, C [B,T,G,Ns] (Ns <= 128; each group serves H / G
    heads) in bf16 or fp32; dt [B,T,H], A, D, dt_bias [H], states [N,H,P,Ns] fp32.
    Returns (y [B,T,H,P], final_state or None)."""
    lead = tuple(x.shape[:-2])
    N, T = _sequences(lead, cu_seqlens)
    dims, ld = _scan_args(x, dt, A, B, C, D, dt_bias, lead)
    H, G, P, Ns = dims
    _opt(initial_state, "initial_state", torch.float32, (N, H, P, Ns))
    dev = _one_device(x, dt, A, B, C, D, dt_bias, initial_state, cu_seqlens, workspace)
    y = torch.empty(lead + (H, P), dtype=x.dtype, device=dev)
    sf = torch.empty((N, H, P, Ns), dtype=torch.float32, device=dev) if output_final_state else None
    nbytes = scan_workspace_bytes(N, T, H, G, P, Ns, cu_seqlens is not None)
    ws = _workspace(nbytes, dev, workspace)
    _call("qdelta_scan_fwd", dev, N, T, _p(cu_seqlens), *dims, _dt(x), int(bool(softplus)),
          *_scan_pointers(x, dt, A, B, C, D, dt_bias, initial_state, ld), _p(y), _p(sf), _p(ws), nbytes)
    return y, sf


def scan_bwd(x, dt, A, B, C, D, dt_bias, initial_state, d_y, d_final_state=None, cu_seqlens=None, softplus=False,
             need_d_initial_state=True, workspace=None):
    """Backward of scan_fwd, from its inputs.  Returns a dict: dx, dB, dC (x's
    type), ddt (of raw), dA, dD and ddt_bias (None without the input),
    d_initial_state (None if not requested), fp32."""
    lead = tuple(x.shape[:-2])
    N, T = _sequences(lead, cu_seqlens)
    dims, ld = _scan_args(x, dt, A, B, C, D, dt_bias, lead)
    H, G, P, Ns = dims
    _opt(initial_state, "initial_state", torch.float32, (N, H, P, Ns))
    _need(d_y, "d_y", x.dtype, lead + (H, P))
    _opt(d_final_state, "d_final_state", torch.float32, (N, H, P, Ns))
    dev = _one_device(x, dt, A, B, C, D, dt_bias, initial_state, cu_seqlens, d_y, d_final_state, workspace)
    new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=dev)      # noqa: E731
    dx, dB, dC = new(*lead, H, P, dtype=x.dtype), new(*lead, G, Ns, dtype=x.dtype), new(*lead, G, Ns, dtype=x.dtype)
    ddt, dA = new(*lead, H), new(H)
    dD = None if D is None else new(H)
    dbias = None if dt_bias is None else new(H)
    ds0 = new(N, H, P, Ns) if need_d_initial_state else None
    nbytes = scan_workspace_bytes(N, T, H, G, P, Ns, cu_seqlens is not None, True)
    ws = _workspace(nbytes, dev, workspace)
    _call("qdelta_scan_bwd", dev, N, T, _p(cu_seqlens), *dims, _dt(x), int(bool(softplus)),
          *_scan_pointers(x, dt, A, B, C, D, dt_bias, initial_state, ld), _p(d_y), _p(d_final_state), _p(dx), _p(ddt),
          _p(dA), _p(dB), _p(dC), _p(dD), _p(dbias), _p(ds0), _p(ws), nbytes)
    return dict(dx=dx, ddt=ddt, dA=dA, dB=dB, dC=dC, dD=dD, ddt_bias=dbias, d_initial_state=ds0)


def scan_step(x, dt, A, B, C, state, D=None, dt_bias=None, softplus=False, out=None, state_out=None):
    """One token of scan_fwd for N sequences: x [N,H,P], dt [N,H], B, C
    [N,G,Ns], state [N,H,P,Ns] fp32, updated in place unless state_out takes
    the new one.  Returns y [N,H,P]."""
    lead = tuple(x.shape[:-2])
    if len(lead) != 1:
        raise ValueError("x must be [N, H, P]")
    dims, ld = _scan_args(x, dt, A, B, C, D, dt_bias, lead)
    H, G, P, Ns = dims
    _need(state, "state", torch.float32, lead + (H, P, Ns))
    new = state if state_out is None else _need(state_out, "state_out", torch.float32, lead + (H, P, Ns))
    y = torch.empty(lead + (H, P), dtype=x.dtype, device=x.device) if out is None else \
        _need(out, "out", x.dtype, lead + (H, P))
    dev = _one_device(x, dt, A, B, C, D, dt_bias, state, new, y)
    _call("qdelta_scan_step", dev, lead[0], *dims, _dt(x), int(bool(softplus)),
          *_scan_pointers(x, dt, A, B, C, D, dt_bias, state, ld), _p(new), _p(y))
    return y
