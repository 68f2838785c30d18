"""mixer's calls on the CPU in 64 bits, from the plain forms (for the tests of the layer's wiring)."""
import numpy as np
import torch

from tests import mixer_reference as ref


def _n(t):
    return None if t is None else t.detach().numpy()


def _t(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a))


def _seqs(x, cu):
    if cu is None:
        return [(i, slice(None)) for i in range(x.shape[0])]
    c = cu.tolist()
    return [(0, slice(c[i], c[i + 1])) for i in range(len(c) - 1)]


def conv_fwd(x, weight, bias=None, initial_state=None, cu_seqlens=None, activation=None):
    y, states = torch.empty_like(x), []
    for i, at in enumerate(_seqs(x, cu_seqlens)):
        yi, si = ref.conv(_n(x[at]), _n(weight), _n(bias), None if initial_state is None else _n(initial_state[i]),
                          activation == "silu")
        y[at] = _t(yi)
        states.append(_t(si))
    return y, torch.stack(states)


def conv_bwd(x, weight, bias, initial_state, d_y, d_final_state=None, cu_seqlens=None, activation=None,
             need_d_initial_state=True):
    dx, dw, db, ds = torch.empty_like(x), 0, 0, []
    for i, at in enumerate(_seqs(x, cu_seqlens)):
        g = ref.conv_grads(_n(x[at]), _n(weight), _n(bias), None if initial_state is None else _n(initial_state[i]),
                           activation == "silu", _n(d_y[at]), None if d_final_state is None else _n(d_final_state[i]))
        dx[at] = _t(g["dx"])
        dw, db = dw + g["dweight"], db + g["dbias"]
        ds.append(_t(g["d_initial_state"]))
    return dict(dx=dx, dweight=_t(dw), dbias=None if bias is None else _t(db),
                d_initial_state=torch.stack(ds) if need_d_initial_state else None)


def norm_fwd(x, weight=None, bias=None, gate=None, eps=1e-5, kind="layer"):
    D = x.shape[-1]
    y, stats = ref.norm(_n(x).reshape(-1, D), _n(weight), _n(bias), None if gate is None else _n(gate).reshape(-1, D), eps,
                        kind == "rms")
    return _t(y).reshape(x.shape), _t(np.concatenate([stats, np.full_like(stats[:, :1], eps)], 1))


def norm_bwd(x, weight, bias, gate, stats, d_y, kind="layer"):
    D = x.shape[-1]
    g = ref.norm_grads(_n(x).reshape(-1, D), _n(weight), _n(bias), None if gate is None else _n(gate).reshape(-1, D),
                       float(stats[0, 2]), kind == "rms", _n(d_y).reshape(-1, D))
    return dict(dx=_t(g["dx"]).reshape(x.shape), dweight=None if weight is None else _t(g["dweight"]),
                dbias=None if bias is None else _t(g["dbias"]),
                dgate=None if gate is None else _t(g["dgate"]).reshape(x.shape))


def scan_fwd(x, dt, A, B, C, D=None, dt_bias=None, initial_state=None, cu_seqlens=None, softplus=False):
    y, states = torch.empty_like(x), []
    for i, at in enumerate(_seqs(x, cu_seqlens)):
        yi, si = ref.scan(_n(x[at]), _n(dt[at]), _n(A), _n(B[at]), _n(C[at]), _n(D), _n(dt_bias),
                          None if initial_state is None else _n(initial_state[i]), softplus)
        y[at] = _t(yi)
        states.append(_t(si))
    return y, torch.stack(states)


def scan_bwd(x, dt, A, B, C, D, dt_bias, initial_state, d_y, d_final_state=None, cu_seqlens=None, softplus=False,
             need_d_initial_state=True):
    out = dict(dx=torch.empty_like(x), ddt=torch.empty_like(dt), dB=torch.empty_like(B), dC=torch.empty_like(C))
    sums, ds = dict(dA=0, dD=0, ddt_bias=0), []
    for i, at in enumerate(_seqs(x, cu_seqlens)):
        g = ref.scan_grads(_n(x[at]), _n(dt[at]), _n(A), _n(B[at]), _n(C[at]), _n(D), _n(dt_bias),
                           None if initial_state is None else _n(initial_state[i]), softplus, _n(d_y[at]),
                           None if d_final_state is None else _n(d_final_state[i]))
        for k in out:
            out[k][at] = _t(g[k])
        for k in sums:
            sums[k] = sums[k] + g[k]
        ds.append(_t(g["d_initial_state"]))
    return dict(**out, dA=_t(sums["dA"]), dD=None if D is None else _t(sums["dD"]),
                ddt_bias=None if dt_bias is None else _t(sums["ddt_bias"]),
                d_initial_state=torch.stack(ds) if need_d_initial_state else None)
