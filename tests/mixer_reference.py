"""Plain 64-bit forms of the operators around the recurrence, token by token, with their gradients from the formulas.

Every function takes one sequence (the scan and the convolution) or all rows (the norm) as numpy arrays.  `mag=True`
gives, in place of each result, the sum of the absolute values of the terms that it is a sum of: what rounding errors
of the terms are relative to."""
import numpy as np


def sigmoid(u):
    return np.exp(-np.logaddexp(0, -u))


def conv(x, w, b, s0, silu, mag=False):
    """x [T, D], w [D, W], b [D], s0 [W-1, D] or None -> y, final state."""
    f = np.abs if mag else (lambda t: t)
    W, (T, D) = w.shape[1], x.shape
    ext = np.concatenate([np.zeros((W - 1, D)) if s0 is None else s0, x])
    u = sum(f(ext[j:j + T] * w[:, j]) for j in range(W)) + (0 if b is None else f(b))
    if silu and mag:
        y = u * 1.1                                    # |SiLU'| <= 1.1
    else:
        y = u * sigmoid(u) if silu else u
    return y, ext[T:]


def conv_grads(x, w, b, s0, silu, dy, dsf, mag=False):
    f = np.abs if mag else (lambda t: t)
    W, (T, D) = w.shape[1], x.shape
    ext = np.concatenate([np.zeros((W - 1, D)) if s0 is None else s0, x])
    u = sum(ext[j:j + T] * w[:, j] for j in range(W)) + (0 if b is None else b)
    du = dy * (sigmoid(u) * (1 + u * (1 - sigmoid(u)))) if silu else dy
    if mag and silu:                                   # |SiLU''| <= 0.5 on the error of u, which is relative to its terms
        du = np.abs(du) + np.abs(dy) * conv(x, w, b, s0, False, mag=True)[0]
    dext = np.zeros_like(ext)
    if dsf is not None:
        dext[T:] += f(dsf)
    dw = np.zeros_like(w)
    for j in range(W):
        dext[j:j + T] += f(w[:, j] * du)
        dw[:, j] = f(du * ext[j:j + T]).sum(0)
    return dict(dx=dext[W - 1:], dweight=dw, dbias=f(du).sum(0), d_initial_state=dext[:W - 1])


def norm(x, w, b, g, eps, rms):
    """x [rows, D] -> y, stats."""
    mean = 0 * x[:, :1] if rms else x.mean(1, keepdims=True)
    r = 1 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)
    y = (x - mean) * r
    y = y * (1 if w is None else w) + (0 if b is None else b)
    if g is not None:
        y = y * g * sigmoid(g)
    return y, np.concatenate([mean, r], 1)


def norm_grads(x, w, b, g, eps, rms, dy, mag=False):
    f = np.abs if mag else (lambda t: t)
    w1 = 1 if w is None else w
    mean, r = (t[:, None] for t in norm(x, None, None, None, eps, rms)[1].T)
    xh = (x - mean) * r
    lin = xh * w1 + (0 if b is None else b)
    d = dy if g is None else dy * g * sigmoid(g)
    if mag:      # the difference x - mean is off relative to its terms, the mean relative to the mean of |x|, however small it is
        xh = (np.abs(x) + np.abs(x).mean(1, keepdims=True)) * r
    res = dict(dweight=f(d * xh).sum(0), dbias=f(d).sum(0))
    if g is not None:
        res["dgate"] = dy * lin * sigmoid(g) * (1 + g * (1 - sigmoid(g)))
        if mag:
            res["dgate"] = np.abs(dy) * (np.abs(xh * w1) + (0 if b is None else np.abs(b))) * 1.1
    e = f(d * w1)
    h = f(xh)
    sign = 1 if mag else -1
    res["dx"] = r * (e + sign * ((0 if rms else e.mean(1, keepdims=True)) + h * (e * h).mean(1, keepdims=True)))
    return res


def _steps(raw, bias, softplus):
    z = raw + (0 if bias is None else bias)
    return z, (np.logaddexp(0, z) if softplus else z)


def scan(x, raw, A, B, C, D, bias, S0, softplus, mag=False):
    """x [T, H, P], raw [T, H], A [H], B, C [T, G, N], S0 [H, P, N] -> y, final state."""
    f = np.abs if mag else (lambda t: t)
    T, H, P = x.shape
    B, C = (np.repeat(t, H // B.shape[1], 1) for t in (B, C))
    _, dt = _steps(raw, bias, softplus)
    S = np.zeros((H, P, B.shape[2])) if S0 is None else f(S0.copy())
    y = np.zeros_like(x)
    for t in range(T):
        S = np.exp(dt[t] * A)[:, None, None] * S + f(dt[t][:, None] * x[t])[:, :, None] * f(B[t])[:, None, :]
        y[t] = np.einsum("hpn,hn->hp", S, f(C[t]))
        if D is not None:
            y[t] += f(D[:, None] * x[t])
    return y, S


def scan_grads(x, raw, A, B, C, D, bias, S0, softplus, dy, dSf, mag=False):
    f = np.abs if mag else (lambda t: t)
    T, H, P = x.shape
    G, N = B.shape[1:]
    Bh, Ch = (f(np.repeat(t, H // G, 1)) for t in (B, C))
    z, dt = _steps(raw, bias, softplus)
    a = np.exp(dt * A)
    x, dy, dtm, Am = f(x), f(dy), f(dt), f(A)
    states = [np.zeros((H, P, N)) if S0 is None else f(S0.copy())]
    for t in range(T):
        states.append(a[t][:, None, None] * states[-1] + (dtm[t][:, None] * x[t])[:, :, None] * Bh[t][:, None, :])
    gr = np.zeros((H, P, N)) if dSf is None else f(dSf.copy())
    res = dict(dx=np.zeros_like(x), ddt=np.zeros_like(dt), dB=np.zeros(B.shape), dC=np.zeros(B.shape), dA=np.zeros(H))
    for t in reversed(range(T)):
        res["dC"][t] = np.einsum("hp,hpn->hn", dy[t], states[t + 1]).reshape(G, -1, N).sum(1)
        gr = gr + dy[t][:, :, None] * Ch[t][:, None, :]
        u = np.einsum("hpn,hn->hp", gr, Bh[t])
        res["dx"][t] = dtm[t][:, None] * u + (0 if D is None else f(D)[:, None] * dy[t])
        res["dB"][t] = (dtm[t][:, None] * np.einsum("hp,hpn->hn", x[t], gr)).reshape(G, -1, N).sum(1)
        dl = a[t] * (gr * states[t]).sum((1, 2))
        res["ddt"][t] = (x[t] * u).sum(1) + Am * dl
        res["dA"] += dtm[t] * dl
        gr = a[t][:, None, None] * gr
    if softplus:
        res["ddt"] *= sigmoid(z)
    res.update(dD=(dy * x).sum((0, 2)), ddt_bias=res["ddt"].sum(0), d_initial_state=gr)
    return res
