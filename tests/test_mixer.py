"""Operators around the recurrence without a GPU: the plain 64-bit forms against differences, the C entry points and
the binding's refusals before any launch (fake, never dereferenced, aligned pointers are used)."""
import os
import re

import numpy as np
import pytest
import torch

from paper_2606_08804_amd import mixer, qdelta
from tests import mixer_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20
OK, EINVAL, EUNSUPPORTED, ENOWORKSPACE = range(4)


def test_library_exports_every_declared_symbol():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "qdelta_mixer.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(qdelta_[a-z0-9_]+)\s*\(", text)))
    assert names == sorted(mixer.EXPORTS)
    for n in names:
        assert hasattr(mixer.lib(), n), n


# ------------------------------------------------------------------ the plain forms against differences

def _differences(loss, args, grads, rng):
    """Directional central differences of loss(args) in each argument that has a gradient."""
    for k, g in grads.items():
        d = rng.normal(size=args[k].shape)
        h = 1e-5
        up, down = ({**args, k: args[k] + s * h * d} for s in (1, -1))
        num = (loss(up) - loss(down)) / (2 * h)
        want = (g * d).sum()
        assert abs(num - want) <= 1e-7 * max(1, abs(want)), (k, num, want)      # h^2 and 2^-53 / h, both about 1e-10


@pytest.mark.parametrize("W,T,silu,state", [(4, 7, True, True), (3, 2, False, True), (2, 1, True, False), (4, 2, True, True)])
def test_conv_gradients_are_the_differences(W, T, silu, state):
    r = np.random.default_rng(W * 10 + T)
    D = 3
    a = dict(x=r.normal(size=(T, D)), w=r.normal(size=(D, W)), b=r.normal(size=D), s0=r.normal(size=(W - 1, D)) if state else None)
    dy, dsf = r.normal(size=(T, D)), r.normal(size=(W - 1, D))

    def loss(v):
        y, sf = ref.conv(v["x"], v["w"], v["b"], v["s0"], silu)
        return (y * dy).sum() + (sf * dsf).sum()
    g = ref.conv_grads(**a, silu=silu, dy=dy, dsf=dsf)
    pairs = dict(x=g["dx"], w=g["dweight"], b=g["dbias"])
    if state:
        pairs["s0"] = g["d_initial_state"]
    _differences(loss, a, pairs, r)


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("gate", [False, True])
def test_norm_gradients_are_the_differences(rms, gate):
    r = np.random.default_rng(rms * 2 + gate)
    a = dict(x=r.normal(size=(3, 5)), w=r.normal(size=5), b=r.normal(size=5), g=r.normal(size=(3, 5)) if gate else None)
    dy = r.normal(size=(3, 5))
    g = ref.norm_grads(**a, eps=1e-3, rms=rms, dy=dy)
    pairs = dict(x=g["dx"], w=g["dweight"], b=g["dbias"])
    if gate:
        pairs["g"] = g["dgate"]
    _differences(lambda v: (ref.norm(**v, eps=1e-3, rms=rms)[0] * dy).sum(), a, pairs, r)


@pytest.mark.parametrize("softplus", [False, True])
def test_scan_gradients_are_the_differences(softplus):
    r = np.random.default_rng(5 + softplus)
    T, H, G, P, N = 6, 4, 2, 3, 5
    a = dict(x=r.normal(size=(T, H, P)), raw=r.uniform(0.1, 0.5, size=(T, H)), A=-r.uniform(0.5, 2, size=H),
             B=r.normal(size=(T, G, N)), C=r.normal(size=(T, G, N)), D=r.normal(size=H), bias=r.uniform(0, 0.2, size=H),
             S0=r.normal(size=(H, P, N)))
    dy, dS = r.normal(size=(T, H, P)), r.normal(size=(H, P, N))

    def loss(v):
        y, S = ref.scan(**v, softplus=softplus)
        return (y * dy).sum() + (S * dS).sum()
    g = ref.scan_grads(**a, softplus=softplus, dy=dy, dSf=dS)
    _differences(loss, a, dict(x=g["dx"], raw=g["ddt"], A=g["dA"], B=g["dB"], C=g["dC"], D=g["dD"], bias=g["ddt_bias"],
                               S0=g["d_initial_state"]), r)


def test_chunk_algebra_of_the_scan_equals_the_tokens():
    """The chunk formulas that the kernels compute, forward and backward, with the decay's gradient without the diagonal."""
    r = np.random.default_rng(11)
    T, P, N = 9, 4, 6
    x, dt, A = r.normal(size=(T, P)), r.uniform(0.01, 0.6, size=T), -1.7
    B, C, S, G = r.normal(size=(T, N)), r.normal(size=(T, N)), r.normal(size=(P, N)), r.normal(size=(P, N))
    dy = r.normal(size=(T, P))
    b = np.cumsum(dt * A)
    low = np.tril(np.ones((T, T)))
    W = np.exp(np.where(low > 0, b[:, None] - b[None], 0)) * low
    K, E, e, tail = C @ B.T, dy @ x.T, np.exp(b), np.exp(b[-1] - b)
    one = lambda t: t[:, None]                                                   # noqa: E731
    y = one(e) * (C @ S.T) + (W * K * dt) @ x
    S1 = e[-1] * S + (x * one(dt * tail)).T @ B
    M = np.tril(W * K * E * dt, -1)
    u = (W * K).T @ dy + one(tail) * (B @ G.T)
    dB = one(dt) * ((W * E).T @ C + one(tail) * (x @ G))
    dC = one(e) * (dy @ S) + (W * E * dt) @ B
    srow, gcol = e * (dy * (C @ S.T)).sum(1), dt * tail * (x * (B @ G.T)).sum(1)
    back = np.cumsum((M.sum(1) - M.sum(0) + srow)[::-1])[::-1]
    dl = back + np.cumsum(gcol) - gcol + e[-1] * (G * S).sum()
    ddt = (x * u).sum(1) + A * dl
    h = lambda t: t[:, None]                                                     # noqa: E731
    args = (h(x), h(dt), np.array([A]), h(B), h(C), None, None, S[None], False)
    y_ref, S_ref = ref.scan(*args)
    g = ref.scan_grads(*args, h(dy), G[None])
    for got, want in [(y, y_ref[:, 0]), (S1, S_ref[0]), (one(dt) * u, g["dx"][:, 0]), (dB, g["dB"][:, 0]),
                      (dC, g["dC"][:, 0]), (ddt, g["ddt"][:, 0]), ((dt * dl).sum(), g["dA"][0]),
                      (e[-1] * G + (dy * one(e)).T @ C, g["d_initial_state"][0])]:
        np.testing.assert_allclose(got, want, rtol=0, atol=1e-12 * max(1, np.abs(want).max()))


# ------------------------------------------------------------------ refusals of the C entry points

def _conv(fn="qdelta_conv_fwd", N=1, T=8, cu=None, D=64, W=4, dtype=1, x=FAKE, ld=64, w=FAKE, b=None, s0=None, y=FAKE, sf=None):
    return mixer.lib().qdelta_conv_fwd(N, T, cu, D, W, dtype, 1, x, ld, w, b, s0, y, sf, None)


def test_conv_refuses_before_launch():
    for bad in (dict(W=1), dict(W=5)):
        assert _conv(**bad) == EUNSUPPORTED
    for bad in (dict(D=0), dict(W=0), dict(ld=63), dict(dtype=5), dict(N=-1), dict(T=-1), dict(x=None), dict(y=None),
                dict(w=None), dict(x=FAKE + 1), dict(b=FAKE + 1), dict(sf=FAKE + 1), dict(N=0, cu=FAKE)):
        assert _conv(**bad) == EINVAL, bad
    assert _conv(N=1 << 20, T=1 << 12) == EUNSUPPORTED
    assert _conv(N=0) == OK
    L = mixer.lib()
    need = mixer.conv_workspace_bytes(1, 200, 64, 4)
    assert need == 7 * 5 * 64 * 4                       # 25 tiles of 8 tokens, four to a workgroup
    assert mixer.conv_workspace_bytes(3, 200, 64, 4, packed=True) == 7 * 5 * 64 * 4     # 28 of them

    def bwd(ws=FAKE, nbytes=need, dy=FAKE, dx=FAKE):
        return L.qdelta_conv_bwd(1, 200, None, 64, 4, 1, 1, FAKE, 64, FAKE, None, None, dy, None, dx, FAKE, None, None, ws, nbytes, None)
    assert bwd(nbytes=need - 1) == ENOWORKSPACE
    assert bwd(ws=None) == bwd(dy=None) == bwd(dx=None) == EINVAL
    assert L.qdelta_conv_step(1, 64, 4, 1, 1, FAKE, 64, FAKE, None, FAKE, None, FAKE, None) == EINVAL
    assert L.qdelta_conv_step(1, 64, 7, 1, 1, FAKE, 64, FAKE, None, FAKE, FAKE, FAKE, None) == EUNSUPPORTED


def test_norm_refuses_before_launch():
    L = mixer.lib()

    def fwd(rows=4, D=64, dtype=1, eps=1e-5, x=FAKE, ldx=64, w=None, b=None, g=None, ldg=64, y=FAKE, stats=None):
        return L.qdelta_norm_fwd(rows, D, dtype, 0, eps, x, ldx, w, b, g, ldg, y, stats, None)
    assert fwd(D=8193, ldx=8193) == EUNSUPPORTED
    for bad in (dict(rows=-1), dict(D=0), dict(ldx=63), dict(g=FAKE, ldg=63), dict(dtype=3), dict(x=None), dict(y=None),
                dict(w=FAKE + 1), dict(stats=FAKE + 2), dict(eps=-1.0), dict(eps=float("nan"))):
        assert fwd(**bad) == EINVAL, bad
    assert fwd(rows=0) == OK
    need = mixer.norm_workspace_bytes(4, 64)

    def bwd(dg=None, g=None, dw=FAKE, ws=FAKE, nbytes=need, stats=FAKE):
        return L.qdelta_norm_bwd(4, 64, 1, 0, FAKE, 64, FAKE, None, g, 64, stats, FAKE, FAKE, dw, None, dg, ws, nbytes, None)
    assert bwd(nbytes=need - 1) == ENOWORKSPACE
    assert bwd(ws=None) == bwd(g=FAKE) == bwd(stats=None) == EINVAL
    assert mixer.norm_workspace_bytes(4, 9000) == 0


def test_scan_refuses_before_launch():
    L = mixer.lib()

    def fwd(N=1, T=64, cu=None, H=4, G=2, P=64, Ns=64, dtype=1, x=FAKE, ldx=256, dt=FAKE, A=FAKE, B=FAKE, ldb=128, C=FAKE,
            ldc=128, D=None, s0=None, y=FAKE, ws=FAKE, nbytes=1 << 40):
        return L.qdelta_scan_fwd(N, T, cu, H, G, P, Ns, dtype, 1, x, ldx, dt, A, B, ldb, C, ldc, D, None, s0, y, None, ws,
                                 nbytes, None)
    for bad in (dict(P=257, ldx=2000), dict(Ns=129, ldb=2000, ldc=2000), dict(N=1 << 15, T=1 << 15)):
        assert fwd(**bad) == EUNSUPPORTED, bad
    for bad in (dict(G=3), dict(G=0), dict(H=0), dict(P=0), dict(Ns=0), dict(dtype=2), dict(ldx=255), dict(ldb=127),
                dict(ldc=127), dict(x=None), dict(dt=None), dict(A=None), dict(B=None), dict(C=None), dict(y=None),
                dict(dt=FAKE + 2), dict(s0=FAKE + 2), dict(x=FAKE + 1), dict(N=-1), dict(N=0, cu=FAKE)):
        assert fwd(**bad) == EINVAL, bad
    assert fwd(N=0) == OK
    need = mixer.scan_workspace_bytes(1, 4096, 2, 1, 64, 64)
    if need:                                             # sequences are cut where one walk would leave the chip idle
        assert fwd(T=4096, H=2, G=1, ldx=128, ldb=64, ldc=64, nbytes=need - 1) == ENOWORKSPACE
    need = mixer.scan_workspace_bytes(1, 64, 4, 2, 64, 64, is_bwd=True)
    assert need >= 2 * 4 * 64 * 64 * 4

    def bwd(nbytes=need, dA=FAKE, ddt=FAKE, dB=FAKE):
        return L.qdelta_scan_bwd(1, 64, None, 4, 2, 64, 64, 1, 1, FAKE, 256, FAKE, FAKE, FAKE, 128, FAKE, 128, None, None, None,
                                 FAKE, None, FAKE, ddt, dA, dB, FAKE, None, None, None, FAKE, nbytes, None)
    assert bwd(nbytes=need - 1) == ENOWORKSPACE
    assert bwd(dA=None) == bwd(ddt=None) == bwd(dB=None) == EINVAL
    assert mixer.scan_workspace_bytes(1, 64, 4, 3, 64, 64) == 0
    assert L.qdelta_scan_step(1, 4, 2, 64, 64, 1, 1, FAKE, 256, FAKE, FAKE, FAKE, 128, FAKE, 128, None, None, None, FAKE, FAKE,
                              None) == EINVAL


# ------------------------------------------------------------------ refusals of the binding

def test_binding_refuses_host_tensors_and_shapes():
    x = torch.zeros(1, 4, 8)
    with pytest.raises(ValueError, match="device tensor"):
        mixer.conv_fwd(x, torch.zeros(8, 4))
    with pytest.raises(ValueError, match="device tensor"):
        mixer.norm_fwd(x)
    with pytest.raises(ValueError, match="kind"):
        mixer.norm_fwd(x, kind="batch")
    with pytest.raises(ValueError, match="leading dimension 1"):
        mixer.conv_fwd(torch.zeros(2, 4, 8), torch.zeros(8, 4), cu_seqlens=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="weight"):
        mixer.conv_fwd(x, torch.zeros(8))
    with pytest.raises(TypeError):
        mixer.norm_fwd(x.half())
    with pytest.raises(ValueError, match="share"):
        mixer.scan_fwd(torch.zeros(1, 4, 3, 8), torch.zeros(1, 4, 3), torch.zeros(3), torch.zeros(1, 4, 2, 8), torch.zeros(1, 4, 2, 8))


class _Fake(torch.Tensor):
    """A host tensor that says it is on the device, for the row checks."""
    is_cuda = True


def _view(t):
    return t.as_subclass(_Fake)


def test_rows_of_views():
    wide = torch.zeros(2, 5, 24)
    assert mixer._rows(_view(wide[..., 8:16]), "x", torch.float32, (2, 5), (8,)) == 24
    assert mixer._rows(_view(wide[:1, :, :8]), "x", torch.float32, (1, 5), (8,)) == 24
    assert mixer._rows(_view(wide[:, :1, :8]), "x", torch.float32, (2, 1), (8,)) == 120
    assert mixer._rows(_view(wide[..., :16].unflatten(2, (2, 8))), "x", torch.float32, (2, 5), (2, 8)) == 24
    assert mixer._rows(_view(wide[:, :0]), "x", torch.float32, (2, 0), (24,)) == 24
    for bad, lead, size in [(wide[:, :4, :8], (2, 4), (8,)), (wide[..., ::2], (2, 5), (12,)), (wide.transpose(0, 1), (5, 2), (24,)),
                            (wide[:, :1].expand(2, 5, 24), (2, 5), (24,)),
                            (wide.unflatten(2, (3, 8))[..., :4], (2, 5), (3, 4))]:
        with pytest.raises(ValueError):
            mixer._rows(_view(bad), "x", torch.float32, lead, size)
    with pytest.raises(TypeError):
        mixer._rows(_view(wide), "x", torch.bfloat16, (2, 5), (24,))
    assert qdelta.QDELTA_F32 == 0


def test_launches_of_two_to_the_32_threads_are_refused():
    L = mixer.lib()
    scan = lambda fn, N, T, H, G, P, cu=None: fn(                                # noqa: E731
        N, T, cu, H, G, P, 16, 1, 1, FAKE, H * P, FAKE, FAKE, FAKE, G * 16, FAKE, G * 16, None, None, None, FAKE, None, FAKE,
        1 << 60, None)
    assert scan(L.qdelta_scan_fwd, 1 << 18, 1, 8, 1, 256) == EUNSUPPORTED        # 2^23 walks of 512 threads
    assert scan(L.qdelta_scan_fwd, 1 << 24, 1, 1, 1, 16) == EUNSUPPORTED         # 2^24 chunks, 256 threads for their gates
    step = lambda N, H, P: L.qdelta_scan_step(                                   # noqa: E731
        N, H, 1, P, 16, 1, 1, FAKE, H * P, FAKE, FAKE, FAKE, 16, FAKE, 16, None, None, FAKE, FAKE, FAKE, None)
    assert step(1 << 17, 16, 128) == EUNSUPPORTED                                # 2^24 workgroups
    assert _conv(N=1 << 24, T=0, cu=FAKE) == EUNSUPPORTED                        # 2^24 final states of 3 x 64 channels
    assert _conv(N=1 << 22, T=1, D=2048, ld=2048) == EUNSUPPORTED
