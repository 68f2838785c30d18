"""Operators around the recurrence on the GPU, against their plain 64-bit forms.

Tolerances: an output of type t is rounded once, eps_t / 2 relative to its value; before that it is a sum in fp32 of
terms whose absolute values add up to `mag`, off by at most K mag: K = 2^-18 (64 roundings of 2^-24) for fp32 products,
and 2^-16 more where a bf16 call takes fp32 values as two bf16 ones (outputs of x's type alone; fp32 outputs are exact
sums of bf16 values)."""
import numpy as np
import pytest
import torch

from paper_2606_08804_amd import mixer
from tests import mixer_reference as ref

pytestmark = pytest.mark.gpu

K32, KSPLIT = 2.0 ** -18, 2.0 ** -16
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def f64(t):
    return None if t is None else t.double().cpu().numpy()


def close(got, want, mag, what, split=False):
    assert got.shape == want.shape, (what, got.shape, want.shape)
    k = K32 + (KSPLIT if split and got.dtype == torch.bfloat16 else 0)
    tol = torch.finfo(got.dtype).eps / 2 * np.abs(want) * (1 + k) + k * mag + 1e-30
    off = np.abs(f64(got) - want)
    assert np.isfinite(f64(got)).all(), (what, "not finite")
    worst = float((off / tol).max()) if off.size else 0.0
    assert worst <= 1, (what, worst, float(off.max()))


def rand(seed, dtype):
    g = torch.Generator("cuda").manual_seed(seed)
    return lambda *s, scale=1.0, t=None: (torch.randn(s, generator=g, device="cuda") * scale).to(t or TYPES[dtype])


def sequences(lens, packed):
    """[(sequence, index of its tokens)] of a dense batch (equal lengths) or a packed one, and cu_seqlens."""
    if not packed:
        return [(i, (i,)) for i in range(len(lens))], None
    cu = np.concatenate([[0], np.cumsum(lens)])
    return [(i, (0, slice(cu[i], cu[i + 1]))) for i in range(len(lens))], torch.tensor(cu, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------------------------------ convolution

CONV = [  # lengths, packed, D, W, silu, state, extra columns of the rows x lies in
    ([1], False, 8, 4, True, True, 0),
    ([3, 3], False, 64, 4, True, False, 0),
    ([7], False, 5, 3, False, True, 0),
    ([33, 33], False, 72, 2, True, True, 8),
    ([130], False, 1000, 4, True, True, 24),
    ([257], False, 129, 4, False, False, 3),
    ([300] * 3, False, 520, 3, True, True, 0),
    ([0, 1, 5, 0, 128, 129, 2], True, 136, 4, True, True, 0),
    ([31, 32, 33, 200], True, 65, 3, True, False, 7),
    ([0], False, 16, 4, True, True, 0),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,packed,D,W,silu,state,extra", CONV)
def test_conv(lens, packed, D, W, silu, state, extra, dtype):
    r = rand(len(lens) * 1000 + D, dtype)
    N, T = len(lens), sum(lens) if packed else lens[0]
    seqs, cu = sequences(lens, packed)
    x = r(1 if packed else N, T, D + extra)[..., :D]
    w, b = r(D, W, scale=0.5), r(D, scale=0.1)
    s0 = r(N, W - 1, D) if state else None
    dy, dsf = r(*x.shape), r(N, W - 1, D)
    act = "silu" if silu else None
    y, sf = mixer.conv_fwd(x, w, b, s0, cu_seqlens=cu, activation=act)
    g = mixer.conv_bwd(x, w, b, s0, dy, dsf, cu_seqlens=cu, activation=act)
    mag = {}
    want = dict(dweight=0, dbias=0)
    for i, at in seqs:
        si = None if s0 is None else f64(s0[i])
        args = (f64(x[at]), f64(w), f64(b), si, silu)
        yr, sr = ref.conv(*args)
        close(y[at], yr, ref.conv(*args, mag=True)[0], "y")
        assert np.array_equal(f64(sf[i]), sr), "the state is a copy"
        gr, gm = (ref.conv_grads(*args, f64(dy[at]), f64(dsf[i]), mag=m) for m in (False, True))
        close(g["dx"][at], gr["dx"], gm["dx"], "dx")
        close(g["d_initial_state"][i], gr["d_initial_state"], gm["d_initial_state"], "d_initial_state")
        for k in ("dweight", "dbias"):
            want[k] = want[k] + gr[k]
            mag[k] = mag.get(k, 0) + gm[k]
    for k in ("dweight", "dbias"):
        close(g[k], want[k], mag[k], k)
    again = mixer.conv_bwd(x, w, b, s0, dy, dsf, cu_seqlens=cu, activation=act)
    for k in g:
        assert torch.equal(g[k], again[k]), (k, "differs from run to run")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,W", [(64, 4), (33, 3), (1000, 2)])
def test_conv_steps_equal_the_prompt(D, W, dtype):
    """Tokens one at a time, from the state of a prompt, in place and into another state."""
    r = rand(D, dtype)
    N, T = 3, 9
    x, w, b, s0 = r(N, T, D), r(D, W), r(D), r(N, W - 1, D)
    y, sf = mixer.conv_fwd(x, w, b, s0, activation="silu")
    _, state = mixer.conv_fwd(x[:, :4].contiguous(), w, b, s0, activation="silu")
    for t in range(4, T):
        before, other = state.clone(), torch.empty_like(state)
        y1 = mixer.conv_step(x[:, t], w, b, state, activation="silu", state_out=other)
        assert torch.equal(state, before)
        y2 = mixer.conv_step(x[:, t], w, b, state, activation="silu")
        assert torch.equal(y1, y2) and torch.equal(state, other)
        assert torch.equal(y1, y[:, t]), t
    assert torch.equal(state, sf)


def test_conv_keeps_a_nan_to_its_window():
    x = torch.randn(1, 70, 16, device="cuda")
    w, b = torch.randn(16, 4, device="cuda"), torch.randn(16, device="cuda")
    y, _ = mixer.conv_fwd(x, w, b, activation="silu")
    x[0, 30, 3] = float("nan")
    z, _ = mixer.conv_fwd(x, w, b, activation="silu")
    assert torch.isnan(z[0, 30:34, 3]).all()
    z[0, 30:34, 3] = y[0, 30:34, 3]
    assert torch.equal(z, y)


# ------------------------------------------------------------------------------------------------ norm

NORM = [  # rows, D, extra columns
    (1, 1, 0), (3, 7, 0), (1, 64, 0), (5, 128, 0), (37, 128, 128), (300, 65, 1), (20, 256, 0), (17, 512, 0), (9, 1003, 0),
    (600, 1024, 8), (7, 2048, 0), (5, 4096, 0), (3, 5000, 0), (2, 8192, 0), (2, 8191, 0), (0, 64, 0), (5000, 16, 0),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,D,extra", NORM)
@pytest.mark.parametrize("kind,gate,affine", [("layer", False, True), ("rms", True, True), ("layer", True, False)])
def test_norm(rows, D, extra, kind, gate, affine, dtype):
    r = rand(rows + D, dtype)
    x, dy = (r(rows, D + extra) * 2 + 0.5)[:, :D], r(rows, D)
    w, b = (r(D), r(D) if kind == "layer" else None) if affine else (None, None)
    g = r(rows, D + 2 * extra)[:, :D] if gate else None
    eps = 1e-3                     # above the rounding of a row of one value's variance (zero)
    y, stats = mixer.norm_fwd(x, w, b, g, eps=eps, kind=kind)
    d = mixer.norm_bwd(x, w, b, g, stats, dy, kind=kind)
    if not rows:
        assert y.shape == x.shape and all(v is None or not v.any() for v in d.values())
        return
    args = (f64(x), f64(w), f64(b), f64(g), eps, kind == "rms")
    yr, sr = ref.norm(*args)
    # terms of y: x and mean times the deviation, w, b; the mean's own error is relative to mean |x|
    rstd = sr[:, 1:]
    big = (np.abs(args[0]) + np.abs(args[0]).mean(1, keepdims=True)) * rstd
    sg = 1 if g is None else np.abs(args[3] * ref.sigmoid(args[3]))
    close(y, yr, (big * (1 if w is None else np.abs(args[1])) + (0 if b is None else np.abs(args[2]))) * sg, "y")
    close(stats, sr, np.concatenate([np.abs(args[0]).mean(1, keepdims=True), rstd * (1 + big.max(1, keepdims=True))], 1), "stats")
    gr, gm = (ref.norm_grads(*args, f64(dy), mag=m) for m in (False, True))
    names = dict(dx=True, dweight=w is not None, dbias=b is not None, dgate=g is not None)
    for k, there in names.items():
        if there:
            close(d[k], gr[k], gm[k], k)
        else:
            assert d[k] is None
    again = mixer.norm_bwd(x, w, b, g, stats, dy, kind=kind)
    for k, there in names.items():
        assert not there or torch.equal(d[k], again[k]), k


def test_norm_large_offset():
    """Rows far from zero: the variance is taken about the mean."""
    x = torch.randn(64, 1024, device="cuda") + 1000
    y, _ = mixer.norm_fwd(x, eps=0.0)
    want, _ = ref.norm(f64(x), None, None, None, 0.0, False)
    # the mean of 1024 values near 1000 is off by at most 2^-24 * 1000 * (10 roundings)
    assert np.abs(f64(y) - want).max() <= 1000 * 10 * 2.0 ** -24 + 2.0 ** -18


# ------------------------------------------------------------------------------------------------ scan

SCAN = [  # lengths, packed, H, G, P, N, state, skip, softplus, extra columns
    ([1], False, 1, 1, 64, 64, True, True, True, 0),
    ([2, 2], False, 2, 1, 16, 16, False, False, True, 0),
    ([63], False, 2, 2, 64, 128, True, True, True, 8),
    ([64, 64], False, 3, 1, 64, 64, True, False, False, 0),
    ([65], False, 4, 2, 32, 48, False, True, True, 16),
    ([130, 130], False, 2, 1, 128, 128, True, True, True, 0),
    ([200], False, 2, 1, 7, 5, True, True, True, 0),
    ([129], False, 1, 1, 256, 32, True, True, True, 0),
    ([100], False, 6, 3, 40, 100, True, True, False, 3),
    ([700], False, 2, 1, 64, 128, True, True, True, 0),
    ([0, 1, 64, 0, 65, 300, 3], True, 4, 2, 64, 64, True, True, True, 0),
    ([2, 500, 61], True, 2, 1, 64, 128, False, False, True, 8),
    ([0, 0], False, 2, 1, 64, 64, True, True, True, 0),
]


def scan_inputs(lens, packed, H, G, P, N, state, skip, extra, dtype, softplus, seed):
    r = rand(seed, dtype)
    n, T = len(lens), sum(lens) if packed else lens[0]
    lead = (1 if packed else n, T)
    f = torch.float32
    wide = r(*lead, H * P + 2 * G * N + extra)
    x = wide[..., :H * P].unflatten(2, (H, P))
    B = wide[..., H * P:H * P + G * N].unflatten(2, (G, N))
    C = wide[..., H * P + G * N:H * P + 2 * G * N].unflatten(2, (G, N))
    if not extra:
        x, B, C = (t.contiguous() for t in (x, B, C))
    raw, bias = r(*lead, H, t=f), r(H, t=f) - 2
    if not softplus:
        raw, bias = raw.abs() * 0.1, None
    A = -r(H, t=f).abs() * 4 - 0.1
    D = r(H, t=f) if skip else None
    s0 = r(n, H, P, N, t=f) if state else None
    return dict(x=x, dt=raw, A=A, B=B, C=C, D=D, dt_bias=bias, initial_state=s0), r(*lead, H, P), r(n, H, P, N, t=f)


NAMES = ("x", "dt", "A", "B", "C", "D", "dt_bias", "initial_state")


def reference_args(d, i, at, softplus):
    one = lambda k: f64(d[k])                                                    # noqa: E731
    return (f64(d["x"][at]), f64(d["dt"][at]), one("A"), f64(d["B"][at]), f64(d["C"][at]), one("D"), one("dt_bias"),
            None if d["initial_state"] is None else f64(d["initial_state"][i]), softplus)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,packed,H,G,P,N,state,skip,softplus,extra", SCAN)
def test_scan(lens, packed, H, G, P, N, state, skip, softplus, extra, dtype):
    d, dy, dsf = scan_inputs(lens, packed, H, G, P, N, state, skip, extra, dtype, softplus, sum(lens) + P + N)
    seqs, cu = sequences(lens, packed)
    y, sf = mixer.scan_fwd(**d, cu_seqlens=cu, softplus=softplus)
    g = mixer.scan_bwd(*(d[k] for k in NAMES), dy, dsf, cu_seqlens=cu, softplus=softplus)
    heads = ("dA", "dD", "ddt_bias")
    want, mag = {k: np.zeros(H) for k in heads}, {k: np.zeros(H) for k in heads}
    for i, at in seqs:
        args = reference_args(d, i, at, softplus)
        (yr, sr), (ym, sm) = (ref.scan(*args, mag=m) for m in (False, True))
        close(y[at], yr, ym, "y", split=True)
        close(sf[i], sr, sm, "final_state")
        gr, gm = (ref.scan_grads(*args, f64(dy[at]), f64(dsf[i]), mag=m) for m in (False, True))
        for k in ("dx", "dB", "dC"):
            close(g[k][at], gr[k], gm[k], k, split=True)
        close(g["ddt"][at], gr["ddt"], gm["ddt"], "ddt")
        close(g["d_initial_state"][i], gr["d_initial_state"], gm["d_initial_state"], "d_initial_state")
        for k in heads:
            want[k], mag[k] = want[k] + gr[k], mag[k] + gm[k]
    for k in heads:
        if g[k] is not None:
            close(g[k], want[k], mag[k], k)
    assert (g["dD"] is None) == (not skip) and (g["ddt_bias"] is None) == (not softplus)
    again = mixer.scan_bwd(*(d[k] for k in NAMES), dy, dsf, cu_seqlens=cu, softplus=softplus)
    for k in g:
        assert g[k] is None or torch.equal(g[k], again[k]), (k, "differs from run to run")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,P,N", [(4, 2, 64, 128), (3, 1, 20, 16), (2, 1, 7, 5), (1, 1, 256, 100)])
def test_scan_steps_equal_the_definition(H, G, P, N, dtype):
    """Single tokens from a prompt's state, in place and into another state."""
    d, _, _ = scan_inputs([80, 80], False, H, G, P, N, True, True, 0, dtype, True, P + N)
    cut = lambda t, s: t[:, s].contiguous()                                      # noqa: E731
    seq = ("x", "dt", "B", "C")
    first = {k: cut(v, slice(0, 70)) if k in seq else v for k, v in d.items()}
    _, state = mixer.scan_fwd(**first, softplus=True)
    ys = []
    for t in range(70, 80):
        one = {k: cut(v, t) if k in seq else v for k, v in d.items() if k != "initial_state"}
        before, other = state.clone(), torch.empty_like(state)
        y1 = mixer.scan_step(**one, state=state, softplus=True, state_out=other)
        assert torch.equal(state, before)
        y2 = mixer.scan_step(**one, state=state, softplus=True)
        assert torch.equal(y1, y2) and torch.equal(state, other)
        ys.append(y1)
    for i in range(2):
        args = reference_args(d, i, (i,), True)
        (yr, sr), (ym, sm) = (ref.scan(*args, mag=m) for m in (False, True))
        close(state[i], sr, sm, "state")
        close(torch.stack(ys, 1)[i], yr[70:], ym[70:], "y")


def test_scan_decay_that_wipes_the_state():
    """A time step that resets the state leaves what comes after it exact (prefix sums near -10^4)."""
    d, dy, dsf = scan_inputs([100], False, 2, 1, 64, 64, True, True, 0, "f32", False, 3)
    d["dt"][0, 40] = 4000.0
    d["x"][0, 40] *= 1e-3
    y, sf = mixer.scan_fwd(**d)
    g = mixer.scan_bwd(*(d[k] for k in NAMES), dy, dsf)
    args = reference_args(d, 0, (0,), False)
    (yr, sr), (ym, sm) = (ref.scan(*args, mag=m) for m in (False, True))
    close(y[0], yr, ym, "y")
    close(sf[0], sr, sm, "state")
    gr, gm = (ref.scan_grads(*args, f64(dy[0]), f64(dsf[0]), mag=m) for m in (False, True))
    for k in ("dx", "dB", "dC", "ddt"):
        close(g[k][0], gr[k], gm[k], k)


# --------------------------------------------------------------------- padding behind the last sequence; many rows

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tokens_behind_the_last_sequence(monkeypatch, dtype):
    """A packed batch in a longer buffer: its results are those without the padding, bit for bit (the padding crosses no
    multiple of 128 tokens, so the tiles are the same), and the padding's rows of the outputs stay as they are."""
    lens, pad = [70, 1, 0, 130], 37
    T, H, G, P, N = sum(lens), 8, 2, 48, 24
    _, cu = sequences(lens, True)
    r = rand(77, dtype)
    nan = lambda t: torch.cat([t, torch.full_like(t[:, :1], float("nan")).expand(-1, pad, *t.shape[2:])], 1)     # noqa: E731
    scan = dict(x=r(1, T, H, P), dt=r(1, T, H, t=torch.float32), B=r(1, T, G, N), C=r(1, T, G, N), dy=r(1, T, H, P))
    fixed = dict(A=-r(H, t=torch.float32).abs() - 0.1, D=r(H, t=torch.float32), dt_bias=r(H, t=torch.float32) - 2)
    conv = dict(x=r(1, T, 72), dy=r(1, T, 72))
    w, b = r(72, 4), r(72)
    empty = torch.empty

    def sevens(*shape, **kw):
        t = empty(*shape, **kw)
        return t.fill_(7) if t.dtype != torch.uint8 else t

    def run(s, c):
        y, S = mixer.scan_fwd(s["x"], s["dt"], fixed["A"], s["B"], s["C"], fixed["D"], fixed["dt_bias"], None, cu, True)
        g = mixer.scan_bwd(s["x"], s["dt"], fixed["A"], s["B"], s["C"], fixed["D"], fixed["dt_bias"], None, s["dy"],
                           cu_seqlens=cu, softplus=True)
        z, rows = mixer.conv_fwd(c["x"], w, b, None, cu, "silu")
        h = mixer.conv_bwd(c["x"], w, b, None, c["dy"], cu_seqlens=cu, activation="silu")
        tokens = [y, g["dx"], g["dB"], g["dC"], g["ddt"], z, h["dx"]]
        return tokens, [S, g["dA"], g["dD"], g["ddt_bias"], g["d_initial_state"], rows, h["dweight"], h["dbias"],
                        h["d_initial_state"]]
    want, want_rest = run(scan, conv)
    padded = [{k: nan(v) for k, v in d.items()} for d in (scan, conv)]
    monkeypatch.setattr(torch, "empty", sevens)
    got, got_rest = run(*padded)
    for a, e in zip(got, want):
        assert torch.equal(a[:, :T], e) and (a[:, T:] == 7).all()
    for a, e in zip(got_rest, want_rest):
        assert torch.equal(a, e) and torch.isfinite(a).all()


def test_norm_of_more_rows_than_a_launch_is_wide():
    """2^27 + 3 rows of 3 values, 16 to a workgroup: 2^23 + 1 workgroups of 256 threads, past the 2^32 of one dimension of a
    launch.  Every row is that of its first copy."""
    rows, D = (1 << 27) + 3, 3
    base = rand(78, "bf16")(1, D)
    y, stats = mixer.norm_fwd(base.expand(rows, D).contiguous())
    one, first = mixer.norm_fwd(base)
    assert (y == one).all() and (stats == first).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_workspaces_are_whole(dtype):
    """A workspace that is a view with gaps or one element expanded is refused before any launch."""
    r = rand(79, dtype)
    x, w, dy = r(2, 40, 24), r(24, 4), r(2, 40, 24)
    nbytes = mixer.conv_workspace_bytes(2, 40, 24, 4)
    for ws in (torch.zeros(1, dtype=torch.uint8, device="cuda").expand(nbytes),
               torch.zeros(2 * nbytes, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError):
            mixer.conv_bwd(x, w, None, None, dy, workspace=ws)
    with pytest.raises(ValueError):
        mixer.conv_bwd(x, w, None, None, dy, workspace=torch.zeros(nbytes, dtype=torch.uint8))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [1, 3, 5, 9, 15, 17, 31, 63, 65, 127, 129, 1023, 2047, 2049, 8191])
def test_norm_rows_of_any_width(D, dtype):
    """Widths about the pieces' and the lanes' edges, the rows between other values that must stay out of the results."""
    r = rand(80 + D, dtype)
    rows = 5
    x, g = r(rows, D + 3)[:, 1:D + 1], r(rows, D + 1)[:, :D]
    w, b, dy = r(D), r(D), r(rows, D)
    y, stats = mixer.norm_fwd(x, w, b, g)
    d = mixer.norm_bwd(x, w, b, g, stats, dy)
    y2, stats2 = mixer.norm_fwd(x.contiguous(), w, b, g.contiguous())
    assert torch.equal(y, y2) and torch.equal(stats, stats2)
    assert all(torch.equal(d[k], v) for k, v in mixer.norm_bwd(x.contiguous(), w, b, g.contiguous(), stats, dy).items())
    n = lambda t: t.double().cpu().numpy()                                       # noqa: E731
    xs, mag = n(x), np.abs(n(x)) + np.abs(n(x)).mean(1, keepdims=True)
    rs = 1 / np.sqrt(((xs - xs.mean(1, keepdims=True)) ** 2).mean(1, keepdims=True) + 1e-5)
    gate = n(g) / (1 + np.exp(-n(g)))
    want = ((xs - xs.mean(1, keepdims=True)) * rs * n(w) + n(b)) * gate
    close(y, want, (mag * rs * np.abs(n(w)) + np.abs(n(b))) * np.abs(gate), "y")
