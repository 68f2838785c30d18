"""Operators around the recurrence at sizes that enter every loop of their kernels: several turns of a tile and several
tiles a wave (convolution), several rows a row group for every number of lanes (norm), several heads and tiles of heads a
workgroup (scan), against 64-bit forms on the GPU.  Each case names the plan that the launch rules give it (for 256 CUs) and
checks it against the size of the workspace, so that a change of a rule cannot move a test off its path unseen.

Tolerances as in test_gpu_mixer (an output is rounded once, eps / 2 of its value, after fp32 sums of terms whose absolute
values add up to `mag`: K = 2^-18, 64 roundings).  Sums over all tokens or rows have more: a wave's tokens (64 at most), four
waves, the workgroups by 16 (64 at most) and 16, beside their terms' own: below 256, 2^-16."""
import math

import pytest
import torch

from paper_2606_08804_amd import mixer

pytestmark = pytest.mark.gpu

K32, KSUM = 2.0 ** -18, 2.0 ** -16
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def close(got, want, mag, what, k=K32):
    assert got.shape == want.shape, (what, got.shape, want.shape)
    tol = torch.finfo(got.dtype).eps / 2 * want.abs() * (1 + k) + k * mag + 1e-30
    assert torch.isfinite(got).all(), (what, "not finite")
    worst = float(((got.double() - want).abs() / tol).max()) if got.numel() else 0.0
    assert worst <= 1, (what, worst)


def rand(seed, dtype):
    g = torch.Generator("cuda").manual_seed(seed)
    return lambda *s, scale=1.0, t=None: (torch.randn(s, generator=g, device="cuda") * scale).to(t or TYPES[dtype])


def up(a, b):
    return -(-a // b)


class Padded:
    """A packed batch [1, T, ...] as sequences [n, longest, ...] in 64 bits, zeros behind each, and back; a dense batch as it
    is.  `real` is [n, longest]."""

    def __init__(self, lens, packed):
        self.packed, self.lens = packed, torch.tensor(lens, device="cuda")
        at = torch.arange(max(lens), device="cuda")
        self.real = at < self.lens[:, None]
        self.cu = torch.tensor([0, *torch.tensor(lens).cumsum(0).tolist()], dtype=torch.int32, device="cuda") if packed else None

    def __call__(self, t):
        if not self.packed:
            return t.double()
        out = torch.zeros(self.real.shape + t.shape[2:], dtype=torch.float64, device="cuda")
        out[self.real] = t[0].double()
        return out

    def back(self, t):
        return t[self.real].unsqueeze(0) if self.packed else t


def sigmoid(u):
    return 1 / (1 + torch.exp(-u))


# ------------------------------------------------------------------------------------------------ convolution

def conv64(x, w, b, s0, dy, dsf, pad, mag):
    f = torch.abs if mag else (lambda t: t)
    x, dy, w, b = pad(x), pad(dy), w.double(), b.double()
    n, T, D = x.shape
    W = w.shape[1]
    ext = torch.cat([s0.double(), x], 1)
    u = b + sum(ext[:, j:j + T] * w[:, j] for j in range(W))
    terms = b.abs() + sum((ext[:, j:j + T] * w[:, j]).abs() for j in range(W)) if mag else None
    sg = sigmoid(u)
    du = dy * sg * (1 + u * (1 - sg))
    if mag:                                    # |SiLU'| <= 1.1 and |SiLU''| <= 0.5 on the error of u
        du = du.abs() + dy.abs() * terms
    rows = (pad.lens[:, None] + torch.arange(W - 1, device="cuda"))[:, :, None].expand(-1, -1, D)
    dext = torch.zeros_like(ext).scatter_add_(1, rows, f(dsf.double()))
    dw = torch.zeros_like(w)
    for j in range(W):
        dext[:, j:j + T] += f(w[:, j] * du)
        dw[:, j] = f(du * ext[:, j:j + T]).sum((0, 1))
    return dict(y=pad.back(1.1 * terms if mag else u * sg), state=torch.gather(ext, 1, rows), dx=pad.back(dext[:, W - 1:]),
                dweight=dw, dbias=f(du).sum((0, 1)), d_initial_state=dext[:, :W - 1])


def conv_plan(lens, packed, D, dtype):
    """Tile of the forward, tile and turns of the backward, workgroups for a group of its channels."""
    tokens, nv = sum(lens), up(D, 8 if dtype == "bf16" else 4)
    slots = lambda L: tokens // L + len(lens) if packed else len(lens) * up(lens[0], L)       # noqa: E731
    L, tile = 64, 32
    while L > 8 and tokens // L * nv < 1 << 17:
        L //= 2
    while tile > 8 and slots(tile) * up(D, 256) < 2048:
        tile //= 2
    groups, most = up(slots(tile), 4), 2048 if D < 512 else max(64, (1 << 20) // D)
    turns = max(1, up(groups, most))
    return L, tile, turns, up(groups, turns)


def ragged(n, most, seed, total=None):
    lens = torch.randint(0, most + 1, (n,), generator=torch.Generator().manual_seed(seed)).tolist()
    lens[:3] = [most, 0, 1]
    return lens if total is None else lens + [max(total - sum(lens), 1)]


CONV = [  # lengths, packed, D, W, type; tiles of the forward and of the backward, its turns
    ([4100] * 4, False, 4104, 4, "bf16", (64, 32, 1)),
    ([4100] * 2, False, 4104, 3, "bf16", (32, 32, 1)),
    ([4100], False, 4101, 4, "bf16", (16, 32, 1)),
    (ragged(40, 300, 1, 16500), True, 4101, 4, "bf16", (64, 32, 1)),
    ([4100] * 2, False, 4104, 4, "f32", (64, 32, 1)),
    ([4100], False, 4101, 2, "f32", (32, 32, 1)),
    (ragged(30, 200, 2, 8300), True, 4104, 4, "f32", (64, 32, 1)),
    ([700] * 2, False, 8192, 4, "bf16", (8, 16, 1)),
    ([700] * 2, False, 8192, 4, "f32", (16, 16, 1)),
    (ragged(1500, 5, 3), True, 4096, 4, "bf16", (8, 32, 2)),
    (ragged(1500, 5, 4), True, 4099, 4, "f32", (16, 32, 2)),
    (ragged(700, 70, 5), True, 6000, 3, "bf16", (64, 32, 3)),
]


@pytest.mark.parametrize("lens,packed,D,W,dtype,plan", CONV)
def test_conv(lens, packed, D, W, dtype, plan):
    groups = conv_plan(lens, packed, D, dtype)
    assert groups[:3] == plan
    T = sum(lens) if packed else lens[0]
    assert mixer.conv_workspace_bytes(len(lens), T, D, W, packed) == groups[3] * (W + 1) * D * 4
    r = rand(D + W, dtype)
    N, lead = len(lens), (1 if packed else len(lens), T)
    x, w, b, s0 = r(*lead, D), r(D, W, scale=0.5), r(D, scale=0.1), r(N, W - 1, D)
    dy, dsf = r(*lead, D), r(N, W - 1, D)
    pad = Padded(lens, packed)
    y, state = mixer.conv_fwd(x, w, b, s0, cu_seqlens=pad.cu, activation="silu")
    g = mixer.conv_bwd(x, w, b, s0, dy, dsf, cu_seqlens=pad.cu, activation="silu")
    want, mag = (conv64(x, w, b, s0, dy, dsf, pad, m) for m in (False, True))
    close(y, want["y"], mag["y"], "y")
    assert torch.equal(state.double(), want["state"]), "the state is a copy"
    for k in g:
        close(g[k], want[k], mag[k], k, KSUM if k in ("dweight", "dbias") else K32)
    again = mixer.conv_bwd(x, w, b, s0, dy, dsf, cu_seqlens=pad.cu, activation="silu")
    assert all(torch.equal(g[k], again[k]) for k in g), "differs from run to run"


# ------------------------------------------------------------------------------------------------ norm

def norm64(x, w, b, g, eps, rms, dy, mag):
    f = torch.abs if mag else (lambda t: t)
    x, w, dy = x.double(), w.double(), dy.double()
    b, g = (None if t is None else t.double() for t in (b, g))
    mean = 0 * x[:, :1] if rms else x.mean(1, keepdim=True)
    r = ((x - mean).square().mean(1, keepdim=True) + eps).rsqrt()
    xh = (x - mean) * r
    if mag:                                    # x - mean is off relative to its terms, the mean relative to the mean of |x|
        xh = (x.abs() + x.abs().mean(1, keepdim=True)) * r
    lin = f(xh * w) + (0 if b is None else f(b))
    s = 1 if g is None else g * sigmoid(g)
    d = f(dy * s)
    res = dict(y=lin * (abs(s) if mag else s), dweight=f(d * xh).sum(0), dbias=None if b is None else d.sum(0), dgate=None)
    if g is not None:
        res["dgate"] = dy.abs() * lin * 1.1 if mag else dy * lin * sigmoid(g) * (1 + g * (1 - sigmoid(g)))
    e, sign = f(d * w), 1 if mag else -1
    res["dx"] = r * (e + sign * ((0 if rms else e.mean(1, keepdim=True)) + xh * (e * xh).mean(1, keepdim=True)))
    return res


def norm_lanes(D, dtype):
    nv = up(D, 8 if dtype == "bf16" else 4)
    return next((lanes, k) for lanes, k in ((8, 1), (16, 1), (32, 1), (64, 1), (64, 2), (64, 4), (256, 2), (256, 4), (256, 8))
                if nv <= lanes * k)


NORM = [(64, (8, 1), (16, 1)), (61, (8, 1), (16, 1)), (128, (16, 1), (32, 1)), (200, (32, 1), (64, 1)), (500, (64, 1), (64, 2)),
        (1000, (64, 2), (64, 4)), (1021, (64, 2), (64, 4)), (2048, (64, 4), (256, 2)), (2045, (64, 4), (256, 2)),
        (4096, (256, 2), (256, 4)), (4099, (256, 4), (256, 8)), (8192, (256, 4), (256, 8)), (8189, (256, 4), (256, 8)),
        (12, (8, 1), (8, 1))]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind,gate", [("layer", False), ("rms", True), ("layer", True), ("rms", False)])
@pytest.mark.parametrize("D,lanes16,lanes32", NORM)
def test_norm_several_rows_a_group(D, lanes16, lanes32, kind, gate, dtype):
    """Three rows for some row groups, two for others."""
    lanes, k = norm_lanes(D, dtype)
    assert (lanes, k) == (lanes16 if dtype == "bf16" else lanes32)
    per = 256 // lanes
    blocks = mixer.norm_workspace_bytes(1 << 20, D) // (8 * D)
    rows = 2 * blocks * per + blocks * per // 2 + 1
    assert mixer.norm_workspace_bytes(rows, D) == 8 * D * blocks
    r = rand(D, dtype)
    x, dy, w = r(rows, D) * 2 + 0.5, r(rows, D), r(D)
    b = r(D) if kind == "layer" else None
    g = r(rows, D) if gate else None
    eps = 1e-3
    y, stats = mixer.norm_fwd(x, w, b, g, eps=eps, kind=kind)
    got = mixer.norm_bwd(x, w, b, g, stats, dy, kind=kind)
    want, mag = (norm64(x, w, b, g, eps, kind == "rms", dy, m) for m in (False, True))
    close(y, want["y"], mag["y"], "y")
    for name in got:
        if got[name] is None:
            assert want[name] is None
        else:
            close(got[name], want[name], mag[name], name, KSUM if name in ("dweight", "dbias") else K32)
    again = mixer.norm_bwd(x, w, b, g, stats, dy, kind=kind)
    assert all(v is None or torch.equal(v, again[name]) for name, v in got.items()), "differs from run to run"


def test_norm_of_workgroups_past_one_dimension():
    """Rows of three bf16 values are one piece: eight lanes, 32 rows a workgroup.  A launch is 2^23 workgroups wide (2^31
    threads), so that of 32 x 2^23 + 3 rows the last three are in its second row of workgroups.  Equal, bit for bit, to calls
    on a sixteenth of the rows each."""
    D = 3
    lanes, _ = norm_lanes(D, "bf16")
    rows = 256 // lanes * (1 << 23) + 3
    g = torch.Generator("cuda").manual_seed(80)
    x = torch.randint(-300, 300, (rows, D), generator=g, device="cuda", dtype=torch.int16).bfloat16()
    y, stats = mixer.norm_fwd(x)
    part = 1 << 24
    for at in range(0, rows, part):
        one, st = mixer.norm_fwd(x[at:at + part])
        assert torch.equal(y[at:at + part], one) and torch.equal(stats[at:at + part], st), at
    assert not torch.equal(y[-1], y[-2])


# ------------------------------------------------------------------------------------------------ scan

def scan64(d, softplus, dy, dsf, pad):
    """The definition by tokens and its gradients, of all sequences side by side; ({name: result}, {name: mag})."""
    two = lambda t: torch.stack([t, t.abs()])                                    # noqa: E731
    x, raw, B, C, dyp = (pad(t) for t in (d["x"], d["dt"], d["B"], d["C"], dy))
    n, T, H, P = x.shape
    G, N = B.shape[2:]
    per = H // G
    A = d["A"].double()
    z = raw + (0 if d["dt_bias"] is None else d["dt_bias"].double())
    dt = (torch.logaddexp(z, torch.zeros_like(z)) if softplus else z) * pad.real[:, :, None]
    a = torch.exp(dt * A)
    x, B, C, dyp, dtm, D = two(x), two(B), two(C), two(dyp), two(dt), None if d["D"] is None else two(d["D"].double())
    Am = two(A)[:, None]
    wide = lambda t: t.repeat_interleave(per, 2)                                 # noqa: E731
    S = torch.zeros(2, n, H, P, N, dtype=torch.float64, device="cuda") if d["initial_state"] is None \
        else two(d["initial_state"].double())
    states, y = [S], torch.zeros_like(x)
    for t in range(T):
        S = a[:, t, :, None, None] * S + (dtm[:, :, t, :, None] * x[:, :, t])[..., None] * wide(B[:, :, t])[..., None, :]
        states.append(S)
        y[:, :, t] = (S * wide(C[:, :, t])[..., None, :]).sum(-1)
    if D is not None:
        y += D[:, None, None, :, None] * x
    Gr = torch.zeros_like(S) if dsf is None else two(dsf.double())
    dx, dd, dB, dC = torch.zeros_like(x), torch.zeros_like(dtm), torch.zeros_like(B), torch.zeros_like(C)
    dA = torch.zeros(2, H, dtype=torch.float64, device="cuda")
    groups = lambda t: t.reshape(2, n, G, per, N).sum(3)                         # noqa: E731
    for t in reversed(range(T)):
        gy = dyp[:, :, t, :, :, None]
        dC[:, :, t] = groups((gy * states[t + 1]).sum(3))
        Gr = Gr + gy * wide(C[:, :, t])[..., None, :]
        u = (Gr * wide(B[:, :, t])[..., None, :]).sum(-1)
        dx[:, :, t] = dtm[:, :, t, :, None] * u
        dB[:, :, t] = groups(dtm[:, :, t, :, None] * (x[:, :, t, :, :, None] * Gr).sum(3))
        dl = a[:, t] * (Gr * states[t]).sum((-1, -2))
        dd[:, :, t] = (x[:, :, t] * u).sum(-1) + Am * dl
        dA += (dtm[:, :, t] * dl).sum(1)
        Gr = a[:, t, :, None, None] * Gr
    if D is not None:
        dx += D[:, None, None, :, None] * dyp
    if softplus:
        dd = dd * sigmoid(z)
    dd = dd * pad.real[:, :, None]
    res = dict(y=y, state=states[-1], dx=dx, ddt=dd, dB=dB, dC=dC, dA=dA, dD=(dyp * x).sum((1, 2, 4)), ddt_bias=dd.sum((1, 2)),
               d_initial_state=Gr)
    return [{k: pad.back(v[i]) if k in ("y", "dx", "ddt", "dB", "dC") else v[i] for k, v in res.items()} for i in (0, 1)]


def scan_bytes(lens, packed, H, G, P, N, seg, splits):
    """Workspace of a backward with these segments (0: whole sequences) and shares of a chunk's heads."""
    r = lambda b: up(b, 256) * 256                                               # noqa: E731
    tokens = sum(lens)
    slots = lambda L: tokens // L + len(lens) if packed else len(lens) * up(lens[0], L)       # noqa: E731
    heads, tiles = slots(64) * H, up(P, 64)
    total = r(heads * 448 * 4) + 2 * r(heads * tiles * 64 * (64 if N <= 64 else 128) * 4) + r(heads * 32)
    if seg:
        total += 4 * r(slots(seg) * H * P * N * 4) + r(slots(seg) * H * 4)
    if splits > 1:
        total += 2 * r(splits * tokens * G * N * 4)
    return total


SCAN = [  # lengths, packed, H, G, P, N; tokens of a segment (fp32; bf16 has 512), workgroups that share a chunk's heads
    (ragged(130, 130, 6), True, 3, 1, 72, 24, 0, 1),             # three heads of two tiles
    (ragged(130, 130, 7), True, 4, 1, 64, 128, 0, 1),            # four heads, whole pieces
    (ragged(130, 130, 8), True, 3, 1, 66, 100, 0, 1),            # three heads of two tiles, rows that are no whole pieces
    ([100] * 50, False, 10, 2, 40, 48, 0, 2),                    # shares of two and three heads
    ([100] * 25, False, 8, 1, 130, 128, 0, 4),                   # shares of two heads of three tiles
    ([4100], False, 12, 4, 16, 16, 256, 1),                      # segments, three heads
    ([4100], False, 6, 2, 64, 128, 128, 2),                      # segments, shares of one and two heads
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,packed,H,G,P,N,seg,splits", SCAN)
def test_scan_several_heads_a_workgroup(lens, packed, H, G, P, N, seg, splits, dtype):
    T = sum(lens) if packed else lens[0]
    assert mixer.scan_workspace_bytes(len(lens), T, H, G, P, N, packed, True) == \
        scan_bytes(lens, packed, H, G, P, N, seg, splits)
    assert H // G > splits
    r, f32 = rand(H * P + N, dtype), torch.float32
    n, lead = len(lens), (1 if packed else len(lens), T)
    d = dict(x=r(*lead, H, P), dt=r(*lead, H, t=f32), A=-r(H, t=f32).abs() - 0.1, B=r(*lead, G, N), C=r(*lead, G, N),
             D=r(H, t=f32), dt_bias=r(H, t=f32) - 2, initial_state=r(n, H, P, N, t=f32))
    dy, dsf = r(*lead, H, P), r(n, H, P, N, t=f32)
    pad = Padded(lens, packed)
    y, state = mixer.scan_fwd(**d, cu_seqlens=pad.cu, softplus=True)
    back = lambda: mixer.scan_bwd(d["x"], d["dt"], d["A"], d["B"], d["C"], d["D"], d["dt_bias"], d["initial_state"], dy, dsf,     # noqa: E731
                                  cu_seqlens=pad.cu, softplus=True)
    got = back()
    want, mag = scan64(d, True, dy, dsf, pad)
    close(y, want["y"], mag["y"], "y")
    close(state, want["state"], mag["state"], "state")
    for k in got:
        close(got[k], want[k], mag[k], k)
    again = back()
    assert all(torch.equal(got[k], again[k]) for k in got), "differs from run to run"
    assert math.prod(got["dB"].shape) == T * lead[0] * G * N


def test_offsets_past_32_bits():
    """2.2e9 values of 8192 a token: the last tokens are those of calls on them alone, with the rows before them as the
    convolution's state and a time step that wipes the scan's.  Bit for bit where a value does not depend on where its tile or
    segment begins; the scan's by 2^-20 of the largest (states are put together in another order)."""
    g = torch.Generator("cuda").manual_seed(81)
    big = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)          # noqa: E731
    D, n, T = 8192, 1000, (1 << 18) + 4100
    x, w, b = big(1, T, D), big(D, 4), big(D)
    last = lambda t: t[:, -n:].contiguous()                                      # noqa: E731
    assert x[:, :-n].numel() > 1 << 31
    y, state = mixer.conv_fwd(x, w, b, activation="silu")
    dx = mixer.conv_bwd(x, w, b, None, x, activation="silu")["dx"]
    before = x[:, -n - 3:-n].contiguous()
    y1, state1 = mixer.conv_fwd(last(x), w, b, before, activation="silu")
    dx1 = mixer.conv_bwd(last(x), w, b, before, last(x), activation="silu")["dx"]
    assert torch.equal(last(y), y1) and torch.equal(state, state1) and torch.equal(last(dx), dx1)

    y, stats = mixer.norm_fwd(x, b)
    dx = mixer.norm_bwd(x, b, None, None, stats, x)["dx"]
    y1, stats1 = mixer.norm_fwd(last(x), b)
    assert torch.equal(last(y), y1) and torch.equal(last(stats), stats1)
    assert torch.equal(last(dx), mixer.norm_bwd(last(x), b, None, None, stats1, last(x))["dx"])

    H, N, at = 64, 16, T // 64 * 64 - 1024
    x = x.unflatten(2, (H, D // H))
    B, C, A = big(1, T, 1, N), big(1, T, 1, N), -torch.ones(H, device="cuda")
    dt = 0.1 * torch.rand(1, T, H, generator=g, device="cuda")
    dt[:, at] = 1000
    last = lambda t: t[:, at:].contiguous()                                      # noqa: E731
    far = lambda a, e: float((a.double() - e.double()).abs().max() / e.double().abs().max())   # noqa: E731
    y, state = mixer.scan_fwd(x, dt, A, B, C)
    y1, state1 = mixer.scan_fwd(last(x), last(dt), A, last(B), last(C))
    assert far(state, state1) <= 2.0 ** -20 and far(last(y), y1) <= 2.0 ** -7    # y: a bf16 rounding to the other side
    got = mixer.scan_bwd(x, dt, A, B, C, None, None, None, x)
    want = mixer.scan_bwd(last(x), last(dt), A, last(B), last(C), None, None, None, last(x))
    for k in ("dx", "dB", "dC"):
        assert far(last(got[k]), want[k]) <= 2.0 ** -7, k
    assert far(last(got["ddt"]), want["ddt"]) <= 2.0 ** -20
