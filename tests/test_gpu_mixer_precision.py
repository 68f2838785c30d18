"""What the operators around the recurrence hold in 32 bits, on inputs that show it: values whose result is known exactly."""
import pytest
import torch

from paper_2606_08804_amd import mixer

pytestmark = pytest.mark.gpu

# Just above the middle between the bf16 values 1 and 1 + 2^-7, by what only the 21st bit holds: it rounds up.  Cut to 16
# bits it is the middle itself, which goes to the even neighbour, 1.
V, PARTS, UP = 1 + 2.0 ** -8 + 2.0 ** -20, (1.0, 2.0 ** -8, 2.0 ** -20), 1 + 2.0 ** -7


@pytest.mark.parametrize("P,N", [(4, 4), (64, 64), (65, 128), (128, 72)])
def test_scan_in_bf16_takes_fp32_values_whole(P, N):
    """One token without decay (A = 0), one product of which is V: everything else is exact, so that the result is V,
    rounded once.  V is the state, the time step, the state's gradient, C . B and dy . x in turn."""
    def zeros(*shape, at=None, parts=None, dtype=torch.bfloat16):
        t = torch.zeros(shape, dtype=dtype, device="cuda")
        for i, v in enumerate(parts or ()):
            t.view(-1)[(at or 0) + i] = v
        return t
    f32, one = torch.float32, (1.0,)
    A = torch.zeros(1, device="cuda")
    p, n = P - 4, N - 4                                    # where the values stand: in the last tile
    sx, sb, ss = (1, 1, 1, P), (1, 1, 1, N), (1, 1, P, N)

    def fwd(x, dt, B, C, s0=None):
        y, _ = mixer.scan_fwd(zeros(*sx, at=p, parts=x), torch.full((1, 1, 1), dt, device="cuda"), A,
                              zeros(*sb, at=n, parts=B), zeros(*sb, at=n, parts=C), None, None,
                              zeros(*ss, at=p * N + n, parts=s0, dtype=f32) if s0 else None)
        return y.view(-1)[p].item()

    def bwd(x, B, C, dy, dsf=None):
        g = mixer.scan_bwd(zeros(*sx, at=p, parts=x), torch.ones(1, 1, 1, device="cuda"), A, zeros(*sb, at=n, parts=B),
                           zeros(*sb, at=n, parts=C), None, None, None, zeros(*sx, at=p, parts=dy),
                           zeros(*ss, at=p * N + n, parts=dsf, dtype=f32) if dsf else None)
        return g
    assert torch.tensor(V).bfloat16().item() == UP
    got = dict(state=fwd(None, 0.0, None, one, (V,)), step=fwd(one, V, one, one),
               scores=fwd(one, 1.0, (1.0, 1.0, 1.0), PARTS),
               dx_of_gradient=bwd(None, one, None, None, (V,))["dx"].view(-1)[p].item(),
               dx_of_scores=bwd(None, (1.0, 1.0, 1.0), PARTS, one)["dx"].view(-1)[p].item(),
               dB=bwd((1.0, 1.0, 1.0), None, one, PARTS)["dB"].view(-1)[n].item(),
               dC=bwd((1.0, 1.0, 1.0), one, None, PARTS)["dC"].view(-1)[n].item())
    assert got == {k: UP for k in got}


# An exponential good to one place (2^-23), 1 + it, a reciprocal good to one place and one or two products: below 2^-21.
K_EXP = 2.0 ** -21
POINTS = torch.cat([torch.linspace(-85, 0, 511), torch.linspace(0.01, 40, 129)])


def _off(got, want, scale=None):
    return float(((got.double().cpu() - want).abs() / (want.abs() if scale is None else scale).clamp(min=1e-37)).max())


@pytest.mark.parametrize("D", [POINTS.numel(), POINTS.numel() - 1])           # rows of whole pieces, and others
def test_silu_in_fp32_is_good_to_the_last_places(D):
    """SiLU and its derivative relative to their own size, far below zero too: the convolution with the taps 0 and 1,
    the norm of rows (1, -1) (mean 0, deviation 1) under the gate."""
    u = POINTS[:D].double()
    sg = 1 / (1 + torch.exp(-u))
    want, slope, terms = u * sg, sg * (1 + u * (1 - sg)), sg * (1 + u.abs())
    x = POINTS[:D].cuda()[None, None]
    w = torch.tensor([0.0, 1.0], device="cuda").repeat(D, 1)
    y, state = mixer.conv_fwd(x, w, activation="silu")
    assert _off(y[0, 0], want) <= K_EXP
    assert _off(mixer.conv_step(x[0], w, None, torch.zeros_like(state), activation="silu")[0], want) <= K_EXP
    dx = mixer.conv_bwd(x, w, None, None, torch.ones_like(x), activation="silu")["dx"]
    assert _off(dx[0, 0], slope, terms) <= 2 * K_EXP                  # two more roundings, and 1 - sg is off by one of 1
    rows = torch.tensor([1.0, -1.0], device="cuda").repeat(D, 1)
    gate = x[0, 0, :, None].expand(D, 2).contiguous()
    y, stats = mixer.norm_fwd(rows, gate=gate, eps=0.0)
    assert (stats == torch.tensor([0.0, 1.0], device="cuda")).all()
    assert _off(y[:, 0], want) <= K_EXP and _off(-y[:, 1], want) <= K_EXP
    dg = mixer.norm_bwd(rows, None, None, gate, stats, torch.ones_like(rows))["dgate"]
    assert _off(dg[:, 0], slope, terms) <= 2 * K_EXP


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_scan_decays_of_the_state_are_good_to_the_last_places(dtype):
    """A state of ones after one token that adds nothing is exp(dt A), for prompts, their state's gradient and single
    tokens; in fp32 the output of the token after one that came in is that as well."""
    H, P, N = 64, 4, 4
    A = -torch.linspace(0.125, 80, H).cuda()
    want = torch.exp(A.double().cpu())
    z = lambda *s, t=dtype: torch.zeros(s, dtype=t, device="cuda")                # noqa: E731
    ones = torch.ones(1, H, P, N, device="cuda")
    dt = torch.ones(1, 1, H, device="cuda")
    args = (z(1, 1, H, P), dt, A, z(1, 1, 1, N), z(1, 1, 1, N))
    _, s = mixer.scan_fwd(*args, initial_state=ones)
    g = mixer.scan_bwd(*args, None, None, ones, z(1, 1, H, P), ones)
    one = ones.clone()
    mixer.scan_step(*(t[0] if t.dim() > 1 else t for t in args), one)
    for got in (s, g["d_initial_state"], one):
        assert (got == got[:, :, :1, :1]).all() and _off(got[0, :, 0, 0], want) <= K_EXP
    if dtype == torch.float32:
        x, B, C = z(1, 2, H, P), z(1, 2, 1, N), z(1, 2, 1, N)
        x[:, 0], B[:, 0], C[:, 1, 0, 0] = 1, 1, 1
        y, _ = mixer.scan_fwd(x, dt.expand(1, 2, H).contiguous(), A, B, C)
        assert not y[:, 0].any() and _off(y[0, 1, :, 0], want) <= 2 * K_EXP       # products in three more roundings


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,H", [(50, 300), (1, 300), (1300, 3)])             # whole sequences; cut into segments
def test_scan_decays_of_prefix_sums_that_32_bits_round(T, H, dtype):
    """The state after T tokens that add nothing is exp(sum dt A) to its last places, also where that sum, here from -1 to
    -80, is no value of fp32 (rounded, it would be off by up to 2^-18): one exponential a chunk and a product a chunk of 21."""
    g = torch.Generator().manual_seed(T)
    dt = (0.5 + torch.rand(1, T, H, generator=g)) / T
    A = -torch.linspace(1, 80, H)
    want = torch.exp((dt.double() * A.double()).sum(1)[0])
    z = lambda *s, t=dtype: torch.zeros(s, dtype=t, device="cuda")                # noqa: E731
    P, N = 4, 4
    ones = torch.ones(1, H, P, N, device="cuda")
    args = (z(1, T, H, P), dt.cuda(), A.cuda(), z(1, T, 1, N), z(1, T, 1, N))
    _, s = mixer.scan_fwd(*args, initial_state=ones)
    back = mixer.scan_bwd(*args, None, None, ones, z(1, T, H, P), ones)["d_initial_state"]
    one = ones.clone()
    if T == 1:
        mixer.scan_step(*(t[0] if t.dim() > 1 else t for t in args), one)
    for got in (s, back, one) if T == 1 else (s, back):
        off = _off(got[0, :, 0, 0], want)
        assert (got == got[:, :, :1, :1]).all() and off <= 21 * 2.0 ** -23, off


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_scan_time_step_without_end(dtype):
    """An infinite time step forgets the state: decay 0, not NaN, in prompts and single tokens (x and B are zero where
    it stands, so that the products with it are NaN there and in what follows; the tokens before are untouched)."""
    g = torch.Generator().manual_seed(3)
    r = lambda *s, t=dtype: torch.randn(*s, generator=g).to(t).cuda()             # noqa: E731
    x, dt, B, C = r(1, 40, 2, 8), r(1, 40, 2, t=torch.float32).abs(), r(1, 40, 1, 8), r(1, 40, 1, 8)
    A = -torch.ones(2, device="cuda")
    y, _ = mixer.scan_fwd(x, dt, A, B, C)
    dt[0, 20, 1] = float("inf")
    z, s = mixer.scan_fwd(x, dt, A, B, C)
    assert torch.equal(z[:, :20], y[:, :20]) and torch.equal(z[:, :, 0], y[:, :, 0]) and torch.isfinite(s[0, 0]).all()


@pytest.mark.parametrize("T", [1, 50, 1300])
def test_scan_growth_past_fp32_is_not_finite(T):
    """dt A > 0 is not expected, and not refused.  A state that grows is exp(sum dt A); past fp32 it becomes an infinity of
    its sign, or, where that happens within a chunk whose weights overflow too (they meet the zeros of x), a NaN."""
    H, P, N = 2, 4, 4
    z = lambda *s: torch.zeros(s, device="cuda")                                 # noqa: E731
    dt, A = torch.full((1, T, H), 1.0 / T).cuda(), torch.tensor([80.0, 100.0]).cuda()
    s0 = torch.tensor([1.0, -1.0], device="cuda").repeat(2)[:, None].expand(1, H, P, N).contiguous()
    args = (z(1, T, H, P), dt, A, z(1, T, 1, N), z(1, T, 1, N))
    _, s = mixer.scan_fwd(*args, initial_state=s0)
    got = [s]
    if T == 1:
        got.append(s0.clone())
        mixer.scan_step(*(t[0] if t.dim() > 1 else t for t in args), got[1])
    want = torch.exp((dt.double().cpu() * A.double().cpu()).sum(1))[0, 0] * s0[0, 0].double().cpu()
    for s in got:
        assert _off(s[0, 0], want) <= 21 * 2.0 ** -23
        assert not torch.isfinite(s[0, 1]).any()
        if T != 50:
            assert torch.equal(s[0, 1], s0[0, 1] * float("inf"))
