"""The operators around the recurrence as a block uses them: convolution, scan and gated norm together, training and
serving; the layer's options; captured graphs; streams."""
import copy

import numpy as np
import pytest
import torch

from paper_2606_08804_amd import layer, mixer
from tests import mixer_oracle, oracle_binding
from tests.gpu_helpers import TOL, normwise

pytestmark = pytest.mark.gpu

H, G, P, N, W = 4, 2, 32, 16, 4
WIDTH = H * P + 2 * G * N


def inputs(B, T, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)                                      # noqa: E731
    act = dict(u=r(B, T, WIDTH), gate=r(B, T, H, P), conv_w=0.5 * r(WIDTH, W), conv_b=0.1 * r(WIDTH), norm_w=1 + 0.1 * r(P))
    f32 = dict(dt=r(B, T, H), A=-r(H).abs() - 0.2, D=r(H), dt_bias=r(H) - 2)
    return {k: v.to(dtype).cuda() for k, v in act.items()} | {k: v.cuda() for k, v in f32.items()}


def split(c):
    B, T = c.shape[:2]
    x, b, m = c.split([H * P, G * N, G * N], dim=-1)
    return x.view(B, T, H, P), b.view(B, T, G, N), m.view(B, T, G, N)


def block(d, ops, cu=None, conv_state=None, state=None):
    c, conv_state = ops.causal_conv(d["u"], d["conv_w"], d["conv_b"], conv_state, cu, "silu")
    x, b, m = split(c)
    y, state = ops.selective_scan(x, d["dt"], d["A"], b, m, d["D"], d["dt_bias"], state, cu, True)
    return ops.row_norm(y, d["norm_w"], None, d["gate"], kind="rms"), conv_state, state


@pytest.mark.parametrize("dtype,packed", [(torch.bfloat16, False), (torch.float32, True)])
def test_training(monkeypatch, dtype, packed):
    """Output and gradients of the three in a row: bit for bit those of the calls made one by one, and in fp32 those of
    the same chain in 64 bits (normwise, 1e-4 as everywhere for fp32)."""
    B, T = (1, 203) if packed else (2, 130)
    cu = torch.tensor([0, 64, 64, 70, 203], dtype=torch.int32) if packed else None
    cg = None if cu is None else cu.cuda()
    d = inputs(B, T, dtype, 7)
    dy = torch.randn(B, T, H, P, generator=torch.Generator().manual_seed(8)).to(dtype)
    leaves = {k: v.clone().requires_grad_() for k, v in d.items()}
    y, _, _ = block(leaves, layer, cg)
    y.backward(dy.cuda())

    c, _ = mixer.conv_fwd(d["u"], d["conv_w"], d["conv_b"], None, cg, "silu")
    x, b, m = split(c)
    o, _ = mixer.scan_fwd(x, d["dt"], d["A"], b, m, d["D"], d["dt_bias"], None, cg, True)
    n, st = mixer.norm_fwd(o, d["norm_w"], None, d["gate"], kind="rms")
    gn = mixer.norm_bwd(o, d["norm_w"], None, d["gate"], st, dy.cuda(), kind="rms")
    gs = mixer.scan_bwd(x, d["dt"], d["A"], b, m, d["D"], d["dt_bias"], None, gn["dx"], None, cg, True)
    dc = torch.cat([gs["dx"].flatten(2), gs["dB"].flatten(2), gs["dC"].flatten(2)], -1)
    gc = mixer.conv_bwd(d["u"], d["conv_w"], d["conv_b"], None, dc, None, cg, "silu")
    assert torch.equal(y, n)
    want = dict(u=gc["dx"], gate=gn["dgate"], conv_w=gc["dweight"], conv_b=gc["dbias"], norm_w=gn["dweight"], dt=gs["ddt"],
                A=gs["dA"], D=gs["dD"], dt_bias=gs["ddt_bias"])
    for k in leaves:
        assert torch.equal(leaves[k].grad, want[k]), k
    if dtype == torch.float32:
        monkeypatch.setattr(layer, "_mixer", mixer_oracle)
        ref = {k: v.detach().cpu().double().requires_grad_() for k, v in d.items()}
        yr, _, _ = block(ref, layer, cu)
        yr.backward(dy.double())
        off = {k: normwise(leaves[k].grad.double().cpu().numpy(), ref[k].grad.numpy()) for k in leaves}
        off["y"] = normwise(y.detach().double().cpu().numpy(), yr.detach().numpy())
        assert max(off.values()) <= TOL["f32"], off


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_prompt_then_single_tokens(dtype):
    """A prompt, then tokens one by one from its states, equal the whole sequence in one call: the same products in
    another order, rounded where the prompt rounds them."""
    B, T, start = 3, 90, 80
    d = inputs(B, T, dtype, 9)
    with torch.no_grad():
        want, conv_end, end = block(d, layer)
        head = {k: v[:, :start].contiguous() if k in ("u", "dt", "gate") else v for k, v in d.items()}
        _, conv_state, state = block(head, layer)
        got = []
        for t in range(start, T):
            c = mixer.conv_step(d["u"][:, t], d["conv_w"], d["conv_b"], conv_state, activation="silu")
            x, b, m = (v[:, 0] for v in split(c.unsqueeze(1)))
            y = mixer.scan_step(x, d["dt"][:, t].contiguous(), d["A"], b, m, state, d["D"], d["dt_bias"], softplus=True)
            got.append(mixer.norm_fwd(y, d["norm_w"], None, d["gate"][:, t].contiguous(), kind="rms")[0])
    tol = TOL["bf16" if dtype == torch.bfloat16 else "f32"]
    assert torch.equal(conv_state, conv_end)
    off = normwise(state.cpu().numpy(), end.cpu().numpy())
    assert off <= TOL["f32"], off
    off = normwise(torch.stack(got, 1).double().cpu().numpy(), want[:, start:].double().cpu().numpy())
    assert off <= tol, off


class Rounded(torch.autograd.Function):
    """Values, and gradients on the way back, as a bf16 tensor holds them."""

    @staticmethod
    def forward(ctx, x):
        return x.bfloat16().double()

    @staticmethod
    def backward(ctx, d):
        return d.bfloat16().double()


class RoundedLinear(torch.nn.Module):
    def __init__(self, linear):
        super().__init__()
        self.weight = linear.weight

    def forward(self, x):
        return Rounded.apply(torch.nn.functional.linear(x, self.weight))


@pytest.mark.parametrize("conv,norm,gate,packed", [(4, "rms", True, False), (3, "layer", False, True)])
def test_layer_options(monkeypatch, conv, norm, gate, packed):
    """The layer with its options against itself in 64 bits.  How far a bf16 layer may be off is taken from the formulas
    themselves: the 64-bit layer again, with what its stages hand on (projections, convolution, recurrence, norm, and
    the gradients there) rounded to bf16.  The kernels make those roundings and smaller ones; two sets of the same
    roundings put the largest error at most 2.5 times apart, and a result is rounded once more, by 2^-8."""
    torch.manual_seed(61)
    m = layer.QDeltaLayer(256, 2, 128, 128, conv_size=conv, out_norm=norm, out_gate=gate).to(torch.bfloat16)
    refs = [copy.deepcopy(m).double() for _ in range(2)]
    g = torch.Generator().manual_seed(62)
    B, T = (1, 270) if packed else (2, 150)
    h, dy = (torch.randn(B, T, 256, generator=g).to(torch.bfloat16) for _ in range(2))
    cu = torch.tensor([0, 70, 71, 270], dtype=torch.int32) if packed else None
    mg, hg = m.cuda(), h.cuda().requires_grad_()
    y = mg(hg, cu_seqlens=None if cu is None else cu.cuda())
    y.backward(dy.cuda())
    torch.cuda.synchronize()
    got = {"y": y.detach(), "h": hg.grad} | {k: p.grad for k, p in mg.named_parameters()}

    monkeypatch.setattr(layer, "_binding", oracle_binding)
    monkeypatch.setattr(layer, "_mixer", mixer_oracle)
    exact = []
    for i, ref in enumerate(refs):
        if i:
            for name in [n for n, c in ref.named_children() if isinstance(c, torch.nn.Linear)]:
                setattr(ref, name, RoundedLinear(getattr(ref, name)))
            conv_f, chunk_f, norm_f = layer.causal_conv, layer.qdelta_chunk, layer.row_norm
            first = lambda f: lambda *a, **k: (lambda r: (Rounded.apply(r[0]),) + r[1:])(f(*a, **k))    # noqa: E731
            monkeypatch.setattr(layer, "causal_conv", first(conv_f))
            monkeypatch.setattr(layer, "qdelta_chunk", first(chunk_f))
            monkeypatch.setattr(layer, "row_norm", lambda *a, **k: Rounded.apply(norm_f(*a, **k)))
        hr = h.double().requires_grad_()
        yr = ref(hr, cu_seqlens=cu)
        yr.backward(dy.double())
        exact.append({"y": yr.detach(), "h": hr.grad} | {k: p.grad for k, p in ref.named_parameters()})
    want, noisy = exact
    off = {}
    for k in got:
        # the scalar bias's gradient sums every (token, head) with cancellation: one bf16 rounding of each summand
        room = 2.5 * normwise(noisy[k].numpy(), want[k].numpy()) + 2.0 ** -8
        off[k] = normwise(got[k].double().cpu().numpy(), want[k].numpy()) / room
    off.pop("lambda_bias")               # compared by its summands in tests/test_gpu_layer.py
    assert max(off.values()) <= 1, off


def calls(d, dy, cu):
    """Everything that a training step and a decode step launch, from fixed inputs to a dict of outputs."""
    c, cs = mixer.conv_fwd(d["u"], d["conv_w"], d["conv_b"], None, cu, "silu")
    x, b, m = split(c)
    y, s = mixer.scan_fwd(x, d["dt"], d["A"], b, m, d["D"], d["dt_bias"], None, cu, True)
    o, st = mixer.norm_fwd(y, d["norm_w"], None, d["gate"], kind="rms")
    gn = mixer.norm_bwd(y, d["norm_w"], None, d["gate"], st, dy, kind="rms")
    gs = mixer.scan_bwd(x, d["dt"], d["A"], b, m, d["D"], d["dt_bias"], None, gn["dx"], None, cu, True)
    dc = torch.cat([gs["dx"].flatten(2), gs["dB"].flatten(2), gs["dC"].flatten(2)], -1)
    gc = mixer.conv_bwd(d["u"], d["conv_w"], d["conv_b"], None, dc, None, cu, "silu")
    n = s.shape[0]
    c1 = mixer.conv_step(d["u"][0, :n], d["conv_w"], d["conv_b"], cs, activation="silu", state_out=torch.empty_like(cs))
    x1, b1, m1 = (v[0] for v in split(c1.unsqueeze(0)))
    y1 = mixer.scan_step(x1, d["dt"][0, :n].contiguous(), d["A"], b1, m1, s, d["D"], d["dt_bias"], softplus=True,
                         state_out=torch.empty_like(s))
    out = dict(o=o, s=s, cs=cs, y1=y1)
    for name, g in (("norm", gn), ("scan", gs), ("conv", gc)):
        out |= {f"{name}.{k}": v for k, v in g.items() if v is not None}
    return out


@pytest.mark.parametrize("T", [50, 900])             # whole sequences; sequences cut into segments
def test_captured_graph_equals_eager(T):
    d = inputs(1, T, torch.bfloat16, 11)
    cu = torch.tensor([0, 10, 10, T], dtype=torch.int32, device="cuda")
    dy = torch.randn(1, T, H, P, generator=torch.Generator().manual_seed(12)).bfloat16().cuda()
    want = {k: v.clone() for k, v in calls(d, dy, cu).items()}
    cap, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    cap.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(cap):
        calls(d, dy, cu)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=cap):
            out = calls(d, dy, cu)
    torch.cuda.current_stream().wait_stream(cap)
    for rep in range(4):
        for v in out.values():
            v.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k, v in out.items():
            assert torch.equal(v, want[k]), (rep, k)
        assert torch.isfinite(torch.randn(1 << 16, device="cuda").sum())      # eager work between replays


def test_two_streams_at_once():
    """Calls of different sizes on two streams, their workspaces their own, equal the calls one after the other."""
    jobs = [(inputs(1, T, torch.bfloat16, T), torch.tensor([0, 10, 10, T], dtype=torch.int32, device="cuda"),
             torch.randn(1, T, H, P, generator=torch.Generator().manual_seed(T)).bfloat16().cuda()) for T in (200, 700)]
    want = [{k: v.clone() for k, v in calls(d, dy, cu).items()} for d, cu, dy in jobs]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in jobs], []
    for s, (d, cu, dy) in zip(streams, jobs):
        with torch.cuda.stream(s):
            got.append(calls(d, dy, cu))
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        for k in b:
            assert torch.equal(a[k], b[k]), k


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("what", ["x", "B", "C", "dt"])
def test_scan_keeps_a_nan_to_what_it_enters(what, dtype):
    """Tokens before a NaN, other heads or components, and other sequences of the packed batch are as without it."""
    g = torch.Generator().manual_seed(13)
    r = lambda *s, t=torch.float32: torch.randn(*s, generator=g).to(t).cuda()           # noqa: E731
    d = dict(x=r(1, 200, 2, 64, t=dtype), dt=r(1, 200, 2).abs() * 0.1, A=-r(2).abs(), B=r(1, 200, 2, 32, t=dtype),
             C=r(1, 200, 2, 32, t=dtype), D=r(2))
    cu = torch.tensor([0, 150, 200], dtype=torch.int32, device="cuda")
    y, s = mixer.scan_fwd(**d, cu_seqlens=cu)
    bad = {k: v.clone() for k, v in d.items()}
    at, head = 75, 1
    (bad[what][0, at, head] if what == "dt" else bad[what][0, at, head, 5:6]).fill_(float("nan"))
    z, f = mixer.scan_fwd(**bad, cu_seqlens=cu)
    assert torch.equal(z[0, :at], y[0, :at]) and torch.equal(z[0, 150:], y[0, 150:]) and torch.equal(z[:, :, 0], y[:, :, 0])
    assert torch.equal(f[1], s[1]) and torch.equal(f[0, 0], s[0, 0])
    assert torch.isnan(z[0, at, head]).any()
    if what == "C":
        assert torch.equal(z[0, at + 1:], y[0, at + 1:]) and torch.equal(f, s)
    else:
        assert torch.isnan(f[0, head]).any()
    if what == "x":
        assert torch.isnan(z[0, at:150, head, 5]).all() and torch.isnan(f[0, head, 5]).all()
        z[0, :, head, 5], f[0, head, 5] = y[0, :, head, 5], s[0, head, 5]
        assert torch.equal(z, y) and torch.equal(f, s)


def test_packing_does_not_change_a_sequence():
    d = inputs(1, 300, torch.bfloat16, 15)
    c = mixer.conv_fwd(d["u"], d["conv_w"], d["conv_b"], activation="silu")[0]
    x, b, m = split(c)
    args = lambda s: (x[:, s], d["dt"][:, s].contiguous(), d["A"], b[:, s], m[:, s], d["D"], d["dt_bias"])   # noqa: E731
    cu = torch.tensor([0, 33, 33, 300], dtype=torch.int32, device="cuda")
    y, s = mixer.scan_fwd(*args(slice(0, 300)), cu_seqlens=cu, softplus=True)
    for i, (a, e) in enumerate([(0, 33), (33, 33), (33, 300)]):
        if e > a:
            yi, si = mixer.scan_fwd(*args(slice(a, e)), softplus=True)
            assert normwise(s[i].cpu().numpy(), si[0].cpu().numpy()) <= 2.0 ** -20       # segments may be cut elsewhere
            assert normwise(y[0, a:e].float().cpu().numpy(), yi[0].float().cpu().numpy()) <= 2.0 ** -7
        else:
            assert not s[i].any()
    assert np.isfinite(y.float().cpu().numpy()).all()
