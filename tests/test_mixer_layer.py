"""The differentiable operators around the recurrence and the layer's options that use them, on the CPU with the
kernels replaced by the plain 64-bit forms: gradcheck compares the gradients through the wiring with differences."""
import pytest
import torch

from paper_2606_08804_amd import layer
from tests import mixer_oracle, oracle_binding


@pytest.fixture(autouse=True)
def plain(monkeypatch):
    monkeypatch.setattr(layer, "_binding", oracle_binding)
    monkeypatch.setattr(layer, "_mixer", mixer_oracle)


def rand(seed):
    g = torch.Generator().manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)


def check(f, xs):
    live = [i for i, x in enumerate(xs) if x is not None]

    def g(*args):
        full = list(xs)
        for i, a in zip(live, args):
            full[i] = a
        return f(*full)
    assert torch.autograd.gradcheck(g, [xs[i].requires_grad_() for i in live], eps=1e-6, atol=1e-7, rtol=1e-6)


CU = torch.tensor([0, 2, 2, 7], dtype=torch.int32)


@pytest.mark.parametrize("packed,bias,state", [(False, True, True), (True, False, True), (True, True, False)])
def test_causal_conv(packed, bias, state):
    r = rand(1)
    B, T, N = (1, 7, 3) if packed else (2, 5, 2)
    xs = [r(B, T, 3), r(3, 4), r(3) if bias else None, r(N, 3, 3) if state else None]
    check(lambda *a: layer.causal_conv(*a, CU if packed else None, "silu"), xs)


@pytest.mark.parametrize("kind,gate,affine", [("layer", True, True), ("rms", False, True), ("layer", False, False)])
def test_row_norm(kind, gate, affine):
    r = rand(2)
    xs = [r(2, 3, 5), r(5) if affine else None, r(5) if affine and kind == "layer" else None, r(2, 3, 5) if gate else None]
    check(lambda *a: layer.row_norm(*a, eps=1e-3, kind=kind), xs)


@pytest.mark.parametrize("packed,extras", [(False, True), (True, True), (True, False)])
def test_selective_scan(packed, extras):
    r = rand(3)
    B, T, N, H, G = (1, 7, 3, 4, 2) if packed else (2, 5, 2, 4, 2)
    xs = [r(B, T, H, 3), r(B, T, H), -r(H).abs() - 0.1, r(B, T, G, 2), r(B, T, G, 2), r(H) if extras else None,
          r(H) if extras else None, r(N, H, 3, 2) if extras else None]
    check(lambda *a: layer.selective_scan(*a, CU if packed else None, True), xs)


@pytest.mark.parametrize("conv,norm,gate", [(4, "rms", True), (2, "layer", False), (3, None, False), (0, "rms", False)])
def test_layer_options(conv, norm, gate):
    torch.manual_seed(4)
    m = layer.QDeltaLayer(6, 2, 4, 3, conv_size=conv, out_norm=norm, out_gate=gate).double()
    names, params = zip(*[(n, p.detach().clone()) for n, p in m.named_parameters()])
    h = torch.randn(2, 4, 6, dtype=torch.float64)
    state = 0.1 * torch.randn(2, 2, 3, 4, dtype=torch.float64)
    rows = torch.randn(2, conv - 1, 2 * 11, dtype=torch.float64) if conv else None

    def f(h, state, rows, *ps):
        y, final = torch.func.functional_call(m, dict(zip(names, ps)), (h,), dict(
            initial_state=(state, rows) if conv else state, output_final_state=True))
        return (y, *final) if conv else (y, final)
    check(f, [h, state, rows, *params])


def test_layer_continues_from_its_state():
    torch.manual_seed(5)
    m = layer.QDeltaLayer(6, 2, 4, 3, conv_size=4, out_norm="layer", out_gate=True).double()
    h = torch.randn(2, 9, 6, dtype=torch.float64)
    y, end = m(h, output_final_state=True)
    y1, mid = m(h[:, :2], output_final_state=True)
    y2, end2 = m(h[:, 2:], initial_state=mid, output_final_state=True)
    assert torch.allclose(torch.cat([y1, y2], 1), y, rtol=1e-12, atol=1e-12)
    for a, b in zip(end, end2):
        assert torch.allclose(a, b, rtol=1e-12, atol=1e-12)


def test_layer_refuses_options():
    for bad in (dict(conv_size=1), dict(conv_size=5), dict(out_norm="batch"), dict(out_gate=True)):
        with pytest.raises(ValueError):
            layer.QDeltaLayer(6, 2, 4, 3, **bad)


def test_layer_without_options_has_its_parameters():
    assert [n for n, _ in layer.QDeltaLayer(6, 2, 4, 3).named_parameters()] == \
        ["lambda_bias", "w_qkv.weight", "w_gates.weight", "w_out.weight"]


def test_second_derivatives_are_refused():
    """The backward passes are kernels without a derivative: a gradient of a gradient raises."""
    r = rand(9)
    x, w = r(1, 5, 3).requires_grad_(), r(3, 4).requires_grad_()
    dt, A, B, C = r(1, 5, 1), -r(1).abs(), r(1, 5, 1, 2), r(1, 5, 1, 2)
    for y in (layer.causal_conv(x, w)[0], layer.row_norm(x, w[:, 0].contiguous()),
              layer.selective_scan(x[:, :, None], dt, A, B, C)[0]):
        g, = torch.autograd.grad(y.square().sum(), x, create_graph=True)
        with pytest.raises(RuntimeError):
            g.sum().backward()
