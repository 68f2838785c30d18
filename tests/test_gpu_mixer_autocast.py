"""The layer's options in mixed precision: fp32 parameters under torch.autocast to bf16."""
import copy

import pytest
import torch

from paper_2606_08804_amd import layer
from tests.gpu_helpers import normwise

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("conv,norm,gate", [(0, None, False), (4, None, False), (0, "layer", False), (2, "rms", False),
                                            (3, "layer", True), (4, "rms", True)])
def test_layer_under_autocast(conv, norm, gate, packed):
    """Autocast rounds each parameter to bf16 where it is used: output, final states and gradients are those of the layer
    held in bf16 (its own scalar bias given a value that bf16 holds), but for the input's gradient, which autocast sums in
    fp32 over the projections and the bf16 layer in bf16: three sums rounded by 2^-8 each at most."""
    torch.manual_seed(71)
    m = layer.QDeltaLayer(256, 2, 128, 128, conv_size=conv, out_norm=norm, out_gate=gate, lambda_bias=-0.75).cuda()
    b = copy.deepcopy(m).to(torch.bfloat16)
    g = torch.Generator().manual_seed(72)
    B, T = (1, 270) if packed else (2, 150)
    cu = torch.tensor([0, 70, 71, 270], dtype=torch.int32, device="cuda") if packed else None
    h, dy = (torch.randn(B, T, 256, generator=g).bfloat16().cuda() for _ in range(2))
    hm, hb = h.float().requires_grad_(), h.clone().requires_grad_()
    with torch.autocast("cuda", dtype=torch.bfloat16):
        y, end = m(hm, cu_seqlens=cu, output_final_state=True)
    y.backward(dy)
    want, end_b = b(hb, cu_seqlens=cu, output_final_state=True)
    want.backward(dy)
    assert y.dtype == torch.bfloat16 and torch.equal(y, want)
    for s, t in zip(end if conv else [end], end_b if conv else [end_b]):
        assert s.dtype == t.dtype and torch.equal(s, t)
    n = lambda t: t.detach().double().cpu().numpy()                              # noqa: E731
    for (name, p), (_, q) in zip(m.named_parameters(), b.named_parameters()):
        assert p.grad.dtype == torch.float32, name
        # the scalar bias's sum is rounded to its own type at the end
        assert normwise(n(p.grad), n(q.grad)) <= (2.0 ** -8 if name == "lambda_bias" else 0.0), name
    assert normwise(n(hm.grad), n(hb.grad)) <= 3 * 2.0 ** -8
