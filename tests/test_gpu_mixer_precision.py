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
