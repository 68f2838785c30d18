"""The layer with the operators around the recurrence as other programs hand it over: pickled before it had options (CPU,
with the recurrence computed by the oracle)."""
import io

import pytest
import torch

from paper_2606_08804_amd import layer
from tests import mixer_oracle, oracle_binding


@pytest.fixture
def plain(monkeypatch):
    monkeypatch.setattr(layer, "_binding", oracle_binding)
    monkeypatch.setattr(layer, "_mixer", mixer_oracle)


def test_layer_pickled_without_options(plain):
    """A module stored whole before conv_size, out_norm and out_gate existed runs as it did."""
    torch.manual_seed(6)
    m = layer.QDeltaLayer(6, 2, 4, 3).double()
    h = torch.randn(2, 5, 6, dtype=torch.float64)
    y, end = m(h, output_final_state=True)
    for name in ("conv_size", "out_norm", "out_gate"):
        m.__dict__.pop(name, None)
    f = io.BytesIO()
    torch.save(m, f)
    f.seek(0)
    old = torch.load(f, weights_only=False)               # what this test has just written
    y2, end2 = old(h, output_final_state=True)
    assert torch.equal(y, y2) and torch.equal(end, end2)
    old.reset_parameters()
    assert old(h).shape == y.shape
