"""What DecoderLayer.pack_gate_up_adapters refuses, without a GPU: nothing is launched on tensors that are not what it says they are."""
from types import SimpleNamespace

import pytest
import torch

from paper_2512_03416_b200 import binding as B
from paper_2512_03416_b200.layer import DecoderLayer


@pytest.mark.parametrize("gate,up", [
    (torch.zeros(2, 128, 16), torch.zeros(2, 128, 16)),                                                      # not 16 bits
    (torch.zeros(2, 256, 16, dtype=torch.bfloat16), torch.zeros(2, 128, 16, dtype=torch.bfloat16)),          # up shorter than gate: read behind its end
    (torch.zeros(2, 128, 16, dtype=torch.bfloat16), torch.zeros(1, 128, 16, dtype=torch.bfloat16)),
    (torch.zeros(2, 128, 16, dtype=torch.bfloat16), torch.zeros(2, 128, 8, dtype=torch.bfloat16)),
    (torch.zeros(2, 128, 16, dtype=torch.bfloat16), torch.zeros(2, 128, 16, dtype=torch.int16)),
    (torch.zeros(128, 16, dtype=torch.bfloat16), torch.zeros(128, 16, dtype=torch.bfloat16)),
    (torch.zeros(2, 128, 16, dtype=torch.bfloat16, device="meta"), torch.zeros(2, 128, 16, dtype=torch.bfloat16, device="meta")),      # elsewhere
])
def test_gate_and_up_that_do_not_fit_are_refused(gate, up, monkeypatch):
    calls = []
    monkeypatch.setattr(B, "ts_pack_gate_up", lambda *a: calls.append(a) or B.TS_OK)
    layer = SimpleNamespace(dec=SimpleNamespace(device=torch.device("cpu"), _stream=lambda: 0))
    with pytest.raises(ValueError):
        DecoderLayer.pack_gate_up_adapters(layer, gate, up)
    assert not calls
