"""Adapters made on one stream and used on another one: they are laid out when their constructor returns."""
import pytest
import torch

from paper_2512_03416_b200 import adapters, binding as B
from paper_2512_03416_b200.adapters import Adapters, adapted_project
from tests.test_gpu_adapters import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", ["plain", "qkv"])
def test_adapters_are_ready_for_any_stream(rows, monkeypatch):
    tokens, which = [1] * 20, [r % 3 for r in range(20)]
    x, w, ad, _ = make(1, tokens, which, 256, 512, 16, 3)
    want = adapted_project(x, w, ad, tokens, which)
    pack = B.ts_adapter_pack

    def late(*args):                                     # the device takes its time over the packing
        torch.cuda._sleep(200_000_000)
        return pack(*args)

    monkeypatch.setattr(adapters.B, "ts_adapter_pack", late)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        again = Adapters(*ad.given, rows)
    got = adapted_project(x, w, again, tokens, which)    # on the default stream, which waits for nothing
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    assert int(again.status.item()) == 0
