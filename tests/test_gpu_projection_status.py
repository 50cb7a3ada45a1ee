"""A wait that ran out in a projection with adapters is seen by who runs the loop (the status is set here, no wait runs out)."""
import json

import pytest

from paper_2512_03416_b200 import binding as B
from paper_2512_03416_b200 import speculative
from paper_2512_03416_b200.decoder import TsError
from tests.test_gpu_sampled_decoding import made

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["q", "o"])
def test_the_loop_raises(name):
    _, ads, sd, _ = made("bf16", 2, 2, 0.5)
    assert min(len(d) for d in sd.generate(2)) >= 2 and sd.projection_status() == 0
    ads[name].status.fill_(B.TS_DEV_TIMEOUT)
    assert sd.projection_status() == B.TS_DEV_TIMEOUT
    with pytest.raises(TsError):
        sd.generate(2)
    ads[name].status.zero_()
    sd.generate(2)
    sd.gemm_status.fill_(B.TS_DEV_TIMEOUT)
    with pytest.raises(TsError):
        sd.generate(2)
    sd.close()


def test_the_command_prints_it(capsys, monkeypatch):
    random_adapters = speculative.random_adapters

    def timed_out(*args):
        ads = random_adapters(*args)
        ads["k"].status.fill_(B.TS_DEV_TIMEOUT)
        return ads

    monkeypatch.setattr(speculative, "random_adapters", timed_out)
    assert speculative.main(["--requests", "2", "--prompt", "20", "--tokens", "4", "--adapters", "2", "--rank", "8"]) == 0
    assert json.loads(capsys.readouterr().out.strip().splitlines()[-1])["gemm_status"] == B.TS_DEV_TIMEOUT
