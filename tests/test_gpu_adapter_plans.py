"""Projections whose plans are as long as the documented limits let them be, against the definition in 64 bits."""
import numpy as np
import pytest

from paper_2512_03416_b200.adapters import adapted_project
from tests.test_gpu_adapters import check, definition, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tile_m", [128, 256])
@pytest.mark.parametrize("rows,tokens,long", [(1024, 8192, 17), (1024, 4096, 17), (1024, 8192, 33), (512, 32768, 65)])
def test_rows_of_two_lengths_up_to_the_limits(rows, tokens, long, tile_m):
    rng = np.random.default_rng(rows + long)
    n = min((tokens - rows) // (long - 1), rows - 1)
    lens = rng.permutation([long] * n + [1] * (rows - n)).tolist()
    lens[0] += tokens - sum(lens)
    which = rng.permutation(rows).tolist()
    x, w, ad, _ = make(rows + long, lens, which, 128, 64, 8, rows)
    y = adapted_project(x, w, ad, lens, which, tile_m=tile_m)
    want, slack = definition(x, w, ad, lens, which, None)
    check(y, want, slack, 64, 8)
    assert int(ad.status.item()) == 0
