"""ts_tree_attention with several times more work units than SMs: every thread block of the tcgen05 kernel takes unit after
unit, so that what it keeps from one to the next (rings, tables, barrier phases) is compared with the definition too."""
import numpy as np
import pytest
import torch

from paper_2512_03416_b200 import workloads as wl
from paper_2512_03416_b200.harness import to_dev
from tests.test_gpu_tree import Case, bf16

pytestmark = pytest.mark.gpu


def _rows(seed, n, least, most, long_ones=()):
    """n rows of 0 to 130 cached tokens (none, one page, whole blocks and one more among them) with least to most nodes, the long ones in between."""
    rng = np.random.default_rng(seed)
    ctx = [int(c) for c in rng.choice([0, 0, 1, 16, 127, 128, 129, 130], n // 2)] + [int(c) for c in rng.integers(0, 131, n - n // 2)]
    ctx = [ctx[i] for i in rng.permutation(n)]
    for i, c in enumerate(long_ones):
        ctx[(i + 1) * n // (len(long_ones) + 1)] = c
    nodes = [int(t) for t in rng.integers(least, most + 1, n)]
    nodes[n // 3] = most
    return list(zip(ctx, nodes))


def _own_powers(c, lo=-10, hi=2):
    """Every (node, head)'s query has a power of two of its own."""
    q = c.rng.standard_normal((c.n, c.hq, c.d)) * 2.0 ** c.rng.integers(lo, hi + 1, (c.n, c.hq, 1))
    c.qb, c.q = bf16(q)


def _outputs(c, times):
    """Steps issued one behind the other, each into its own output."""
    q, k, v = to_dev(c.qb), to_dev(c.kb), to_dev(c.vb)
    mask = None if c.mask is None else torch.from_numpy(c.mask.view(np.int64)).cuda()
    outs = [torch.full((c.n, c.hq, c.d), 0x7FC0, dtype=torch.int16, device="cuda") for _ in range(times)]
    torch.cuda.synchronize()
    for out in outs:
        c.dec.tree_attention(c.slots, c.nodes, c.ctx, q, k, v, out, mask=mask)
    assert c.dec.device_status() == 0
    return outs


# (query heads, KV heads), rows, least and most nodes: the queries of a KV head in half a tile, one, two tiles, several units
UNITS = [((16, 4), 90, 5, 16), ((16, 4), 90, 17, 32), ((16, 4), 90, 33, 64), ((16, 4), 90, 1, 64), ((32, 2), 100, 1, 64), ((9, 3), 80, 1, 64),
         ((32, 4), 100, 1, 9)]


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,n,least,most", UNITS, ids=lambda v: str(v))
@pytest.mark.parametrize("long_ones", [(), (2500, 700, 5000)], ids=["short", "some-long"])
def test_many_units(heads, n, least, most, long_ones, cache):
    c = Case((*heads, 128), cache, _rows(n + most, n, least, most, long_ones), masks="tree", seed=most)
    _own_powers(c)
    outs = _outputs(c, 6)
    c.check(wl.bf16_bits_to_f32(outs[0].cpu().numpy().view(np.uint16)).astype(np.float64))
    assert all(torch.equal(outs[0], o) for o in outs[1:]), "another bit pattern in another step"


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("masks", [None, "none", "any"])
def test_masks_of_many_units(masks, cache):
    c = Case((16, 4, 128), cache, _rows(7, 90, 1, 40), masks=masks, seed=21)
    _own_powers(c)
    got = c.check()
    if masks == "none":
        alone = np.repeat([x == 0 for x in c.ctx], c.nodes)
        assert (got[alone] == 0).all()


def test_many_units_of_pieces():
    """Pieces of split rows as units of a few blocks, and their merge."""
    c = Case((16, 4, 128), "e4m3", [(3000 + 97 * i, 9 + i) for i in range(24)], masks="tree", seed=31)
    _own_powers(c)
    before = c.dec.velocity()["kernel_launches"]
    c.check()
    assert c.dec.velocity()["kernel_launches"] - before == 2
