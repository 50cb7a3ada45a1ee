"""Layer steps with adapters whose plans are as long as they get: they are served, or refused with nothing changed."""
import numpy as np
import pytest
import torch

from paper_2512_03416_b200 import workloads as wl
from paper_2512_03416_b200.adapters import Adapters
from paper_2512_03416_b200.harness import LoadedBatch, to_dev
from paper_2512_03416_b200.layer import DecoderLayer
from tests.test_gpu_layer_adapters import adapter, bits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("only", ["qkv", "o", "gate_up", "down"])
def test_a_step_of_the_longest_plans_is_served_or_leaves_everything_as_it_was(only):
    """1024 rows of 1 and 17 new tokens, 8192 in all, each with an adapter of its own, on one projection: those behind the attention too are
    planned before anything is enqueued."""
    rng = np.random.default_rng(5)
    s, hidden, inter, rank, rows = wl.Shape(2, 2, 128), 128, 128, 8, 1024
    lens = rng.permutation([17] * 448 + [1] * 576)
    b = wl.make_batch("plans", s, [3] * rows, lens.tolist(), seed=1, chunk_size=8192)
    lb = LoadedBatch(b)
    shapes = dict(w_norm1=(hidden,), w_qkv=(768, hidden), w_o=(hidden, 256), w_norm2=(hidden,), w_gate=(inter, hidden), w_up=(inter, hidden), w_down=(hidden, inter))
    layer = DecoderLayer(lb.dec, **{k: to_dev(bits(rng, v, 0.1)) for k, v in shapes.items()}, max_position=64)
    out_in = dict(qkv=(768, hidden), o=(hidden, 256), gate_up=(2 * inter, hidden), down=(hidden, inter))[only]
    a, bb = adapter(rng, rows, rank, *out_in)
    layer.set_adapters(**{only: Adapters(to_dev(a), to_dev(bb), None, only if only in ("qkv", "gate_up") else "plain")})
    x = to_dev(bits(rng, (b.n_tokens, hidden), 1.0))
    plain, got = torch.full_like(x, 0x7FC0), torch.full_like(x, 0x7FC0)
    layer.step(lb.slots, b.q_len.tolist(), b.ctx_len.tolist(), x, plain, keep_len=True)
    torch.cuda.synchronize()
    pool = lb.dec.pool.clone()
    try:
        layer.step(lb.slots, b.q_len.tolist(), b.ctx_len.tolist(), x, got, adapters=rng.permutation(rows).tolist())
    except RuntimeError:
        torch.cuda.synchronize()
        assert [lb.dec.block_table(slot)[1] for slot in lb.slots] == [3] * rows
        assert torch.equal(lb.dec.pool, pool) and bool((got == 0x7FC0).all())
    else:
        torch.cuda.synchronize()
        assert [lb.dec.block_table(slot)[1] for slot in lb.slots] == (3 + lens).tolist()
        assert torch.isfinite(got.view(torch.bfloat16).float()).all() and not torch.equal(got, plain)
        assert lb.dec.device_status() == 0
    layer.close()
