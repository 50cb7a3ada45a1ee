"""Sizes and refusals of the adapters' entry points that need no GPU."""
import ctypes

import pytest

from paper_2512_03416_b200 import binding as B


def config(chunk_size, max_requests=64):
    cfg = B.ts_config()
    cfg.chunk_size, cfg.max_requests = chunk_size, max_requests
    return cfg


def layer_bytes(cfg, *ranks, count=4):
    kept = [None if r is None else B.ts_adapters(count, r, 1, 1, 1, None) for r in ranks]
    return B.ts_layer_adapters_workspace_bytes(cfg, B.ts_layer_adapters(*[None if a is None else ctypes.pointer(a) for a in kept], None, 0))


def test_a_layers_workspace_serves_its_widest_projection_and_the_longest_adapted_step():
    one = layer_bytes(config(2112), 16, None, None, None)
    assert one >= B.ts_adapter_workspace_bytes(2112, 64, 4, 16) > 0
    assert layer_bytes(config(2112), 16, None, 64, 8) == layer_bytes(config(2112), None, None, 64, None) > one
    assert layer_bytes(config(40000), 16, None, None, None) == layer_bytes(config(32768), 16, None, None, None) > one      # longer steps have no adapters
    assert layer_bytes(config(2112), None, None, None, None) == 0


@pytest.mark.parametrize("cfg,rank,count", [((0,), 16, 4), ((64, 0), 16, 4), ((64,), 12, 4), ((64,), 264, 4), ((64,), 0, 4), ((64,), 16, 0), ((64,), 16, 65537)])
def test_a_layers_workspace_of_what_is_not_served_is_none(cfg, rank, count):
    assert layer_bytes(config(*cfg), None, rank, None, None, count=count) == 0


def test_workspace_grows_with_every_argument():
    base = (300, 20, 8, 32)
    size = B.ts_adapter_workspace_bytes(*base)
    for i, more in enumerate((301, 21, 9, 40)):
        args = list(base)
        args[i] = more
        assert B.ts_adapter_workspace_bytes(*args) >= size > 0
    for args in ((0, 1, 1, 8), (1, 0, 1, 8), (1, 1, 0, 8), (1, 1, 1, 4), (1, 1, 1, 260), (40000, 1, 1, 8), (9000, 513, 1, 8), (2000, 1025, 1, 8)):
        assert B.ts_adapter_workspace_bytes(*args) == 0


def test_packed_sizes():
    assert B.ts_adapter_packed_bytes(3, 130, 24) == 3 * 32 * 256 * 2 and B.ts_adapter_packed_bytes(1, 128, 72) == 128 * 128 * 2
    for args in ((0, 128, 8), (1, 0, 8), (1, 128, 12), (1, 128, 264)):
        assert B.ts_adapter_packed_bytes(*args) == 0
