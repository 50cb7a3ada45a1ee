"""A context's first page copy sets up nothing that copies do not use: it needs the pool alone."""
import numpy as np
import pytest
import torch

from paper_2512_03416_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["bf16", "e4m3", "both"])
def test_pages_of_a_context_without_a_workspace(cache):
    n, hkv, d = 12, 2, 64
    pool = torch.randint(-2 ** 15, 2 ** 15, (n, 2 * hkv * 16 * d), dtype=torch.int16, device="cuda") if cache != "e4m3" else None
    values, scales = (torch.randint(0, 127, (n, 2 * hkv * 16 * k), dtype=torch.uint8, device="cuda") for k in (d, 1)) if cache != "bf16" else (None, None)
    cfg = B.ts_config(4, hkv, d, 16, n, 4, 6, 512, 0, 0, 0, 0.0, 0, 0, None if pool is None else pool.data_ptr(), 0 if pool is None else pool.numel() * 2, None, 0, 0, 0)
    rc, h = B.ts_create(cfg)
    assert rc == B.TS_OK
    if values is not None:
        assert B.ts_cache8_attach(h, B.ts_cache8(values.data_ptr(), values.numel(), scales.data_ptr(), scales.numel())) == B.TS_OK
    regions = [t for t in (pool, values, scales) if t is not None]
    before = [t.clone() for t in regions]
    stream = torch.cuda.current_stream().cuda_stream
    src, dst = np.array([3, 3, 7], dtype=np.int32), np.array([0, 11, 5], dtype=np.int32)
    assert B.ts_copy_pages(h, src, dst, stream) == B.TS_OK
    _, slot = B.ts_request_add(h, 1, 20, 0)
    assert B.ts_alloc_pages(h, slot, 20, 0) == B.TS_OK and B.ts_request_set_len(h, slot, 20) == B.TS_OK
    out = np.zeros(1, dtype=np.int32)
    assert B.ts_request_fork(h, np.array([slot], dtype=np.int32), None, np.array([2]), out, stream) == B.TS_OK
    (_, own, _), (_, fork, _) = B.ts_block_table(h, slot), B.ts_block_table(h, int(out[0]))
    assert own[0] == fork[0] and own[1] != fork[1]
    torch.cuda.synchronize()
    for t, want in zip(regions, before):
        for a, b in ((3, 0), (3, 11), (7, 5)):
            want[b] = want[a]
        want[fork[1]] = want[own[1]]
        assert torch.equal(t, want)
    assert B.ts_destroy(h) == B.TS_OK
