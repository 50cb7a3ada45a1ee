"""Host side of the tree, cache and log probability calls: mask words, sizes and refusals (no device needed)."""
import ctypes

import numpy as np
import pytest

from paper_2512_03416_b200 import binding as B
from tests import tree_oracle as O


def _ctx(**kw):
    cfg = B.ts_config()
    for k, v in dict(dict(n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=16, n_pages=64, max_requests=4, max_pages_per_req=16), **kw).items():
        setattr(cfg, k, v)
    rc, h = B.ts_create(cfg)
    assert rc == B.TS_OK
    return cfg, h


def test_tree_masks():
    #   0        3
    #  / \       |
    # 1   2      4
    #     |
    #     5
    rc, m = B.ts_tree_masks([-1, 0, 0, -1, 3, 2])
    assert rc == B.TS_OK and m == [0b1, 0b11, 0b101, 0b1000, 0b11000, 0b100101]
    rc, m = B.ts_tree_masks(list(range(-1, 63)))                    # a chain of 64
    assert rc == B.TS_OK and m == [(2 << i) - 1 for i in range(64)]
    assert B.ts_tree_masks([]) == (B.TS_OK, [])
    for bad in ([0], [-2], [-1, 1], [-1, 2], [-1] * 65):
        assert B.ts_tree_masks(bad)[0] == B.TS_ERR_INVALID


def test_cache8_sizes():
    cfg, h = _ctx()
    assert B.ts_cache8_value_bytes(cfg) == 64 * 2 * 2 * 16 * 128 and B.ts_cache8_scale_bytes(cfg) == 64 * 2 * 2 * 16
    n, s = B.ts_cache8_value_bytes(cfg), B.ts_cache8_scale_bytes(cfg)
    ok = B.ts_cache8(1 << 20, n, 1 << 24, s)
    assert B.ts_cache8_attach(h, ok) == B.TS_OK
    for bad, code in ((B.ts_cache8(None, n, 1 << 24, s), B.TS_ERR_INVALID), (B.ts_cache8(1 << 20, n, None, s), B.TS_ERR_INVALID),
                      (B.ts_cache8((1 << 20) + 16, n, 1 << 24, s), B.TS_ERR_INVALID), (B.ts_cache8(1 << 20, n - 1, 1 << 24, s), B.TS_ERR_WORKSPACE),
                      (B.ts_cache8(1 << 20, n, 1 << 24, s - 1), B.TS_ERR_WORKSPACE)):
        assert B.ts_cache8_attach(h, bad) == code
    bad_cfg = B.ts_config()
    assert B.ts_cache8_value_bytes(bad_cfg) == 0 and B.ts_cache8_scale_bytes(bad_cfg) == 0
    B.ts_destroy(h)


def _calls(h, slots, lens, ctx, q=16, k=16, v=16, out=16, cache=0, mask=0, source=0, n_source=100):
    st, keep = B.make_step(slots, lens, ctx, q, k, v, out)
    return (B.ts_tree_attention(h, st, cache, mask, 0), B.ts_cache_append(h, st, cache, source, n_source, 0), B.ts_cache_read(h, st, cache, k, v, 0))


def test_refusals():
    cfg, h = _ctx()
    slots = [B.ts_request_add(h, r, 10, 10)[1] for r in range(3)]
    for s in slots:
        assert B.ts_alloc_pages(h, s, 100) == B.TS_OK
    assert B.ts_request_set_len(h, slots[0], 100) == B.TS_OK
    bad, short, cuda = B.TS_ERR_INVALID, B.TS_ERR_TABLE_SHORT, B.TS_ERR_CUDA
    # valid calls get as far as the device, which this context has no memory on
    assert _calls(h, slots[1:], [3, 64], [0, 0]) == (cuda, cuda, cuda)
    assert _calls(h, slots[1:2], [65], [0])[0] == bad                  # more nodes than a mask word has bits
    assert _calls(h, slots[1:2], [0], [0]) == (bad, B.TS_OK, B.TS_OK)  # no node; no token is nothing to do
    assert _calls(h, slots[1:2], [-1], [0]) == (bad, bad, bad)
    assert _calls(h, slots[:1], [1], [99])[:2] == (bad, bad)           # not the cached length
    assert _calls(h, slots[:1], [1], [99])[2] == cuda                  # a read may start anywhere
    assert _calls(h, slots[:1], [13], [100]) == (cuda, short, short)   # nodes need no room in the table, tokens do
    assert _calls(h, slots[:1], [2], [-1]) == (bad, bad, bad)
    assert _calls(h, [slots[1]] * 2, [1, 1], [0, 0]) == (bad, bad, bad)
    assert _calls(h, [3], [1], [0]) == (bad, bad, bad)                 # not a live slot
    assert _calls(h, [-1], [1], [0]) == (bad, bad, bad)
    assert _calls(h, slots[1:2], [1], [0], cache=1) == (bad, bad, bad)     # no 8-bit cache attached
    assert _calls(h, slots[1:2], [1], [0], cache=2) == (bad, bad, bad)
    for name in ("q", "k", "v", "out"):
        for value in (0, 8):                                           # missing, misaligned
            got = _calls(h, slots[1:2], [1], [0], **{name: value})
            assert got[0] == bad
            assert got[1:] == ((bad, bad) if name in "kv" else (cuda, cuda))
    assert _calls(h, slots[1:2], [1], [0], mask=4)[0] == bad
    assert _calls(h, slots[1:2], [1], [0], source=6)[1] == bad
    assert _calls(h, slots[1:2], [1], [0], source=16, n_source=-1)[1] == bad
    assert _calls(h, [], [], []) == (B.TS_OK, B.TS_OK, B.TS_OK)
    assert B.ts_tree_attention(None, B.make_step([], [], [])[0], 0, 0, 0) == bad
    assert B.lib().ts_cache_append(h, None, 0, None, 0, None) == bad
    # a refused call changes nothing
    assert [B.ts_block_table(h, s)[2] for s in slots] == [100, 0, 0]
    assert B.ts_velocity(h)[1]["kernel_launches"] == 0
    # appending nothing advances nothing
    st, keep = B.make_step(slots, [0, 0, 0], [100, 0, 0])
    assert B.ts_cache_append(h, st, 0, 0, 0, 0) == B.TS_OK
    B.ts_destroy(h)


def test_logprobs_refusals():
    good = dict(device=0, n_rows=0, vocab=100, dtype=B.TS_F32, logits=256, row_stride=100, scale=256, tokens=256, n_given=1, n_top=2, logprob=256,
                rank=256, entropy=256, top_logprob=256, top_token=256)
    assert B.ts_token_logprobs(B.ts_logprobs(**good), 0) == B.TS_OK     # no rows: nothing to do
    bad = B.TS_ERR_INVALID
    for change, code in ((dict(n_rows=-1), bad), (dict(vocab=0), bad), (dict(row_stride=99), bad), (dict(n_given=9), bad), (dict(n_given=-1), bad),
                         (dict(n_top=33), bad), (dict(n_top=-1), bad), (dict(dtype=2), B.TS_ERR_UNSUPPORTED),
                         (dict(vocab=(1 << 30) + 1, row_stride=1 << 31), B.TS_ERR_UNSUPPORTED)):
        assert B.ts_token_logprobs(B.ts_logprobs(**dict(good, **change)), 0) == code, change
    for change in (dict(logits=0), dict(logits=258), dict(tokens=0), dict(logprob=0), dict(top_logprob=0), dict(top_token=0), dict(scale=258),
                   dict(tokens=257), dict(entropy=2), dict(rank=1)):
        assert B.ts_token_logprobs(B.ts_logprobs(**dict(good, n_rows=1, **change)), 0) == bad, change
    assert B.lib().ts_token_logprobs(None, None) == bad


def test_the_oracle_of_the_format():
    """Closed forms: exact codes, ties to the even mantissa, the boundary of the scale, saturation."""
    assert O.E4M3[0x7E] == 448 and O.E4M3[0x01] == 2.0 ** -9 and O.E4M3[0x38] == 1.0
    codes, b = O.quantise_row(np.array([448.0, 1.0, -1.0, 1.0625, 1.1875, 0.0, 2.0 ** -9, 2.0 ** -10, 1.5 * 2.0 ** -9]))
    assert b == 127 and list(codes) == [0x7E, 0x38, 0xB8, 0x38, 0x3A, 0, 1, 0, 2]
    assert O.quantise_row(np.array([448.5]))[1] == 128 and O.quantise_row(np.array([224.0]))[1] == 126 and O.quantise_row(np.zeros(3))[1] == 127
    assert O.quantise_row(np.array([2.0 ** 100, 1.0])) [1] == 62 + 127 and list(O.quantise_row(np.array([2.0 ** 100]))[0]) == [0x7E]


def test_the_oracle_of_the_logprobs():
    lp, rank, ent, top_lp, top = O.token_logprobs(np.log(np.array([0.25, 0.5, 0.25])), 1.0, [2, 1, 5], 5)
    assert np.allclose(lp[:2], np.log([0.25, 0.5])) and np.isnan(lp[2]) and list(rank) == [2, 0, -1]
    assert np.isclose(ent, 1.5 * np.log(2)) and list(top) == [1, 0, 2, -1, -1]


@pytest.mark.parametrize("hq,hkv", [(1, 1), (6, 2)])
def test_the_oracle_of_the_attention(hq, hkv):
    rng = np.random.default_rng(0)
    v = rng.standard_normal((3, hkv, 4))
    seen = np.array([[1, 0, 0], [1, 1, 1], [0, 0, 0]], bool)
    out, _ = O.attention(np.zeros((3, hq, 4)), rng.standard_normal((3, hkv, 4)), v, seen, 1.0)
    g = hq // hkv
    for h in range(hq):                                              # one key: its V; equal scores: the mean; none: zeros
        assert np.allclose(out[0, h], v[0, h // g]) and np.allclose(out[1, h], v[:, h // g].mean(0)) and (out[2, h] == 0).all()
    assert ctypes.sizeof(B.ts_cache8) == 32


def test_types_of_tensors():
    """16-bit tensors are bf16, or bit patterns of it; masks are 64-bit words. A float16 or float64 tensor is not taken for one by its size."""
    import types

    import torch

    from paper_2512_03416_b200.decoder import Decoder
    dec = Decoder.__new__(Decoder)                                 # its checks alone: no device
    dec.ctx, dec.device, dec.cache = None, torch.device("cpu"), B.TS_CACHE_BF16
    dec.cfg = types.SimpleNamespace(n_q_heads=4, n_kv_heads=2, head_dim=64)
    for dtype in (torch.bfloat16, torch.int16, torch.uint16):
        t = torch.zeros((3, 2, 64), dtype=dtype)
        assert dec._tokens(t, 2, "k") == t.data_ptr()
    for dtype in (torch.float16, torch.int8, torch.float32):
        with pytest.raises(ValueError):
            dec._tokens(torch.zeros((3, 2, 64), dtype=dtype), 2, "k")
    q, k = (torch.zeros((3, h, 64), dtype=torch.bfloat16) for h in (4, 2))
    dec._stream = lambda: 0
    for mask in (torch.zeros(3, dtype=torch.float64), torch.zeros(3, dtype=torch.complex64), torch.zeros(3, dtype=torch.int32),
                 torch.zeros(2, dtype=torch.int64)):
        with pytest.raises(ValueError):
            dec.tree_attention([0], [3], [0], q, k, k, q, mask=mask)


def test_logprobs_of_too_many_rows():
    """Row numbers of a call, and those a block looks ahead to, fit into 32 bits."""
    args = dict(device=0, vocab=100, dtype=B.TS_F32, logits=256, row_stride=100, scale=None, tokens=256, n_given=1, n_top=2, logprob=256,
                rank=256, entropy=256, top_logprob=256, top_token=256)
    for n_rows in ((1 << 30) + 1, (1 << 31) - 1):
        assert B.ts_token_logprobs(B.ts_logprobs(**dict(args, n_rows=n_rows)), 0) == B.TS_ERR_UNSUPPORTED
