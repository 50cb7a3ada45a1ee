"""ts_cache_append and ts_cache_read over both caches, byte for byte."""
import numpy as np
import pytest
import torch

from paper_2512_03416_b200 import binding as B
from paper_2512_03416_b200 import workloads as wl
from paper_2512_03416_b200.decoder import Decoder, TsError
from paper_2512_03416_b200.harness import to_dev
from tests import tree_oracle as O

pytestmark = pytest.mark.gpu


def _image(dec):
    """(values [page, kv, head, slot, d], scales [page, kv, head, slot]) as they lie in memory."""
    c = dec.cfg
    torch.cuda.synchronize()
    shape = (c.n_pages, 2, c.n_kv_heads, 16, c.head_dim)
    if dec.pool is not None:
        return dec.pool.cpu().numpy().view(np.uint16).reshape(shape), None
    return dec.cache8_values.cpu().numpy().reshape(shape), dec.cache8_scales.cpu().numpy().reshape(shape[:-1])


def _values(bits):
    return wl.bf16_bits_to_f32(bits).astype(np.float64)


def _special(rng, n, hkv, d):
    """Rows of all sizes, zeros, subnormals, values between codes, infinities and NaN."""
    x = rng.standard_normal((n, hkv, d)) * 2.0 ** rng.integers(-6, 7, (n, hkv, 1))
    bits = wl.f32_to_bf16_bits(x.astype(np.float32))
    flat = bits.reshape(n * hkv, d)
    for i in range(0, len(flat), 7):
        kind = (i // 7) % 8
        if kind == 0:
            flat[i] = 0
        elif kind == 1:
            flat[i, 3] = 0x7FC0
        elif kind == 2:
            flat[i, 5] = 0xFF80
        elif kind == 3:
            flat[i] = rng.integers(0, 0x80, d)                       # subnormal in bf16: below the smallest scale
        elif kind == 4:
            flat[i] = rng.integers(0x7E00, 0x7F80, d)                # above the largest
        elif kind == 5:
            flat[i] = wl.f32_to_bf16_bits((448 * 2.0 ** (i % 9) * np.ones(d)).astype(np.float32)) + (i // 56) % 2   # at 448 * 2^E and right behind
        elif kind == 6:
            flat[i] = wl.f32_to_bf16_bits(np.linspace(-448, 448, d).astype(np.float32))
        else:
            flat[i, 1:] = 0x8000
            flat[i, 0] = 0x8000 if i % 2 else 0x3F80
    return bits


CASES = [((4, 2, 64), [(0, 1)]), ((1, 1, 64), [(3, 20), (0, 0), (16, 16)]), ((6, 3, 64), [(15, 2), (1, 100), (0, 33)]),
         ((2, 1, 128), [(7, 9), (0, 1)]), ((8, 8, 128), [(0, 17), (31, 1), (5, 64), (0, 0)]), ((10, 5, 128), [(100, 200)])]


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("shape,rows", CASES, ids=lambda v: str(v))
def test_written_and_read_back(shape, rows, cache):
    hq, hkv, d = shape
    rng = np.random.default_rng(sum(c + t for c, t in rows) + d)
    pages = [-(-(c + t) // 16) for c, t in rows]
    dec = Decoder(hq, hkv, d, n_pages=sum(pages) + 4, max_requests=len(rows), max_pages_per_req=max(pages + [1]), alloc_shuffle_seed=7, cache=cache,
                  nan_fill=True)
    slots = []
    for r, (c, t) in enumerate(rows):
        slots.append(dec.request_add(r, c + t))
        dec.alloc_pages(slots[-1], c + t)
        dec.request_set_len(slots[-1], c)
    ctx, new = [c for c, _ in rows], [t for _, t in rows]
    n = sum(new)
    k, v = _special(rng, n, hkv, d), _special(rng, n, hkv, d)[::-1].copy()
    values, scales = _image(dec)
    values = values.copy()
    scales = None if scales is None else scales.copy()
    dec.cache_append(slots, new, ctx, to_dev(k), to_dev(v))
    want = np.empty((2, n, hkv, d))
    tok = 0
    for r, (c, t) in enumerate(rows):
        table, cached = dec.block_table(slots[r])
        assert cached == c + t
        for i in range(t):
            page, slot = table[(c + i) // 16], (c + i) % 16
            for kv, x in enumerate((k, v)):
                for h in range(hkv):
                    if cache == "bf16":
                        values[page, kv, h, slot] = x[tok, h]
                        want[kv, tok, h] = _values(x[tok, h])
                    else:
                        codes, scale = O.quantise_row(_values(x[tok, h]))
                        values[page, kv, h, slot], scales[page, kv, h, slot] = codes, scale
                        want[kv, tok, h] = O.E4M3[codes] * 2.0 ** (scale - 127) if scale != 255 else np.nan
            tok += 1
    got_values, got_scales = _image(dec)
    if scales is not None:
        assert np.array_equal(got_scales, scales)
        # the codes of a row of NaN are of no interest; rows nobody wrote are (they hold 255 too)
        written = np.zeros(scales.shape, bool)
        for r, (c, t) in enumerate(rows):
            for i in range(c, c + t):
                written[dec.block_table(slots[r])[0][i // 16], :, :, i % 16] = True
        got_values = np.where((written & (scales == 255))[..., None], values, got_values)
    assert np.array_equal(got_values, values), "pages differ, or others were written"
    ko, vo = (torch.full((n + 2, hkv, d), 0x1234, dtype=torch.int16, device="cuda") for _ in range(2))
    dec.cache_read(slots, ctx, new, ko, vo)
    for kv, t in enumerate((ko, vo)):
        bits = t.cpu().numpy().view(np.uint16)
        assert (bits[n:] == 0x1234).all()
        assert np.array_equal(_values(bits[:n]), want[kv], equal_nan=True)
    assert dec.device_status() == 0


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_accepted_path(cache):
    """Tokens named by source; an index outside skips its token, and says so."""
    dec = Decoder(8, 2, 128, n_pages=40, max_requests=4, max_pages_per_req=10, alloc_shuffle_seed=3, cache=cache, nan_fill=True)
    rng = np.random.default_rng(2)
    k, v = (rng.integers(-3, 4, (30, 2, 128)).astype(np.float32) for _ in range(2))
    slots = [dec.request_add(r, 50) for r in range(3)]
    for s, c in zip(slots, (14, 0, 40)):
        dec.alloc_pages(s, 60)
        dec.request_set_len(s, c)
    source = [0, 3, 7, 12, 29, 29, 4]
    dk, dv = (to_dev(wl.f32_to_bf16_bits(x)) for x in (k, v))
    dec.cache_append(slots, [3, 0, 4], [14, 0, 40], dk, dv, source=torch.tensor(source, dtype=torch.int32, device="cuda"))
    assert [dec.block_table(s)[1] for s in slots] == [17, 0, 44]
    ko, vo = (torch.empty((7, 2, 128), dtype=torch.int16, device="cuda") for _ in range(2))
    dec.cache_read(slots, [14, 0, 40], [3, 0, 4], ko, vo)
    assert np.array_equal(_values(ko.cpu().numpy().view(np.uint16)), k[source]) and np.array_equal(_values(vo.cpu().numpy().view(np.uint16)), v[source])
    assert dec.device_status() == 0
    before, _ = _image(dec)
    dec.cache_append(slots[:1], [2], [17], dk, dv, source=torch.tensor([30, -1], dtype=torch.int32, device="cuda"))
    assert dec.device_status() == B.TS_DEV_BAD_INDEX
    assert np.array_equal(before, _image(dec)[0])


def test_bf16_append_is_kv_append():
    a, b = (Decoder(8, 2, 64, n_pages=40, max_requests=3, max_pages_per_req=10, nan_fill=True) for _ in range(2))
    rng = np.random.default_rng(3)
    k, v = (to_dev(rng.integers(0, 1 << 16, (45, 2, 64)).astype(np.uint16)) for _ in range(2))
    for dec in (a, b):
        for r in range(3):
            dec.alloc_pages(dec.request_add(r, 30), 30)
    a.kv_append([0, 1, 2], [10, 30, 5], [0, 0, 0], k, v)
    b.cache_append([0, 1, 2], [10, 30, 5], [0, 0, 0], k, v)
    torch.cuda.synchronize()
    assert torch.equal(a.pool, b.pool)


def test_mixed_steps_need_a_pool():
    dec = Decoder(8, 2, 128, n_pages=8, max_requests=1, max_pages_per_req=4, cache="e4m3")
    slot = dec.request_add(0, 4)
    dec.alloc_pages(slot, 4)
    q, k = (torch.zeros((1, h, 128), dtype=torch.int16, device="cuda") for h in (8, 2))
    with pytest.raises(TsError) as e:
        dec.mixed_step([slot], [1], [0], q, k, k, torch.empty_like(q))
    assert e.value.code == B.TS_ERR_CUDA


def test_checks_of_tensors():
    dec = Decoder(8, 2, 128, n_pages=8, max_requests=2, max_pages_per_req=4, cache="e4m3")
    slot = dec.request_add(0, 4)
    dec.alloc_pages(slot, 40)
    q, k = (torch.zeros((3, h, 128), dtype=torch.bfloat16, device="cuda") for h in (8, 2))
    out = torch.empty_like(q)
    mask = torch.zeros(3, dtype=torch.int64, device="cuda")
    bad = [lambda: dec.tree_attention([slot], [4], [0], q, k, k, out), lambda: dec.tree_attention([slot], [3], [0], q.float(), k, k, out),
           lambda: dec.tree_attention([slot], [3], [0], k, k, k, out), lambda: dec.tree_attention([slot], [3], [0], q, k, k, out, mask=mask[:2]),
           lambda: dec.tree_attention([slot], [3], [0], q, k, k, out, mask=mask.int()), lambda: dec.tree_attention([slot], [3], [0], q, k.cpu(), k, out),
           lambda: dec.tree_attention([slot], [1], [0], q[:, ::2], k, k, out), lambda: dec.cache_append([slot], [4], [0], k, k),
           lambda: dec.cache_append([slot], [2], [0], k, k, source=torch.zeros(2, dtype=torch.int64, device="cuda")),
           lambda: dec.cache_append([slot], [2], [0], k, k, source=torch.zeros(1, dtype=torch.int32, device="cuda")),
           lambda: dec.cache_read([slot], [0], [4], k, k)]
    for f in bad:
        with pytest.raises((ValueError, TsError)):
            f()
    with pytest.raises(TsError):
        dec.tree_attention([slot], [3], [1], q, k, k, out)            # not the cached length
    with pytest.raises(ValueError):
        Decoder(8, 2, 128, n_pages=8, max_requests=2, max_pages_per_req=4, cache="int8")


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("rows", [60, 700, 4095, 4096, 9000])
def test_many_rows(rows, cache):
    """One call for thousands of requests: more row arrays than launch parameters (768 words) and than a thread block's default shared memory
    (4095 rows) hold. 0 to 2 tokens each, then a tree step of a node each."""
    dec = Decoder(2, 1, 64, n_pages=rows, max_requests=rows, max_pages_per_req=1, alloc_shuffle_seed=5, cache=cache, nan_fill=True)
    rng = np.random.default_rng(rows)
    count = [int(x) for x in rng.integers(0, 3, rows)]
    slots = [dec.request_add(r, 4) for r in range(rows)]
    for s in slots:
        dec.alloc_pages(s, 4)
    n = sum(count)
    k, v = (rng.integers(-3, 4, (n, 1, 64)).astype(np.float32) for _ in range(2))          # exact in 8 bits
    dec.cache_append(slots, count, [0] * rows, to_dev(wl.f32_to_bf16_bits(k)), to_dev(wl.f32_to_bf16_bits(v)))
    ko, vo = (torch.empty((n, 1, 64), dtype=torch.int16, device="cuda") for _ in range(2))
    dec.cache_read(slots, [0] * rows, count, ko, vo)
    assert np.array_equal(_values(ko.cpu().numpy().view(np.uint16)), k) and np.array_equal(_values(vo.cpu().numpy().view(np.uint16)), v)
    q = torch.zeros((rows, 2, 64), dtype=torch.bfloat16, device="cuda")                   # equal scores: the mean of V
    out = torch.empty_like(q)
    v1 = torch.ones((rows, 1, 64), dtype=torch.bfloat16, device="cuda")
    dec.tree_attention(slots, [1] * rows, count, q, v1, v1, out)
    assert dec.device_status() == 0
    first = np.concatenate([[0], np.cumsum(count)])
    want = np.stack([(v[a:b].sum(0) + 1) / (b - a + 1) for a, b in zip(first[:-1], first[1:])])
    assert np.abs(out.float().cpu().numpy() - want).max() <= 2.0 ** -7 * 4
