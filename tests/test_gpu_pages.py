"""Cache pages copied, forked and compacted: the pool bit for bit, and steps over shared pages against the same requests with pages of their own."""
import numpy as np
import pytest
import torch

from paper_2512_03416_b200 import binding as B
from paper_2512_03416_b200.decoder import Decoder, TsError

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")


SHAPES = [(4, 2, 64), (3, 1, 128), (32, 8, 128)]


def decoder(shape, cache, n_pages, requests=16, width=16, seed=1, **more):
    dec = Decoder(*shape, n_pages=n_pages, max_requests=requests, max_pages_per_req=width, cache=cache, **more)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if cache == "bf16":
        dec.pool.copy_(torch.randn(dec.pool.shape, generator=gen, device="cuda").to(torch.bfloat16).view(torch.int16))
    else:
        dec.cache8_values.copy_(torch.randint(0, 127, dec.cache8_values.shape, generator=gen, device="cuda", dtype=torch.uint8))
        dec.cache8_scales.copy_(torch.randint(118, 126, dec.cache8_scales.shape, generator=gen, device="cuda", dtype=torch.uint8))
    return dec


def regions(dec):
    n = dec.cfg.n_pages
    return [t.view(n, -1) for t in (dec.pool, dec.cache8_values, dec.cache8_scales) if t is not None]


def request(dec, tokens, table=None):
    s = dec.request_add(0, tokens)
    dec.alloc_pages(s, tokens) if table is None else dec.block_table_set(s, table)
    dec.request_set_len(s, tokens)
    return s


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("count", [0, 1, 7, 385, 4000])
def test_copied_pages_and_no_others(shape, cache, count):
    if count == 4000 and shape[1] == 8:
        count = 500
    dec = decoder(shape, cache, n_pages=2 * count + 5)
    before = [t.clone() for t in regions(dec)]
    order = torch.randperm(2 * count + 5, generator=torch.Generator().manual_seed(count)).numpy()
    src, dst = order[:count], order[count:2 * count]
    dec.copy_pages(src, dst)
    for t, want in zip(regions(dec), before):
        want[torch.from_numpy(dst).cuda()] = want[torch.from_numpy(src).cuda()]
        assert torch.equal(t, want)
    assert dec.device_status() == 0


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_one_page_may_be_copied_to_many(cache):
    dec = decoder((4, 2, 64), cache, n_pages=40)
    dec.copy_pages([3] * 20, list(range(10, 30)))
    for t in regions(dec):
        assert (t[10:30] == t[3]).all() and not torch.equal(t[30], t[3])


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("shape", SHAPES)
def test_forks_read_what_their_parent_held(shape, cache):
    """Each fork, at lengths inside pages, at their ends and of nothing, goes on with tokens of its own; every request's cache is then its parent's prefix and
    those, and the parent's is untouched."""
    hkv, d = shape[1], shape[2]
    dec = decoder(shape, cache, n_pages=120, alloc_shuffle_seed=5)
    lens = [37, 64, 5]
    parents = [request(dec, n) for n in lens]
    at = [0, 1, 16, 31, 32, 37, 64, 48, 5, 5]
    of = [0, 0, 0, 0, 0, 0, 1, 1, 2, 2]
    kids = dec.fork([parents[i] for i in of], range(10), at)

    def read(slots, first, count):
        k, v = (torch.empty(sum(count), hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        dec.cache_read(list(slots), first, count, k, v)
        return [torch.stack(x) for x in zip(k.split(count), v.split(count))]

    held = read(parents, [0] * 3, lens)
    for got, i, n in zip(read(kids, [0] * 10, at), of, at):
        assert torch.equal(got, held[i][:, :n])
    gen = torch.Generator(device="cuda").manual_seed(2)
    k, v = (torch.randn(200, hkv, d, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    everyone, had = parents + kids.tolist(), lens + at
    more = [1 + (3 * r) % 19 for r in range(13)]
    for s, n, m in zip(everyone, had, more):
        dec.alloc_pages(s, n + m)
    dec.cache_append(everyone, more, had, k, v)
    start = np.concatenate([[0], np.cumsum(more)])
    both = [torch.stack([x[a:b] for x in (k, v)]) for a, b in zip(start[:-1], start[1:])]
    new = read(everyone, had, more)
    for r in range(13):
        if cache == "bf16":
            assert torch.equal(new[r], both[r])
        else:                                            # half a step of e4m3: 2^-4 of a value, 2^-10 of a unit that is at most 2^-7.8 of the row's largest
            x, y = both[r].float(), new[r].float()
            assert ((x - y).abs() <= 2.0 ** -4 * x.abs() + 2.0 ** -17 * x.abs().amax(-1, keepdim=True)).all()
    for got, i, n in zip(read(everyone, [0] * 13, had), [0, 1, 2] + of, had):
        assert torch.equal(got, held[i][:, :n])
    dec.requests_free(everyone)
    assert dec.velocity()["pages_free"] == 120 and dec.device_status() == 0


def test_a_mixed_step_over_shared_pages_is_that_over_copies():
    shape = (32, 8, 128)
    a, b = (decoder(shape, "bf16", n_pages=200, width=24, chunk_size=256) for _ in range(2))
    lens = [200, 131, 16]
    of, at = [0, 0, 1, 1, 2], [200, 190, 131, 112, 16]
    own = [request(a, n) for n in lens]
    kids = a.fork([own[i] for i in of], range(5), at).tolist()
    for s, n in zip(own + kids, lens + at):
        a.alloc_pages(s, n + 40)
    tables = a.block_tables(own + kids)
    others = []
    for r, n in enumerate(lens + at):                     # the same contents, every page a request's own
        s = request(b, n + 40)
        b.request_set_len(s, n)
        others.append(s)
    pa, pb = a.pool.view(200, -1), b.pool.view(200, -1)
    for r, s in enumerate(others):
        mine = b.block_table(s)[0]
        pb[torch.from_numpy(mine).long().cuda()] = pa[torch.from_numpy(tables[r][:len(mine)]).long().cuda()]
    q_len = [1, 1, 40, 1, 1, 17, 1, 1]
    n = sum(q_len)
    gen = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (torch.randn(n, h, 128, generator=gen, device="cuda").to(torch.bfloat16).view(torch.int16) for h in (32, 8, 8))
    outs = [torch.empty_like(q) for _ in range(2)]
    for dec, slots, out in ((a, own + kids, outs[0]), (b, others, outs[1])):
        dec.mixed_step(slots, q_len, lens + at, q, k, v, out)
        assert dec.device_status() == 0
    assert torch.equal(outs[0], outs[1])
    a.request_set_len(kids[0], 100)
    with pytest.raises(TsError) as e:
        a.mixed_step([kids[0]], [1], [100], q[:1], k[:1], v[:1], outs[0][:1])
    assert e.value.code == B.TS_ERR_SHARED_PAGE


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_compacting_keeps_every_request(cache):
    shape, n_pages = (4, 2, 64), 300
    dec = decoder(shape, cache, n_pages=n_pages, alloc_shuffle_seed=9, requests=32, width=20)
    lens = [300, 17, 160, 45, 250, 9]
    slots = [request(dec, n) for n in lens]
    kids = dec.fork(slots, range(6), [n // 2 for n in lens]).tolist()
    dec.requests_free([slots.pop(2)])
    lens = lens[:2] + lens[3:]
    everyone, had = slots + kids, lens + [150, 8, 80, 22, 125, 4]
    old = [t.clone() for t in regions(dec)]
    tables = dec.block_tables(everyone)
    k, v = (torch.empty(sum(had), 2, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    dec.cache_read(everyone, [0] * len(had), had, k, v)          # the device has the tables of before
    live = len(set(tables[tables >= 0].tolist()))
    first, used = dec.compact(5)
    assert len(first) == 5 and used > live
    rest, used = dec.compact()
    assert used == live and dec.compact()[0].size == 0
    moved = dict(np.concatenate([first, rest]).tolist())
    after = dec.block_tables(everyone)
    assert (after == np.vectorize(lambda p: moved.get(p, p))(tables)).all() and after.max() == live - 1
    for t, o in zip(regions(dec), old):
        for x, y in zip(after[after >= 0].tolist(), tables[tables >= 0].tolist()):
            assert torch.equal(t[x], o[y])
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    dec.cache_read(everyone, [0] * len(had), had, k2, v2)
    assert torch.equal(k, k2) and torch.equal(v, v2)
    new = request(dec, 320)                               # free pages are free, and once
    assert not set(dec.block_table(new)[0].tolist()) & set(after[after >= 0].tolist())
    dec.requests_free(everyone + [new])
    assert dec.velocity()["pages_free"] == n_pages


def test_copies_follow_the_stream_and_a_graph():
    dec = decoder((4, 2, 64), "bf16", n_pages=64)
    pool = dec.pool.view(64, -1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pool[1] = 77
        dec.copy_pages([1], [2])
    side.synchronize()
    assert (pool[2] == 77).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dec.copy_pages([1], [5])
    pool[1] = 78
    graph.replay()
    torch.cuda.synchronize()
    assert (pool[5] == 78).all() and (pool[2] == 77).all()


def test_refusals():
    dec = decoder((4, 2, 64), "bf16", n_pages=8)
    before = dec.pool.clone()
    s = request(dec, 20)
    for call in (lambda: dec.copy_pages([0], [8]), lambda: dec.copy_pages([1, 2], [3, 3]), lambda: dec.copy_pages([1], [1]), lambda: dec.fork([s], [0], [21]),
                 lambda: dec.fork([s] * 7, range(7)), lambda: dec.requests_free([s, s])):
        with pytest.raises(TsError):
            call()
    for call in (lambda: dec.copy_pages([0, 1], [2]), lambda: dec.fork([s], [0, 1]), lambda: dec.fork([s], [0], [1, 2])):
        with pytest.raises(ValueError):
            call()
    assert torch.equal(before, dec.pool) and dec.velocity()["pages_free"] == 6
