"""ts_tree_attention over both caches against its definition in 64 bits: shapes, lengths, masks, what masked places may hold."""
import math

import numpy as np
import pytest
import torch

from paper_2512_03416_b200 import binding as B
from paper_2512_03416_b200 import workloads as wl
from paper_2512_03416_b200.decoder import Decoder
from paper_2512_03416_b200.harness import to_dev
from tests import tree_oracle as O

pytestmark = pytest.mark.gpu


def _need_gpu():
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required")


def bf16(x):
    """float array -> (bits, the float64 values they stand for)."""
    b = wl.f32_to_bf16_bits(np.asarray(x, np.float32))
    return b, wl.bf16_bits_to_f32(b).astype(np.float64)


class Case:
    """A decoder whose cache holds random context (everything else NaN), drafted nodes, and what they must give."""

    def __init__(self, shape, cache, rows, masks="tree", seed=0, k_size=1.0, v_size=lambda rng, n: np.ones(n), extra=0):
        _need_gpu()
        self.hq, self.hkv, self.d = shape
        self.rows, self.cache = rows, cache
        rng = self.rng = np.random.default_rng(seed)
        self.ctx, self.nodes = [c for c, _ in rows], [t for _, t in rows]
        n = self.n = sum(self.nodes)
        pages = [-(-c // 16) for c in self.ctx]
        self.dec = Decoder(self.hq, self.hkv, self.d, n_pages=sum(pages) + 3, max_requests=len(rows) + extra, max_pages_per_req=max(pages + [1]),
                           alloc_shuffle_seed=seed + 1, cache=cache, nan_fill=True)
        self.k, self.v, self.slots = [], [], []
        for r, c in enumerate(self.ctx):
            slot = self.dec.request_add(r, c)
            self.slots.append(slot)
            kb, kf = bf16(rng.standard_normal((c, self.hkv, self.d)) * k_size)
            vb, vf = bf16(rng.standard_normal((c, self.hkv, self.d)) * v_size(rng, c)[:, None, None])
            if c:
                self.dec.alloc_pages(slot, c)
                self.dec.cache_append([slot], [c], [0], to_dev(kb), to_dev(vb))
                if cache == "e4m3":                              # what the cache holds now, read back
                    ko, vo = (torch.empty((c, self.hkv, self.d), dtype=torch.int16, device="cuda") for _ in range(2))
                    self.dec.cache_read([slot], [0], [c], ko, vo)
                    kf, vf = (wl.bf16_bits_to_f32(t.cpu().numpy().view(np.uint16)).astype(np.float64) for t in (ko, vo))
            self.k.append(kf)
            self.v.append(vf)
        self.qb, self.q = bf16(rng.standard_normal((n, self.hq, self.d)))
        self.kb, self.kn = bf16(rng.standard_normal((n, self.hkv, self.d)) * k_size)
        self.vb, self.vn = bf16(rng.standard_normal((n, self.hkv, self.d)) * v_size(rng, n)[:, None, None])
        self.mask = None if masks is None else np.array([m for t in self.nodes for m in self._masks(masks, t)], np.uint64)

    def _masks(self, kind, t):
        if kind == "tree":
            rc, m = B.ts_tree_masks([-1 if i == 0 else int(self.rng.integers(-1, i)) for i in range(t)])
            assert rc == B.TS_OK
            return m
        if kind == "none":
            return [0] * t
        if kind == "any":                                       # any bits, those behind the last node too
            return [int(x) for x in self.rng.integers(0, 1 << 63, t, dtype=np.uint64) * 2 + self.rng.integers(0, 2, t, dtype=np.uint64)]
        raise ValueError(kind)

    def run(self):
        out = torch.full((self.n, self.hq, self.d), 0x7FC0, dtype=torch.int16, device="cuda")
        mask = None if self.mask is None else torch.from_numpy(self.mask.view(np.int64)).cuda()
        self.dec.tree_attention(self.slots, self.nodes, self.ctx, to_dev(self.qb), to_dev(self.kb), to_dev(self.vb), out, mask=mask)
        assert self.dec.device_status() == 0
        return wl.bf16_bits_to_f32(out.cpu().numpy().view(np.uint16)).astype(np.float64)

    def seen(self, r):
        t, c, first = self.nodes[r], self.ctx[r], sum(self.nodes[:r])
        s = np.ones((t, c + t), bool)
        for i in range(t):
            bits = (2 << i) - 1 if self.mask is None else int(self.mask[first + i])
            s[i, c:] = [(bits >> j) & 1 for j in range(t)]
        return s

    def want(self):
        outs, bounds = [], []
        for r in range(len(self.rows)):
            a, b = sum(self.nodes[:r]), sum(self.nodes[:r + 1])
            o, w = O.attention(self.q[a:b], np.concatenate([self.k[r], self.kn[a:b]]), np.concatenate([self.v[r], self.vn[a:b]]), self.seen(r),
                               1 / math.sqrt(self.d))
            outs.append(o)
            bounds.append(w)
        return np.concatenate(outs), np.concatenate(bounds)

    def check(self, got=None):
        """Weights are rounded to 8 significant bits (2^-9 of each) and so is the result; scores, sums and the exponentials are
        fp32. Twice that of sum p|v| is the bound, 2^-8 + 2^-8 |out|."""
        got = self.run() if got is None else got
        want, bound = self.want()
        assert np.isfinite(got).all()
        over = np.abs(got - want) - 2.0 ** -8 * (bound + np.abs(want))
        assert over.max() <= 0, (np.unravel_index(over.argmax(), over.shape), over.max())
        return got


SHAPES = [(4, 2, 64), (3, 3, 64), (16, 1, 64), (6, 2, 64), (2, 2, 128), (32, 8, 128), (16, 1, 128), (20, 4, 128), (64, 8, 128), (9, 3, 128)]
ROWS = [[(0, 1)], [(1, 1), (15, 1), (16, 1), (17, 1)], [(0, 64)], [(1, 3), (0, 2), (16, 17), (33, 64), (300, 1)], [(129, 16), (40, 5)]]


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("rows", ROWS, ids=lambda r: "_".join(f"{c}+{t}" for c, t in r))
def test_shapes_and_lengths(shape, cache, rows):
    Case(shape, cache, rows, seed=sum(c + t for c, t in rows)).check()


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("shape,rows", [((8, 2, 64), [(5000, 7), (0, 3), (1200, 64)]), ((8, 2, 128), [(9000, 1)]), ((16, 2, 128), [(6001, 33), (70, 2)]),
                                        ((8, 1, 128), [(3000, 64), (2999, 63)]), ((4, 1, 128), [(20000, 64)])], ids=lambda v: str(v))
def test_split_rows(shape, cache, rows):
    """Long rows, which are split over thread blocks and merged."""
    c = Case(shape, cache, rows, seed=3)
    before = c.dec.velocity()["kernel_launches"]
    got = c.check()
    assert c.dec.velocity()["kernel_launches"] - before >= 2     # with the merge
    assert np.array_equal(got, c.run()), "another bit pattern the second time"


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("shape", [(8, 2, 64), (32, 8, 128), (16, 1, 128)], ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("masks", [None, "none", "any"])
def test_masks(shape, cache, masks):
    """Chains, nodes that see no node (with and without cached tokens: then the output is zero), and any bits."""
    c = Case(shape, cache, [(0, 5), (31, 40), (0, 1), (64, 64), (2500, 30)], masks=masks, seed=11)
    got = c.check()
    if masks == "none":
        assert (got[:5] == 0).all() and (got[45] == 0).all()


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("shape", [(8, 2, 64), (32, 8, 128)], ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("nodes", [3, 40])
def test_what_is_not_seen_may_hold_anything(shape, cache, nodes):
    """Node 1's K and V are infinities and NaN: only its viewers may notice."""
    c = Case(shape, cache, [(20, nodes), (0, nodes)], masks="tree", seed=5)
    for r in range(2):
        first = r * nodes
        for i in range(nodes):                                   # nobody sees node 1 but node 1 itself and node 2
            m = int(c.mask[first + i]) & ~2
            c.mask[first + i] = m | (2 if i in (1, 2) else 0)
        c.kb[first + 1] = np.where(np.arange(c.d) % 2, 0x7F80, 0x7FC0)
        c.vb[first + 1] = np.where(np.arange(c.d) % 2, 0xFF80, 0x7FC0)
    got = c.run()
    want, bound = c.want()                                       # of the values from before
    for i in range(2 * nodes):
        if i % nodes in (1, 2):
            assert np.isnan(got[i]).all()
        else:
            assert (np.abs(got[i] - want[i]) <= 2.0 ** -8 * (bound[i] + np.abs(want[i]))).all(), i


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("nodes", [2, 40])
def test_infinite_v_of_a_seen_node(cache, nodes):
    c = Case((32, 8, 128), cache, [(20, nodes)], masks=None, seed=6)
    c.vb[1, 3, 5] = 0x7F80                                       # one element of one head
    got = c.run()
    want, bound = c.want()
    heads = np.arange(32) // 4 == 3
    assert np.isnan(got[1:, heads]).all()
    ok = np.abs(got - want) <= 2.0 ** -8 * (bound + np.abs(want))
    assert ok[0].all() and ok[1:, ~heads].all()


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("nodes", [1, 6, 33])
def test_sizes_of_values(cache, nodes):
    """V rows whose sizes span 2^60 (2^14 within 32 neighbouring keys), K and Q that make single keys dominate: weights down to
    2^-100 of the largest."""
    for seed, k_size in ((1, 0.01), (2, 1.0), (3, 6.0)):
        Case((8, 2, 128), cache, [(700, nodes), (0, nodes)], seed=seed, k_size=k_size,
             v_size=lambda rng, n: 2.0 ** (np.repeat(rng.integers(-40, 7, n // 32 + 1), 32)[:n] + rng.integers(0, 15, n))).check()


@pytest.mark.parametrize("nodes", [1, 40])
def test_a_row_of_nan_in_the_cache(nodes):
    """One cached token's V (then K) holds a NaN: it is seen by all nodes of its row, and of that KV head alone."""
    for which in (0, 1):
        c = Case((8, 2, 128), "e4m3", [(100, nodes), (50, nodes)], seed=12)
        kb, vb = (to_dev(wl.f32_to_bf16_bits(c.rng.standard_normal((1, 2, 128)).astype(np.float32))) for _ in range(2))
        (vb, kb)[which][0, 1, 7] = 0x7FC0
        c.dec.request_set_len(c.slots[0], 99)
        c.dec.cache_append([c.slots[0]], [1], [99], kb, vb)
        got = c.run()
        assert np.isnan(got[:nodes, 4:]).all() and np.isfinite(got[:nodes, :4]).all() and np.isfinite(got[nodes:]).all()


@pytest.mark.parametrize("nodes", [1, 12, 64])
def test_many_small_weights_next_to_a_large_one(nodes):
    """One key at 2^19 times the weight of 16000 others, all with the same V: what the small ones carry together is 3 %."""
    c = Case((8, 2, 128), "e4m3", [(16000, nodes)], masks="none", seed=8)
    d = c.d
    kb = np.zeros((16000, 2, d))
    kb[77, :, 0] = 2.0
    vb = np.ones((16000, 2, d))
    vb[77] = 0.0
    slot = c.slots[0]
    c.dec.request_set_len(slot, 0)
    c.dec.cache_append([slot], [16000], [0], to_dev(bf16(kb)[0]), to_dev(bf16(vb)[0]))
    q = np.zeros((c.n, c.hq, d))
    q[:, :, 0] = 19 * math.log(2) * math.sqrt(d) / 2
    c.qb, c.q = bf16(q)
    c.k, c.v = [kb], [vb]
    c.check()


def test_one_node_is_a_decode_row():
    c = Case((32, 8, 128), "bf16", [(500, 1), (16, 1), (3000, 1)], masks=None, seed=4)
    got = c.check()
    for s, ctx in zip(c.slots, c.ctx):
        c.dec.alloc_pages(s, ctx + 1)
    out = torch.empty((c.n, c.hq, c.d), dtype=torch.int16, device="cuda")
    c.dec.mixed_step(c.slots, [1] * 3, c.ctx, to_dev(c.qb), to_dev(c.kb), to_dev(c.vb), out)
    c.check(wl.bf16_bits_to_f32(out.cpu().numpy().view(np.uint16)).astype(np.float64))
    assert np.abs(got).max() > 0


def test_another_stream():
    c = Case((8, 2, 128), "e4m3", [(900, 20)], seed=9)
    want = c.check()
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        assert np.array_equal(c.run(), want)


def test_large_page_numbers():
    """Pages whose byte offset passes 2^32 in both caches."""
    for cache in ("bf16", "e4m3"):
        n_pages = (1 << 32) // (2 * 8 * 16 * 128) + 300            # 8-bit: 32 KB a page
        dec = Decoder(32, 8, 128, n_pages=n_pages, max_requests=1, max_pages_per_req=8, cache=cache)
        slot = dec.request_add(0, 100)
        dec.block_table_set(slot, [n_pages - 1, 5, n_pages - 7, n_pages - 100, 0, n_pages - 2, 9])
        rng = np.random.default_rng(1)
        kb, kf = bf16(rng.integers(-3, 4, (101, 8, 128)))          # small whole numbers: exact in 8 bits
        vb, vf = bf16(rng.integers(-3, 4, (101, 8, 128)))
        qb, qf = bf16(rng.standard_normal((1, 32, 128)) / 8)
        dec.cache_append([slot], [100], [0], to_dev(kb[:100]), to_dev(vb[:100]))
        out = torch.empty((1, 32, 128), dtype=torch.int16, device="cuda")
        dec.tree_attention([slot], [1], [100], to_dev(qb), to_dev(kb[100:]), to_dev(vb[100:]), out)
        got = wl.bf16_bits_to_f32(out.cpu().numpy().view(np.uint16)).astype(np.float64)
        want, bound = O.attention(qf, kf, vf, np.ones((1, 101), bool), 128 ** -0.5)
        assert (np.abs(got - want) <= 2.0 ** -8 * (bound + np.abs(want))).all()
        dec.close()
        del dec
        torch.cuda.empty_cache()


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("shape,nodes", [((8, 2, 128), 3), ((8, 2, 128), 6), ((16, 2, 128), 2), ((16, 1, 128), 2)], ids=lambda v: str(v))
@pytest.mark.parametrize("keys", [150, 399, 401, 4100])
def test_few_nodes_of_short_and_long_rows(shape, nodes, cache, keys):
    """Nine to 32 queries per KV head, of rows on both sides of the lengths that choose a step's kernel."""
    Case(shape, cache, [(keys, nodes), (keys - 3, 1), (keys + 3, nodes)], seed=keys + nodes).check()


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("shape", [(8, 2, 64), (8, 2, 128), (16, 1, 128)], ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("nodes", [1, 3, 40])
def test_queries_that_are_not_finite(shape, nodes, cache):
    """A query with an infinity or a NaN has no softmax, not even where all its scores are -inf: NaN where it sees a key, zeros where it sees
    none, and nothing of it in the other queries. Long and short rows, whichever kernel they are on."""
    c = Case(shape, cache, [(37, nodes), (0, nodes), (2300, nodes)], masks="tree", seed=41)
    c.mask[nodes] = 0                                            # the second row's first node sees nothing
    bad = np.zeros((c.n, c.hq), bool)
    for r, node in enumerate((0, 0, nodes - 1)):
        for h, (at, bits) in enumerate(((0, 0x7F80), (c.d - 1, 0xFF80), (17, 0x7FC0))):
            c.qb[r * nodes + node, h, at] = bits
            bad[r * nodes + node, h] = True
    # -inf times what is above 0 in all keys: every score is -inf
    for x in [*c.k, c.kn]:
        x[:, 0, 0] = 1.0
    c.kb[:, 0, 0] = 0x3F80
    for r, ctx in enumerate(c.ctx):
        if ctx:
            kb, vb = bf16(c.k[r])[0], bf16(c.v[r])[0]
            c.dec.request_set_len(c.slots[r], 0)
            c.dec.cache_append([c.slots[r]], [ctx], [0], to_dev(kb), to_dev(vb))
            if cache == "e4m3":
                ko, vo = (torch.empty((ctx, c.hkv, c.d), dtype=torch.int16, device="cuda") for _ in range(2))
                c.dec.cache_read([c.slots[r]], [0], [ctx], ko, vo)
                c.k[r], c.v[r] = (wl.bf16_bits_to_f32(t.cpu().numpy().view(np.uint16)).astype(np.float64) for t in (ko, vo))
    c.qb[0, 0] = c.qb[nodes, 0] = 0
    c.qb[0, 0, 0] = c.qb[nodes, 0, 0] = 0xFF80
    got = c.run()
    want, bound = c.want()                                       # of the finite queries from before
    ok = np.abs(got - want) <= 2.0 ** -8 * (bound + np.abs(want))
    assert ok[~bad].all()
    blind = np.zeros((c.n, c.hq), bool)
    blind[nodes] = True
    assert np.isnan(got[bad & ~blind]).all()
    assert (got[blind] == 0).all()


@pytest.mark.parametrize("nodes", [2, 5, 40])
def test_infinite_k_of_a_seen_node(nodes):
    """Over the 8-bit cache, whose codes have no infinities: the node's viewers get NaN, whichever kernel they are on."""
    c = Case((16, 4, 128), "e4m3", [(20, nodes), (2100, nodes)], masks=None, seed=43)
    for r in range(2):
        c.kb[r * nodes + 1, r, 5] = (0x7F80, 0xFF80)[r]
    got = c.run()
    want, bound = c.want()
    ok = np.abs(got - want) <= 2.0 ** -8 * (bound + np.abs(want))
    for r in range(2):
        heads = np.arange(16) // 4 == r
        mine = slice(r * nodes, (r + 1) * nodes)
        assert np.isnan(got[mine][1:, heads]).all()
        assert ok[mine][0].all() and ok[mine][:, ~heads].all()


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nodes", [1, 6, 12, 33])
@pytest.mark.parametrize("size", [-6, -20, -40])
def test_v_rows_of_zeros(size, nodes, d, cache):
    """Some cached tokens and nodes, and a stretch of 40 tokens, whose V is zero, among small ones: zeros are smaller than any of them."""
    def v_size(rng, n):
        i = np.arange(n)
        return np.where((i % 7 == 3) | ((i >= 200) & (i < 240)), 0.0, 2.0 ** size)
    Case((8, 2, d), cache, [(700, nodes), (0, nodes), (2100, nodes), (5, nodes)], seed=51, v_size=v_size).check()


@pytest.mark.parametrize("nodes", [1, 33])
def test_nothing_but_zeros(nodes):
    c = Case((8, 2, 128), "e4m3", [(300, nodes), (0, nodes)], seed=52, v_size=lambda rng, n: np.zeros(n))
    assert (c.check() == 0).all()
