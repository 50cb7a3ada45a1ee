"""Bookkeeping of shared pages without a GPU: forks at page ends copy nothing, uses are counted, writes into shared pages are refused."""
import numpy as np
import pytest

from paper_2512_03416_b200 import binding as B


def ctx(n_pages=64, max_requests=16, width=16, reserved=0):
    cfg = B.ts_config(4, 2, 64, 16, n_pages, max_requests, width, 512, reserved, 0, 0, 0.0, 0, 0, None, 0, None, 0, 0, 0)
    rc, h = B.ts_create(cfg)
    assert rc == B.TS_OK
    return h


def i32(*a):
    return np.array(a, dtype=np.int32)


def fork(h, slots, lens=None):
    out = np.full(len(slots), -9, dtype=np.int32)
    rc = B.ts_request_fork(h, i32(*slots), None if lens is None else i32(*lens), np.arange(100, 100 + len(slots)), out, 0)
    return rc, out.tolist()


def request(h, tokens, room=None):
    _, s = B.ts_request_add(h, 1, tokens, 0)
    assert B.ts_alloc_pages(h, s, tokens if room is None else room, 0) == B.TS_OK and B.ts_request_set_len(h, s, tokens) == B.TS_OK
    return s


def plan(h, slot, q, c):
    st, keep = B.make_step([slot], [q], [c])
    return B.ts_plan_step(h, st)[0]


def free_pages(h):
    return B.ts_velocity(h)[1]["pages_free"]


def test_forks_share_whole_pages_and_the_last_use_frees_them():
    h = ctx()
    a = request(h, 48, 80)
    assert free_pages(h) == 59
    rc, (b, c) = fork(h, [a, a], [48, 32])
    assert rc == B.TS_OK and free_pages(h) == 59
    ta, tb, tc = (B.ts_block_table(h, s) for s in (a, b, c))
    assert tb[1] == ta[1][:3] and tc[1] == ta[1][:2] and (tb[2], tc[2]) == (48, 32)
    rc, (d,) = fork(h, [b])
    assert rc == B.TS_OK and B.ts_block_table(h, d)[1] == ta[1][:3]
    assert B.ts_request_free(h, a) == B.TS_OK and free_pages(h) == 61            # what only a held
    assert B.ts_requests_free(h, i32(b, d)) == B.TS_OK and free_pages(h) == 62
    assert B.ts_requests_free(h, i32(c)) == B.TS_OK and free_pages(h) == 64
    s = request(h, 64 * 16 // 4)
    pages = B.ts_block_table(h, s)[1]
    assert len(set(pages)) == 16
    B.ts_destroy(h)


def test_writes_into_shared_pages_are_refused_until_they_are_not():
    h = ctx()
    a = request(h, 32, 64)
    _, (b,) = fork(h, [a])
    assert plan(h, a, 1, 32) == B.TS_OK                                          # a's next page is its own
    assert plan(h, b, 1, 32) == B.TS_ERR_TABLE_SHORT
    assert B.ts_alloc_pages(h, b, 40, 0) == B.TS_OK and plan(h, b, 8, 32) == B.TS_OK
    assert B.ts_request_set_len(h, b, 20) == B.TS_OK
    assert plan(h, b, 1, 20) == plan(h, b, 20, 20) == B.TS_ERR_SHARED_PAGE
    st, keep = B.make_step([b], [1], [20])
    assert B.ts_cache_append(h, st, B.TS_CACHE_BF16, 0, 0, 0) == B.TS_ERR_SHARED_PAGE
    assert B.ts_kv_append(h, st, 0) == B.TS_ERR_SHARED_PAGE
    assert B.ts_request_free(h, a) == B.TS_OK
    assert plan(h, b, 1, 20) == B.TS_OK
    B.ts_destroy(h)


def test_fork_refusals_change_nothing():
    h = ctx(n_pages=8, max_requests=3)
    a = request(h, 32)
    before = B.ts_velocity(h)
    for slots, lens in (([a], [33]), ([a], [-1]), ([5], None), ([-1], None), ([a, 2], None)):
        assert fork(h, slots, lens)[0] == B.TS_ERR_INVALID
    assert fork(h, [a, a, a])[0] == B.TS_ERR_NO_SLOT
    assert fork(h, [a], [20])[0] == B.TS_ERR_CUDA                                # a page to copy, and no pool
    assert B.ts_velocity(h) == before and fork(h, [a, a])[0] == B.TS_OK
    B.ts_destroy(h)
    h = ctx(n_pages=4, max_requests=8, reserved=1)
    a = request(h, 17)
    assert fork(h, [a, a])[0] == B.TS_ERR_NO_PAGES
    assert B.ts_requests_free(h, i32(a, a)) == B.ts_requests_free(h, i32(a, 7)) == B.TS_ERR_INVALID
    assert B.ts_block_table(h, a)[2] == 17
    assert fork(h, [])[0] == B.TS_OK and B.ts_requests_free(h, i32()) == B.TS_OK
    B.ts_destroy(h)


def test_tables_set_by_hand_and_shared_pages():
    h = ctx()
    a = request(h, 32)
    _, (b,) = fork(h, [a])
    p, q = B.ts_block_table(h, a)[1]
    assert B.ts_block_table_set(h, b, [q, p, 40]) == B.TS_OK                     # its own pages in another order
    c = request(h, 16)
    assert B.ts_block_table_set(h, c, [p]) == B.TS_ERR_INVALID                   # another's
    assert B.ts_block_table_set(h, a, [50, 51]) == B.TS_OK and B.ts_block_table_set(h, c, [p]) == B.TS_ERR_INVALID
    assert B.ts_block_table_set(h, b, [41]) == B.TS_OK and B.ts_block_table_set(h, c, [p, q, 40]) == B.TS_OK
    assert free_pages(h) == 64 - 6
    B.ts_destroy(h)


def test_copy_refusals():
    h = ctx()
    a = request(h, 32)
    fork(h, [a])
    p = B.ts_block_table(h, a)[1][0]
    for src, dst in (((3,), (64,)), ((-1,), (3,)), ((3, 4), (5, 5)), ((3,), (3,)), ((3, 4), (5, 3))):
        assert B.ts_copy_pages(h, i32(*src), i32(*dst), 0) == B.TS_ERR_INVALID
    assert B.ts_copy_pages(h, i32(20), i32(p), 0) == B.TS_ERR_SHARED_PAGE
    assert B.ts_copy_pages(h, i32(20), i32(21), 0) == B.TS_ERR_CUDA              # no pool
    assert B.ts_copy_pages(h, i32(), i32(), 0) == B.TS_OK
    out = np.zeros((1, 2), dtype=np.int32)
    assert B.ts_block_tables(h, i32(a), out) == B.TS_OK and out.tolist() == [B.ts_block_table(h, a)[1]]
    assert B.ts_block_tables(h, i32(a), out[:, :1].copy()) == B.TS_ERR_TABLE_SHORT
    assert B.ts_block_tables(h, i32(9), out) == B.TS_ERR_INVALID
    B.ts_destroy(h)


def test_compacting_a_compact_pool_moves_nothing():
    h = ctx()
    a = request(h, 48)
    moves = np.empty((64, 2), dtype=np.int32)
    assert B.ts_compact_pages(h, 64, moves, 0) == (B.TS_OK, 0, 3)
    assert B.ts_compact_pages(h, -1, moves, 0)[0] == B.TS_ERR_INVALID
    assert B.ts_block_table_set(h, a, [40, 0, 41]) == B.TS_OK
    assert B.ts_compact_pages(h, 64, moves, 0)[0] == B.TS_ERR_CUDA and B.ts_block_table(h, a)[1] == [40, 0, 41]    # no pool
    assert B.ts_compact_pages(h, 0, moves, 0) == (B.TS_OK, 0, 42)
    B.ts_destroy(h)


@pytest.mark.parametrize("seed", range(4))
def test_counts_hold_over_random_calls(seed):
    rng, h, live = np.random.default_rng(seed), ctx(n_pages=40, max_requests=12), []
    for _ in range(400):
        what = rng.integers(0, 4)
        if what == 0:
            rc, s = B.ts_request_add(h, 1, 0, 0)
            if rc == B.TS_OK:
                n = int(rng.integers(0, 6)) * 16
                if B.ts_alloc_pages(h, s, n, 0) == B.TS_OK:
                    B.ts_request_set_len(h, s, n)
                live.append(s)
        elif what == 1 and live:
            rc, new = fork(h, [int(rng.choice(live)) for _ in range(int(rng.integers(1, 4)))])
            assert rc in (B.TS_OK, B.TS_ERR_NO_SLOT)
            live += new if rc == B.TS_OK else []
        elif what == 2 and live:
            B.ts_request_free(h, live.pop(int(rng.integers(0, len(live)))))
        elif live:
            s = int(rng.choice(live))
            B.ts_alloc_pages(h, s, 16 * int(rng.integers(0, 8)), 0)
        used = set().union(*[B.ts_block_table(h, s)[1] for s in live]) if live else set()
        assert B.ts_velocity(h)[1]["pages_in_use"] == len(used)
    B.ts_destroy(h)


@pytest.mark.parametrize("seed", range(4))
def test_requests_freed_together_leave_what_they_leave_one_by_one(seed):
    """Forks of forks at any lengths, freed in any order: the free pages come in the same order, so that new requests get the same pages."""
    tables = []
    for together in (False, True):
        rng, h = np.random.default_rng(seed), ctx(n_pages=60, max_requests=40)
        live = [request(h, 16 * int(rng.integers(1, 9))) for _ in range(3)]
        for _ in range(12):
            s = int(rng.choice(live))
            rc, new = fork(h, [s] * 3, [16 * int(rng.integers(0, B.ts_block_table(h, s)[2] // 16 + 1)) for _ in range(3)])
            assert rc == B.TS_OK
            live += new
            B.ts_alloc_pages(h, new[0], B.ts_block_table(h, new[0])[2] + 16, 0)
        gone = rng.permutation(live)[:int(rng.integers(5, 30))] if seed % 2 else np.array(live[3:][::-1])
        gone = gone.astype(np.int32)
        if together:
            assert B.ts_requests_free(h, gone) == B.TS_OK
        else:
            for s in gone:
                assert B.ts_request_free(h, int(s)) == B.TS_OK
        rest = [s for s in live if s not in gone]
        used = set().union(*[B.ts_block_table(h, s)[1] for s in rest]) if rest else set()
        assert free_pages(h) == 60 - len(used)
        new = [request(h, 16 * k) for k in (3, 1, 5)]
        tables.append([B.ts_block_table(h, s)[1] for s in new] + [new])
        B.ts_requests_free(h, i32(*rest, *new))
        assert free_pages(h) == 60
        B.ts_destroy(h)
    assert tables[0] == tables[1]
