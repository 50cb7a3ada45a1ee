"""How the tokens of a call with adapters are divided (ts_adapter_plan, host only): every call within the documented limits has a plan."""
import numpy as np
import pytest

from paper_2512_03416_b200 import binding as B

MANY_ROWS, LONG = (1024, 8192), (512, 32768)          # rows, tokens


def tiles_of(tokens):
    """Tokens of a tile that a product of so many can have: 128, or those of a pair's where it takes up to three tiles more than need be."""
    least = -(-tokens // 256)
    return sorted({128} | {(-(-tokens // m) + 15) // 16 * 16 for m in range(least, least + 4)})


def plain(tokens, which, tile):
    """Entries and, per adapter, tokens, counted token by token."""
    of = np.repeat(which, tokens)
    entries = sum(len(set(of[t:t + tile].tolist()) - {-1}) for t in range(0, len(of), tile))
    return entries, np.bincount(of[of >= 0], minlength=max(which) + 1)


def check(tokens, which):
    m, count = sum(tokens), max(max(which) + 1, 1)
    for tile in tiles_of(m):
        rc, (entries, groups, group, words) = B.ts_adapter_plan(m, tile, tokens, which, count)
        assert rc == B.TS_OK, (len(tokens), m, tile)
        want, per = plain(tokens, which, tile)
        assert entries == want and group in (16, 64) and groups == sum(-(-int(n) // group) for n in per)
        assert words <= 7936


def mixed(rng, rows, tokens, long):
    """So many rows and tokens, of rows of 1 and of `long` tokens and one of what is left."""
    n = min((tokens - rows) // (long - 1), rows - 1)
    lens = [long] * n + [1] * (rows - n)
    lens[-1] += min(tokens - sum(lens), long)
    return rng.permutation(lens).tolist()


@pytest.mark.parametrize("rows,tokens", [MANY_ROWS, LONG, (920, 8192), (1024, 4096), (1024, 1024), (513, 8192), (512, 512)])
@pytest.mark.parametrize("long", [2, 15, 16, 17, 18, 33, 49, 64, 65, 129])
def test_rows_of_two_lengths_up_to_the_limits(rows, tokens, long):
    rng = np.random.default_rng(rows + long)
    lens = mixed(rng, rows, tokens, long)
    for which in (range(rows), rng.permutation(rows), np.arange(rows) % 7 - 1, np.arange(rows) // 2, rng.integers(-1, rows, rows)):
        check(lens, [int(a) for a in which])


@pytest.mark.parametrize("seed", range(60))
def test_rows_of_any_lengths_up_to_the_limits(seed):
    rng = np.random.default_rng(seed)
    most_rows, most_tokens = MANY_ROWS if seed % 2 else LONG
    rows = most_rows if seed % 3 else int(rng.integers(1, most_rows + 1))
    cuts = np.sort(rng.choice(np.arange(1, most_tokens), rows - 1, replace=False))
    lens = np.diff(np.concatenate([[0], cuts, [most_tokens]])).tolist()
    check(lens, rng.permutation(rows).tolist())
    check(lens, rng.integers(-1, max(1, rows // int(rng.integers(1, 9))), rows).tolist())


def test_the_mix_with_the_longest_plan():
    """8410 words in groups of 16: it has to be groups of 64."""
    lens = np.random.default_rng(1).permutation([17] * 448 + [1] * 576).tolist()
    rc, (entries, groups, group, words) = B.ts_adapter_plan(8192, 128, lens, list(range(1024)), 1024)
    assert rc == B.TS_OK and group == 64 and groups == 1024 and words <= 7936
    check(lens, list(range(1024)))


def test_refusals():
    ok = (100, 128, [50, 50], [0, -1], 1)
    assert B.ts_adapter_plan(*ok)[0] == B.TS_OK
    for i, bad in ((0, 0), (0, 99), (1, 0), (1, 24), (1, 272), (2, [100]), (2, [100, 0]), (2, [101, -1]), (3, [1, 0]), (3, [0, -2]), (4, 0), (4, 65537)):
        args = list(ok)
        args[i] = bad
        assert B.ts_adapter_plan(*args)[0] == B.TS_ERR_INVALID, (i, bad)
    for rows, tokens in ((1025, 1025), (513, 8193), (512, 32769)):
        lens = [1] * (rows - 1) + [tokens - rows + 1]
        assert B.ts_adapter_plan(tokens, 128, lens, [0] * rows, 1)[0] == B.TS_ERR_UNSUPPORTED
