"""Projections with an adapter per request against the definition in 64 bits, on every kernel that a product can take, and the
decoder layer with adapters against the layer oracle with the adapters merged into its weights."""
import math

import numpy as np
import pytest
import torch

from paper_2512_03416_b200 import binding as B
from paper_2512_03416_b200.adapters import Adapters, adapted_project, stack_adapters
from paper_2512_03416_b200.decoder import TsError

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")


def make(seed, tokens, which, n, k, rank, count, residual=False, scale=True):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * std).to(torch.bfloat16)

    m = sum(tokens)
    a, b = normal(count, rank, k, std=k ** -0.5), normal(count, n, rank, std=rank ** -0.5)
    s = 0.5 + torch.rand(count, generator=gen, device="cuda") if scale else None
    return normal(m, k), normal(n, k, std=k ** -0.5), made(a, b, s), (normal(m, n) if residual else None)


def made(a, b, scale=None):
    ad = Adapters(a, b, scale)
    ad.given = (a, b, scale)                             # what the definition is taken of
    return ad


def definition(x, w, ad, tokens, which, residual):
    """y in 64 bits and, per element, how far rounding u to bf16 may move it: half a step 2^-9 of every |u| times |B|."""
    a, b, s = ad.given
    y, slack, at = x.double() @ w.double().T, torch.zeros(x.shape[0], w.shape[0], dtype=torch.float64, device="cuda"), 0
    for t, i in zip(tokens, which):
        if i >= 0:
            u = (x[at:at + t].double() @ a[i].double().T) * (1.0 if s is None else float(s[i]))
            y[at:at + t] += u @ b[i].double().T
            slack[at:at + t] = 2.0 ** -8 * u.abs() @ b[i].double().abs().T
        at += t
    return (y if residual is None else y + residual.double()), slack


def check(got, want, slack, k, rank):
    """A sum of k + rank + 1 products in fp32 is off by less than (k + rank) 2^-23 of the sum of their magnitudes, which for these inputs
    (unit variance) stays below 2 sqrt(k): 1e-4 covers it up to k = 16384 many times over. The result is rounded to bf16 once: 2^-8."""
    assert torch.isfinite(got.float()).all()
    err = (got.double() - want).abs()
    over = err - (2.0 ** -8 * want.abs() + slack + 1e-4 * (1 + want.abs()))
    assert float(over.max()) <= 0, float(over.max())


ROWS = {
    "one": ([1], [0]),
    "none_between": ([1, 2, 1, 5], [1, -1, 0, 1]),
    "decode_64": ([1] * 64, [(7 * r) % 11 for r in range(64)]),
    "decode_own": ([1] * 40, list(range(40))),
    "shared_apart": ([1] * 130, [r % 2 * 3 for r in range(130)]),
    "chunks": ([33, 1, 257, 1, 1, 128, 100], [0, 2, 1, -1, 2, 0, 2]),
    "long": ([1] * 9 + [600], [-1, 0, 1, 2, 0, 1, 2, -1, 2, 1]),
}


@pytest.mark.parametrize("tile_m", [0, 128, 256])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("n,k,rank", [(512, 1024, 16), (264, 72, 8), (640, 520, 24), (1024, 2048, 64), (256, 264, 136)])
def test_project_matches_the_definition(rows, n, k, rank, tile_m):
    tokens, which = ROWS[rows]
    x, w, ad, r = make(n + k + rank + sum(tokens), tokens, which, n, k, rank, max(which) + 1, residual=n == 640, scale=rank != 64)
    y = adapted_project(x, w, ad, tokens, which, residual=r, tile_m=tile_m)
    want, slack = definition(x, w, ad, tokens, which, r)
    assert int(ad.status.item()) == 0
    check(y, want, slack, k, rank)


def test_tokens_without_an_adapter_are_those_of_the_plain_product():
    """Zeros added to a sum leave it: a request without an adapter gets the bits that any adapters beside it leave."""
    tokens, which = ROWS["chunks"]
    x, w, ad, _ = make(3, tokens, which, 512, 1024, 32, 3)
    y = adapted_project(x, w, ad, tokens, which, tile_m=256)
    plain = adapted_project(x, w, ad, tokens, [-1] * len(tokens), tile_m=256)
    at = sum(tokens[:3])
    assert torch.equal(y[at], plain[at]) and not torch.equal(y[0], plain[0])


def test_foreign_nan_stays_with_its_adapter_and_its_tokens():
    tokens, which = [3, 1, 70, 2], [0, 1, 2, -1]
    x, w, ad, _ = make(4, tokens, which, 384, 512, 16, 3)
    clean = adapted_project(x, w, ad, tokens, which)
    ad.given[0][1].fill_(math.nan)
    x[5] = math.inf
    y = adapted_project(x, w, ad, tokens, which)
    bad = ~torch.isfinite(y.float()).all(1)
    assert bad.nonzero().flatten().tolist() == [3, 5]
    keep = ~bad
    assert torch.equal(y[keep], clean[keep])


def test_equal_calls_give_equal_bits_and_a_captured_call_follows_its_inputs():
    tokens, which = ROWS["decode_64"]
    x, w, ad, r = make(5, tokens, which, 1024, 2048, 16, 11, residual=True)
    first = adapted_project(x, w, ad, tokens, which, residual=r)
    for _ in range(3):
        assert torch.equal(adapted_project(x, w, ad, tokens, which, residual=r), first)
    out = torch.empty_like(first)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        adapted_project(x, w, ad, tokens, which, residual=r, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        adapted_project(x, w, ad, tokens, which, residual=r, out=out)
    x2 = torch.flip(x, [0])
    want = adapted_project(x2, w, ad, tokens, which, residual=r)
    x.copy_(x2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_an_adapter_changed_in_place_counts_from_the_next_call_on():
    """a and scale are not copied: a call reads what the work enqueued in front of it has written."""
    tokens, which = [1] * 64, [r % 16 for r in range(64)]
    x, w, ad, _ = make(8, tokens, which, 512, 4096, 32, 16)
    a, b, s = ad.given
    others = [(torch.randn_like(a.float()) / 64).to(torch.bfloat16) for _ in range(4)]
    torch.cuda.synchronize()
    got = []
    for o in others:
        a.copy_(o)
        s.mul_(1.25)
        got.append((adapted_project(x, w, ad, tokens, which), s.clone()))
    for y, o, scale in ((y, o, scale) for (y, scale), o in zip(got, others)):
        assert torch.equal(y, adapted_project(x, w, made(o, b, scale), tokens, which))


def test_stacked_adapters_are_those_of_the_parts():
    gen = torch.Generator(device="cuda").manual_seed(6)
    parts = [((torch.randn(2, r, 256, generator=gen, device="cuda") / 16).to(torch.bfloat16), (torch.randn(2, n, r, generator=gen, device="cuda") / 4).to(torch.bfloat16))
             for r, n in ((8, 256), (16, 64), (8, 64))]
    a, b = stack_adapters(parts)
    x, w = (torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16) for s in ((5, 256), (384, 256)))
    y = adapted_project(x, w / 16, Adapters(a, b), [2, 3], [1, 0])
    at = 0
    for part in parts:
        n = part[1].shape[1]
        alone = adapted_project(x, (w / 16)[at:at + n].contiguous(), made(*part), [2, 3], [1, 0])
        want, slack = definition(x, (w / 16)[at:at + n], made(*part), [2, 3], [1, 0], None)
        check(y[:, at:at + n], want, slack, 256, 32)
        check(alone, want, slack, 256, 16)
        at += n


def test_refusals():
    x, w, ad, _ = make(7, [4], [0], 256, 64, 8, 2)
    for tokens, which in (([4], [2]), ([4], [-2]), ([3], [0]), ([4, 1], [0, 0]), ([4, 0], [0, 0]), ([5, -1], [0, 0])):
        with pytest.raises(TsError):
            adapted_project(x, w, ad, tokens, which)
    with pytest.raises(ValueError):
        adapted_project(x, w, ad, [4], [0, 0])
    with pytest.raises(ValueError):
        adapted_project(x[:, :56], w, ad, [4], [0])
    with pytest.raises(ValueError):
        adapted_project(x, w.float(), ad, [4], [0])
    with pytest.raises(ValueError):
        Adapters(torch.zeros(1, 12, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 256, 12, dtype=torch.bfloat16, device="cuda"))
    for bad in (math.nan, math.inf, -math.inf):          # B is in the products of tokens that it is not for
        a, b, _ = ad.given
        b = b.clone()
        b[1, 255, 7] = bad
        for form in (b, b.view(torch.int16)):
            with pytest.raises(ValueError):
                Adapters(a, form)
    assert B.ts_adapter_workspace_bytes(4, 1, 2, 12) == 0 and B.ts_adapter_workspace_bytes(4000, 1025, 2, 8) == 0
    need = B.ts_adapter_workspace_bytes(4, 1, 2, 8)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    rc = B.ts_adapter_project(0, 4, 256, 64, x.data_ptr(), w.data_ptr(), 0, w.data_ptr(), ad.args, 1, [4], [0], ws.data_ptr(), need - 1, 0,
                              ad.status.data_ptr(), 0)
    assert rc == B.TS_ERR_WORKSPACE
    assert adapted_project(x[:0], w, ad, [], []).shape == (0, 256)


@pytest.mark.parametrize("rows,tokens", [(1024, 1), (512, 64), (300, 27)])
def test_as_many_rows_as_are_served(rows, tokens):
    """The longest plans: every row another adapter than its neighbours, or its own."""
    for which in ([r % 7 - 1 for r in range(rows)], list(range(rows))):
        count = max(which) + 1
        x, w, ad, _ = make(rows, [tokens] * rows, which, 128, 64, 8, count)
        y = adapted_project(x, w, ad, [tokens] * rows, which)
        want, slack = definition(x, w, ad, [tokens] * rows, which, None)
        check(y, want, slack, 64, 8)
        assert int(ad.status.item()) == 0
    with pytest.raises(TsError):
        adapted_project(x.new_zeros(9000, 64), w, ad, [9] * 1000, [0] * 1000)
