"""Verification of drafted tokens against a walk in 64 bits: emitted tokens and paths exactly, log probabilities to fp32."""
import math

import numpy as np
import pytest
import torch

from paper_2512_03416_b200 import binding as B
from paper_2512_03416_b200.verify import verify_tokens
from tests.verify_oracle import walk

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")


def trees(rng, nodes, kind):
    out = []
    for n in nodes:
        if kind == "chain":
            out.append([-1] + list(range(n - 1)))
        elif kind == "star":
            out.append([-1] + [0] * (n - 1))
        else:
            out.append([-1] + [int(rng.integers(0, i)) for i in range(1, n)])
    return out


def make(seed, nodes, vocab, dtype, kind, drawn, noise=0.7, spread=2.0, scales=True):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    parents, n = trees(rng, nodes, kind), sum(nodes)
    x = torch.randn(n, vocab, generator=gen, device="cuda") * spread
    if vocab > 8:
        likely = torch.randint(0, vocab, (n, 6), generator=gen, device="cuda")
        x.scatter_add_(1, likely, 12 * torch.rand(n, 6, generator=gen, device="cuda"))
    d = (x + noise * torch.randn(n, vocab, generator=gen, device="cuda")).to(dtype)
    x = x.to(dtype)
    tokens, at = torch.zeros(n, dtype=torch.int32, device="cuda"), 0
    for t in parents:
        for i, p in enumerate(t):
            if p >= 0:
                row = d[at + p].float()
                tokens[at + i] = int(torch.multinomial(torch.softmax(row, 0), 1, generator=gen)) if drawn else int(torch.topk(row, min(vocab, i + 1)).indices[-1])
        at += len(t)
    flat = torch.tensor([p for t in parents for p in t], dtype=torch.int32, device="cuda")
    u = torch.rand(n, generator=gen, device="cuda")
    v = torch.rand(len(nodes), generator=gen, device="cuda")
    s = (0.7 + 0.6 * torch.rand(n, generator=gen, device="cuda")) if scales else None
    return dict(logits=x, tokens=tokens, parents=flat, n_nodes=list(nodes), u_accept=u, u_sample=v, draft=d if drawn else None, scale=s,
                draft_scale=s.flip(0).contiguous() if scales and drawn else None)


def check(a, got=None, least=1e-11):
    """Tokens, counts and paths are the walk's wherever no comparison is nearer to its border than `least` (sums of up to 2e5 terms in 64 bits differ by less,
    2e5 * 2^-53 = 2e-11 at most, in practice a thousandth). Log probabilities: fp32 sums of V terms of one sign are off by 2^-23 of themselves and the
    exponentials by 2^-22, their logarithm by 1e-6; the product of a logit and its scale by 2^-24 of it, of up to 60."""
    got = verify_tokens(**a) if got is None else got
    emitted, count, path, lp = (t.cpu().numpy() for t in got)
    host = {k: v.double().cpu().numpy() if torch.is_tensor(v) else v for k, v in a.items()}
    one = np.ones(len(host["tokens"]))
    scale, dscale = host["scale"] if a["scale"] is not None else one, host["draft_scale"] if a["draft_scale"] is not None else one
    at, accepted = 0, 0
    for r, n in enumerate(a["n_nodes"]):
        rows = slice(at, at + n)
        want, nodes, wlp, near = walk(host["logits"][rows], None if a["draft"] is None else host["draft"][rows], host["tokens"][rows].astype(int),
                                      host["parents"][rows].astype(int), host["u_accept"][rows], host["u_sample"][r], scale[rows], dscale[rows])
        if near > least:
            c = int(count[r])
            assert c == len(want) and emitted[rows][:c].tolist() == want, (r, near, emitted[rows].tolist(), want)
            assert path[rows][:c].tolist() == [at + i for i in nodes]
            assert (emitted[rows][c:] == -1).all() and (path[rows][c:] == -1).all() and (lp[rows][c:] == 0).all()
            np.testing.assert_allclose(lp[rows][:c], wlp, rtol=3e-7, atol=1.2e-5)
            accepted += c - 1
        at += n
    return accepted


@pytest.mark.parametrize("drawn", [False, True], ids=["given", "drawn"])
@pytest.mark.parametrize("kind", ["chain", "star", "tree"])
@pytest.mark.parametrize("vocab,dtype,nodes", [
    (1, torch.float32, [1, 3]), (2, torch.bfloat16, [5] * 40), (7, torch.float32, [9] * 30), (255, torch.bfloat16, [1, 2, 64, 17]), (1000, torch.float32, [6] * 50),
    (32000, torch.bfloat16, [8]), (32001, torch.bfloat16, [5, 1, 7]), (50257, torch.float32, [12, 3, 30]), (131072, torch.bfloat16, [4] * 40)])
def test_tokens_are_those_of_the_walk(vocab, dtype, nodes, kind, drawn):
    check(make(vocab + len(nodes), nodes, vocab, dtype, kind, drawn))


@pytest.mark.parametrize("drawn", [False, True], ids=["given", "drawn"])
def test_flat_distributions_of_many_tokens(drawn):
    """Every border of the cumulative sum is 5e-6 from the next: a sum off by 1e-7 would draw a neighbour now and then."""
    for seed in range(3):
        check(make(seed, [3] * 60, 200003, torch.float32, "star", drawn, spread=0.3, noise=0.02))


def test_a_draft_like_the_model_is_accepted():
    a = make(1, [10] * 8, 4000, torch.float32, "chain", True, scales=False)
    a["draft"] = a["logits"].clone()
    got = verify_tokens(**a)
    assert (got.count == 10).all()
    for noise in (1e-3, 1e-6):                           # what is left of nearly equal distributions is small differences
        check(make(2, [6] * 40, 4000, torch.float32, "star", True, noise=noise))


def test_what_is_emitted_is_distributed_as_the_model(trials=40000):
    """The first emitted token over many requests of one distribution, drafts from another: counts within 6 standard deviations."""
    gen = torch.Generator(device="cuda").manual_seed(11)
    vocab, nodes = 12, 3
    row, drow = torch.randn(vocab, generator=gen, device="cuda") * 1.5, torch.randn(vocab, generator=gen, device="cuda") * 1.5
    n = trials * nodes
    q = torch.softmax(drow.double(), 0)
    tokens = torch.multinomial(q, n, replacement=True, generator=gen).int()
    for draft in (drow.expand(n, vocab).contiguous(), None):
        got = verify_tokens(row.expand(n, vocab).contiguous(), tokens, torch.tensor([-1, 0, 0], dtype=torch.int32, device="cuda").repeat(trials), [nodes] * trials,
                            torch.rand(n, generator=gen, device="cuda"), torch.rand(trials, generator=gen, device="cuda"), draft=draft)
        seen = torch.bincount(got.emitted[::nodes].long(), minlength=vocab).double()
        p = torch.softmax(row.double(), 0)
        assert float(((seen - trials * p).abs() / (trials * p * (1 - p)).sqrt()).max()) < 6


def test_masked_tokens_and_rows_that_are_no_distribution():
    inf, nan = math.inf, math.nan
    a = make(3, [4] * 12, 500, torch.float32, "chain", True, scales=False)
    x, d = a["logits"], a["draft"]
    x[0:4, 100:] = -inf                                  # the draft allows what the model does not
    d[4:8, 250:] = -inf                                  # and the other way round
    x[8:12] = -inf
    x[8:12, 77] = -3e38                                  # one token left, of the type's lowest values
    x[12, 5] = nan
    x[16, 5] = inf
    x[20] = -inf
    d[24, 9] = nan
    d[31] = nan                                          # of a node without children: not read
    x[32:36] = 3e38                                      # one size: flat
    x[36:40] *= 1e4                                      # one token has it all
    d[40] = -inf
    d[44:48] = 1e30
    check(a)
    got = verify_tokens(**a)
    e, lp = got.emitted.view(12, 4), got.logprob.view(12, 4)
    for r in (3, 4, 5, 6, 10):
        assert e[r, 0] == -1 and torch.isnan(lp[r, 0]) and got.count[r] == 1
    assert (e[2, :1] == 77).all()
    for dtype in (torch.bfloat16,):
        b = {k: (v.to(dtype) if k in ("logits", "draft") else v) for k, v in a.items()}
        check(b)


def test_borders_of_the_random_numbers():
    a = make(4, [3] * 6, 300, torch.float32, "star", False, scales=False)
    a["logits"][:, :10] = -math.inf
    a["logits"][:, 290:] = -math.inf
    a["tokens"][:] = 0                                   # impossible: never accepted
    a["u_accept"].zero_()
    a["u_sample"].copy_(torch.tensor([0.0, 1.0, 2.0, math.nan, 1 - 2.0 ** -24, 0.5]))
    got = verify_tokens(**a)
    first = got.emitted.view(6, 3)[:, 0].tolist()
    assert first[0] == 10 and first[1] == first[2] == first[3] == 289 and first[4] <= 289 and (got.count == 1).all()
    a["tokens"][:] = torch.tensor([0, -1, 300], dtype=torch.int32, device="cuda").repeat(6)      # no such tokens
    a["parents"][:] = torch.tensor([-1, 0, 5], dtype=torch.int32, device="cuda").repeat(6)
    assert torch.equal(verify_tokens(**a).emitted.view(6, 3)[:, 0], got.emitted.view(6, 3)[:, 0])
    b = make(5, [4], 300, torch.float32, "star", False, scales=False)
    b["tokens"][:] = 7                                   # one token given three times
    b["u_accept"].fill_(1.0)
    check(b)
    assert int(verify_tokens(**b).emitted[0]) != 7


def test_strided_and_unaligned_rows():
    a = make(6, [5, 1, 9], 1001, torch.bfloat16, "tree", True)
    want = verify_tokens(**a)
    for pad, off in ((0, 1), (7, 0), (23, 3)):
        b = dict(a)
        for name, extra in (("logits", 0), ("draft", 1)):
            n, v = a[name].shape
            store = torch.full((n * (v + pad) + off + extra + pad,), math.nan, dtype=torch.bfloat16, device="cuda")
            view = store[off + extra:off + extra + n * (v + pad)].view(n, v + pad)[:, :v]
            view.copy_(a[name])
            b[name] = view
        got = verify_tokens(**b)
        check(b, got)                                    # (sums are cut at 16-byte boundaries: log probabilities may differ in their last bits)
        assert all(torch.equal(x, y) for x, y in zip(got[:3], want[:3]))


def test_many_requests_streams_and_a_captured_call():
    a = make(7, [1 + r % 4 for r in range(1700)], 600, torch.float32, "chain", True)
    want = verify_tokens(**a)
    check(a, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = verify_tokens(**a)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(other, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        inside = verify_tokens(**a)
    a["u_sample"].copy_(a["u_sample"].flip(0))
    graph.replay()
    torch.cuda.synchronize()
    check(a, inside)


def test_refusals():
    a = make(8, [3, 2], 100, torch.float32, "chain", True)
    for change in (dict(n_nodes=[3, 3]), dict(n_nodes=[5]), dict(tokens=a["tokens"].long()), dict(draft=a["draft"].to(torch.bfloat16)),
                   dict(u_sample=a["u_accept"]), dict(scale=a["scale"].double()), dict(logits=a["logits"].half()), dict(logits=a["logits"].t()),
                   dict(parents=a["parents"].cpu())):
        with pytest.raises(ValueError):
            verify_tokens(**{**a, **change})
    big = make(9, [33, 32], 10, torch.float32, "chain", False)
    for nodes in ([65], [0, 65], [66, -1]):
        with pytest.raises(RuntimeError):
            verify_tokens(**{**big, "n_nodes": nodes, "u_sample": big["u_sample"][:len(nodes)].contiguous()})
    args = B.ts_verify(0, 1, 0, B.TS_F32)
    assert B.ts_verify_tokens(args, 0) == B.TS_ERR_INVALID
    empty = verify_tokens(a["logits"][:0], a["tokens"][:0], a["parents"][:0], [], a["u_accept"][:0], a["u_sample"][:0])
    assert all(t.numel() == 0 for t in empty)
