"""Tests of drafts near their border where a thread sums a long part of a row: as many requests as leave each one thread block, rows of up to 2^20
logits whose weights are of one size, so that roundings of a sum do not cancel."""
import pytest
import torch

from paper_2512_03416_b200.verify import verify_tokens

pytestmark = pytest.mark.gpu

REQUESTS = 300                               # more than an SM's blocks of 128 threads can be doubled for: one block a request


def rows(kind, vocab, dtype, r, gen):
    """The model's and the draft's row of request r, the drafted token is 5."""
    at = torch.arange(vocab, device="cuda", dtype=torch.float32)
    if kind == "flat":                       # weights 2^-0.3 to 2^-4 of the token's own
        x, d = torch.full_like(at, -0.2 - 0.01 * r), torch.full_like(at, -25.0)
        x[5] = d[5] = 0.0
    elif kind == "unlikely":                 # the drafted token is the reference and e^60 below the rest: references move
        x, d = torch.full_like(at, 0.01 * r), torch.full_like(at, 0.005 * r)
        x[5], d[5] = -60.0, -59.0 - 0.005 * r
    else:                                    # rising, by less than a rounding of a factor from tile to tile
        x = at * ((69.0 + 0.01 * r) / vocab)
        d = x.clone()
        d[5] += 0.5
    return x.to(dtype), d.to(dtype)


@pytest.mark.parametrize("kind,vocab,dtype", [("flat", 262144, torch.bfloat16), ("flat", 1 << 20, torch.bfloat16), ("flat", 300007, torch.float32),
                                              ("unlikely", 1 << 19, torch.bfloat16), ("rising", 400001, torch.float32)])
def test_drafts_near_their_border_over_long_rows(kind, vocab, dtype):
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    n = 2 * REQUESTS
    x, d = (torch.zeros(n, vocab, dtype=dtype, device="cuda") for _ in range(2))
    lp, lq = (torch.empty(REQUESTS, dtype=torch.float64, device="cuda") for _ in range(2))
    for r in range(REQUESTS):
        x[2 * r], d[2 * r] = rows(kind, vocab, dtype, r, gen)
        for row, out in ((x[2 * r].double(), lp), (d[2 * r].double(), lq)):
            out[r] = row[5] - torch.logsumexp(row, 0)
    # random numbers from 1e-6 to 1e-4 of the border, on either side; in fp32 they are 6e-8 from where they were put
    off = 10.0 ** (-6 + 2 * torch.rand(REQUESTS, generator=gen, device="cuda", dtype=torch.float64))
    off[1::2] *= -1
    u = torch.rand(n, generator=gen, device="cuda")
    u[1::2] = (torch.exp(lp - lq) * (1 + off)).float()
    assert float(u.max()) < 1
    want = torch.log(u[1::2].double()) + lq < lp         # in 64 bits: logarithms of up to 100, off by 1e-14
    assert torch.equal(want, off < 0)
    tokens = torch.full((n,), 5, dtype=torch.int32, device="cuda")
    parents = torch.tensor([-1, 0], dtype=torch.int32, device="cuda").repeat(REQUESTS)
    got = verify_tokens(x, tokens, parents, [2] * REQUESTS, u, torch.rand(REQUESTS, generator=gen, device="cuda"), draft=d)
    assert torch.equal(got.count == 2, want), off[(got.count == 2) != want].abs().max()
    # A sum of weights is off by 8.6e-6 of itself at most, 2.7e-5 where references move (chains of 64 terms, lanes, warps, exponents' roundings); the
    # exponent of the token, up to 104, by two roundings of 2^-18 times ln 2, there also by 2^-23 of itself; the result by 2^-24.
    slack = 8.6e-6 + 5.3e-6 if kind == "flat" else 2.7e-5 + 1.3e-5
    emitted, logprob = got.emitted.view(-1, 2)[:, 0], got.logprob.view(-1, 2)[:, 0].double()
    exact = torch.stack([x[2 * r, int(t)].double() for r, t in enumerate(emitted.tolist())]) - x[::2, 5].double() + lp
    assert bool(((logprob - exact).abs() <= slack + 2.0 ** -24 * exact.abs()).all()), (logprob - exact).abs().max()
