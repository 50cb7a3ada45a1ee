"""Drafts so unlikely that their weights are below fp32's range, next to a draft's probability of the same kind that is not: decided as in 64 bits."""
import math

import pytest
import torch

from paper_2512_03416_b200.verify import verify_tokens

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("far", [9.5, -9.5, 0.5])
@pytest.mark.parametrize("vocab,requests", [(1000, 300), (1000, 40), (50000, 4)])
def test_weights_below_the_range_of_fp32(vocab, requests, far):
    """far: logarithm of q over p of the drafted token, whose logit lies 60 to 120 below all others."""
    gen = torch.Generator(device="cuda").manual_seed(vocab + requests)
    n, t = 2 * requests, vocab - 3
    x = torch.zeros(n, vocab, device="cuda")
    d = torch.zeros(n, vocab, device="cuda")
    x[::2, t] = -60 - 60 * torch.rand(requests, generator=gen, device="cuda")
    d[::2, t] = x[::2, t] + far
    u = torch.rand(n, generator=gen, device="cuda")
    near = torch.where(torch.arange(requests, device="cuda") % 2 == 0, 0.7, 1.4)
    u[1::2] = torch.clamp(math.exp(-far) * near, max=1 - 2.0 ** -24)
    u[1::8] = 0                                          # accepted whatever q
    lp, lq = (a[::2, t].double() - torch.logsumexp(a[::2].double(), 1) for a in (x, d))
    want = torch.log(u[1::2].double()) + lq < lp         # exponents up to 170: nothing underflows in logarithms
    tokens = torch.full((n,), t, dtype=torch.int32, device="cuda")
    parents = torch.tensor([-1, 0], dtype=torch.int32, device="cuda").repeat(requests)
    got = verify_tokens(x, tokens, parents, [2] * requests, u, torch.rand(requests, generator=gen, device="cuda"), draft=d)
    assert torch.equal(got.count == 2, want), (x[::2, t][(got.count == 2) != want], want.sum())
    first, logprob = got.emitted[::2], got.logprob[::2].double()
    assert bool((first[want] == t).all()) and bool((first[~want] >= 0).all())
    # the exponent, up to 174, rounded twice to 2^-17, and short by 2^-23 of itself where references move; a sum 2.7e-5 off; the result 2^-24
    exact = x[::2].gather(1, first.long()[:, None])[:, 0].double() - torch.logsumexp(x[::2].double(), 1)
    assert bool(((logprob - exact).abs() <= 2.7e-5 + 1.5e-5 + 2.0 ** -22 * exact.abs()).all())
