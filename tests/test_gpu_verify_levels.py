"""Verification where a request has one thread block, level after level: long chains of accepted drafts over short rows, many requests at once."""
import pytest
import torch

from paper_2512_03416_b200.verify import verify_tokens
from tests.test_gpu_verify import check

pytestmark = pytest.mark.gpu


def chains(seed, requests, nodes, vocab, dtype, drawn):
    """Chains whose drafts are likely enough that most are accepted one after the other; a token of the draft's, drawn or given, at every node."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = requests * nodes
    x = torch.randn(n, vocab, generator=gen, device="cuda")
    likely = torch.randint(0, vocab, (n, 1), generator=gen, device="cuda")
    x.scatter_(1, likely, 14.0)                          # p of some 0.99999 - vocab e^-14
    d = (x + 0.05 * torch.randn(n, vocab, generator=gen, device="cuda")).to(dtype)
    tokens = torch.zeros(requests, nodes, dtype=torch.int32, device="cuda")
    tokens[:, 1:] = likely.view(requests, nodes)[:, :-1].int()
    parents = torch.arange(-1, nodes - 1, dtype=torch.int32, device="cuda").repeat(requests)
    return dict(logits=x.to(dtype), tokens=tokens.view(-1), parents=parents, n_nodes=[nodes] * requests, u_accept=torch.rand(n, generator=gen, device="cuda"),
                u_sample=torch.rand(requests, generator=gen, device="cuda"), draft=d if drawn else None, scale=None, draft_scale=None)


@pytest.mark.parametrize("drawn", [False, True], ids=["given", "drawn"])
@pytest.mark.parametrize("vocab,dtype,requests,nodes", [(257, torch.bfloat16, 600, 64), (600, torch.float32, 340, 40), (1000, torch.bfloat16, 300, 64), (1000, torch.float32, 12, 64)])
def test_long_accepted_chains_of_requests_of_one_block(vocab, dtype, requests, nodes, drawn):
    a = chains(vocab + requests, requests, nodes, vocab, dtype, drawn)
    got = verify_tokens(**a)
    accepted = check(a, got)
    assert accepted > requests * nodes * 0.8             # the levels that this is about are walked
    for _ in range(4):                                   # sums in a fixed order: whichever warp is first
        assert all(torch.equal(x, y) or (x.isnan() == y.isnan()).all() and torch.equal(x.nan_to_num(), y.nan_to_num()) for x, y in zip(verify_tokens(**a), got))
