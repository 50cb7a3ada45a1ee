"""ts_token_logprobs against its definition in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2512_03416_b200.logprobs import token_logprobs
from tests import tree_oracle as O

pytestmark = pytest.mark.gpu


def _check(logits, tokens=None, n_top=0, scale=None):
    """Whole numbers must be equal. In fp32 y log2(e) carries 2^-23 of its size, the sums of up to 2^17 terms less than
    2^-20 of theirs, of which the logarithm makes an absolute error; the entropy's terms are as large as the spread of y."""
    r = token_logprobs(logits, tokens, n_top, scale)
    torch.cuda.synchronize()
    x = logits.double().cpu().numpy()
    given = np.zeros((len(x), 0), int) if tokens is None else tokens.view(len(x), -1).cpu().numpy()
    for i in range(len(x)):
        s = 1.0 if scale is None else float(scale[i])
        lp, rank, ent, top_lp, top = O.token_logprobs(x[i], s, given[i], n_top)
        fin = np.abs(x[i][np.isfinite(x[i])]) * s
        tol = 2.0 ** -19 * (1 + (fin.max() if len(fin) else 0))
        assert np.array_equal(r.rank[i].cpu().numpy(), rank), (i, given[i])
        assert np.array_equal(r.top_token[i].cpu().numpy(), top), i
        for got, want, what in ((r.logprob[i], lp, "logprob"), (r.top_logprob[i], top_lp, "top"), (r.entropy[i:i + 1], np.array([ent]), "entropy")):
            got = got.cpu().numpy().astype(np.float64)
            same = (got == want) | (np.isnan(got) & np.isnan(want))
            with np.errstate(invalid="ignore"):
                assert (same | (np.abs(got - want) <= tol)).all(), (what, i, got, want)
    return r


def _logits(rows, vocab, dtype, seed=0, size=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(rows, vocab, generator=g, device="cuda") * size).to(dtype)


def _tokens(rows, given, vocab, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + 100)
    return torch.randint(0, vocab, (rows, given), generator=g, device="cuda", dtype=torch.int32)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 31, 33, 1000, 4095, 4096, 4097, 8193, 32000, 50001, 131072, 200003])
@pytest.mark.parametrize("rows,given,n_top", [(1, 1, 20), (3, 8, 32), (40, 2, 1), (2, 0, 5), (5, 3, 0)])
def test_sizes(rows, vocab, dtype, given, n_top):
    _check(_logits(rows, vocab, dtype, vocab), _tokens(rows, given, vocab) if given else None, n_top)


@pytest.mark.parametrize("rows", [150, 600])
def test_many_rows(rows):
    _check(_logits(rows, 3001, torch.bfloat16), _tokens(rows, 1, 3001), 4)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [65, 5000, 40000])
def test_strides_and_alignment(vocab, dtype):
    """Rows that start anywhere in a 16-byte block, with neighbours that must not be looked at."""
    wide = torch.full((6, vocab + 37), 1e4, dtype=dtype, device="cuda")
    for start in (0, 1, 3, 8, 13):
        wide.fill_(float("nan"))
        view = wide[:, start:start + vocab]
        view.copy_(_logits(6, vocab, dtype, start))
        _check(view, _tokens(6, 2, vocab), 7)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [40, 5000, 70001])
def test_masked_and_odd_logits(vocab, dtype):
    inf = float("inf")
    x = _logits(12, vocab, dtype, 5)
    x[0] = -inf                                                    # nothing is left
    x[1, 3:] = -inf                                                # three tokens are left: the next ones go by index
    x[2] = 1.5                                                     # all alike
    x[3, vocab // 2] = float("nan")
    x[4, 7] = inf
    x[5, ::2] = torch.finfo(dtype).min                             # masked by the type's lowest value
    x[6] = torch.arange(vocab, device="cuda") * (60.0 / vocab)     # ascending
    x[7] = -torch.arange(vocab, device="cuda") * (60.0 / vocab)
    x[8] = float("nan")
    x[9, 5:] = float("nan")                                        # fewer numbers than alternatives
    x[10] = torch.where(torch.arange(vocab, device="cuda") % 2 == 0, 0.0, -0.0)
    x[11] = -inf
    x[11, vocab - 1] = -3.0
    tokens = _tokens(12, 5, vocab)
    tokens[:, 1] = vocab - 1
    tokens[:, 2] = 0
    tokens[:, 3] = torch.tensor([vocab, -1, 1 << 30, -(1 << 31)] * 3, dtype=torch.int32, device="cuda")
    for n_top in (1, 6, 32):
        _check(x, tokens, n_top)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [1, 400])
def test_best_tokens_in_one_place(dtype, rows):
    """The best tokens all in the blocks that one or few threads read, in ascending order: more candidates than the list holds."""
    n = 8 if dtype == torch.bfloat16 else 4
    x = _logits(rows, 300000, dtype, 6, 0.5)
    block = torch.arange(300000, device="cuda") // n
    for r in range(0, rows, 50):
        part = block % 512 < 1 + r // 50
        x[r, part] = (10 + torch.arange(300000, device="cuda")[part] * 1e-4).to(dtype)
    _check(x[::50].contiguous() if rows > 1 else x, None, 32)
    if rows > 1:
        r = token_logprobs(x, None, 32)
        one = token_logprobs(x[:1], None, 32)
        assert torch.equal(r.top_token[0], one.top_token[0])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_scales_and_sizes(dtype):
    x = _logits(8, 9000, dtype, 7)
    x[4:] *= 300                                                    # hundreds of nats apart, positive and negative
    x[6] += 2000
    x[7] -= 2000
    _check(x, _tokens(8, 4, 9000), 10, torch.tensor([0.25, 1, 2, 10, 0.01, 1, 1, 1], device="cuda"))


def test_single_values_rise():
    """A reference that has to move again and again: every block's values exceed all earlier ones by more than 2^64."""
    x = (torch.arange(200000, device="cuda") // 4096 * 70.0)[None].contiguous()
    _check(x, _tokens(1, 3, 200000), 5)


def test_same_bits_again_and_on_another_stream():
    x, t = _logits(30, 60001, torch.bfloat16, 8), _tokens(30, 3, 60001)
    a = token_logprobs(x, t, 9)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        b = token_logprobs(x, t, 9)
    st.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_refusals():
    x = _logits(2, 100, torch.float32)
    t = _tokens(2, 1, 100)
    for f in (lambda: token_logprobs(x.half()), lambda: token_logprobs(x.cpu()), lambda: token_logprobs(x.t()), lambda: token_logprobs(x[0]),
              lambda: token_logprobs(x, t.long()), lambda: token_logprobs(x, t[:1]), lambda: token_logprobs(x, _tokens(2, 9, 100)),
              lambda: token_logprobs(x, n_top=33), lambda: token_logprobs(x, n_top=-1), lambda: token_logprobs(x, scale=torch.ones(3, device="cuda")),
              lambda: token_logprobs(x[:, :0]), lambda: token_logprobs(x[:1].expand(2, 100))):
        with pytest.raises(ValueError):
            f()
    r = token_logprobs(x[:0], t[:0], 3)
    assert r.logprob.shape == (0, 1) and r.top_token.shape == (0, 3)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,vocab,n_top", [(200, 40000, 3), (200, 40000, 12), (40, 131072, 5), (160, 131072, 20), (3, 50001, 9)])
def test_alternatives_with_equal_logits(rows, vocab, n_top, dtype):
    """A few dozen logits of few sizes in front of all others, anywhere in the row: the lower index of equal ones comes first."""
    g = torch.Generator(device="cuda").manual_seed(rows + vocab + n_top)
    x = torch.randn(rows, vocab, generator=g, device="cuda").clamp(max=2.0)
    at = torch.randint(0, vocab, (rows, 40), generator=g, device="cuda")
    x.scatter_(1, at, 4.0 + torch.randint(0, 4, (rows, 40), generator=g, device="cuda").float() * 0.5)
    _check(x.to(dtype), None, n_top)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("above", [12.0, 16.0, 20.0])
def test_likely_tokens(above, dtype):
    """One logit far above the others: its log probability is near 0, and the reference of the sums, a logit from the row's beginning,
    far from it. The weight's exponent is rounded once, and the same in the sum; the weight itself carries 2^-22, the sum of up to
    2^15 smaller ones (which are less than an e-th) 2^-23, the logarithm's part and the last products 2^-23: 2^-20 in all."""
    x = _logits(20, 32000, torch.float32, seed=int(above), size=0.5)
    at = _tokens(20, 1, 32000)
    x.scatter_(1, at.long(), above + torch.arange(20, device="cuda").view(20, 1) * 0.0625)
    x = x.to(dtype)
    r = token_logprobs(x, at, 1)
    want = torch.log_softmax(x.double(), -1).gather(1, at.long())
    assert (r.top_token == at).all()
    assert ((r.logprob.double() - want).abs() <= 2.0 ** -20).all()
    assert ((r.top_logprob.double() - want).abs() <= 2.0 ** -20).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,vocab", [(1, 4096), (1, 8192), (1, 16384), (1, 16391), (37, 4100), (18, 17000)])
def test_short_shares_of_a_cluster(rows, vocab, dtype):
    """Rows shared by clusters whose blocks have one or two 16-byte blocks per thread: the pass is as short as it gets. Many such calls in a
    row, behind each other's ends, give the same bits."""
    x, t = _logits(rows, vocab, dtype, vocab + rows), _tokens(rows, 3, vocab)
    want = _check(x, t, 32)
    many = [token_logprobs(x, t, 32) for _ in range(300)]
    torch.cuda.synchronize()
    for r in many:
        assert all(torch.equal(p, q) for p, q in zip(want, r))


def _entropy_bound(y):
    """For y = scale x of a row, in nats. H = ln S - sum e u / S with u = log e. The sums' reference r is a logit no more than 2.8 (4 log2) below
    the largest one: the largest itself where the second is further behind. With A = E|y - r|, Q = E(y - r)^2: the exponents' factor and
    roundings (2^-23 of them) move the entropy by less than 2^-22 Q, the exponentials (2^-22) and the sums (2^-21) by less than 2^-20 (1 + A)."""
    y = np.sort(y[np.isfinite(y)])[::-1]
    d = y[0] - y
    p = np.exp(-d) / np.exp(-d).sum()
    near = 2.8 if len(y) > 1 and d[1] < 2.8 else 0.0
    return 2.0 ** -20 * (1 + (p * d).sum() + near) + 2.0 ** -22 * ((p * d * d).sum() + near * near)


def _check_entropy(x, scale=None):
    r = token_logprobs(x, None, 0, scale)
    for i, (row, got) in enumerate(zip(x.double().cpu().numpy(), r.entropy.cpu().numpy().astype(np.float64))):
        s = 1.0 if scale is None else float(scale[i])
        want = O.token_logprobs(row, s, [], 0)[2]
        assert got >= 0 and abs(got - want) <= _entropy_bound(row * s), (i, got, want, _entropy_bound(row * s))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [1, 300, 32000, 131072])
@pytest.mark.parametrize("offset", [0.0, 100.0, -100.0, 2000.0, -1e5])
def test_entropy_of_rows_far_from_zero(offset, vocab, dtype):
    """What is added to all logits is no part of the entropy."""
    for size in (0.3, 2.5, 40.0):
        _check_entropy((_logits(6, vocab, torch.float32, vocab, size) + offset).to(dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [3, 200])
def test_entropy_of_likely_tokens(rows, dtype):
    """One logit 8 to 40 nats above the others, rows far from zero among them: entropies down to nothing."""
    x = _logits(rows, 32000, torch.float32, 17, 0.5)
    at = _tokens(rows, 1, 32000, 3).long()
    x.scatter_(1, at, 8.0 + torch.arange(rows, device="cuda").view(rows, 1) * (32.0 / rows))
    _check_entropy(x.to(dtype))
    _check_entropy((x + 1000).to(dtype))
    _check_entropy(x.to(dtype), torch.linspace(0.5, 3.0, rows, device="cuda"))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [50, 40000])
def test_logits_of_the_largest_sizes(vocab, dtype):
    """One number of any size among logits of -inf has all the probability; and numbers whose product with the scale is beyond fp32."""
    sizes = [-(2.0 ** 127), -(2.0 ** 126), -(2.0 ** 125), -(2.0 ** 124), -1e30, 0.0, 2.0 ** 100, 2.0 ** 125, 2.0 ** 126, 2.0 ** 127]
    for scale in (0.25, 1.0, 1000.0):
        x = torch.full((len(sizes), vocab), -float("inf"), device="cuda")
        at = _tokens(len(sizes), 1, vocab, 9)
        x.scatter_(1, at.long(), torch.tensor(sizes, device="cuda").view(-1, 1))
        r = token_logprobs(x.to(dtype), at, 1, torch.full((len(sizes),), scale, device="cuda"))
        assert (r.logprob == 0).all() and (r.top_logprob == 0).all() and (r.entropy == 0).all() and (r.top_token == at).all()
    x = (-torch.arange(vocab, device="cuda", dtype=torch.float64) * 2.0 ** 100 + 2.0 ** 121)[None].to(dtype)      # y to 2^130, 2^109 apart and more
    t = torch.tensor([[0, vocab - 1]], dtype=torch.int32, device="cuda")
    for row in (x, -x):
        r = token_logprobs(row, t, 1, torch.full((1,), 512.0, device="cuda"))
        lp = O.token_logprobs(row[0].double().cpu().numpy(), 512.0, t[0].cpu().numpy(), 1)
        assert np.allclose(r.logprob[0].cpu().numpy(), lp[0], rtol=2.0 ** -20, atol=2.0 ** -20)
        assert np.array_equal(r.top_token[0].cpu().numpy(), lp[4]) and abs(float(r.entropy[0]) - lp[2]) <= 2.0 ** -18


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("offset", [-1e9, -1e10, -3e30, 1e7])
def test_rows_masked_throughout(offset, dtype):
    """Every token at the same number of any size, some tokens 2^-7 of it above or below: what is left is a distribution like any other."""
    x = torch.full((3, 20001), offset, device="cuda", dtype=torch.float64)
    x[1, ::3] *= 1 + 2.0 ** -7
    x[2, 5:9] *= 1 - 2.0 ** -7
    x, t = x.to(dtype), _tokens(3, 2, 20001)
    _check(x, t, 4)
    _check_entropy(x)


def test_references_on_both_sides_of_where_they_count_as_huge():
    """Logits times log2(e) around 2^20, a few nats apart: parts of a row refer to logits on either side."""
    base = 2.0 ** 20 / 1.4426950408889634
    x = (base + _logits(4, 60000, torch.float32, 23, 3.0)).contiguous()
    x[1] = -x[1]
    x[2] *= 1024.0
    x[3] = torch.cat([torch.linspace(base - 12, base + 6, 59999, device="cuda"), torch.tensor([base - 30.0], device="cuda")])
    scale = torch.tensor([1.0, 1.0, 1.0 / 1024, 1.0], device="cuda")
    r = token_logprobs(x, None, 3, scale)
    for i in range(4):
        _, _, ent, top_lp, top = O.token_logprobs(x[i].double().cpu().numpy(), float(scale[i]), [], 3)
        assert np.array_equal(r.top_token[i].cpu().numpy(), top)
        assert np.abs(r.top_logprob[i].cpu().numpy() - top_lp).max() <= 2.0 ** -18 and abs(float(r.entropy[i]) - ent) <= 2.0 ** -16, i
