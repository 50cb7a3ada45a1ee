"""The loop fork -> projections with adapters -> tree attention -> verification by sampling -> accepted path into the cache."""
import json
import math

import numpy as np
import pytest
import torch

from paper_2512_03416_b200 import speculative
from paper_2512_03416_b200.adapters import Adapters
from paper_2512_03416_b200.speculative import SpeculativeDecoder, main, random_adapters, random_weights

pytestmark = pytest.mark.gpu
HQ, HKV, D, HIDDEN, VOCAB = 8, 2, 128, 256, 512
PROMPTS, WHICH = ([3], [5, 6, 7, 8, 9], list(range(100, 141))), (1, -1, 0)


class Kept(Adapters):
    def __init__(self, a, b):
        super().__init__(a, b)
        self.given = a, b


def made(cache, depth, width, temperature, seed=3, attention=0.5, forks=2):
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required")
    w = random_weights(VOCAB, HIDDEN, HQ, HKV, D, seed=7, attention=attention)
    speculative.Adapters = Kept
    try:
        ads = random_adapters(w, 2, 16, seed=8)
    finally:
        speculative.Adapters = Adapters
    sd = SpeculativeDecoder(w, HQ, HKV, D, max_requests=3 * (1 + forks), max_tokens=160, depth=depth, width=width, cache=cache, temperature=temperature,
                            seed=seed, adapters=ads)
    for p, a in zip(PROMPTS, WHICH):
        sd.add(p, a)
    of = list(range(3))
    for i in range(3):
        of += [i] * len(sd.fork(i, forks)) if forks else []
    return w, ads, sd, of


def logits64(w, ads, which, tokens, first):
    """float64 logits after tokens[: first + 1], ... with the request's adapters merged into the weights."""
    m = [t.double().cpu().numpy() for t in w]
    if which >= 0:
        for i, name in ((1, "q"), (2, "k"), (3, "v"), (4, "o")):
            a, b = ads[name].given
            m[i] = m[i] + (b[which].double() @ a[which].double()).cpu().numpy()
    x = m[0][tokens]
    q, k, v = ((x @ a.T).reshape(len(tokens), -1, D) for a in m[1:4])
    out = np.zeros((len(tokens) - first, HQ, D))
    for i in range(first, len(tokens)):
        for h in range(HQ):
            s = k[:i + 1, h * HKV // HQ] @ q[i, h] / math.sqrt(D)
            p = np.exp(s - s.max())
            out[i - first, h] = (p / p.sum()) @ v[:i + 1, h * HKV // HQ]
    return (x[first:] + out.reshape(len(out), -1) @ m[4].T) @ m[5].T


@pytest.mark.parametrize("cache,tol", [("bf16", 0.15), ("e4m3", 0.7)])
@pytest.mark.parametrize("depth,width", [(3, 2), (4, 1), (1, 8)])
def test_log_probabilities_are_those_of_each_requests_own_model(cache, tol, depth, width):
    """What a fork with an adapter emits has the log probability that its own weights give it after its own tokens. tol: of one logit, as derived for the greedy
    loop; an adapter adds a twentieth to a projection's variance and the rounding of u, 2^-8 of that part. Temperature 0.7 divides all."""
    w, ads, sd, of = made(cache, depth, width, 0.7)
    done = sd.generate(16)
    assert len(done) == 9 and int(sd.gemm_status.item()) == 0 and all(int(a.status.item()) == 0 for a in ads.values())
    for r, i in enumerate(of):
        tokens = list(PROMPTS[i]) + [t for t, _ in done[r]]
        assert len(done[r]) >= 16 and sd.cached[r] == len(tokens) - 1 and sd.last[r] == tokens[-1]
        ref = logits64(w, ads, WHICH[i], tokens[:-1], len(PROMPTS[i]) - 1) / 0.7
        for row, (token, lp) in zip(ref, done[r]):
            true = row[token] - row.max() - math.log(np.exp(row - row.max()).sum())
            assert abs(lp - true) <= 2 * tol / 0.7
    assert len({tuple(t for t, _ in d) for d in done}) > 6      # samples of one prompt part ways
    sd.close()


def test_runs_are_repeatable_and_forks_leave_their_parent_alone():
    runs = []
    for forks in (0, 2):
        _, _, sd, _ = made("bf16", 3, 2, 0.0, forks=forks)      # greedy: every fork emits what its parent does
        runs.append(sd.generate(12))
        sd.close()
    for r in range(3):
        n = min(len(runs[0][r]), len(runs[1][r]))
        assert [t for t, _ in runs[0][r]][:n] == [t for t, _ in runs[1][r]][:n]
        for f in (3 + 2 * r, 4 + 2 * r):
            assert [t for t, _ in runs[1][f]][:n] == [t for t, _ in runs[1][r]][:n]
    again = []
    for seed in (3, 3, 4):
        _, _, sd, _ = made("bf16", 3, 2, 1.0, seed=seed)
        again.append(sd.generate(12))
        sd.close()
    assert again[0] == again[1] != again[2]


def test_refusals():
    w, ads, sd, _ = made("bf16", 2, 2, 0.5)
    with pytest.raises(ValueError):
        sd.add([1], 2)
    with pytest.raises(RuntimeError):
        sd.fork(0, 1)                                           # no slot left
    sd.close()
    with pytest.raises(ValueError):
        SpeculativeDecoder(w, HQ, HKV, D, 1, 64, temperature=-1.0)
    plain = SpeculativeDecoder(w, HQ, HKV, D, 1, 64)
    with pytest.raises(ValueError):
        plain.add([1], 0)
    plain.close()


def test_logits_that_are_no_distribution_end_the_loop_with_an_error():
    w, _, sd, _ = made("bf16", 2, 2, 0.5)
    sd.step()
    cached = list(sd.cached)
    w.w_head[7].fill_(math.nan)
    with pytest.raises(FloatingPointError):
        sd.step()
    assert sd.cached == cached
    sd.close()


def test_command(capsys):
    assert main(["--requests", "2", "--samples", "2", "--prompt", "20", "--tokens", "4", "--temperature", "0.8", "--adapters", "2", "--rank", "8"]) == 0
    line = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    assert line["gemm_status"] == 0 and line["requests"] == 4 and line["tokens"] >= 16
