"""The loop draft -> tree attention -> log probabilities -> accepted path into the cache: what it emits is the model's own
greedy choice after everything emitted before, and its cache holds the tokens that were emitted."""
import math

import numpy as np
import pytest
import torch

from paper_2512_03416_b200 import binding as B
from paper_2512_03416_b200.decoder import TsError
from paper_2512_03416_b200.speculative import SpeculativeDecoder, main, random_weights

pytestmark = pytest.mark.gpu
HQ, HKV, D, HIDDEN, VOCAB = 8, 2, 128, 256, 512
PROMPTS = ([3], [5, 6, 7, 8, 9], list(range(100, 141)))


def decode(cache, attention, depth, width, n_tokens):
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required")
    w = random_weights(VOCAB, HIDDEN, HQ, HKV, D, seed=7, attention=attention)
    sd = SpeculativeDecoder(w, HQ, HKV, D, max_requests=3, max_tokens=160, depth=depth, width=width, cache=cache)
    for p in PROMPTS:
        sd.add(p)
    return w, sd, sd.generate(n_tokens)


def logits64(w, tokens, first):
    """float64 logits after tokens[: first + 1], [: first + 2], ...: every token attends to itself and those before."""
    m = [t.double().cpu().numpy() for t in w]
    x = m[0][tokens]
    q, k, v = ((x @ a.T).reshape(len(tokens), -1, D) for a in m[1:4])
    out = np.zeros((len(tokens) - first, HQ, D))
    for i in range(first, len(tokens)):
        for h in range(HQ):
            s = k[:i + 1, h * HKV // HQ] @ q[i, h] / math.sqrt(D)
            p = np.exp(s - s.max())
            out[i - first, h] = (p / p.sum()) @ v[:i + 1, h * HKV // HQ]
    return (x[first:] + out.reshape(len(out), -1) @ m[4].T) @ m[5].T


# Tolerance of one logit (rms 4.1, the largest of 512 about 14). Its own rounding to bf16: half a step, 2^-5 below 16 and 2^-4
# below 32. y = x + attention has rms 1.1 and carries roundings of x W_o^T + x (2^-9 relative) and, at a tenth of that, those of
# the attention's inputs and output: 0.002 rms at most 0.004 with all of them, times 4 for the head, times 5 standard deviations:
# 0.08. Together 0.15. Eight-bit keys and values differ by 2^-5 of their size on average: 3 % of an attention output of 0.5 * 0.3
# (weights over several tokens), from the values and once more from the weights, makes 0.007, times 4 times 5 = 0.14 more; a short
# context (one to three tokens: the request of one token) does not average, attention 0.5, 0.02: 0.4 more.
TOL = {"bf16": 0.15, "e4m3": 0.7}


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("attention,depth,width", [(0.5, 3, 2), (0.1, 4, 1), (0.5, 1, 8), (0.5, 9, 7)])
def test_emits_the_greedy_choice(cache, attention, depth, width):
    w, sd, done = decode(cache, attention, depth, width, 24)
    assert int(sd.gemm_status.item()) == 0
    for r, p in enumerate(PROMPTS):
        tokens = p + [t for t, _ in done[r]]
        assert len(done[r]) >= 24 and sd.cached[r] == len(tokens) - 1 and sd.last[r] == tokens[-1]
        ref = logits64(w, tokens[:-1], len(p) - 1)
        assert len(ref) == len(done[r])
        for row, (token, lp) in zip(ref, done[r]):
            assert row[token] >= row.max() - 2 * TOL[cache]
            true = row[token] - row.max() - math.log(np.exp(row - row.max()).sum())
            assert abs(lp - true) <= 2 * TOL[cache]
    sd.close()


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_the_cache_holds_what_was_emitted(cache):
    w, sd, done = decode(cache, 0.1, 4, 2, 30)
    for r, p in enumerate(PROMPTS):
        n = sd.cached[r]
        tokens = (p + [t for t, _ in done[r]])[:n]
        k = torch.empty((n, HKV, D), dtype=torch.bfloat16, device="cuda")
        v = torch.empty_like(k)
        sd.dec.cache_read([sd.slots[r]], [0], [n], k, v)
        x = w.embed[torch.tensor(tokens, device="cuda")].double()
        # bf16: a rounding to nearest and the sum's order, 2^-8; 8 bits: half a step of 2^-3 besides, and the step below the
        # smallest normal code, 2^-9 of a scale that is at most 2^-7 of the row's largest
        rel = 2.0 ** -8 if cache == "bf16" else 2.0 ** -4 + 2.0 ** -8
        for got, m in ((k, w.w_k), (v, w.w_v)):
            want = (x @ m.double().T).view(n, HKV, D)
            most = want.abs().amax(-1, keepdim=True)
            assert bool(((got.double() - want).abs() <= rel * want.abs() + 2.0 ** -15 * most).all())
    sd.close()


def test_several_tokens_per_step():
    """With little attention the draft is nearly the model: most levels are accepted."""
    _, sd, _ = decode("bf16", 0.1, 4, 2, 1)
    steps = [sum(len(e) for e in sd.step()) for _ in range(8)]
    assert sum(steps) >= 8 * 3 * 2.5
    sd.close()


def test_refusals():
    w, sd, _ = decode("bf16", 0.5, 2, 2, 1)
    for depth, width in ((0, 2), (2, 0), (2, 9), (8, 8)):
        with pytest.raises(ValueError):
            SpeculativeDecoder(w, HQ, HKV, D, 1, 64, depth=depth, width=width)
    with pytest.raises(ValueError):
        sd.add([])
    with pytest.raises(ValueError):
        sd.add([1] * 161)
    with pytest.raises(TsError) as e:
        sd.add([1])                                            # a fourth request of three
    assert e.value.code == B.TS_ERR_NO_SLOT
    sd.close()


def test_command(capsys):
    import json
    assert main(["--requests", "3", "--prompt", "20", "--tokens", "4"]) == 0
    line = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    assert line["gemm_status"] == 0 and line["tokens"] >= 12 and 1 <= line["tokens_per_request_and_step"] <= 4
