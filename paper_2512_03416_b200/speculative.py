"""Speculative decoding on the decoder's cache: every iteration drafts a small tree of tokens per request, verifies all of
them in one step (ts_tree_attention -> logits -> ts_token_logprobs) and writes the accepted path behind the cached tokens
(ts_cache_append). The model is one attention layer between an embedding and a head, without positions:
    x = embed[token],   y = x + attention(x W_q, x W_k, x W_v) W_o,   logits = y W_head
and its draft leaves the attention out (logits = x W_head), so that a draft depends on one token only. Projections run
through ts_gemm_bf16, PyTorch looks embeddings up and holds the memory.

With a temperature, drafts are drawn and verified by sampling (ts_verify_tokens), a request may be continued several times from one
prompt (ts_request_fork shares its pages), and requests may have low-rank adapters of their own on the attention's projections
(ts_adapter_project).

    python -m paper_2512_03416_b200.speculative --requests 32 --prompt 1000 --tokens 64 --cache e4m3
    python -m paper_2512_03416_b200.speculative --requests 8 --samples 4 --temperature 0.8 --adapters 8 --rank 16
"""
from __future__ import annotations

import argparse
import functools
import json
import operator
from typing import Dict, List, NamedTuple, Optional

import numpy as np
import torch

from . import binding as B
from .adapters import Adapters, adapted_project
from .decoder import Decoder, TsError, _check, _raw_stream
from .logprobs import token_logprobs
from .verify import verify_tokens


class Weights(NamedTuple):
    """bf16 CUDA tensors [out features, in features]."""
    embed: torch.Tensor          # [vocab, hidden]
    w_q: torch.Tensor            # [Hq D, hidden]
    w_k: torch.Tensor            # [Hkv D, hidden]
    w_v: torch.Tensor            # [Hkv D, hidden]
    w_o: torch.Tensor            # [hidden, Hq D]
    w_head: torch.Tensor         # [vocab, hidden]


def random_weights(vocab: int, hidden: int, n_q_heads: int, n_kv_heads: int, head_dim: int, seed: int, device: int = 0,
                   attention: float = 0.5) -> Weights:
    """attention: the attention's share of y next to x; the larger it is, the more often the draft is wrong."""
    gen = torch.Generator(device=f"cuda:{device}").manual_seed(seed)

    def normal(rows, cols, std):
        return (torch.randn(rows, cols, generator=gen, device=f"cuda:{device}") * std).to(torch.bfloat16)

    hq, hkv = n_q_heads * head_dim, n_kv_heads * head_dim
    return Weights(normal(vocab, hidden, 1.0), normal(hq, hidden, hidden ** -0.5), normal(hkv, hidden, hidden ** -0.5),
                   normal(hkv, hidden, hidden ** -0.5), normal(hidden, hq, attention * hq ** -0.5),
                   normal(vocab, hidden, 4 * hidden ** -0.5))


def random_adapters(weights: Weights, count: int, rank: int, seed: int, strength: float = 0.3) -> Dict[str, Adapters]:
    """count adapters for each of the attention's projections; strength: their part of a projection's result."""
    gen = torch.Generator(device=weights.w_q.device).manual_seed(seed)

    def normal(*shape, std):
        return (torch.randn(*shape, generator=gen, device=weights.w_q.device) * std).to(torch.bfloat16)

    out = {}
    for name, w in (("q", weights.w_q), ("k", weights.w_k), ("v", weights.w_v), ("o", weights.w_o)):
        n, k = w.shape
        std = strength * float(w.float().std()) * k ** 0.5
        out[name] = Adapters(normal(count, rank, k, std=k ** -0.5), normal(count, n, rank, std=std * rank ** -0.5))
    return out


class SpeculativeDecoder:
    """Decoding of several requests at once. A tree has depth levels of width tokens below the last emitted token; the
    first token of a level carries the next level. temperature 0: greedy, levels are the draft's likeliest tokens, and what is emitted is what one
    token per step would give. Otherwise levels are drawn from the draft's distribution, and what is emitted is distributed as samples of one
    token per step are. adapters: of the projections q, k, v, o (random_adapters; those that are not there have none)."""

    def __init__(self, weights: Weights, n_q_heads: int, n_kv_heads: int, head_dim: int, max_requests: int, max_tokens: int,
                 depth: int = 3, width: int = 2, cache: str = "bf16", device: int = 0, temperature: float = 0.0, seed: int = 0,
                 adapters: Optional[Dict[str, Adapters]] = None):
        if not (depth >= 1 and 1 <= width <= 8 and 1 + depth * width <= 64):
            raise ValueError("a tree has 1 to 8 tokens per level and at most 64 in all")
        if temperature < 0:
            raise ValueError("a temperature is not negative")
        self.w, self.depth, self.width, self.nodes = weights, depth, width, 1 + depth * width
        pages = -(-max_tokens // 16)
        self.dec = Decoder(n_q_heads, n_kv_heads, head_dim, n_pages=pages * max_requests, max_requests=max_requests,
                           max_pages_per_req=pages, cache=cache, device=device)
        self.device = self.dec.device
        self.max_tokens = max_tokens
        # node 0 is the last emitted token; level l holds the nodes 1 + l width .., all children of one node
        self.carrier = [0] + [1 + l * width for l in range(depth - 1)]            # that level's parent
        parents = [-1] + [p for p in self.carrier for _ in range(width)]
        rc, words = B.ts_tree_masks(parents)
        _check(rc, "ts_tree_masks")
        self.words = np.array(words, dtype=np.uint64).astype(np.int64)
        self.gemm_status = torch.zeros(1, dtype=torch.int32, device=self.device)
        self.slots: List[int] = []
        self.cached: List[int] = []
        self.last: List[int] = []            # emitted (or given), not cached yet: the next tree's first node
        self.masks = None
        self.temperature, self.adapters = temperature, adapters or {}
        self.adapter: List[int] = []         # of each request, -1: none
        self.parents = torch.tensor(parents, dtype=torch.int32, device=self.device)
        self.random = torch.Generator(device=self.device).manual_seed(seed)

    def _project(self, x: torch.Tensor, w: torch.Tensor, residual=None, name: str = "", rows=(), which=()) -> torch.Tensor:
        """rows, which: tokens and adapter of each request, for a projection that has adapters."""
        if name in self.adapters and any(a >= 0 for a in which):
            return adapted_project(x, w, self.adapters[name], rows, which, residual=residual)
        out = torch.empty((x.shape[0], w.shape[0]), dtype=torch.bfloat16, device=self.device)
        _check(B.ts_gemm_bf16(self.device.index, x.shape[0], w.shape[0], x.shape[1], x.data_ptr(), w.data_ptr(),
                              0 if residual is None else residual.data_ptr(), out.data_ptr(), 0, self.gemm_status.data_ptr(),
                              _raw_stream(self.device.index)), "ts_gemm_bf16")
        return out

    def _heads(self, x: torch.Tensor, w: torch.Tensor, *adapted) -> torch.Tensor:
        return self._project(x, w, None, *adapted).view(x.shape[0], -1, self.dec.cfg.head_dim)

    def add(self, prompt, adapter: int = -1) -> int:
        """Cache the prompt's tokens but the last one, which becomes the first tree's first node. Returns the request's index."""
        if adapter < -1 or any(adapter >= a.count for a in self.adapters.values()) or (adapter >= 0 and not self.adapters):
            raise ValueError(f"there is no adapter {adapter}")
        prompt = [int(t) for t in prompt]
        if not 1 <= len(prompt) <= self.max_tokens:
            raise ValueError(f"a prompt has 1 to {self.max_tokens} tokens")
        slot = self.dec.request_add(len(self.slots), len(prompt))
        n = len(prompt) - 1
        if n:
            self.dec.alloc_pages(slot, n)
            x = self.w.embed[torch.tensor(prompt[:-1], device=self.device)]
            self.dec.cache_append([slot], [n], [0], self._heads(x, self.w.w_k, "k", [n], [adapter]), self._heads(x, self.w.w_v, "v", [n], [adapter]))
        return self._added(slot, n, prompt[-1], adapter)

    def _added(self, slot: int, cached: int, last: int, adapter: int) -> int:
        self.slots.append(slot)
        self.cached.append(cached)
        self.last.append(last)
        self.adapter.append(adapter)
        self.masks = torch.from_numpy(np.tile(self.words, len(self.slots))).to(self.device)
        return len(self.slots) - 1

    def fork(self, index: int, copies: int) -> List[int]:
        """Further requests that go on from where request `index` is, its cached tokens shared. Returns their indices."""
        slots = self.dec.fork([self.slots[index]] * copies, range(len(self.slots), len(self.slots) + copies))
        return [self._added(int(s), self.cached[index], self.last[index], self.adapter[index]) for s in slots]

    def _draft(self) -> torch.Tensor:
        """int32 [requests, nodes]: the last token of each request, then the levels."""
        tree = torch.empty((len(self.slots), self.nodes), dtype=torch.int32, device=self.device)
        tree[:, 0] = torch.tensor(self.last, dtype=torch.int32, device=self.device)
        for l, parent in enumerate(self.carrier):
            logits = self._project(self.w.embed[tree[:, parent]], self.w.w_head)
            tree[:, 1 + l * self.width:1 + (l + 1) * self.width] = token_logprobs(logits, n_top=self.width).top_token
        return tree

    def _uniform(self, n: int) -> torch.Tensor:
        return torch.rand(n, generator=self.random, device=self.device)

    def _draw(self):
        """_draft with the levels drawn, each token by itself, and the draft's logits [requests * nodes, vocab] (rows of nodes with children)."""
        R, W = len(self.slots), self.width
        tree = torch.empty((R, self.nodes), dtype=torch.int32, device=self.device)
        tree[:, 0] = torch.tensor(self.last, dtype=torch.int32, device=self.device)
        draft = torch.empty((R, self.nodes, self.w.w_head.shape[0]), dtype=torch.bfloat16, device=self.device)
        for l, parent in enumerate(self.carrier):
            draft[:, parent] = self._project(self.w.embed[tree[:, parent]], self.w.w_head)
            rows = draft[:, parent].repeat_interleave(W, 0)
            none = torch.full((R * W,), -1, dtype=torch.int32, device=self.device)
            drawn = verify_tokens(rows, none, none, [1] * (R * W), self._uniform(R * W), self._uniform(R * W), scale=self._scale(R * W))
            tree[:, 1 + l * W:1 + (l + 1) * W] = drawn.emitted.view(R, W)
        return tree, draft.view(R * self.nodes, -1)

    def _scale(self, n: int) -> torch.Tensor:
        return torch.full((n,), 1.0 / self.temperature, device=self.device)

    def _sampled(self, tree, draft, logits, k, v) -> List[List[tuple]]:
        R, T = len(self.slots), self.nodes
        scale = self._scale(R * T)
        got = verify_tokens(logits, tree.view(-1), self.parents.repeat(R), [T] * R, self._uniform(R * T), self._uniform(R), draft=draft, scale=scale, draft_scale=scale)
        counts = got.count.tolist()
        keep = got.path >= 0                                     # count of each request, in order: what the cache takes
        tokens, lps = got.emitted[keep].tolist(), got.logprob[keep].tolist()
        if -1 in tokens:
            raise FloatingPointError("logits or draft logits that are no distribution")
        for r in range(R):
            self.dec.alloc_pages(self.slots[r], self.cached[r] + counts[r])
        self.dec.cache_append(self.slots, counts, self.cached, k, v, source=got.path[keep])
        emitted, at = [], 0
        for r, n in enumerate(counts):
            emitted.append(list(zip(tokens[at:at + n], lps[at:at + n])))
            self.cached[r] += n
            self.last[r] = tokens[at + n - 1]
            at += n
        return emitted

    def step(self) -> List[List[tuple]]:
        """One iteration. Returns each request's newly emitted (token, log probability) pairs, at least one."""
        R, T, W = len(self.slots), self.nodes, self.width
        tree, draft = self._draw() if self.temperature > 0 else (self._draft(), None)
        x = self.w.embed[tree.view(-1)]
        rows = [T] * R
        q, k, v = (self._heads(x, w, name, rows, self.adapter) for name, w in (("q", self.w.w_q), ("k", self.w.w_k), ("v", self.w.w_v)))
        out = torch.empty_like(q)
        self.dec.tree_attention(self.slots, rows, self.cached, q, k, v, out, self.masks)
        logits = self._project(self._project(out.view(R * T, -1), self.w.w_o, x, "o", rows, self.adapter), self.w.w_head)
        if self.temperature > 0:
            return self._sampled(tree, draft, logits, k, v)
        # the drafted children of each node, -1 where it has none: a child of rank 0 is what the model would emit there
        given = torch.full((R, T, W), -1, dtype=torch.int32, device=self.device)
        given[:, self.carrier] = tree[:, 1:].view(R, self.depth, W)
        lp = token_logprobs(logits, given.view(R * T, W), n_top=1)
        rank = lp.rank.view(R, T, W).cpu().numpy()
        best, best_lp = lp.top_token.view(R, T).cpu().numpy(), lp.top_logprob.view(R, T).cpu().numpy()
        emitted, source, counts = [], [], []
        for r in range(R):
            path = [0]
            for l, parent in enumerate(self.carrier):
                hit = np.flatnonzero(rank[r, parent] == 0) if path[-1] == parent else ()
                if len(hit) == 0:
                    break
                path.append(1 + l * W + int(hit[0]))
            emitted.append([(int(best[r, n]), float(best_lp[r, n])) for n in path])
            source += [r * T + n for n in path]
            counts.append(len(path))
            self.dec.alloc_pages(self.slots[r], self.cached[r] + len(path))
        self.dec.cache_append(self.slots, counts, self.cached, k, v,
                              source=torch.tensor(source, dtype=torch.int32, device=self.device))
        for r in range(R):
            self.cached[r] += counts[r]
            self.last[r] = emitted[r][-1][0]
        return emitted

    def generate(self, n_tokens: int) -> List[List[tuple]]:
        """At least n_tokens further (token, log probability) pairs per request."""
        done: List[List[tuple]] = [[] for _ in self.slots]
        while min(len(d) for d in done) < n_tokens:
            for d, new in zip(done, self.step()):
                d += new
        if self.projection_status():
            raise TsError(B.TS_ERR_DEVICE_TIMEOUT, "a projection")
        return done

    def projection_status(self) -> int:
        """TS_DEV_TIMEOUT where a bounded wait of a projection ran out, of one with adapters too (whose status other users of these adapters share).
        Waits for the steps."""
        return functools.reduce(operator.or_, (int(s.item()) for s in [self.gemm_status] + [a.status for a in self.adapters.values()]))

    def close(self) -> None:
        self.dec.close()


def main(argv=None) -> int:
    ap = argparse.ArgumentParser(description=__doc__.split(":")[0])
    ap.add_argument("--requests", type=int, default=32)
    ap.add_argument("--prompt", type=int, default=1000)
    ap.add_argument("--tokens", type=int, default=64, help="to emit per request, at least")
    ap.add_argument("--depth", type=int, default=3)
    ap.add_argument("--width", type=int, default=2)
    ap.add_argument("--cache", choices=("bf16", "e4m3"), default="e4m3")
    ap.add_argument("--seed", type=int, default=1)
    ap.add_argument("--temperature", type=float, default=0.0, help="0: greedy")
    ap.add_argument("--samples", type=int, default=1, help="continuations of each request (with a temperature)")
    ap.add_argument("--adapters", type=int, default=0, help="low-rank adapters, request r uses r modulo this")
    ap.add_argument("--rank", type=int, default=16)
    a = ap.parse_args(argv)
    hidden, vocab, hq, hkv, d = 1024, 32000, 32, 8, 128
    weights = random_weights(vocab, hidden, hq, hkv, d, a.seed)
    sd = SpeculativeDecoder(weights, hq, hkv, d, a.requests * a.samples,
                            a.prompt + (a.tokens + 3) * (a.depth + 1), a.depth, a.width, a.cache, temperature=a.temperature, seed=a.seed,
                            adapters=random_adapters(weights, a.adapters, a.rank, a.seed) if a.adapters else None)
    rng = np.random.default_rng(a.seed)
    for r in range(a.requests):
        sd.add(rng.integers(0, vocab, a.prompt), r % a.adapters if a.adapters else -1)
    for r in range(a.requests):
        if a.samples > 1:
            sd.fork(r, a.samples - 1)
    a.requests *= a.samples
    for _ in range(3):
        sd.step()
    start, stop = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    steps = tokens = 0
    while tokens < a.tokens * a.requests:
        tokens += sum(len(e) for e in sd.step())
        steps += 1
    stop.record()
    stop.synchronize()
    ms = start.elapsed_time(stop)
    print(json.dumps({"requests": a.requests, "prompt": a.prompt, "cache": a.cache, "nodes_per_tree": sd.nodes, "steps": steps,
                      "tokens": tokens, "tokens_per_request_and_step": round(tokens / steps / a.requests, 3),
                      "ms_per_step": round(ms / steps, 4), "tokens_per_s": round(tokens / ms * 1e3, 1),
                      "gemm_status": sd.projection_status(), "data": "synthetic, random weights"}))
    sd.close()
    return 0


if __name__ == "__main__":
    raise SystemExit(main())
