"""Speculative decoding on the decoder's cache: every iteration drafts a small tree of tokens per request, verifies all of
them in one step (ts_tree_attention -> logits -> ts_token_logprobs) and writes the accepted path behind the cached tokens
(ts_cache_append). The model is one attention layer between an embedding and a head, without positions:
    x = embed[token],   y = x + attention(x W_q, x W_k, x W_v) W_o,   logits = y W_head
and its draft leaves the attention out (logits = x W_head), so that a draft depends on one token only. Projections run
through ts_gemm_bf16, PyTorch looks embeddings up and holds the memory.

    python -m paper_2512_03416_b200.speculative --requests 32 --prompt 1000 --tokens 64 --cache e4m3
"""
from __future__ import annotations

import argparse
import json
from typing import List, NamedTuple

import numpy as np
import torch

from . import binding as B
from .decoder import Decoder, _check, _raw_stream
from .logprobs import token_logprobs


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


class SpeculativeDecoder:
    """Greedy decoding of several requests at once. A tree has depth levels of width tokens below the last emitted token; the
    first (likeliest) token of a level carries the next level. What is emitted is what one token per step would give."""

    def __init__(self, weights: Weights, n_q_heads: int, n_kv_heads: int, head_dim: int, max_requests: int, max_tokens: int,
                 depth: int = 3, width: int = 2, cache: str = "bf16", device: int = 0):
        if not (depth >= 1 and 1 <= width <= 8 and 1 + depth * width <= 64):
            raise ValueError("a tree has 1 to 8 tokens per level and at most 64 in all")
        self.w, self.depth, self.width, self.nodes = weights, depth, width, 1 + depth * width
        pages = -(-max_tokens // 16)
        self.dec = Decoder(n_q_heads, n_kv_heads, head_dim, n_pages=pages * max_requests, max_requests=max_requests,
                           max_pages_per_req=pages, cache=cache, device=device)
        self.device = self.dec.device
        self.max_tokens = max_tokens
        # node 0 is the last emitted token; level l holds the nodes 1 + l width .., all children of one node
        self.carrier = [0] + [1 + l * width for l in range(depth - 1)]            # that level's parent
        rc, words = B.ts_tree_masks([-1] + [p for p in self.carrier for _ in range(width)])
        _check(rc, "ts_tree_masks")
        self.words = np.array(words, dtype=np.uint64).astype(np.int64)
        self.gemm_status = torch.zeros(1, dtype=torch.int32, device=self.device)
        self.slots: List[int] = []
        self.cached: List[int] = []
        self.last: List[int] = []            # emitted (or given), not cached yet: the next tree's first node
        self.masks = None

    def _project(self, x: torch.Tensor, w: torch.Tensor, residual=None) -> torch.Tensor:
        out = torch.empty((x.shape[0], w.shape[0]), dtype=torch.bfloat16, device=self.device)
        _check(B.ts_gemm_bf16(self.device.index, x.shape[0], w.shape[0], x.shape[1], x.data_ptr(), w.data_ptr(),
                              0 if residual is None else residual.data_ptr(), out.data_ptr(), 0, self.gemm_status.data_ptr(),
                              _raw_stream(self.device.index)), "ts_gemm_bf16")
        return out

    def _heads(self, x: torch.Tensor, w: torch.Tensor) -> torch.Tensor:
        return self._project(x, w).view(x.shape[0], -1, self.dec.cfg.head_dim)

    def add(self, prompt) -> int:
        """Cache the prompt's tokens but the last one, which becomes the first tree's first node. Returns the request's index."""
        prompt = [int(t) for t in prompt]
        if not 1 <= len(prompt) <= self.max_tokens:
            raise ValueError(f"a prompt has 1 to {self.max_tokens} tokens")
        slot = self.dec.request_add(len(self.slots), len(prompt))
        n = len(prompt) - 1
        if n:
            self.dec.alloc_pages(slot, n)
            x = self.w.embed[torch.tensor(prompt[:-1], device=self.device)]
            self.dec.cache_append([slot], [n], [0], self._heads(x, self.w.w_k), self._heads(x, self.w.w_v))
        self.slots.append(slot)
        self.cached.append(n)
        self.last.append(prompt[-1])
        self.masks = torch.from_numpy(np.tile(self.words, len(self.slots))).to(self.device)
        return len(self.slots) - 1

    def _draft(self) -> torch.Tensor:
        """int32 [requests, nodes]: the last token of each request, then the levels."""
        tree = torch.empty((len(self.slots), self.nodes), dtype=torch.int32, device=self.device)
        tree[:, 0] = torch.tensor(self.last, dtype=torch.int32, device=self.device)
        for l, parent in enumerate(self.carrier):
            logits = self._project(self.w.embed[tree[:, parent]], self.w.w_head)
            tree[:, 1 + l * self.width:1 + (l + 1) * self.width] = token_logprobs(logits, n_top=self.width).top_token
        return tree

    def step(self) -> List[List[tuple]]:
        """One iteration. Returns each request's newly emitted (token, log probability) pairs, at least one."""
        R, T, W = len(self.slots), self.nodes, self.width
        tree = self._draft()
        x = self.w.embed[tree.view(-1)]
        q, k, v = self._heads(x, self.w.w_q), self._heads(x, self.w.w_k), self._heads(x, self.w.w_v)
        out = torch.empty_like(q)
        self.dec.tree_attention(self.slots, [T] * R, self.cached, q, k, v, out, self.masks)
        logits = self._project(self._project(out.view(R * T, -1), self.w.w_o, x), self.w.w_head)
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
        return done

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
    a = ap.parse_args(argv)
    hidden, vocab, hq, hkv, d = 1024, 32000, 32, 8, 128
    sd = SpeculativeDecoder(random_weights(vocab, hidden, hq, hkv, d, a.seed), hq, hkv, d, a.requests,
                            a.prompt + (a.tokens + 3) * (a.depth + 1), a.depth, a.width, a.cache)
    rng = np.random.default_rng(a.seed)
    for _ in range(a.requests):
        sd.add(rng.integers(0, vocab, a.prompt))
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
                      "gemm_status": int(sd.gemm_status.item()), "data": "synthetic, random weights"}))
    sd.close()
    return 0


if __name__ == "__main__":
    raise SystemExit(main())
