"""What is timed of the operators for requests that are not alike: a projection with a low-rank adapter per request, drafted
tokens verified against the model's probabilities from given random numbers, and cache pages copied and shared between requests.

A decoder that samples several continuations per request from drafts runs them in turn: Decoder.fork of the prompt,
adapted_project around Decoder.tree_attention, verify_tokens of the logits, Decoder.cache_append of the accepted path, and
Decoder.requests_free. Shapes are those of workloads.py and of the 8B-shaped layer of bench.py (hidden 4096, intermediate 14336).

Plain form: elementary torch operations in 32 bits (probabilities that are compared or summed along a vocabulary in 64).
exact(): the definition in 64 bits.
"""
import math

import numpy as np
import torch

own = False

TINY, SHAPE_8B, SHAPE_70B = (4, 2, 64), (32, 8, 128), (64, 8, 128)
PAGE = 16


def _adapt(n, k, rank, adapters, decode, chunks, longest=1, residual=False, none=0.0, lens=1):
    """decode: requests of one token; chunks: requests of 2 to longest tokens; none: share of requests without an adapter;
    lens: seed of lengths and adapters."""
    return {"kind": "adapt", "n": n, "k": k, "rank": rank, "adapters": adapters, "decode": decode, "chunks": chunks, "longest": longest,
            "residual": residual, "none": none, "lens": lens}


def _verify(requests, nodes, vocab, dtype, chain, drawn, ragged=False, lens=1):
    """nodes: of each request's tree (ragged: 1 to nodes), the last emitted token among them; chain: each node has one child;
    drawn: drafts are drawn from a draft model's distribution, which is given too (else they are its likeliest tokens)."""
    return {"kind": "verify", "requests": requests, "nodes": nodes, "vocab": vocab, "dtype": dtype, "chain": chain, "drawn": drawn, "ragged": ragged,
            "lens": lens}


def _pages(shape, how, cache, count, tokens, copies=1, lens=1):
    """how: "copy" `count` pages to others, "fork" `count` requests of up to `tokens` cached tokens `copies` times and free the copies."""
    return {"kind": "pages", "hkv": shape[1], "hq": shape[0], "d": shape[2], "how": how, "cache": cache, "count": count, "tokens": tokens, "copies": copies,
            "lens": lens}


def listed():
    c = [
        # the smallest step of a small model: launches count
        ("adapt_tiny", _adapt(384, 256, 8, 3, 2, 1, 3)),
        # the ordinary decode batch, every request with an adapter of its own, query/key/value projection
        ("adapt_64_qkv_8b", _adapt(6144, 4096, 16, 64, 64, 0)),
        # a larger decode batch of the larger model, adapters shared by some requests, output projection
        ("adapt_192_out_70b", _adapt(8192, 8192, 32, 48, 192, 0, residual=True, none=0.1)),
        # the burst step: decode requests next to a prompt's chunk, gate and up projection, rank 64
        ("adapt_2112_gate_up_8b", _adapt(28672, 4096, 64, 16, 64, 1, 2048)),
        # chunks of several prompts, odd lengths and rank, down projection
        ("adapt_chunks_down_8b", _adapt(4096, 14336, 24, 5, 3, 9, 333, residual=True, none=0.2)),
        # one request's draft of three tokens: latency
        ("verify_1x4", _verify(1, 4, 32000, "bf16", True, True)),
        # the ordinary decode batch, chains of five drafted tokens drawn from a draft model
        ("verify_64x6_drawn", _verify(64, 6, 131072, "bf16", True, True)),
        # trees of drawn tokens, 32-bit logits of a vocabulary of odd size
        ("verify_48x25_drawn_f32", _verify(48, 25, 100003, "f32", False, True, ragged=True)),
        # a large decode batch, trees of a draft's likeliest tokens
        ("verify_256x8_likeliest", _verify(256, 8, 131072, "bf16", False, False)),
        # four samples of each request of a decode batch
        ("fork_64x4_8b", _pages(SHAPE_8B, "fork", "bf16", 64, 2048, 4)),
        # pages of an 8-bit cache moved together
        ("copy8_1000_8b", _pages(SHAPE_8B, "copy", "e4m3", 1000, 0)),
        # a long prompt's pages copied
        ("copy_4096_70b", _pages(SHAPE_70B, "copy", "bf16", 4096, 0)),
    ]
    return [dict(v, name=k) for k, v in c]


def _log(rng, lo, hi):
    """An integer from lo to hi, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 6.4e12, w["flops"] / 1.2e15)


def draw(rng):
    limit = {"adapt": 0, "verify": 0, "pages": 0}
    for c in listed():
        limit[c["kind"]] = max(limit[c["kind"]], _cost(c))
    while True:
        kind, lens = rng.choice(["adapt", "adapt", "adapt", "verify", "verify", "verify", "pages"]), rng.randrange(1 << 20)
        if kind == "adapt":
            n, k = rng.choice([(6144, 4096), (4096, 4096), (28672, 4096), (4096, 14336), (10240, 8192), (8192, 8192), (384, 256), (264, 520)])
            chunks = rng.choice([0, 0, 1, _log(rng, 2, 16)])
            c = _adapt(n, k, rng.choice([8, 16, 16, 24, 32, 40, 64, 128]), _log(rng, 1, 96), _log(rng, 1, 256) if not chunks or rng.random() < 0.7 else 0, chunks,
                       _log(rng, 2, 2048) if chunks else 1, rng.random() < 0.5, rng.choice([0.0, 0.0, 0.3]), lens)
        elif kind == "verify":
            c = _verify(_log(rng, 1, 256), _log(rng, 1, 32), _log(rng, 1000, 200003), rng.choice(["bf16", "f32"]), rng.random() < 0.4,
                        rng.random() < 0.6, rng.random() < 0.5, lens)
        else:
            how = rng.choice(["copy", "fork"])
            c = _pages(rng.choice([TINY, SHAPE_8B, SHAPE_70B]), how, rng.choice(["bf16", "e4m3"]), _log(rng, 1, 4096 if how == "copy" else 64),
                       _log(rng, 1, 4096), _log(rng, 1, 8), lens)
        if _cost(c) <= limit[kind] and (kind != "verify" or sum(_nodes(c)) * c["vocab"] <= 300_000_000):
            return c


# ------------------------------------------------------------------------------------------ sizes of a case
def _rows(case):
    """(tokens, adapter or -1) per request, in the order of the step."""
    rng = np.random.default_rng(case["lens"])
    tokens = [1] * case["decode"] + [int(rng.integers((case["longest"] + 2) // 2, case["longest"] + 1)) if case["longest"] > 2 else 2
                                     for _ in range(case["chunks"])]
    if case["chunks"] == 1 and case["longest"] > 1:
        tokens[-1] = case["longest"]
    adapter = [-1 if rng.random() < case["none"] else r % case["adapters"] for r in range(len(tokens))]
    return tokens, rng.permutation(adapter).tolist()


def _nodes(case):
    rng = np.random.default_rng(case["lens"])
    return [int(rng.integers(1, case["nodes"] + 1)) if case["ragged"] else case["nodes"] for _ in range(case["requests"])]


WIDEST = 4


def _parents(case):
    """Per request the parent of each node (-1: the first): the one in front (chain) or any in front that has fewer than WIDEST children."""
    rng = np.random.default_rng(case["lens"] + 1)
    out = []
    for n in _nodes(case):
        p, children = [-1], [0] * n
        for i in range(1, n):
            j = i - 1
            if not case["chain"]:
                j = int(rng.choice([x for x in range(i) if children[x] < WIDEST]))
            children[j] += 1
            p.append(j)
        out.append(p)
    return out


def _cached(case):
    rng = np.random.default_rng(case["lens"])
    return [int(rng.integers((case["tokens"] + 1) // 2, case["tokens"] + 1)) for _ in range(case["count"])]


def _page_bytes(case):
    return 2 * case["hkv"] * PAGE * (2 * case["d"] if case["cache"] == "bf16" else case["d"] + 1)


def work(case):
    if case["kind"] == "adapt":
        tokens, adapter = _rows(case)
        m, n, k, rank = sum(tokens), case["n"], case["k"], case["rank"]
        adapted = sum(t for t, a in zip(tokens, adapter) if a >= 0)
        used = len(set(adapter) - {-1})
        return {"bytes": 2.0 * (m * k + n * k + m * n * (2 if case["residual"] else 1) + used * rank * (n + k)),
                "flops": 2.0 * m * n * k + 2.0 * adapted * rank * (n + k)}
    if case["kind"] == "verify":
        # the first node's row (and the draft's) of each request has to be read, whatever is accepted; of the others, the ones on the accepted path
        values = float(case["requests"] * case["vocab"] * (2 if case["drawn"] else 1))
        return {"bytes": values * (2 if case["dtype"] == "bf16" else 4) + 20.0 * sum(_nodes(case)), "flops": 6.0 * values}
    lengths = _cached(case) if case["how"] == "fork" else []
    copied = case["count"] if case["how"] == "copy" else case["copies"] * sum(t % PAGE != 0 for t in lengths)
    return {"bytes": 2.0 * copied * _page_bytes(case) + 8.0 * copied + 8.0 * case["copies"] * sum(-(-t // PAGE) for t in lengths), "flops": 0.0}


# ------------------------------------------------------------------------------------------ inputs
class _State:
    pass


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = _State()
    s.case = case

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=gen, device="cuda", dtype=torch.bfloat16) * std)

    if case["kind"] == "adapt":
        s.tokens, s.adapter = _rows(case)
        m, n, k, rank, count = sum(s.tokens), case["n"], case["k"], case["rank"], case["adapters"]
        s.x, s.w = normal(m, k), normal(n, k, std=k ** -0.5)
        s.a, s.b = normal(count, rank, k, std=k ** -0.5), normal(count, n, rank, std=0.5 * rank ** -0.5)
        s.scale = 0.5 + torch.rand(count, generator=gen, device="cuda")
        s.residual = normal(m, n) if case["residual"] else None
        if own:
            from paper_2512_03416_b200.adapters import Adapters
            s.adapters = Adapters(s.a, s.b, s.scale)
        return s

    if case["kind"] == "verify":
        s.nodes, parents, v = _nodes(case), _parents(case), case["vocab"]
        n, dtype = sum(s.nodes), torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        first = np.concatenate([[0], np.cumsum(s.nodes)])
        s.logits, s.draft = (torch.empty(n, v, device="cuda", dtype=dtype) for _ in range(2))
        for i in range(0, n, 64):                                # rows of a model: a few likely tokens; the draft's are near them
            x = torch.randn(min(64, n - i), v, generator=gen, device="cuda") * 2
            likely = torch.randint(0, v, (x.shape[0], 12), generator=gen, device="cuda")
            x.scatter_add_(1, likely, 15 * torch.rand(likely.shape, generator=gen, device="cuda"))
            s.logits[i:i + 64] = x
            s.draft[i:i + 64] = x + 0.7 * torch.randn(x.shape, generator=gen, device="cuda")
        s.parents = torch.tensor([p for t in parents for p in t], dtype=torch.int32, device="cuda")
        s.tokens = torch.randint(0, v, (n,), generator=gen, device="cuda", dtype=torch.int32)
        above = [(int(first[r]) + i, int(first[r]) + p, sum(x == p for x in t[:i])) for r, t in enumerate(parents) for i, p in enumerate(t) if p >= 0]
        for i in range(0, len(above), 64):
            node, parent, sibling = (torch.tensor(x, device="cuda") for x in zip(*above[i:i + 64]))
            row = s.draft[parent].float()
            if case["drawn"]:                                    # independent draws from the draft's distribution
                e = torch.empty_like(row).exponential_(generator=gen)
                s.tokens[node] = (row - torch.log(e)).argmax(-1).int()
            else:
                s.tokens[node] = torch.topk(row, WIDEST, -1).indices.gather(1, sibling[:, None])[:, 0].int()
        if not case["drawn"]:
            s.draft = None
        s.u_accept, s.u_sample = (torch.rand(x, generator=gen, device="cuda") for x in (n, len(s.nodes)))
        s.scale = 0.8 + 0.4 * torch.rand(n, generator=gen, device="cuda")
        s.draft_scale = s.scale.clone() if case["drawn"] else None
        depths = [0]
        for t in parents:
            d = []
            for p in t:
                d.append(d[p] + 1 if p >= 0 else 0)
            depths.append(max(d))
        s.depth, s.widest = max(depths), max([max((t.count(p) for p in t if p >= 0), default=0) for t in parents])
        return s

    hkv, d, cpu = case["hkv"], case["d"], torch.Generator().manual_seed(seed)
    if case["how"] == "copy":
        n_pages = 2 * case["count"] + case["count"] // 4
        order = torch.randperm(n_pages, generator=cpu)
        s.src, s.dst = order[:case["count"]], order[case["count"]:2 * case["count"]]
    else:
        lengths = _cached(case)
        held = [-(-t // PAGE) for t in lengths]
        n_pages = sum(held) + case["copies"] * case["count"] + 8
        order = torch.randperm(n_pages, generator=cpu).tolist()
        tables, at = [], 0
        for h in held:
            tables.append(order[at:at + h])
            at += h
        free = sorted(order[at:])                                # a decoder's new pages are the lowest free ones
        s.src = torch.tensor([t[-1] for t, n in zip(tables, lengths) if n % PAGE for _ in range(case["copies"])], dtype=torch.int64)
        s.dst = torch.tensor(free[:len(s.src)], dtype=torch.int64)
        s.tables = torch.tensor([t + [-1] * (max(held) - len(t)) for t in tables], dtype=torch.int32)
        s.ends = torch.tensor([h - 1 for h, n in zip(held, lengths) if n % PAGE for _ in range(case["copies"])])
        s.partial = torch.tensor([r * case["copies"] + i for r, n in enumerate(lengths) if n % PAGE for i in range(case["copies"])], dtype=torch.int64)
        s.uses = torch.zeros(n_pages, dtype=torch.int32)
        s.uses[order[:at]] = 1
    shape = (n_pages, 2, hkv, PAGE, d)
    if case["cache"] == "bf16":
        s.pool = normal(*shape)
    else:
        # codes of numbers and, in powers of two, what rows are scaled by
        s.codes = torch.randint(0, 0x7f, shape, generator=gen, device="cuda", dtype=torch.uint8)
        s.scales = torch.randint(110, 130, shape[:-1], generator=gen, device="cuda", dtype=torch.uint8)
    if own:
        from paper_2512_03416_b200.decoder import Decoder
        copies = case["copies"] if case["how"] == "fork" else 0
        longest = max(held) if copies else 1
        s.dec = Decoder(case["hq"], hkv, d, n_pages=n_pages, max_requests=case["count"] * (1 + copies), max_pages_per_req=longest, cache=case["cache"])
        if case["cache"] == "bf16":
            s.dec.pool.copy_(s.pool.view(torch.int16).view(-1))
            s.pool = s.dec.pool.view(torch.bfloat16).view(shape)
        else:
            s.dec.cache8_values.copy_(s.codes.view(-1))
            s.dec.cache8_scales.copy_(s.scales.view(-1))
            s.codes, s.scales = s.dec.cache8_values.view(shape), s.dec.cache8_scales.view(shape[:-1])
        s.src, s.dst = s.src.numpy().astype(np.int32), s.dst.numpy().astype(np.int32)
        if copies:
            slots = []
            for r, table in enumerate(tables):
                slots.append(s.dec.request_add(r, lengths[r]))
                s.dec.block_table_set(slots[r], table)
                s.dec.request_set_len(slots[r], lengths[r])
            s.parents = np.repeat(np.array(slots, dtype=np.int32), copies)
            s.ids = np.arange(len(slots), len(slots) + len(s.parents), dtype=np.int64)
    else:
        s.src, s.dst = s.src.cuda(), s.dst.cuda()
        if case["how"] == "fork":
            s.tables, s.ends, s.partial, s.uses = s.tables.cuda(), s.ends.cuda(), s.partial.cuda(), s.uses.cuda()
            s.parents = torch.arange(case["count"], device="cuda").repeat_interleave(case["copies"])
    return s


# ------------------------------------------------------------------------------------------ one pass
def _run_own(s):
    c = s.case
    if c["kind"] == "adapt":
        from paper_2512_03416_b200.adapters import adapted_project
        return {"y": adapted_project(s.x, s.w, s.adapters, s.tokens, s.adapter, residual=s.residual)}
    if c["kind"] == "verify":
        from paper_2512_03416_b200.verify import verify_tokens
        r = verify_tokens(s.logits, s.tokens, s.parents, s.nodes, s.u_accept, s.u_sample, draft=s.draft, scale=s.scale, draft_scale=s.draft_scale)
        return {"emitted": r.emitted, "count": r.count, "path": r.path, "logprob": r.logprob}
    out = {"pool": s.pool} if c["cache"] == "bf16" else {"codes": s.codes, "scales": s.scales}
    if c["how"] == "copy":
        s.dec.copy_pages(s.src, s.dst)
        return out
    slots = s.dec.fork(s.parents, s.ids)
    out["tables"] = s.dec.block_tables(slots)
    s.dec.requests_free(slots[::-1])
    return out


def _adapt_plain(s):
    n, k, rank, count = s.case["n"], s.case["k"], s.case["rank"], s.case["adapters"]
    x = s.x.float()
    y = x @ s.w.float().T
    which = torch.tensor(s.adapter, device="cuda").repeat_interleave(torch.tensor(s.tokens, device="cuda"))
    of = torch.arange(count, device="cuda").repeat_interleave(rank)                    # the adapter of each of all the ranks
    u = (x @ s.a.float().view(-1, k).T) * s.scale.repeat_interleave(rank)
    u = u * (which[:, None] == of)
    y += u @ s.b.float().transpose(1, 2).reshape(-1, n)
    if s.residual is not None:
        y += s.residual.float()
    return {"y": y.to(torch.bfloat16)}


def _verify_plain(s):
    """All requests at once, level after level."""
    n, v, dev = len(s.tokens), s.case["vocab"], s.tokens.device
    nodes = torch.tensor(s.nodes, device=dev)
    first = torch.cumsum(nodes, 0) - nodes
    start = first.repeat_interleave(nodes)
    above = torch.where(s.parents >= 0, s.parents + start, -1)
    emitted, path = (torch.full((n + 1,), -1, dtype=torch.int32, device=dev) for _ in range(2))          # the last place is nobody's
    logprob, count = torch.zeros(n + 1, device=dev), torch.zeros(len(nodes), dtype=torch.int32, device=dev)
    at, live = first, torch.ones(len(nodes), dtype=torch.bool, device=dev)
    token = s.tokens.long()
    for level in range(s.depth + 1):
        x = s.logits[at].double() * s.scale[at, None].double()
        logp = x - torch.logsumexp(x, -1, keepdim=True)
        r = torch.exp(logp)
        if s.draft is not None:
            y = s.draft[at].double() * s.draft_scale[at, None].double()
            q = torch.exp(y - torch.logsumexp(y, -1, keepdim=True))
        chosen = torch.full_like(at, -1)
        mine = above[None, :] == at[:, None]
        order = torch.cumsum(mine, -1) - 1
        for j in range(s.widest):
            hit = mine & (order == j)
            child = torch.where(hit.any(-1), hit.int().argmax(-1), -1)
            tok = token[child.clamp(min=0)][:, None]
            asked = live & (chosen < 0) & (child >= 0)
            chance = s.u_accept[child.clamp(min=0)].double() * (q.gather(1, tok)[:, 0] if s.draft is not None else 1.0)
            yes = asked & (chance < r.gather(1, tok)[:, 0])
            chosen = torch.where(yes, child, chosen)
            less = (r - q).clamp(min=0) if s.draft is not None else r.scatter(1, tok, 0.0)
            total = less.sum(-1, keepdim=True)
            r = torch.where((asked & ~yes)[:, None] & (total > 0), less / total, r)
        cdf = torch.cumsum(r, -1)
        drawn = (cdf <= s.u_sample[:, None].double() * cdf[:, -1:]).sum(-1).clamp(max=v - 1)
        out = torch.where(chosen >= 0, token[chosen.clamp(min=0)], drawn)
        to = torch.where(live, first + level, n)
        emitted[to], path[to] = out.int(), at.int()
        logprob[to] = logp.gather(1, out[:, None])[:, 0].float()
        count += live.int()
        live = live & (chosen >= 0)
        at = torch.where(live, chosen, at)
    return {"emitted": emitted[:n], "count": count, "path": path[:n], "logprob": logprob[:n]}


def run(s):
    if own:
        return _run_own(s)
    if s.case["kind"] == "adapt":
        return _adapt_plain(s)
    if s.case["kind"] == "verify":
        return _verify_plain(s)
    if s.case["cache"] == "bf16":
        s.pool[s.dst] = s.pool[s.src]
        out = {"pool": s.pool}
    else:
        s.codes[s.dst], s.scales[s.dst] = s.codes[s.src], s.scales[s.src]
        out = {"codes": s.codes, "scales": s.scales}
    if s.case["how"] == "fork":
        tables = s.tables[s.parents]
        tables[s.partial, s.ends] = s.dst.int()
        held = tables[tables >= 0].long()
        s.uses.index_add_(0, held, torch.ones_like(held, dtype=torch.int32))           # the copies' requests hold them
        s.uses.index_add_(0, held, torch.full_like(held, -1, dtype=torch.int32))       # and are freed
        out["tables"] = tables
    return out


# ------------------------------------------------------------------------------------------ the definition, in 64 bits
def _walk(s, r, first, parents):
    """One request: the logarithms of the model's probabilities of what it emits."""
    node, out = 0, []
    while True:
        x = s.logits[first + node].double() * float(s.scale[first + node])
        p = torch.softmax(x, 0)
        left = p
        if s.draft is not None:
            q = torch.softmax(s.draft[first + node].double() * float(s.draft_scale[first + node]), 0)
        found = None
        for c in [i for i, a in enumerate(parents) if a == node]:
            t = int(s.tokens[first + c])
            if s.draft is None:
                q = torch.zeros_like(p)
                q[t] = 1.0
            if float(s.u_accept[first + c]) * float(q[t]) < float(left[t]):
                found = c
                break
            rest = torch.relu(left - q)
            if float(rest.sum()) > 0:
                left = rest / rest.sum()
        if found is None:
            upto = torch.cumsum(left, 0)
            t = int((upto > float(s.u_sample[r]) * float(upto[-1])).nonzero()[0])
        out.append(float(torch.log_softmax(x, 0)[t]))
        if found is None:
            return out
        node = found


def exact(case, seed):
    global own
    keep, own = own, False                                     # the inputs alone
    try:
        s = prepare(case, seed)
    finally:
        own = keep
    if case["kind"] == "adapt":
        ys, at = [], 0
        for t, a in zip(s.tokens, s.adapter):
            x = s.x[at:at + t].double()
            w = torch.zeros(t, case["n"], dtype=torch.float64, device="cuda")
            if a >= 0:
                w = float(s.scale[a]) * ((x @ s.a[a].double().T) @ s.b[a].double().T)
            if s.residual is not None:
                w += s.residual[at:at + t].double()
            ys.append(w)
            at += t
        return {"y": torch.cat(ys) + s.x.double() @ s.w.double().T}
    if case["kind"] == "verify":
        lp, at = torch.zeros(len(s.tokens), dtype=torch.float64), 0
        for r, t in enumerate(_parents(case)):
            for i, x in enumerate(_walk(s, r, at, t)):
                lp[at + i] = x
            at += len(t)
        return {"emitted": None, "count": None, "path": None, "logprob": lp}
    if case["cache"] != "bf16":
        return None
    want = s.pool.double()                                       # copies are exact
    for a, b in zip(s.src.tolist(), s.dst.tolist()):
        want[b] = s.pool[a].double()
    return {"pool": want, "tables": None} if case["how"] == "fork" else {"pool": want}
