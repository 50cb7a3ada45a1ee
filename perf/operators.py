"""What is timed of the operators around drafted tokens: attention for a tree of them over the paged KV cache
(bf16 or 8 bit), the cache written in 8 bits and read back, and log probabilities of given tokens.

A decoder that verifies drafts runs these one after the other: Decoder.tree_attention over the nodes of every
request's draft, token_logprobs of the logits, and Decoder.cache_append of the accepted path. Shapes are those of
workloads.py (the tiny, the 8B-shaped and the 70B-shaped layer), contexts lognormal as in its decode batches.

Plain form: elementary torch operations in 32 bits. exact(): the definition in 64 bits.
"""
import math

import numpy as np
import torch

own = False

TINY, SHAPE_8B, SHAPE_70B = (4, 2, 64), (32, 8, 128), (64, 8, 128)
PAGE = 16


def _tree(shape, cache, rows, median, longest, nodes, ragged=False, shortest=128, lens=2):
    """rows, median, shortest, longest: requests and their cached tokens (lognormal, sigma 1, clipped); nodes: drafted
    tokens of each (ragged: 1 to nodes); lens: seed of the lengths."""
    return {"kind": "tree", "hq": shape[0], "hkv": shape[1], "d": shape[2], "cache": cache, "rows": rows, "median": median,
            "shortest": min(shortest, longest), "longest": longest, "nodes": nodes, "ragged": ragged, "lens": lens}


def _cache(shape, how, cache, rows, tokens, lens=2):
    """how: "write" a chunk of up to `tokens` tokens per row and read it back, "commit" 1 to 6 of `tokens` drafted tokens per
    row and read them back, "read" up to `tokens` tokens per row."""
    return {"kind": "cache", "hq": shape[0], "hkv": shape[1], "d": shape[2], "how": how, "cache": cache, "rows": rows, "tokens": tokens,
            "lens": lens}


def _logprobs(rows, vocab, dtype, top, given):
    return {"kind": "logprobs", "rows": rows, "vocab": vocab, "dtype": dtype, "top": top, "given": given}


def listed():
    c = [
        # the smallest verification: a small model, short drafts, where latency and launches count
        ("tree_tiny", _tree(TINY, "bf16", 4, 64, 128, 5, shortest=16, lens=1)),
        # one long conversation with a full tree: the cache has to be split over the chip
        ("tree_long_8b", _tree(SHAPE_8B, "bf16", 1, 32768, 32768, 64, shortest=32768)),
        # the ordinary decode batch, sixteen drafted tokens each
        ("tree_64x16_8b", _tree(SHAPE_8B, "bf16", 64, 2048, 8192, 16)),
        # large trees of odd size on the larger model: the tensor cores' case
        ("tree_48x61_70b", _tree(SHAPE_70B, "bf16", 48, 1200, 10240, 61, shortest=16, lens=5)),
        # plain decode over the 8-bit cache: one token per request
        ("decode8_64_8b", _tree(SHAPE_8B, "e4m3", 64, 2048, 8192, 1)),
        # the ordinary decode batch over the 8-bit cache, drafts of uneven length
        ("tree8_64x16_8b", _tree(SHAPE_8B, "e4m3", 64, 2048, 8192, 16, ragged=True)),
        # larger trees on the larger model over the 8-bit cache
        ("tree8_96x25_70b", _tree(SHAPE_70B, "e4m3", 96, 1200, 10240, 25, shortest=16, lens=6)),
        # the accepted paths of a decode batch go into the cache
        ("commit8_64_8b", _cache(SHAPE_8B, "commit", "e4m3", 64, 16)),
        # prompts' chunks are written in 8 bits and read back (handed to another instance)
        ("write8_4x8192_8b", _cache(SHAPE_8B, "write", "e4m3", 4, 8192)),
        # one request's next token: alternatives for the client
        ("logprobs_1x32000", _logprobs(1, 32000, "bf16", 20, 1)),
        # a decode batch's verification
        ("logprobs_1024x131072", _logprobs(1024, 131072, "bf16", 5, 3)),
        # a prompt's log probabilities from 32-bit logits, a vocabulary of odd size
        ("logprobs_2000x100003_f32", _logprobs(2000, 100003, "f32", 20, 1)),
    ]
    return [dict(v, name=k) for k, v in c]


def _log(rng, lo, hi):
    """An integer from lo to hi, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 6.5e12, w["flops"] / 1.2e15)


def draw(rng):
    limit = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["tree", "tree", "tree8", "tree8", "decode8", "tiny", "cache", "cache", "logprobs", "logprobs"])
        shape, lens = rng.choice([SHAPE_8B, SHAPE_70B]), rng.randrange(1 << 20)
        median, longest = _log(rng, 64, 4096), rng.choice([8192, 10240, 16384, 32768])
        if kind in ("tree", "tree8"):
            c = _tree(shape, "e4m3" if kind == "tree8" else "bf16", _log(rng, 1, 128), median, longest, _log(rng, 2, 64), rng.random() < 0.5,
                      16, lens)
        elif kind == "decode8":
            c = _tree(shape, "e4m3", _log(rng, 1, 256), median, longest, 1, False, 16, lens)
        elif kind == "tiny":
            c = _tree(TINY, rng.choice(["bf16", "e4m3"]), _log(rng, 1, 32), _log(rng, 16, 256), 512, _log(rng, 1, 64), rng.random() < 0.5, 1, lens)
        elif kind == "cache":
            how = rng.choice(["write", "commit", "read"])
            tokens = _log(rng, 6, 64) if how == "commit" else _log(rng, 1, 8192)
            c = _cache(rng.choice([TINY, SHAPE_8B, SHAPE_70B]), how, rng.choice(["bf16", "e4m3", "e4m3"]), _log(rng, 1, 64), tokens, lens)
        else:
            c = _logprobs(_log(rng, 1, 4096), _log(rng, 1000, 200003), rng.choice(["bf16", "f32"]), rng.choice([0, 1, 5, 20, 32]), rng.randint(1, 4))
        if _cost(c) <= limit:
            return c


# ------------------------------------------------------------------------------------------ sizes of a case
def _lengths(case):
    """(cached tokens, new tokens) per row."""
    rng = np.random.default_rng(case["lens"])
    if case["kind"] == "tree":
        ctx = [int(min(max(round(case["median"] * math.exp(rng.standard_normal())), case["shortest"]), case["longest"]))
               for _ in range(case["rows"])]
        nodes = [int(rng.integers(1, case["nodes"] + 1)) if case["ragged"] else case["nodes"] for _ in range(case["rows"])]
        return ctx, nodes
    ctx = [int(rng.integers(0, 64)) for _ in range(case["rows"])]                       # in front of the tokens: pages are shared with them
    if case["how"] == "commit":
        return ctx, [case["tokens"]] * case["rows"]
    return ctx, [int(rng.integers((case["tokens"] + 1) // 2, case["tokens"] + 1)) for _ in range(case["rows"])]


def _accepted(case):
    """"commit": per row the drafted tokens that are accepted, in order."""
    rng = np.random.default_rng(case["lens"] + 1)
    return [sorted(rng.choice(case["tokens"], size=int(rng.integers(1, min(6, case["tokens"]) + 1)), replace=False).tolist())
            for _ in range(case["rows"])]


def _trees(case):
    """Per row: the set of nodes each node sees as a bit mask (itself and its ancestors); parents are drawn among the nodes in front."""
    rng = np.random.default_rng(case["lens"] + 2)
    out = []
    for n in _lengths(case)[1]:
        masks = []
        for i in range(n):
            p = int(rng.integers(-1, i)) if i else -1
            masks.append((masks[p] if p >= 0 else 0) | 1 << i)
        out.append(masks)
    return out


def work(case):
    """Everything the operator reads and writes once; flops of the visible (query, key) pairs."""
    if case["kind"] == "logprobs":
        n = case["rows"] * case["vocab"]
        return {"bytes": float(n * (2 if case["dtype"] == "bf16" else 4) + case["rows"] * (12 * case["given"] + 8 * case["top"] + 4)), "flops": 5.0 * n}
    ctx, new = _lengths(case)
    hq, hkv, d, n = case["hq"], case["hkv"], case["d"], sum(new)
    wide, token = 2 * hkv * d * 2, 2 * hkv * d * 2 if case["cache"] == "bf16" else 2 * hkv * (d + 1)
    if case["kind"] == "cache":
        n = sum(len(a) for a in _accepted(case)) if case["how"] == "commit" else n
        # written: read wide, stored, read again, handed out wide
        return {"bytes": float(n * (wide + token) * (1 if case["how"] == "read" else 2)), "flops": 2.0 * n * hkv * d}
    pairs = sum(t * c for c, t in zip(ctx, new)) + sum(m.bit_count() for t in _trees(case) for m in t)
    return {"bytes": float(sum(ctx) * token + n * wide + 2 * n * hq * d * 2 + 8 * n), "flops": 4.0 * d * hq * pairs}


# ------------------------------------------------------------------------------------------ inputs
class _State:
    pass


def _power(E):
    """2^E in 32 bits, exactly (pow need not be)."""
    return (E.int() + 127 << 23).view(torch.float32)


def _quantise(x):
    """[..., D] -> e4m3 codes (uint8) and the bytes E + 127 of the powers of two they are scaled by."""
    x = x.float()
    most = x.abs().amax(-1)
    m, e = torch.frexp(most)                                   # most = m 2^e, 0.5 <= m < 1; 448 = 0.875 2^9
    E = (e - 9 + (m > 0.875)).clamp(-62, 62)
    E = torch.where(most == 0, torch.zeros_like(E), E)
    codes = (x * _power(-E)[..., None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    return codes, (E + 127).to(torch.uint8)


def _dequantise(codes, scales):
    return codes.view(torch.float8_e4m3fn).float() * _power(scales.int() - 127)[..., None]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = _State()
    s.case = case

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.bfloat16)

    if case["kind"] == "logprobs":
        n, v = case["rows"], case["vocab"]
        x = torch.empty(n, v, device="cuda", dtype=torch.bfloat16 if case["dtype"] == "bf16" else torch.float32).normal_(0, 2.5, generator=gen)
        # most rows of a language model have a few likely tokens: lift some by 0 to 14
        likely = torch.randint(0, v, (n, 6), generator=gen, device="cuda")
        lift = 14 * torch.rand(n, 6, generator=gen, device="cuda")
        x.scatter_add_(1, likely, lift.to(x.dtype))
        s.logits = x
        # the tokens asked for: the first is a likely one, the others are any
        s.tokens = torch.randint(0, v, (n, case["given"]), generator=gen, device="cuda", dtype=torch.int32)
        s.tokens[:, 0] = likely[:, 0].int()
        return s

    ctx, new = _lengths(case)
    hq, hkv, d, n = case["hq"], case["hkv"], case["d"], sum(new)
    grown = [len(a) for a in _accepted(case)] if case["kind"] == "cache" and case["how"] == "commit" else new
    pages = [-(-(c + t) // PAGE) for c, t in zip(ctx, grown)]
    n_pages = -(-5 * sum(pages) // 4)                           # a pool a quarter larger than the live pages, in shuffled order
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).tolist()
    s.ctx, s.new, s.tables, at = ctx, new, [], 0
    for p in pages:
        s.tables.append(order[at:at + p])
        at += p
    s.pool = normal(n_pages, 2, hkv, PAGE, d)                   # the cached context
    if case["cache"] == "e4m3":
        s.codes = torch.empty(s.pool.shape, dtype=torch.uint8, device="cuda")
        s.scales = torch.empty(s.pool.shape[:-1], dtype=torch.uint8, device="cuda")
        for i in range(0, n_pages, 1024):
            s.codes[i:i + 1024], s.scales[i:i + 1024] = _quantise(s.pool[i:i + 1024])
        s.pool = None
    s.k_new, s.v_new = normal(n, hkv, d), normal(n, hkv, d)
    if case["kind"] == "tree":
        s.q = normal(n, hq, d)
        s.out = torch.empty_like(s.q)
        flat = np.array([m for t in _trees(case) for m in t], dtype=np.uint64).view(np.int64)
        s.mask = torch.from_numpy(flat).cuda()
    else:
        if case["how"] == "commit":
            first = np.concatenate([[0], np.cumsum(new)])
            s.source = torch.tensor([int(first[r]) + i for r, a in enumerate(_accepted(case)) for i in a], dtype=torch.int32, device="cuda")
        else:
            s.source = None
        s.count, s.total = grown, sum(grown)
        s.k_out = torch.empty(s.total, hkv, d, dtype=torch.bfloat16, device="cuda")
        s.v_out = torch.empty_like(s.k_out)
    if own:
        from paper_2512_03416_b200.decoder import Decoder
        s.dec = Decoder(hq, hkv, d, n_pages=n_pages, max_requests=len(ctx), max_pages_per_req=max(pages), cache=case["cache"])
        if case["cache"] == "e4m3":
            s.dec.cache8_values.copy_(s.codes.view(-1))
            s.dec.cache8_scales.copy_(s.scales.view(-1))
            s.codes = s.scales = None
        else:
            s.dec.pool.copy_(s.pool.view(torch.int16).view(-1))
            s.pool = None
        s.slots = []
        for r, table in enumerate(s.tables):
            slot = s.dec.request_add(r, ctx[r] + grown[r])
            s.dec.block_table_set(slot, table)
            s.dec.request_set_len(slot, ctx[r])
            s.slots.append(slot)
    else:
        s.tables = [torch.tensor(t, dtype=torch.int64, device="cuda") for t in s.tables]
    return s


# ------------------------------------------------------------------------------------------ one pass
def _run_own(s):
    c = s.case
    if c["kind"] == "logprobs":
        from paper_2512_03416_b200.logprobs import token_logprobs
        r = token_logprobs(s.logits, s.tokens, n_top=c["top"])
        return {"logprob": r.logprob, "rank": r.rank, "entropy": r.entropy, "top_logprob": r.top_logprob, "top_token": r.top_token}
    if c["kind"] == "tree":
        s.dec.tree_attention(s.slots, s.new, s.ctx, s.q, s.k_new, s.v_new, s.out, mask=s.mask)
        return {"out": s.out}
    if c["how"] != "read":
        s.dec.cache_append(s.slots, s.count, s.ctx, s.k_new, s.v_new, source=s.source, keep_len=True)
    s.dec.cache_read(s.slots, s.ctx, s.count, s.k_out, s.v_out)
    return {"k": s.k_out, "v": s.v_out}


def _gather(s, table, first, count):
    """K and V [count, hkv, d] of a request's tokens first, first + 1, ... in 32 bits."""
    pos = torch.arange(first, first + count, device="cuda")
    page, slot = table[pos // PAGE], pos % PAGE
    if s.case["cache"] == "bf16":
        both = s.pool[page, :, :, slot].float()
    else:
        both = _dequantise(s.codes[page, :, :, slot], s.scales[page, :, :, slot])
    return both[:, 0], both[:, 1]


def _attend(case, q, k, v, mask, ctx):
    """q [t, hq, d], k and v [keys, hkv, d], mask [t] bits of the keys from ctx on -> [t, hq, d]."""
    t, hq, d = q.shape
    hkv, n = k.shape[1], k.shape[0]
    q = q.view(t, hkv, hq // hkv, d).permute(1, 0, 2, 3).reshape(hkv, -1, d)              # [hkv, t * g, d]
    s = torch.matmul(q, k.permute(1, 2, 0)) * d ** -0.5                                    # [hkv, t * g, keys]
    seen = torch.ones(t, n, dtype=torch.bool, device=q.device)
    seen[:, ctx:] = (mask[:, None] >> torch.arange(n - ctx, device=q.device)) & 1 != 0
    s = s.masked_fill(~seen.repeat_interleave(hq // hkv, 0), -math.inf)
    p = torch.exp(s - s.amax(-1, keepdim=True))
    o = torch.matmul(p, v.permute(1, 0, 2)) / p.sum(-1, keepdim=True)
    return o.view(hkv, t, hq // hkv, d).permute(1, 0, 2, 3).reshape(t, hq, d)


def _run_plain(s):
    c = s.case
    if c["kind"] == "logprobs":
        parts = []
        for i in range(0, c["rows"], 256):
            x, tok = s.logits[i:i + 256].float(), s.tokens[i:i + 256].long()
            m = x.amax(-1, keepdim=True)
            e = torch.exp(x - m)
            z = e.sum(-1, keepdim=True)
            lse = m + torch.log(z)
            at = x.gather(1, tok)
            index = torch.arange(c["vocab"], device=x.device)
            rank = torch.stack([((x > at[:, j:j + 1]) | ((x == at[:, j:j + 1]) & (index < tok[:, j:j + 1]))).sum(-1) for j in range(c["given"])], 1)
            # the shift by the maximum keeps the difference of two large numbers out of the entropy
            entropy = torch.log(z[:, 0]) - (e * (x - m)).sum(-1) / z[:, 0]
            if c["top"]:
                top, which = torch.sort(x, dim=-1, descending=True, stable=True)              # equal values: lowest index first
                top, which = top[:, :c["top"]] - lse, which[:, :c["top"]]
            else:
                top, which = x[:, :0], tok[:, :0]
            parts.append((at - lse, rank.int(), entropy, top, which.int()))
        names = ("logprob", "rank", "entropy", "top_logprob", "top_token")
        return {name: torch.cat([p[j] for p in parts]) for j, name in enumerate(names)}
    at = np.concatenate([[0], np.cumsum(s.new)]).tolist()
    if c["kind"] == "tree":
        outs = []
        for r, ctx in enumerate(s.ctx):
            a, b = at[r], at[r + 1]
            k, v = _gather(s, s.tables[r], 0, ctx)
            k, v = torch.cat([k, s.k_new[a:b].float()]), torch.cat([v, s.v_new[a:b].float()])
            outs.append(_attend(c, s.q[a:b].float(), k, v, s.mask[a:b], ctx))
        return {"out": torch.cat(outs).to(torch.bfloat16)}
    if c["how"] != "read":
        k, v = (s.k_new, s.v_new) if s.source is None else (s.k_new[s.source.long()], s.v_new[s.source.long()])
        pos = torch.cat([torch.arange(f, f + n, device="cuda") for f, n in zip(s.ctx, s.count)])
        page = torch.cat([s.tables[r][torch.arange(f, f + n, device="cuda") // PAGE] for r, (f, n) in enumerate(zip(s.ctx, s.count))])
        if c["cache"] == "bf16":
            s.pool[page, 0, :, pos % PAGE], s.pool[page, 1, :, pos % PAGE] = k, v
        else:
            for i, x in enumerate((k, v)):
                s.codes[page, i, :, pos % PAGE], s.scales[page, i, :, pos % PAGE] = _quantise(x)
    both = [_gather(s, s.tables[r], f, n) for r, (f, n) in enumerate(zip(s.ctx, s.count))]
    return {"k": torch.cat([b[0] for b in both]).to(torch.bfloat16), "v": torch.cat([b[1] for b in both]).to(torch.bfloat16)}


def run(s):
    return _run_own(s) if own else _run_plain(s)


# ------------------------------------------------------------------------------------------ the definition, in 64 bits
def _value_of_codes():
    """The 256 values of e4m3: sign, 4 bits of exponent (bias 7), 3 of mantissa; 0x7f and 0xff are no numbers."""
    v = []
    for b in range(256):
        e, m = b >> 3 & 15, b & 7
        x = math.nan if e == 15 and m == 7 else (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6
        v.append(-x if b >> 7 else x)
    return v


def _nearest_code(x):
    """x (64 bits, magnitude up to 448) rounded to e4m3, ties to the even mantissa."""
    step = torch.full_like(x, 2.0 ** -9)                       # of the numbers below 2^-5
    for e in range(-5, 9):
        step[x.abs() >= 2.0 ** e] = 2.0 ** (e - 3)
    return torch.round(x / step) * step


def exact(case, seed):
    global own
    keep, own = own, False                                     # the inputs alone
    try:
        s = prepare(case, seed)
    finally:
        own = keep
    if case["kind"] == "logprobs":
        lp, ent, top = [], [], []
        for i in range(0, case["rows"], 128):
            x = s.logits[i:i + 128].double()
            lse = torch.logsumexp(x, -1, keepdim=True)
            p = torch.exp(x - lse)
            lp.append(torch.gather(x - lse, 1, s.tokens[i:i + 128].long()))
            ent.append(-(p * (x - lse)).sum(-1))
            top.append(torch.topk(x - lse, case["top"], -1).values)
        return {"logprob": torch.cat(lp), "rank": None, "entropy": torch.cat(ent), "top_logprob": torch.cat(top), "top_token": None}
    if case["cache"] == "e4m3":
        table = torch.tensor(_value_of_codes(), dtype=torch.float64, device="cuda")
        power = torch.tensor([2.0 ** (b - 127) for b in range(256)], dtype=torch.float64, device="cuda")
    where = [(torch.arange(c + n, device="cuda")) for c, n in zip(s.ctx, s.new if case["kind"] == "tree" else s.count)]

    def cached(r, pos):                                         # [tokens, 2, hkv, d]
        page, slot = s.tables[r][pos // PAGE], pos % PAGE
        if case["cache"] == "bf16":
            return s.pool[page, :, :, slot].double()
        return table[s.codes[page, :, :, slot].long()] * power[s.scales[page, :, :, slot].long()][..., None]

    first = 0
    if case["kind"] == "cache":
        ks, vs = [], []
        for r, (f, n) in enumerate(zip(s.ctx, s.count)):
            if case["how"] == "read":
                both = cached(r, where[r][f:])
            else:
                rows = s.source[first:first + n].long() if s.source is not None else torch.arange(first, first + n, device="cuda")
                both = torch.stack([s.k_new[rows], s.v_new[rows]], 1).double()
                if case["cache"] == "e4m3":
                    unit = power[(torch.ceil(torch.log2(both.abs().amax(-1, keepdim=True) / 448)).clamp(-62, 62) + 127).long()]
                    both = _nearest_code(both / unit) * unit
            ks.append(both[:, 0])
            vs.append(both[:, 1])
            first += n
        return {"k": torch.cat(ks), "v": torch.cat(vs)}
    outs, g = [], case["hq"] // case["hkv"]
    for r, (c, n) in enumerate(zip(s.ctx, s.new)):
        old = cached(r, where[r][:c])
        new = torch.stack([s.k_new[first:first + n], s.v_new[first:first + n]], 1).double()
        kv = torch.cat([old, new])
        bits = [[(m >> j) & 1 for j in range(n)] for m in s.mask[first:first + n].tolist()]
        hidden = torch.cat([torch.zeros(n, c, device="cuda"), 1.0 - torch.tensor(bits, dtype=torch.float32, device="cuda")], 1) > 0
        out = torch.empty(n, case["hq"], case["d"], dtype=torch.float64, device="cuda")
        for h in range(case["hq"]):
            score = s.q[first:first + n, h].double() @ kv[:, 0, h // g].T / math.sqrt(case["d"])
            score[hidden] = -math.inf
            out[:, h] = torch.softmax(score, -1) @ kv[:, 1, h // g]
        outs.append(out)
        first += n
    return {"out": torch.cat(outs)}
