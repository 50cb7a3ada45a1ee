"""The walk of a verification in 64 bits, one request at a time, from the definition (numpy)."""
import numpy as np


def softmax(row, scale):
    y = np.asarray(row, np.float64) * float(scale)
    if np.isnan(y).any() or (y == np.inf).any() or (y == -np.inf).all():
        return None
    e = np.exp(y - y.max())
    return e / e.sum()


def walk(logits, draft, tokens, parents, u_accept, u_sample, scale, draft_scale):
    """Arrays of one request. Returns (emitted tokens, nodes walked, log probabilities, how near the nearest decision was): the last is the least
    distance of a comparison from its border, as a probability."""
    vocab = logits.shape[1]
    node, emitted, path, lp, near = 0, [], [], [], np.inf
    while True:
        path.append(node)
        kids = [i for i in range(node + 1, len(tokens)) if parents[i] == node and 0 <= tokens[i] < vocab]
        p = softmax(logits[node], scale[node])
        q = softmax(draft[node], draft_scale[node]) if draft is not None and kids else None
        if p is None or (draft is not None and kids and q is None):
            return emitted + [-1], path, lp + [np.nan], near
        r, chosen, seen = p, None, set()
        for i in kids:
            t = int(tokens[i])
            if draft is None:
                if t in seen:
                    continue
                seen.add(t)
                need, less = float(u_accept[i]), r.copy()
                less[t] = 0.0
            else:
                need, less = float(u_accept[i]) * q[t], np.maximum(r - q, 0.0)
            near = min(near, abs(need - r[t]))
            if need < r[t]:
                chosen = i
                break
            if less.sum() > 0:
                r = less / less.sum()
        if chosen is None:
            cdf = np.cumsum(r)
            want = float(u_sample) * cdf[-1]
            near = min(near, np.abs(cdf - want).min())
            hit = np.flatnonzero(cdf > want)
            t = int(hit[0]) if len(hit) else int(np.flatnonzero(r)[-1])
        else:
            t = int(tokens[chosen])
        emitted.append(t)
        with np.errstate(divide="ignore"):
            lp.append(float(np.log(p[t])))
        if chosen is None:
            return emitted, path, lp, near
        node = chosen
