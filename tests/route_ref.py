"""The wide gate's choice from its definition, in 64 bits and one token after the other: an expert whose logit is -inf or NaN is
masked; masked experts come after all others and are equal, groups with fewer than group_best others after those that have them, groups with
none after those, and equal values go to the smaller id."""
import math

INF = float("inf")


def clean(l):
    """Logits with -inf in the place of NaN."""
    return l.masked_fill(l != l, -INF)


def scores(row, sigmoid):
    if sigmoid:
        return [1 / (1 + math.exp(-x)) if x > -709.0 else 0.0 for x in row]
    top = max(row)
    e = [math.exp(x - top) if x > -INF else 0.0 for x in row]
    total = sum(e)
    return [x / total if total > 0 else 0.0 for x in e]


def choose(r, row, bias=None):
    """(ids, their scores) of one token's logits for the router r (a binding's struct)."""
    row, S = [x if x == x else -INF for x in row], r.E // r.n_groups
    live = [x > -INF for x in row]
    s = scores(row, r.score == 1)
    v = [x + b for x, b in zip(s, bias)] if bias is not None else row
    best = lambda e: (False, -v[e], e) if live[e] else (True, 0.0, e)
    open_ = list(range(r.E))
    if r.n_groups > 1:
        def rank(g):
            of = [(v if r.group_best == 1 or bias is not None else s)[e] for e in range(g * S, g * S + S) if live[e]]
            value = sum(sorted(of, reverse=True)[:r.group_best]) if len(of) >= r.group_best else -INF
            return not of, -value, g
        groups = sorted(range(r.n_groups), key=rank)[:r.top_groups]
        open_ = [e for e in open_ if e // S in groups]
    ids = sorted(open_, key=best)[:r.k]
    return ids, [s[e] for e in ids]


def route(r, l, bias=None):
    """Choices and weights of every row of l."""
    idx, w = [], []
    b = None if bias is None else bias.double().tolist()
    for row in l.double().tolist():
        ids, s = choose(r, row, b)
        total = sum(s) if r.renormalise else 1.0
        idx.append(ids)
        w.append([r.scale * x / total if total > 0 else 0.0 for x in s])
    return idx, w
