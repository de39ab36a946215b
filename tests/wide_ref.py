"""Plain 64-bit forms of the wide gate, the 8-bit format and clipping, written from their definitions (CPU torch)."""
import math

import torch

INF = float("inf")


def scores(l, sigmoid):
    l = l.double()
    if sigmoid:
        return torch.sigmoid(l)
    top = l.max(1, keepdim=True).values
    e = torch.exp(l - torch.where(top == -INF, torch.zeros_like(top), top))
    s = e.sum(1, keepdim=True)
    return e / torch.where(s > 0, s, torch.ones_like(s))


def route(r, l, bias=None, mask=None):
    """Choices and weights of the router r (a binding's struct), one token after the other."""
    S = r.E // r.n_groups
    p = scores(l, r.score == 1)
    idx, w = torch.full((r.T, r.k), -1, dtype=torch.int32), torch.zeros(r.T, r.k, dtype=torch.float64)
    for t in range(r.T):
        if mask is not None and not mask[t]:
            continue
        live = [float(l[t, e]) > -INF for e in range(r.E)]
        sums = [float(p[t, e]) + (0.0 if bias is None else float(bias[e])) for e in range(r.E)]
        v = [(float(l[t, e]) if bias is None else sums[e]) if live[e] else -INF for e in range(r.E)]
        open_ = range(r.E)
        if r.n_groups > 1:
            value = []
            for g in range(r.n_groups):
                of = (v if r.group_best == 1 else [s if a else -INF for s, a in zip(sums, live)])[g * S:(g + 1) * S]
                value.append(sum(sorted(of, reverse=True)[:r.group_best]))
            groups = sorted(range(r.n_groups), key=lambda g: (-value[g], g))[:r.top_groups]
            open_ = [e for e in range(r.E) if e // S in groups]
        chosen = sorted(open_, key=lambda e: (-v[e], e))[:r.k]
        s = [float(p[t, e]) for e in chosen]
        total = sum(s) if r.renormalise else 1.0
        for j, e in enumerate(chosen):
            idx[t, j] = e
            w[t, j] = r.scale * s[j] / total if total > 0 else 0.0
    return idx, w


def route_grad(r, l, idx, dw):
    """Gradient by torch's autograd in 64 bits on an independent statement of the weights."""
    x = torch.nan_to_num(l.double(), neginf=-1e300).requires_grad_()
    p = torch.sigmoid(x) if r.score == 1 else torch.softmax(x, 1)
    ok = (idx >= 0) & (idx < r.E)
    ok = ok & (l.gather(1, torch.where(ok, idx, 0).long()) > -INF)
    s = p.gather(1, torch.where(ok, idx, 0).long()) * ok
    if r.renormalise:
        total = s.sum(1, keepdim=True)
        s = s / torch.where(total > 0, total, torch.ones_like(total))
    torch.where(ok, r.scale * s * dw.double(), torch.zeros_like(s)).sum().backward()
    return x.grad


def up(n, m):
    return -(-n // m) * m


def unit(e):
    return torch.pow(torch.tensor(2.0, dtype=torch.float64), e.double())


def exponent(top):
    """Smallest e >= -127 with top * 2^-e <= 448; 0 for 0; 120 at least where top is not finite."""
    out = torch.zeros(top.shape, dtype=torch.int64)
    for i, v in enumerate(top.reshape(-1).tolist()):
        if not math.isfinite(v):
            e = 120
        elif v == 0:
            e = 0
        else:
            e = math.frexp(v)[1] - 9
            while v > 448.0 * 2.0 ** e:
                e += 1
        out.view(-1)[i] = max(e, -127)
    return out


def e4m3(v):
    """Values of at most 448 (or not finite: NaN) rounded to e4m3, ties to even."""
    _, e = torch.frexp(v.abs())
    step = unit((e - 4).clamp(min=-9))
    return torch.where(torch.isfinite(v), torch.round(v / step) * step, torch.full_like(v, float("nan")))


def quantise_rows(x):
    rows, K = x.shape
    Kp = up(K, 128)
    b = torch.zeros(rows, Kp, dtype=torch.float64)
    b[:, :K] = x.double()
    b = b.reshape(rows, Kp // 128, 128)
    top = torch.where(torch.isnan(b), torch.full_like(b, INF), b.abs()).amax(2)
    e = exponent(top)
    byte = torch.full((rows, up(Kp // 128, 4)), 127, dtype=torch.uint8)
    byte[:, :Kp // 128] = (e + 127).to(torch.uint8)
    return e4m3(b / unit(e)[:, :, None]).reshape(rows, Kp), byte


def quantise_weights(W):
    E, K, N = W.shape
    Kp, Np = up(K, 128), up(N, 128)
    b = torch.zeros(E, Np, Kp, dtype=torch.float64)
    b[:, :N, :K] = W.double().transpose(1, 2)
    b = b.reshape(E, Np // 128, 128, Kp // 128, 128)
    top = torch.where(torch.isnan(b), torch.full_like(b, INF), b.abs()).amax(dim=(2, 4))
    e = exponent(top)
    byte = torch.full((E, Np // 128, up(Kp // 128, 4)), 127, dtype=torch.uint8)
    byte[:, :, :Kp // 128] = (e + 127).to(torch.uint8)
    return e4m3(b / unit(e)[:, :, None, :, None]).reshape(E, Np, Kp), byte


def wide_rows(q, byte):
    """64-bit values of 8-bit rows [.., Kp] with a byte per row and 128 entries."""
    n = q.shape[-1] // 128
    v = q.double().reshape(*q.shape[:-1], n, 128) * unit(byte[..., :n].long() - 127)[..., None]
    return v.reshape(q.shape)


def wide_weights(q, byte):
    """64-bit matrices [E, Kp, Np] of 8-bit weights [E, Np, Kp]."""
    v = wide_rows(q, byte.repeat_interleave(128, 1))
    return v.transpose(1, 2)


def act(z, gelu):
    return 0.5 * z * torch.erfc(-z * math.sqrt(0.5)) if gelu else torch.relu(z)
