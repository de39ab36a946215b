"""The operators around a many-expert layer, as measurable cases: routing over groups of experts (forward, and forward
with backward), quantising rows and weights to 8 bits, the experts' block on 8-bit operands, the whole serving pass
built from them, and the global norm and clipping of gradients.

`own` chooses who computes: the plain forms below, or the framework's entry points.  Definitions:

* Routing.  Scores s of a token's logits l: softmax, or the logistic function of each.  An expert's value is s + bias (in
  64 bits), or l itself without a bias.  With groups of E / n_groups consecutive experts, a group's value is the sum of
  its group_best largest values (of s where there is no bias and more than one is summed), and only experts of the
  top_groups groups with the largest values can be chosen.  The k experts with the largest values are chosen, best
  first; ties go to the lower id.  The weights are scale * s / (sum of the chosen s), or scale * s.  A masked (padded)
  token has choices -1 and weights 0.
* 8 bits.  A block of 128 consecutive entries of a row (of 128 x 128 of a weight matrix) shares one exponent e, the
  smallest with max |x| * 2^-e <= 448, held as e + 127 in a byte; the values are x * 2^-e rounded to e4m3.  Rows are
  padded with zeros to a multiple of 128, their exponents to a multiple of 4; weights are held transposed, [N, K].
* Clipping.  norm = sqrt(sum of all squares); gradients are multiplied by max_norm / norm if norm > max_norm.
"""
import math

import torch

own = False

_T = {"f32": torch.float32, "bf16": torch.bfloat16}
_INF = float("inf")


# ---- cases --------------------------------------------------------------------------------------------------------
def _route(name, T, E, k, score="sigmoid", bias=True, groups=1, top=1, best=1, renorm=True, scale=1.0, pad=0.0, train=False):
    return {"name": name, "op": "route", "T": T, "E": E, "k": k, "score": score, "bias": bias, "groups": groups, "top": top,
            "best": best, "renorm": renorm, "scale": scale, "pad": pad, "train": train}


def _ffn(name, T, k, d, f, E, act="gelu", skew=0.0):
    return {"name": name, "op": "ffn", "T": T, "k": k, "d": d, "f": f, "E": E, "act": act, "skew": skew}


def _serve(name, T, k, d, f, E, groups, top, best, act="gelu", pad=0.0):
    return {"name": name, "op": "serve", "T": T, "k": k, "d": d, "f": f, "E": E, "groups": groups, "top": top, "best": best,
            "act": act, "score": "sigmoid", "bias": True, "renorm": True, "scale": 1.5, "pad": pad}


def _clip(name, tensors, n32, n16, share):
    return {"name": name, "op": "clip", "tensors": tensors, "n32": n32, "n16": n16, "share": share}


def listed():
    return [
        # One step of a decoder: a handful of tokens, many experts in groups; latency is all there is.
        _route("route_decode", 24, 128, 6, groups=8, top=3, best=2, scale=2.0),
        # Training the existing layer's kind of gate (softmax, top-2), a ragged batch with padding: forward and backward.
        _route("route_train_softmax", 5003, 60, 2, score="softmax", bias=False, pad=0.15, train=True),
        # Training a wide gate with a balancing bias on a large batch.
        _route("route_train_wide", 65536, 256, 8, groups=8, top=4, best=2, scale=2.5, train=True),
        # Activations on their way into the experts, no size a multiple of a block or a tile.
        {"name": "quantise_rows_ragged", "op": "rows", "rows": 3001, "K": 776, "dtype": "bf16"},
        # A large batch of wide activations.
        {"name": "quantise_rows_large", "op": "rows", "rows": 65536, "K": 2048, "dtype": "bf16"},
        # All first matrices of the 32-expert layer, from their fp32 masters.
        {"name": "quantise_weights", "op": "weights", "E": 32, "K": 1024, "N": 4096, "dtype": "f32"},
        # The 32-expert layer's block with a few rows per expert: the weights' stream.
        _ffn("ffn_few_rows", 61, 2, 1024, 4096, 32),
        # Sizes that are no multiple of any tile, popular and unpopular experts.
        _ffn("ffn_ragged", 5003, 2, 776, 3080, 6, act="relu", skew=1.1),
        # A big share of wide experts: matrix instructions.
        _ffn("ffn_large", 65536, 2, 2048, 8192, 16),
        # Serving: a full batch of prompts through router, experts and mixture, some of it padding.
        _serve("serve_prompts", 8192, 4, 1024, 4096, 64, 8, 4, 2, pad=0.1),
        # Gradients of a small model: many tensors of any length, held in one buffer without alignment.
        _clip("clip_many_small", 157, 1500000, 700000, 0.4),
        # The expert matrices' fp32 gradients of the 32-expert layer beside a larger model's bf16 ones.
        _clip("clip_large", 24, 270000000, 130000000, 0.4),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _mult8(rng, lo, hi):
    return max(8, 8 * (_log_int(rng, lo, hi) // 8))


def draw(rng):
    op = rng.choice(("route", "route", "rows", "weights", "ffn", "ffn", "serve", "clip"))
    if op == "route":
        groups = rng.choice((1, 1, 2, 4, 8, 16))
        size = rng.randint(max(2, -(-8 // groups)), 256 // groups)
        E, best = groups * size, rng.choice((1, 2))
        top = rng.randint(1, groups)
        c = _route("", _log_int(rng, 1, 65536), E, rng.randint(1, min(8, top * size)), score=rng.choice(("softmax", "sigmoid")),
                   bias=rng.random() < 0.6, groups=groups, top=top, best=best, renorm=rng.random() < 0.75,
                   scale=rng.choice((1.0, 2.5)), pad=rng.choice((0.0, 0.0, 0.2)), train=rng.random() < 0.6)
    elif op == "rows":
        c = {"op": op, "rows": _log_int(rng, 1, 65536), "K": _mult8(rng, 64, 2048), "dtype": rng.choice(("f32", "bf16"))}
    elif op == "weights":
        c = {"op": op, "E": _log_int(rng, 1, 32), "K": _mult8(rng, 64, 2048), "N": _mult8(rng, 64, 2048),
             "dtype": rng.choice(("f32", "bf16"))}
    elif op == "ffn":
        while True:
            c = _ffn("", _log_int(rng, 1, 65536), rng.choice((1, 2, 4, 8)), _mult8(rng, 128, 2048), _mult8(rng, 256, 8192),
                     _log_int(rng, 8, 128), act=rng.choice(("gelu", "gelu", "relu")), skew=rng.choice((0.0, 0.0, 1.1)))
            if c["T"] * c["k"] * c["d"] * c["f"] <= 131072 * 2048 * 8192 // 4 and c["E"] * c["d"] * c["f"] <= 1 << 29 \
                    and c["T"] * c["k"] <= 131072:
                break
    elif op == "serve":
        while True:
            groups = rng.choice((1, 2, 4, 8))
            size = rng.randint(max(2, -(-8 // groups)), 128 // groups)
            top = rng.randint(max(1, -(-8 // size)) if size * groups >= 8 else groups, groups)
            c = _serve("", _log_int(rng, 1, 16384), rng.choice((1, 2, 4, 8)), _mult8(rng, 128, 2048), _mult8(rng, 256, 8192),
                       groups * size, groups, top, rng.choice((1, 2)), act=rng.choice(("gelu", "relu")),
                       pad=rng.choice((0.0, 0.2)))
            if c["k"] <= top * size and c["T"] * c["k"] * c["d"] * c["f"] <= 131072 * 2048 * 8192 // 8 \
                    and c["E"] * c["d"] * c["f"] <= 1 << 29 and c["T"] * c["k"] <= 65536:
                break
    else:
        n = _log_int(rng, 1000, 200000000)
        part = rng.choice((0.0, 0.4, 0.8, 1.0))
        c = _clip("", rng.randint(1, 400), int(n * part), n - int(n * part), rng.choice((0.3, 2.0)))
    c.pop("name", None)
    return c


# ---- inputs -------------------------------------------------------------------------------------------------------
def _up(n, m):
    return -(-n // m) * m


def _logits(c, g, dev):
    """A trained gate's logits: spread like N(0, 1.5), experts differently popular."""
    l = torch.randn(c["T"], c["E"], generator=g, device=dev) * 1.5
    return l + 0.5 * torch.randn(c["E"], generator=g, device=dev)


def _route_state(c, g, dev):
    T, k = c["T"], c["k"]
    s = {"logits": _logits(c, g, dev), "bias": None, "mask": None}
    if c["bias"]:       # what a balancing rule leaves behind: a few hundredths against the popular experts
        s["bias"] = torch.randn(c["E"], generator=g, device=dev) * 0.05
    if c["pad"]:        # sequences of 128 tokens end early
        at = torch.arange(T, device=dev)
        ends = 128 * (1 - 2 * c["pad"] * torch.rand(-(-T // 128), generator=g, device=dev))
        s["mask"] = ((at % 128) < ends[at // 128]).to(torch.uint8)
    if c.get("train"):
        s["dgate_w"] = torch.randn(T, k, generator=g, device=dev)
        s["dlogits"] = torch.empty(T, c["E"], device=dev)
    s["expert_idx"] = torch.empty(T, k, dtype=torch.int32, device=dev)
    s["gate_w"] = torch.empty(T, k, device=dev)
    return s


def _weights8(c, g, dev, rows, cols):
    """E matrices [rows, cols] ~ N(0, 0.02) in 8 bits as a serving program holds them."""
    E, Kp, Np = c["E"], _up(rows, 128), _up(cols, 128)
    q = torch.empty(E, Np, Kp, dtype=torch.float8_e4m3fn, device=dev)
    e = torch.empty(E, Np // 128, _up(Kp // 128, 4), dtype=torch.uint8, device=dev)
    for i in range(E):
        w = torch.randn(rows, cols, generator=g, device=dev) * 0.02
        q[i], e[i] = _plain_weights(w)
    return q, e


def prepare(case, seed):
    c = case
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    s = {"case": c}
    if c["op"] == "route":
        s.update(_route_state(c, g, dev))
    elif c["op"] in ("rows", "weights"):
        if c["op"] == "rows":
            # activations behind a norm: a few columns much larger than the others
            x = torch.randn(c["rows"], c["K"], generator=g, device=dev)
            x *= torch.exp(torch.randn(c["K"], generator=g, device=dev))
            s["x"] = x.to(_T[c["dtype"]])
            rows, Kp = (c["rows"],), _up(c["K"], 128)
            blocks = rows
        else:
            s["x"] = (torch.randn(c["E"], c["K"], c["N"], generator=g, device=dev) * 0.02).to(_T[c["dtype"]])
            Kp, Np = _up(c["K"], 128), _up(c["N"], 128)
            rows, blocks = (c["E"], Np), (c["E"], Np // 128)
        s["q"] = torch.empty(*rows, Kp, dtype=torch.float8_e4m3fn, device=dev)
        s["e"] = torch.empty(*blocks, _up(Kp // 128, 4), dtype=torch.uint8, device=dev)
    elif c["op"] in ("ffn", "serve"):
        T, k, d, f, E = c["T"], c["k"], c["d"], c["f"], c["E"]
        s["W1"], s["W1e"] = _weights8(c, g, dev, d, f)
        s["W2"], s["W2e"] = _weights8(c, g, dev, f, d)
        x = torch.randn(T * k if c["op"] == "ffn" else T, d, generator=g, device=dev).to(torch.bfloat16)
        if c["op"] == "ffn":
            share = torch.arange(1, E + 1, dtype=torch.float64) ** -c["skew"]
            at = torch.rand(T * k, generator=g, device=dev, dtype=torch.float64).cpu()
            e = torch.bucketize(at, torch.cumsum(share / share.sum(), 0)).clamp_(max=E - 1)
            s["counts"] = torch.bincount(e, minlength=E).tolist()
            start = [0]
            for n in s["counts"]:
                start.append(start[-1] + n)
            s["start"] = torch.tensor(start, dtype=torch.int32, device=dev)
            s["x"], s["xe"] = _plain_rows(x)
            if own:
                from paper_2109_10465_amd import binding as B
                s["shape"] = B.make_fp8_shape(T, d, f, E, k, B.BF16, B.GELU if c["act"] == "gelu" else B.RELU)
                s["h"] = torch.empty(T * k, _up(f, 128), dtype=torch.float8_e4m3fn, device=dev)
                s["he"] = torch.empty(T * k, _up(_up(f, 128) // 128, 4), dtype=torch.uint8, device=dev)
                s["y"] = torch.empty(T * k, d, dtype=torch.bfloat16, device=dev)
        else:
            s["x"] = x
            s.update(_route_state(c, g, dev))
            if own:
                from paper_2109_10465_amd import binding as B
                from paper_2109_10465_amd.layer import Fp8MoELayer
                s["layer"] = Fp8MoELayer(T, d, f, E, k, B.BF16, B.GELU if c["act"] == "gelu" else B.RELU,
                                         (s["W1"], s["W1e"]), (s["W2"], s["W2e"]), score=B.SIGMOID, n_groups=c["groups"],
                                         top_groups=c["top"], group_best=c["best"], renormalise=c["renorm"], scale=c["scale"])
    else:
        r = torch.Generator()
        r.manual_seed(seed)
        s["tensors"] = []
        for name, n in (("f32", c["n32"]), ("bf16", c["n16"])):
            if n:
                s[name] = (torch.randn(n, generator=g, device=dev) * 1e-3).to(_T[name])
                s[name + "_out"] = torch.empty_like(s[name])
                # cut anywhere: a bucket of gradients of parameters of any length, an empty one among them
                cuts = sorted(torch.randint(0, n + 1, (max(0, c["tensors"] // 2 - 1),), generator=r).tolist())
                for a, b in zip([0] + cuts, cuts + [n]):
                    s["tensors"].append((s[name][a:b], s[name + "_out"][a:b]))
        s["max_norm"] = 1e-3 * math.sqrt(c["n32"] + c["n16"]) * c["share"]
        s["norm"] = torch.empty(1, device=dev)
        if own:
            from paper_2109_10465_amd import binding as B
            s["grads"] = B.make_grads(s["tensors"])
            s["ws"] = torch.empty(B.moe_grad_workspace_bytes(s["grads"]), dtype=torch.uint8, device=dev)
    if own and c["op"] == "route":
        from paper_2109_10465_amd import binding as B
        s["router"] = B.make_router(c["T"], c["E"], c["k"], B.SIGMOID if c["score"] == "sigmoid" else B.SOFTMAX, c["groups"],
                                    c["top"], c["best"], c["renorm"], c["scale"])
    return s


# ---- plain forms --------------------------------------------------------------------------------------------------
def _plain_scores(l, score):
    """Scores in 64 bits, where a border between two choices needs them; an expert with a logit of -inf scores 0."""
    l = l.double()
    if score == "sigmoid":
        return 1 / (1 + torch.exp(-l))
    top = l.max(1, keepdim=True).values
    e = torch.exp(l - torch.where(top == -_INF, torch.zeros_like(top), top))
    return e / e.sum(1, keepdim=True).clamp(min=1e-300)


def _plain_route(c, s):
    l, bias, T, E, k = s["logits"], s["bias"], c["T"], c["E"], c["k"]
    p = _plain_scores(l, c["score"])
    dead = ~(l > -_INF)
    sums = p if bias is None else p + bias.double()
    v = l.double() if bias is None else sums
    v, sums = v.masked_fill(dead, -1e300), sums.masked_fill(dead, -_INF)
    if c["groups"] > 1:
        G = c["groups"]
        by = (v if c["best"] == 1 else sums).reshape(T, G, E // G)
        gv = torch.sort(by, dim=2, descending=True).values[:, :, :c["best"]].sum(2)
        chosen = torch.sort(gv, dim=1, descending=True, stable=True).indices[:, :c["top"]]
        keep = torch.zeros(T, G, dtype=torch.bool, device=l.device).scatter_(1, chosen, True)
        v = v.reshape(T, G, E // G).masked_fill(~keep[:, :, None], -_INF).reshape(T, E)
    idx = torch.sort(v, dim=1, descending=True, stable=True).indices[:, :k]
    w = p.gather(1, idx)
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True).clamp(min=1e-300)
    w = w * c["scale"]
    if s["mask"] is not None:
        off = s["mask"][:, None] == 0
        idx, w = idx.masked_fill(off, -1), w.masked_fill(off, 0.0)
    return idx.to(torch.int32), w.float()


def _plain_route_bwd(c, s, idx):
    l = s["logits"]
    live = (idx >= 0).all(1, keepdim=True)
    at = idx.clamp(min=0).long()
    p = _plain_scores(l, c["score"]).float()
    ps, dw = p.gather(1, at), s["dgate_w"] * c["scale"]
    if c["renorm"]:
        S = ps.sum(1, keepdim=True).clamp(min=1e-30)
        ds = (dw - (dw * ps).sum(1, keepdim=True) / S) / S
    else:
        ds = dw
    if c["score"] == "sigmoid":
        other = 1 / (1 + torch.exp(l.gather(1, at)))
        out = torch.zeros_like(l).scatter_(1, at, ds * ps * other)
    else:
        out = -p * (ds * ps).sum(1, keepdim=True)
        out = out.scatter_add_(1, at, ds * ps)
    return out.masked_fill(~live, 0.0)


def _plain_exponent(top):
    """Smallest e with top * 2^-e <= 448 = 0.875 * 2^9; 0 for a block of zeros."""
    m, e = torch.frexp(top)
    return torch.where(top > 0, e - 9 + (m > 0.875).int(), torch.zeros_like(e)).clamp(min=-127)


def _pow2(e):
    """2^e as a product of two powers that fp32 holds."""
    a = torch.div(e, 2, rounding_mode="floor")
    bits = lambda n: ((n + 127) << 23).to(torch.int32).view(torch.float32)
    return bits(a) * bits(e - a)


def _plain_rows(x):
    rows, K = x.shape
    Kp = _up(K, 128)
    b = torch.zeros(rows, Kp, device=x.device)
    b[:, :K] = x.float()
    b = b.reshape(rows, Kp // 128, 128)
    e = _plain_exponent(b.abs().amax(2))
    q = (b * _pow2(-e)[:, :, None]).to(torch.float8_e4m3fn).reshape(rows, Kp)
    out = torch.full((rows, _up(Kp // 128, 4)), 127, dtype=torch.uint8, device=x.device)
    out[:, :Kp // 128] = (e + 127).to(torch.uint8)
    return q, out


def _plain_weights(w):
    K, N = w.shape
    Kp, Np = _up(K, 128), _up(N, 128)
    b = torch.zeros(Np, Kp, device=w.device)
    b[:N, :K] = w.float().t()
    b = b.reshape(Np // 128, 128, Kp // 128, 128)
    e = _plain_exponent(b.abs().amax(dim=(1, 3)))
    q = (b * _pow2(-e)[:, None, :, None]).to(torch.float8_e4m3fn).reshape(Np, Kp)
    out = torch.full((Np // 128, _up(Kp // 128, 4)), 127, dtype=torch.uint8, device=w.device)
    out[:, :Kp // 128] = (e + 127).to(torch.uint8)
    return q, out


def _wide_rows(q, e):
    n = q.shape[1] // 128
    return (q.float().reshape(-1, n, 128) * _pow2(e[:, :n].int() - 127)[:, :, None]).reshape(q.shape)


def _wide_weights(q, e):
    n, m = q.shape[0] // 128, q.shape[1] // 128
    return (q.float().reshape(n, 128, m, 128) * _pow2(e[:, :m].int() - 127)[:, None, :, None]).reshape(q.shape)


def _plain_act(z, act):
    if act == "relu":
        return torch.relu(z)
    return 0.5 * z * torch.erfc(-z * math.sqrt(0.5))


def _plain_block(c, s, x, e):
    """One expert's rows through its two matrices."""
    h = _plain_act(_wide_rows(*x) @ _wide_weights(s["W1"][e], s["W1e"][e]).t(), c["act"])
    return (_wide_rows(*_plain_rows(h)) @ _wide_weights(s["W2"][e], s["W2e"][e]).t())[:, :c["d"]]


def _plain_ffn(c, s):
    y = torch.empty(c["T"] * c["k"], c["d"], dtype=torch.bfloat16, device=s["x"].device)
    a = 0
    for e, n in enumerate(s["counts"]):
        if n:
            y[a:a + n] = _plain_block(c, s, (s["x"][a:a + n], s["xe"][a:a + n]), e).to(torch.bfloat16)
            a += n
    return y


def _plain_serve(c, s):
    idx, w = _plain_route(c, s)
    q, e = _plain_rows(s["x"])
    y = torch.zeros(c["T"], c["d"], device=q.device)
    order = torch.sort(idx.reshape(-1), stable=True).indices
    counts = torch.bincount(idx.reshape(-1).long() + 1, minlength=c["E"] + 1).tolist()
    yd = torch.zeros(c["T"] * c["k"], c["d"], device=q.device)
    a = counts[0]
    for x, n in enumerate(counts[1:]):
        if n:
            at = order[a:a + n]
            t = at // c["k"]
            yd[at] = _plain_block(c, s, (q[t], e[t]), x)
            a += n
    for j in range(c["k"]):
        y += w[:, j:j + 1] * yd.reshape(c["T"], c["k"], -1)[:, j]
    return {"y": y.to(torch.bfloat16), "expert_idx": idx, "gate_w": w}


def _plain_clip(c, s):
    total = torch.zeros((), dtype=torch.float64, device=s["norm"].device)
    for g, _ in s["tensors"]:
        total += g.double().square().sum()
    norm = total.sqrt()
    factor = torch.where(norm > s["max_norm"], s["max_norm"] / norm, torch.ones_like(norm)).float()
    for g, o in s["tensors"]:
        o.copy_(g.float() * factor)
    s["norm"].copy_(norm.reshape(1))
    return {"norm": s["norm"], **{n: s[n + "_out"] for n in ("f32", "bf16") if n in s}}


def run(state):
    s, c = state, state["case"]
    if own:
        from paper_2109_10465_amd import binding as B
    if c["op"] == "route":
        if not own:
            idx, w = _plain_route(c, s)
            out = {"expert_idx": idx, "gate_w": w}
            if c["train"]:
                out["dlogits"] = _plain_route_bwd(c, s, idx)
            return out
        B.moe_router_fwd(s["router"], s["logits"], s["bias"], s["mask"], s["expert_idx"], s["gate_w"])
        out = {"expert_idx": s["expert_idx"], "gate_w": s["gate_w"]}
        if c["train"]:
            B.moe_router_bwd(s["router"], s["logits"], s["expert_idx"], s["dgate_w"], s["dlogits"])
            out["dlogits"] = s["dlogits"]
        return out
    if c["op"] == "rows":
        if not own:
            q, e = _plain_rows(s["x"])
            return {"q": q, "e": e}
        B.moe_quantise_rows_fp8(c["rows"], c["K"], s["x"], s["q"], s["e"])
        return {"q": s["q"], "e": s["e"]}
    if c["op"] == "weights":
        if not own:
            for i in range(c["E"]):
                s["q"][i], s["e"][i] = _plain_weights(s["x"][i])
        else:
            B.moe_quantise_weights_fp8(c["E"], c["K"], c["N"], s["x"], s["q"], s["e"])
        return {"q": s["q"], "e": s["e"]}
    if c["op"] == "ffn":
        if not own:
            return {"y": _plain_ffn(c, s)}
        B.moe_expert_ffn_fwd_fp8(s["shape"], s["x"], s["xe"], s["start"], s["W1"], s["W1e"], s["W2"], s["W2e"], s["h"], s["he"],
                                 s["y"])
        return {"y": s["y"]}
    if c["op"] == "serve":
        if not own:
            return _plain_serve(c, s)
        layer = s["layer"]
        y = layer.forward(s["x"], logits=s["logits"], select_bias=s["bias"], token_mask=s["mask"])
        return {"y": y, "expert_idx": layer.expert_idx, "gate_w": layer.gate_w}
    if not own:
        return _plain_clip(c, s)
    B.moe_clip_grads(s["grads"], s["max_norm"], s["norm"], s["ws"])
    return {"norm": s["norm"], **{n: s[n + "_out"] for n in ("f32", "bf16") if n in s}}


# ---- 64 bits ------------------------------------------------------------------------------------------------------
def _grid8(v):
    """Nearest e4m3 number, ties to even, of values that are at most 448."""
    _, e = torch.frexp(v.abs())
    step = _unit64((e - 4).clamp(min=-9))
    return torch.round(v / step) * step


def _unit64(e):
    """2^e in 64 bits, |e| < 1022."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _held(x):
    """Rows [n, K] in 64 bits as their 8-bit form stands for them: whole blocks of 128, not padded."""
    out = torch.empty_like(x)
    for a in range(0, x.shape[1], 128):
        b = x[:, a:a + 128]
        top = b.abs().amax(1, keepdim=True)
        e = torch.ceil(torch.log2(torch.where(top > 0, top, torch.full_like(top, 448.0)) / 448))
        unit = _unit64(e)
        # log2 may be off next to a power of two
        unit = torch.where(top > 448 * unit, 2 * unit, torch.where(top <= 224 * unit, unit / 2, unit))
        unit = torch.where(top > 0, unit, torch.ones_like(unit))
        out[:, a:a + 128] = _grid8(b / unit) * unit
    return out


def _stands(q, e, rows):
    """64-bit values of 8-bit data [n, K] whose exponents are shared by `rows` rows and 128 columns."""
    v = q.double()
    unit = _unit64(e.int() - 127)
    unit = unit.repeat_interleave(rows, 0).repeat_interleave(128, 1)
    return v * unit[:v.shape[0], :v.shape[1]]


def _exact_route(c, s):
    l, T, E, k, G = s["logits"].double(), c["T"], c["E"], c["k"], c["groups"]
    p = torch.sigmoid(l) if c["score"] == "sigmoid" else torch.softmax(l, 1)
    v = l if s["bias"] is None else p + s["bias"].double()
    left = v.clone()
    if G > 1:
        gv = (v if c["best"] == 1 else p if s["bias"] is None else v).reshape(T, G, -1).topk(c["best"], 2).values.sum(2)
        # the number of groups in front of each one
        ahead = torch.zeros(T, G, dtype=torch.int32, device=l.device)
        for i in range(G):
            o = gv[:, i:i + 1]
            ahead += (o > gv) | ((o == gv) & (torch.arange(G, device=l.device) > i))
        left[(ahead >= c["top"]).repeat_interleave(E // G, 1)] = -_INF
    idx = torch.empty(T, k, dtype=torch.int64, device=l.device)
    for j in range(k):
        top = left.max(1, keepdim=True).values
        idx[:, j:j + 1] = torch.where(left == top, torch.arange(E, device=l.device), E).min(1, keepdim=True).values
        left.scatter_(1, idx[:, j:j + 1], -_INF)
    mine = p.gather(1, idx)
    w = c["scale"] * (mine / mine.sum(1, keepdim=True) if c["renorm"] else mine)
    if s["mask"] is not None:
        idx[s["mask"] == 0] = -1
        w[s["mask"] == 0] = 0
    return idx, w


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "route":
        idx, w = _exact_route(c, s)
        out = {"expert_idx": idx.int(), "gate_w": w}
        if c["train"]:
            l = s["logits"].double().requires_grad_()
            p = torch.sigmoid(l) if c["score"] == "sigmoid" else torch.softmax(l, 1)
            m = p.gather(1, idx.clamp(min=0))
            o = c["scale"] * (m / m.sum(1, keepdim=True) if c["renorm"] else m)
            (o * s["dgate_w"].double() * (idx >= 0)).sum().backward()
            out["dlogits"] = l.grad
        return out
    if c["op"] == "rows":
        x = s["x"].double()
        e = torch.stack([_exact_byte(x[:, a:a + 128].abs().amax(1)) for a in range(0, x.shape[1], 128)], 1)
        q = torch.zeros(s["q"].shape, dtype=torch.float64, device=x.device)
        q[:, :x.shape[1]] = _grid8(x * _unit64(127 - e.int()).repeat_interleave(128, 1)[:, :x.shape[1]])
        full = torch.full(s["e"].shape, 127, dtype=torch.uint8, device=x.device)
        full[:, :e.shape[1]] = e
        return {"q": q, "e": full}
    if c["op"] == "weights":
        full = torch.full(s["e"].shape, 127, dtype=torch.uint8, device=s["x"].device)
        q = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["x"].device)
        for i in range(c["E"]):
            w = s["x"][i].double()
            for a in range(0, c["K"], 128):
                for b in range(0, c["N"], 128):
                    t = w[a:a + 128, b:b + 128]
                    e = _exact_byte(t.abs().max())
                    full[i, b // 128, a // 128] = e
                    q[i, b:b + t.shape[1], a:a + t.shape[0]] = _grid8(t * _unit64(127 - e.int())).t()
        return {"q": q, "e": full}
    if c["op"] in ("ffn", "serve"):
        d, f = c["d"], c["f"]

        def block(x, e):
            z = x @ _stands(s["W1"][e], s["W1e"][e], 128)[:f, :d].t()
            h = torch.relu(z) if c["act"] == "relu" else torch.nn.functional.gelu(z)
            return _held(h) @ _stands(s["W2"][e], s["W2e"][e], 128)[:d, :f].t()

        if c["op"] == "ffn":
            y, a = torch.empty(c["T"] * c["k"], d, dtype=torch.float64, device=s["x"].device), 0
            for e, n in enumerate(s["counts"]):
                for b in range(a, a + n, 8192):
                    o = slice(b, min(b + 8192, a + n))
                    y[o] = block(_stands(s["x"][o], s["xe"][o], 1)[:, :d], e)
                a += n
            return {"y": y}
        idx, w = _exact_route(c, s)
        x = _held(s["x"].double())
        y = torch.zeros(c["T"], d, dtype=torch.float64, device=x.device)
        for e in range(c["E"]):
            t, j = torch.nonzero(idx == e, as_tuple=True)
            if len(t):
                y.index_add_(0, t, w[t, j][:, None] * block(x[t], e))
        return {"y": y, "expert_idx": idx.int(), "gate_w": w}
    norm = math.sqrt(sum(float(s[n].double().square().sum()) for n in ("f32", "bf16") if n in s))
    by = s["max_norm"] / norm if norm > s["max_norm"] else 1.0
    return {"norm": torch.tensor([norm], dtype=torch.float64), **{n: s[n].double() * by for n in ("f32", "bf16") if n in s}}


def _exact_byte(top):
    m, e = torch.frexp(top)
    return (torch.where(top > 0, e - 9 + (m > 0.875).int(), torch.zeros_like(e)).clamp(min=-127) + 127).to(torch.uint8)


# ---- what a pass cannot do without --------------------------------------------------------------------------------
def _touched(c):
    """Expected number of experts that get rows, the choices taken as drawn from the popularity."""
    E, R = c["E"], c["T"] * c["k"]
    share = [(i + 1.0) ** -c.get("skew", 0.0) for i in range(E)]
    return sum(1.0 - (1.0 - v / sum(share)) ** R for v in share)


def work(case):
    c = case
    if c["op"] == "route":
        T, E, k = c["T"], c["E"], c["k"]
        n = 4 * T * E + 8 * T * k + (4 * E if c["bias"] else 0) + (T if c["pad"] else 0)
        if c["train"]:
            n += 4 * T * k + 4 * T * E
        return {"bytes": n, "flops": T * E * (8 if c["train"] else 4)}
    if c["op"] == "rows":
        n = c["rows"] * c["K"]
        return {"bytes": n * (3 if c["dtype"] == "bf16" else 5) + n // 128, "flops": 3 * n}
    if c["op"] == "weights":
        n = c["E"] * c["K"] * c["N"]
        return {"bytes": n * (3 if c["dtype"] == "bf16" else 5), "flops": 3 * n}
    if c["op"] in ("ffn", "serve"):
        R = c["T"] * c["k"] * (1.0 - c.get("pad", 0.0))
        n = 2 * c["d"] * c["f"] * _touched(c)
        n += R * c["d"] * 3 if c["op"] == "ffn" else 4 * c["T"] * c["d"] + 4 * c["T"] * c["E"] + 8 * R
        return {"bytes": n, "flops": 4.0 * R * c["d"] * c["f"]}
    return {"bytes": 8 * c["n32"] + 4 * c["n16"], "flops": 3 * (c["n32"] + c["n16"])}
