"""The wide gate on the GPU against its definition in 64 bits: choices exactly, weights and gradients within the roundings
of their fp32 formulas; the sort of the choices and the bias update exactly."""
import numpy as np
import pytest
import torch

from paper_2109_10465_amd import binding as B

import wide_ref as R

pytestmark = pytest.mark.gpu


def inputs(r, seed, bias, kind="normal", pad=0.0):
    rng = np.random.default_rng(seed)
    l = rng.standard_normal((r.T, r.E)).astype(np.float32) * np.float32(1.5)
    if kind == "ties":
        l = np.round(l)
    elif kind == "huge":
        l *= np.float32(300.0)
    elif kind == "low":          # all scores far below what fp32 holds of a logistic function
        l -= np.float32(120.0)
    elif kind == "masked":       # experts that are switched off, by -inf and by the type's lowest value; whole rows of either
        l[rng.random(l.shape) < 0.5] = -np.inf
        l[rng.random(l.shape) < 0.1] = np.finfo(np.float32).min
        l[::5] = -np.inf
        l[3::7] = np.finfo(np.float32).min
    b = rng.standard_normal(r.E).astype(np.float32) * np.float32(0.05) if bias else None
    if bias and kind == "ties":
        b[:] = np.round(b * 20) / 20
    m = (rng.random(r.T) >= pad).astype(np.uint8) if pad else None
    return [None if a is None else torch.from_numpy(a) for a in (l, b, m)]


def cuda(t):
    return None if t is None else t.cuda()


def forward(r, l, b, m):
    idx = torch.full((r.T, r.k), -7, dtype=torch.int32, device="cuda")
    w = torch.full((r.T, r.k), -7.0, device="cuda")
    B.moe_router_fwd(r, cuda(l), cuda(b), cuda(m), idx, w)
    torch.cuda.synchronize()
    return idx, w


def check(r, seed, bias, kind="normal", pad=0.0):
    l, b, m = inputs(r, seed, bias, kind, pad)
    print(f"[gpu] router T={r.T} E={r.E} k={r.k} score={r.score} groups={r.n_groups}/{r.top_groups}/{r.group_best} "
          f"renorm={r.renormalise} bias={bias} {kind}", flush=True)
    idx, w = forward(r, l, b, m)
    ref_idx, ref_w = R.route(r, l, b, m)
    assert torch.equal(idx.cpu(), ref_idx)
    # a weight: an exponential's argument off by |l - most| 2^-24 (at most 0.37 2^-24 of the largest weight after the
    # exponential), exponential, sum of 8, division, scale: below 16 roundings of 2^-24 of the largest weight, which is
    # at most scale
    assert (w.cpu().double() - ref_w).abs().max() <= abs(r.scale) * 16 * 2.0 ** -24
    dw = torch.from_numpy(np.random.default_rng(seed + 1).standard_normal((r.T, r.k)).astype(np.float32))
    dl = torch.full((r.T, r.E), -7.0, device="cuda")
    B.moe_router_bwd(r, cuda(l), idx, cuda(dw), dl)
    torch.cuda.synchronize()
    ref = R.route_grad(r, l, ref_idx, dw)
    # q = c r (dw - mean): r within 16 roundings, the mean of at most 8 terms within 16 + 8, difference and products 4:
    # below 64 roundings of 2^-24 of scale * 2 max |dw|; a softmax's dense part adds as much once more
    assert (dl.cpu().double() - ref).abs().max() <= abs(r.scale) * 2 * float(dw.abs().max()) * 128 * 2.0 ** -24
    if m is not None:
        assert not dl.cpu()[m == 0].any()


SIZES = [(1, 8, 1, 1, 1, 1), (1, 256, 8, 8, 4, 2), (3, 1, 1, 1, 1, 1), (7, 2, 2, 1, 1, 1), (65, 5, 3, 1, 1, 1), (33, 60, 2, 1, 1, 1),
         (130, 8, 8, 4, 4, 2), (50, 128, 6, 8, 3, 2), (40, 96, 8, 16, 5, 1), (17, 255, 8, 5, 2, 2), (21, 119, 7, 17, 9, 2),
         (19, 192, 4, 64, 40, 2), (23, 64, 5, 64, 33, 1), (29, 252, 8, 36, 7, 2), (31, 256, 8, 1, 1, 1), (12, 250, 3, 10, 1, 1),
         (9, 256, 8, 2, 1, 2)]


@pytest.mark.parametrize("score", [B.SOFTMAX, B.SIGMOID])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_sizes(size, score):
    T, E, k, groups, top, best = size
    for i, (bias, renorm, scale) in enumerate(((False, True, 1.0), (True, True, 2.5), (True, False, 1.0), (False, False, -0.5))):
        check(B.make_router(T, E, k, score, groups, top, best, renorm, scale), i, bias)


@pytest.mark.parametrize("kind", ["ties", "huge", "low", "masked"])
@pytest.mark.parametrize("score", [B.SOFTMAX, B.SIGMOID])
@pytest.mark.parametrize("bias", [False, True])
def test_values(kind, score, bias):
    for groups, top, best in ((1, 1, 1), (8, 3, 1), (8, 3, 2), (7, 2, 2)):
        E = 56 if groups == 7 else 64
        for renorm in (True, False):
            check(B.make_router(60, E, 6, score, groups, top, best, renorm, 1.0), 3, bias, kind, pad=0.2)


def test_inputs_that_start_anywhere():
    r = B.make_router(33, 64, 6, B.SIGMOID, 8, 3, 2)
    l, b, m = inputs(r, 4, True, pad=0.3)
    want = forward(r, l, b, m)
    off = lambda t, n: torch.cat([torch.zeros(n, dtype=t.dtype), t.reshape(-1)]).cuda()[n:].reshape(t.shape)
    for i, j in ((1, 0), (0, 3), (2, 2)):
        got = forward(r, off(l, i), off(b, j), off(m, 1))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_near_ties_are_decided_in_64_bits():
    """Two experts whose score + bias differ by less than fp32 can tell, in every order."""
    T, E = 256, 32
    rng = np.random.default_rng(5)
    l = torch.from_numpy(rng.standard_normal((T, E)).astype(np.float32))
    r = B.make_router(T, E, 2, B.SIGMOID)
    b = torch.zeros(E)
    for t in range(T):          # expert 7's logit one step of fp32 beside expert 3's, both in front
        l[t, 3] = 4.0 + t / 64
        l[t, 7] = torch.nextafter(l[t, 3], torch.tensor(9.0 if t % 3 else 0.0))
        if t % 5 == 0:
            l[t, 7] = l[t, 3]
    for bias in (b, b + 0.25):
        idx, _ = forward(r, l, bias, None)
        ref, _ = R.route(r, l, bias, None)
        assert torch.equal(idx.cpu(), ref)


@pytest.mark.parametrize("E,k,score", [(16, 1, B.SOFTMAX), (24, 3, B.SIGMOID), (64, 8, B.SOFTMAX), (136, 2, B.SIGMOID), (256, 8, B.SIGMOID)])
def test_near_ties_of_equal_places(E, k, score):
    """The same entry of two lanes' eights, a step of fp32 apart or equal: once at every rank, the last and the one behind it too."""
    T, rng = 512, np.random.default_rng(E)
    l = rng.standard_normal((T, E)).astype(np.float32)
    for t in range(T):
        rank = t % (k + 1)
        e = int(np.argsort(-l[t])[rank])
        o = (e + 8 * int(rng.integers(1, E // 8))) % (E // 8 * 8)
        l[t, o] = (l[t, e], np.nextafter(l[t, e], np.float32(9)), np.nextafter(l[t, e], np.float32(-9)))[t // (k + 1) % 3]
    l = torch.from_numpy(l)
    b = torch.zeros(E)
    mask = torch.from_numpy((rng.random(T) < 0.9).astype(np.uint8))
    for bias in (None, b):
        for m in (None, mask):
            r = B.make_router(T, E, k, score)
            got, ref = forward(r, l, bias, m)[0].cpu(), R.route(r, l, bias, m)[0]
            assert torch.equal(got, ref), (got != ref).any(1).nonzero()[:5].tolist()


@pytest.mark.parametrize("how", ["shifted", "cancelled"])
def test_groups_that_differ_by_little(how):
    """Sums of a group's best two that differ by less than keys of 32 bits can tell: logits far from 0 whose softmax does not
    mind, and biases that take the scores away."""
    T, E, G = 512, 64, 4
    rng = np.random.default_rng(11)
    l = rng.standard_normal((T, E)).astype(np.float32)
    l[:, ::16] += np.float32(4.0)               # a group's best
    b = None
    if how == "shifted":
        l += np.float32(200.0)
        for t in range(T):                      # groups that are another one's copy but for a few steps of fp32
            l[t, 48:] = np.roll(l[t, 32:48], 5)
            l[t, 16:32] = np.roll(l[t, :16], 3)
            for e in (19, 53):
                for _ in range(1 + t % 5):
                    l[t, e] = np.nextafter(l[t, e], np.float32(300 if t % 2 else 0))
    else:
        b = np.zeros(E, dtype=np.float32)
        b[::16] = 5.0
        b[1::16] = np.float32([-5.9, -5.90001, -5.900004, -5.9])
        b[2:16] = b[18:32] = b[34:48] = b[50:] = -20.0
        l[:, 1:16] = l[:, 1:2]
        for q in range(1, 4):
            l[:, 16 * q:16 * q + 16] = l[:, :16]
        l[:, 16] += (rng.standard_normal(T) * 1e-4).astype(np.float32)
        for q in range(4):
            l[:, 16 * q:16 * q + 16] = np.roll(l[:, 16 * q:16 * q + 16], 2 * q + 1, 1)
            b[16 * q:16 * q + 16] = np.roll(b[16 * q:16 * q + 16], 2 * q + 1)
    l, b = torch.from_numpy(l), None if b is None else torch.from_numpy(b)
    for top in (1, 3):
        r = B.make_router(T, E, 2, B.SOFTMAX if b is None else B.SIGMOID, G, top, 2)
        got, ref = forward(r, l, b, None)[0].cpu(), R.route(r, l, b, None)[0]
        assert torch.equal(got, ref), (got != ref).any(1).sum().item()


def test_gradient_against_differences():
    r = B.make_router(16, 24, 3, B.SIGMOID, 4, 2, 2, True, 1.5)
    l, b, _ = inputs(r, 11, True)
    idx, w = forward(r, l, b, None)
    dw = torch.randn(r.T, r.k, generator=torch.Generator().manual_seed(1))
    dl = torch.empty(r.T, r.E, device="cuda")
    B.moe_router_bwd(r, cuda(l), idx, cuda(dw), dl)
    h = 2.0 ** -6
    for e in range(r.E):
        out = []
        for s in (h, -h):
            x = l.double()
            x[:, e] += s
            p = torch.sigmoid(x).gather(1, idx.cpu().long())
            out.append((r.scale * p / p.sum(1, keepdim=True) * dw).sum(1))
        num = (out[0] - out[1]) / (2 * h)
        # third derivative of a ratio of logistic functions below 2: h^2 / 6 * 2 per choice
        assert (num - dl.cpu().double()[:, e]).abs().max() <= h * h / 3 * r.scale * float(dw.abs().sum(1).max()) + 1e-5


def test_non_finite_logits_give_indices_in_range():
    for groups, top, best, bias in ((1, 1, 1, False), (8, 2, 2, True), (8, 2, 1, False), (1, 1, 1, True)):
        r = B.make_router(64, 64, 8, B.SOFTMAX if groups == 1 else B.SIGMOID, groups, top, best)
        l, b, _ = inputs(r, 2, bias)
        rng = np.random.default_rng(3)
        for v in (np.nan, np.inf, -np.inf):
            l[torch.from_numpy(rng.random((64, 64)) < 0.3)] = v
        l[:8] = np.nan
        l[8:16] = np.inf
        idx, _ = forward(r, l, b, None)
        i = idx.cpu()
        assert ((i >= 0) & (i < 64)).all()
        assert all(len(set(row.tolist())) == 8 for row in i)


@pytest.mark.parametrize("T,k,E", [(1, 1, 1), (1, 8, 256), (5, 3, 7), (64, 2, 4), (1023, 1, 256), (1025, 1, 3), (1024, 8, 256), (1025, 8, 256), (700, 4, 90), (4000, 8, 60),
                                   (9001, 7, 200), (70000, 2, 256)])
@pytest.mark.parametrize("kind", ["even", "one", "some"])
def test_sort(T, k, E, kind):
    rng = np.random.default_rng(T + k)
    idx = rng.integers(0, E, (T, k)).astype(np.int32)
    if kind == "one":
        idx[:] = E - 1
    elif kind == "some":        # padding, and choices of nobody
        idx[rng.random((T, k)) < 0.3] = -1
        idx[rng.random((T, k)) < 0.01] = E
    r = B.make_router(T, E, k)
    row = torch.full((T, k), -7, dtype=torch.int32, device="cuda")
    start = torch.full((E + 2,), -7, dtype=torch.int32, device="cuda")
    ws = torch.full((B.moe_sort_workspace_bytes(r),), 0x55, dtype=torch.uint8, device="cuda")
    print(f"[gpu] sort T={T} k={k} E={E} {kind}", flush=True)
    B.moe_sort_choices(r, torch.from_numpy(idx).cuda(), row, start, ws)
    torch.cuda.synchronize()
    flat = idx.reshape(-1)
    ok = (flat >= 0) & (flat < E)
    want = np.full(T * k, -1, np.int32)
    want[np.nonzero(ok)[0][np.argsort(flat[ok], kind="stable")]] = np.arange(ok.sum(), dtype=np.int32)
    counts = np.bincount(flat[ok], minlength=E)
    assert np.array_equal(row.cpu().numpy().reshape(-1), want)
    assert start.cpu().tolist() == [0] + np.cumsum(counts).tolist() + [-7]


def test_bias_update():
    for counts in ([3, 5, 4, 4], [0, 0, 9], [7], [1 << 20, (1 << 20) + 1]):
        E = len(counts)
        r = B.make_router(max(1, sum(counts)), E, 1)
        start = torch.tensor([0] + np.cumsum(counts).tolist(), dtype=torch.int32, device="cuda")
        bias = torch.linspace(-1, 1, E).cuda()
        want = bias.cpu().clone()
        for e, n in enumerate(counts):
            if n * E != sum(counts):
                want[e] += 0.125 if n * E < sum(counts) else -0.125
        B.moe_router_bias_update(r, start, 0.125, bias)
        assert torch.equal(bias.cpu(), want)


def test_more_tokens_than_a_launch_has():
    T = (1 << 25) + 5
    r = B.make_router(T, 8, 1, B.SOFTMAX, renormalise=False)
    l = torch.randn((T, 8), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    mask = torch.ones(T, dtype=torch.uint8, device="cuda")
    mask[T - 2] = mask[7] = 0
    idx, w = torch.empty((T, 1), dtype=torch.int32, device="cuda"), torch.empty((T, 1), device="cuda")
    B.moe_router_fwd(r, l, None, mask, idx, w)
    dw, dl = torch.ones((T, 1), device="cuda"), torch.empty_like(l)
    B.moe_router_bwd(r, l, idx, dw, dl)
    torch.cuda.synchronize()
    on = mask != 0
    assert (idx[~on] == -1).all() and (w[~on] == 0).all() and (dl[~on] == 0).all()
    assert torch.equal(l.gather(1, idx.long().clamp(min=0))[on, 0], l.amax(1)[on])
    for at in (slice(0, 7), slice((1 << 25) - 4, (1 << 25) + 3)):
        s = torch.softmax(l[at].double(), 1)
        best, e = s.max(1, keepdim=True)
        want = -best * s
        want.scatter_add_(1, e, best)
        # (scores of at most 1 from exponentials within 2^-20)
        assert (w[at].double() - best).abs().max() <= 2.0 ** -18 and (dl[at].double() - want).abs().max() <= 2.0 ** -18


def test_captured_and_replayed_on_another_stream():
    r = B.make_router(300, 96, 4, B.SIGMOID, 8, 3, 2, True, 2.0)
    l, b, m = inputs(r, 8, True, pad=0.1)
    l, b, m = cuda(l), cuda(b), cuda(m)
    dw = torch.randn(r.T, r.k, device="cuda")
    buf = lambda *s, dt=torch.int32: torch.zeros(*s, dtype=dt, device="cuda")
    idx, w, dl = buf(r.T, r.k), buf(r.T, r.k, dt=torch.float32), buf(r.T, r.E, dt=torch.float32)
    row, start = buf(r.T, r.k), buf(r.E + 1)
    ws = buf(B.moe_sort_workspace_bytes(r), dt=torch.uint8)

    def run():
        B.moe_router_fwd(r, l, b, m, idx, w)
        B.moe_sort_choices(r, idx, row, start, ws)
        B.moe_router_bwd(r, l, idx, dw, dl)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for seed in range(3):
        l.copy_(inputs(r, 20 + seed, True)[0])
        run()
        torch.cuda.synchronize()
        want = [t.clone() for t in (idx, w, dl, row, start)]
        for t in (idx, w, dl, row, start):
            t.fill_(-3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip((idx, w, dl, row, start), want))
