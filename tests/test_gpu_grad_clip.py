"""Global norm and clipping of gradients against 64 bits."""
import numpy as np
import pytest
import torch

from paper_2109_10465_amd import binding as B
from paper_2109_10465_amd import inputs as I
from paper_2109_10465_amd.layer import MoELayer

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def clip(pairs, max_norm):
    g = B.make_grads(pairs)
    norm = torch.full((1,), -7.0, device="cuda")
    ws = torch.full((B.moe_grad_workspace_bytes(g),), 0xff, dtype=torch.uint8, device="cuda")
    B.moe_clip_grads(g, max_norm, norm, ws)
    torch.cuda.synchronize()
    return float(norm)


def check(tensors, max_norm, place=False):
    """tensors: inputs (views of any alignment); outputs lie in buffers of their own with guards around them."""
    want_norm = float(torch.stack([t.double().square().sum().cpu() for t in tensors] + [torch.zeros((), dtype=torch.float64)]).sum().sqrt())
    src = [t.clone() for t in tensors]
    if place:
        pairs = [(t, t) for t in tensors]
    else:
        guard = [torch.full((t.numel() + 16,), 3.0, dtype=t.dtype, device="cuda") for t in tensors]
        pairs = [(t, g[(i * 5) % 9:][:t.numel()]) for i, (t, g) in enumerate(zip(tensors, guard))]
    norm = clip(pairs, max_norm)
    # one rounding of the root's result
    assert abs(norm - want_norm) <= 2.0 ** -23 * want_norm
    f = max_norm / want_norm if want_norm > max_norm else 1.0
    for s, (_, o) in zip(src, pairs):
        got, want = o.double().cpu(), s.double().cpu() * f
        # the norm's rounding, the factor's, the product's; then the type's
        tol = 4 * 2.0 ** -24 + (2.0 ** -8 if s.dtype == BF16 else 0.0)
        assert ((got - want).abs() <= tol * want.abs() + 1e-45).all()
        if f == 1.0:
            assert torch.equal(o, s)
    if not place:
        for i, (t, g) in enumerate(zip(src, guard)):
            a = (i * 5) % 9
            assert (g[:a] == 3.0).all() and (g[a + t.numel():] == 3.0).all()
            assert torch.equal(tensors[i], t)


def make(sizes, seed, std=1e-2, offset=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        dt = BF16 if i % 3 == 1 else F32
        base = (torch.randn(n + 16, generator=gen, device="cuda") * std).to(dt)
        out.append(base[(i * 3 + offset) % 9:][:n])
    return out


@pytest.mark.parametrize("sizes", [(1,), (0,), (3, 0, 5), (7, 8, 9, 15, 16, 17), (255, 256, 257, 1000), (16383, 16384, 16385),
                                   (100001, 250007, 99999), (5_000_000, 3_000_003)], ids=lambda s: f"{len(s)}x{s[-1]}")
@pytest.mark.parametrize("share", [0.3, 2.0])
@pytest.mark.parametrize("place", [False, True])
def test_sizes(sizes, share, place):
    print(f"[gpu] clip {sizes} {share} {place}", flush=True)
    check(make(sizes, 1), 1e-2 * max(1, sum(sizes)) ** 0.5 * share, place)


@pytest.mark.parametrize("count", [0, 1, 95, 96, 97, 193, 400])
def test_many_tensors(count):
    rng = np.random.default_rng(count)
    sizes = [int(v) for v in rng.integers(0, 3000, count)]
    check(make(sizes, 2, offset=1), 0.5)


@pytest.mark.parametrize("std", [1e-30, 1e25])
def test_squares_beyond_fp32(std):
    check(make((1000, 1001, 5000), 3, std=std), std * 10)


def test_norm_alone_and_zero_limit():
    t = make((5000, 777, 123457), 4)
    g = B.make_grads([(x, None) for x in t])
    norm, ws = torch.empty(1, device="cuda"), torch.empty(B.moe_grad_workspace_bytes(g), dtype=torch.uint8, device="cuda")
    B.moe_grad_norm(g, norm, ws)
    want = float(sum(x.double().square().sum() for x in t).sqrt())
    assert abs(float(norm) - want) <= 2.0 ** -23 * want
    outs = [torch.ones_like(x) for x in t]
    clip(list(zip(t, outs)), 0.0)
    assert not any(o.any() for o in outs)
    zeros = [torch.zeros(100, device="cuda")]
    assert clip([(zeros[0], zeros[0])], 0.0) == 0.0 and not zeros[0].any()


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_a_norm_that_is_not_finite_leaves_the_gradients(bad):
    t = make((5000, 777), 5)
    t[1][3] = bad
    src = [x.clone() for x in t]
    outs = [torch.zeros_like(x) for x in t]
    norm = clip(list(zip(t, outs)), 1e-3)
    assert not np.isfinite(norm)
    for o, s in zip(outs, src):
        assert torch.equal(torch.nan_to_num(o), torch.nan_to_num(s)) and torch.equal(torch.isnan(o), torch.isnan(s))


def test_tensors_of_several_launches():
    check(make([16384 + i for i in range(330)], 4), 0.3, True)      # more sums than a clipping launch adds up itself


def test_same_result_every_time_and_captured():
    t = make((3_000_001, 70_001, 55), 6)
    outs = [torch.empty_like(x) for x in t]
    g = B.make_grads(list(zip(t, outs)))
    norm, ws = torch.empty(1, device="cuda"), torch.empty(B.moe_grad_workspace_bytes(g), dtype=torch.uint8, device="cuda")
    run = lambda: B.moe_clip_grads(g, 0.4, norm, ws)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for seed in range(3):
        for x in t:
            x.copy_(torch.randn(x.shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * 0.01)
        run()
        torch.cuda.synchronize()
        want = [x.clone() for x in (norm, *outs)]
        for x in (norm, *outs):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((norm, *outs), want))


def test_a_layers_gradients_with_others():
    w = I.small("clip", 200, 64, 136, 4, 2, 60, I.BF16, I.GELU)
    d = I.make_inputs(w, seed=1)
    layer = MoELayer(w.T, w.d_model, w.d_ff, w.E, w.k, w.capacity, w.dtype, w.act)
    up = lambda a, dt=BF16: torch.from_numpy(np.ascontiguousarray(a)).cuda().to(dt)
    layer.step(up(d["x"]), up(d["Wg"], F32), None, up(d["W1"]), up(d["W2"]), up(d["rts_keys"], F32), up(d["dy"]))
    other = torch.randn(1001, device="cuda").to(BF16)
    grads = [layer.dWg, layer.dW1, layer.dW2, other]
    src = [g.clone() for g in grads]
    want = float(sum(g.double().square().sum() for g in src).sqrt())
    norm = layer.clip_gradients(0.25 * want, [other])
    assert abs(float(norm) - want) <= 2.0 ** -23 * want
    for g, s in zip(grads, src):
        tol = 2.0 ** -8 + 2.0 ** -21 if g.dtype == BF16 else 2.0 ** -21
        assert ((g.double() - 0.25 * s.double()).abs() <= tol * 0.25 * s.double().abs()).all()
    # a captured call keeps what it works with: later calls have other norms, and more tensors
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = layer.clip_gradients(0.25 * want, [other])
    big = [torch.full((300_000,), 1e-3, device="cuda") for _ in range(40)]
    for again in range(3):
        later = layer.clip_gradients(1e9, (b for b in big))
        for g, s in zip(grads, src):
            g.copy_(s)
        graph.replay()
        torch.cuda.synchronize()
        assert float(captured) == float(norm) and float(later) != float(norm)
        assert (grads[1].double() - 0.25 * src[1].double()).abs().max() <= 2.0 ** -7 * src[1].double().abs().max()
    with pytest.raises(B.MoeError):
        layer.clip_gradients(1.0, [torch.zeros(4)])
