"""8-bit operands on the GPU: the format exactly, products within the roundings of their fp32 sums, the block on its own
8-bit hidden activation, and the whole pass."""
import numpy as np
import pytest
import torch

from paper_2109_10465_amd import binding as B
from paper_2109_10465_amd.layer import Fp8MoELayer

import wide_ref as R

pytestmark = pytest.mark.gpu

F8, U8 = torch.float8_e4m3fn, torch.uint8


def same(q, want):
    got = q.cpu().view(F8).double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))


def values(shape, seed, dtype, kind="normal"):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal(shape)
    if kind == "wide":          # every exponent that the type has, zeros, subnormal numbers
        x = np.ldexp(x, rng.integers(-148, 124, shape[:-1] + (1,)))
    elif kind == "spread":      # many exponents in one block
        x = np.ldexp(x, rng.integers(-20, 8, shape))
    elif kind == "edges":       # magnitudes on and beside 448 * 2^n, and halves of e4m3 steps
        x = np.sign(x) * np.exp2(rng.integers(-3, 3, shape)) * rng.choice([448.0, 447.9999, 448.0001, 1.0, 1.0625, 1.1875, 17.0], shape)
    x = x.astype(np.float32)
    if kind != "normal":
        x[..., :3] = 0.0
        x.reshape(-1, shape[-1])[::7] = 0.0
    return torch.from_numpy(x).to(dtype)


@pytest.mark.parametrize("rows,K", [(1, 8), (1, 128), (3, 136), (17, 512), (5, 520), (100, 776), (333, 2048)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["normal", "wide", "spread", "edges"])
def test_rows(rows, K, dtype, kind):
    x = values((rows, K), rows + K, dtype, kind)
    q = torch.full((rows + 1, B.fp8_padded(K)), 0x55, dtype=U8, device="cuda")
    b = torch.full((rows + 1, B.fp8_scale_bytes(K)), 0x55, dtype=U8, device="cuda")
    print(f"[gpu] quantise rows {rows} {K} {dtype} {kind}", flush=True)
    B.moe_quantise_rows_fp8(rows, K, x.cuda(), q, b)
    torch.cuda.synchronize()
    wq, wb = R.quantise_rows(x)
    assert torch.equal(b.cpu()[:rows], wb)
    same(q[:rows], wq)
    assert (q[rows] == 0x55).all() and (b[rows] == 0x55).all()


@pytest.mark.parametrize("E,K,N", [(1, 8, 8), (2, 128, 128), (3, 136, 264), (1, 520, 72), (2, 72, 520), (4, 1024, 256)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["normal", "spread", "edges"])
def test_weights(E, K, N, dtype, kind):
    W = values((E, K, N), K + N, dtype, kind)
    print(f"[gpu] quantise weights {E} {K} {N} {dtype} {kind}", flush=True)
    q, b = Fp8MoELayer.quantise_weights(W.cuda())
    torch.cuda.synchronize()
    wq, wb = R.quantise_weights(W)
    assert torch.equal(b.cpu(), wb)
    same(q, wq)


def test_values_that_are_not_finite():
    x = values((6, 384), 1, torch.float32)
    x[0, 5], x[1, 130], x[2, 300], x[3, 0], x[3, 383] = np.inf, -np.inf, np.nan, np.nan, np.inf
    q = torch.empty(6, 384, dtype=F8, device="cuda")
    b = torch.empty(6, 4, dtype=U8, device="cuda")
    B.moe_quantise_rows_fp8(6, 384, x.cuda(), q, b)
    torch.cuda.synchronize()
    wq, wb = R.quantise_rows(x)
    assert torch.equal(b.cpu(), wb)
    same(q, wq)


def starts(counts):
    return torch.tensor([0] + np.cumsum(counts).tolist(), dtype=torch.int32, device="cuda")


def operands(counts, K, N, seed, rows=None, wstd=0.05):
    """8-bit rows and weights; the rows behind the last expert's hold NaN, as does the data that no row of a product reads."""
    n = sum(counts)
    rows = n if rows is None else rows
    x = values((max(rows, 1), K), seed, torch.float32, "normal")
    xq, xb = R.quantise_rows(x)
    xq[n:] = float("nan")
    wq, wb = R.quantise_weights(values((len(counts), K, N), seed + 1, torch.float32) * wstd)
    return [t.to(F8).cuda() if t.dtype == torch.float64 else t.cuda() for t in (xq, xb, wq, wb)]


def exact_product(xq, xb, wq, wb, counts, N):
    """The product in 64 bits, and how far the matrix instructions' sums may be off: of 8 neighbouring products each but the
    largest loses less than 2^-13 of the largest (bounded by the largest factors), and the K / 8 sums are added in fp32
    (cut off at worst: 2^-23 of the sum of magnitudes each)."""
    x, w = R.wide_rows(xq.cpu(), xb.cpu()), R.wide_weights(wq.cpu(), wb.cpu())
    K = x.shape[1]
    y, off, a = torch.zeros(x.shape[0], N, dtype=torch.float64), torch.zeros(x.shape[0], N, dtype=torch.float64), 0
    for e, n in enumerate(counts):
        if n:
            xe, we = x[a:a + n], w[e][:, :N]
            y[a:a + n] = xe @ we
            off[a:a + n] = 7 * 2.0 ** -13 * (xe.abs().reshape(n, K // 8, 8).amax(2) @ we.abs().reshape(K // 8, 8, N).amax(1))
            off[a:a + n] += K / 8 * 2.0 ** -23 * (xe.abs() @ we.abs())
        a += n
    return y, off


def close(got, want, off):
    """... and the result's own rounding on top."""
    u = 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -24
    assert ((got.cpu().double() - want).abs() <= off + u * (want.abs() + off)).all()


COUNTS = [(1,), (3, 0, 2), (0, 0, 40, 1), (33, 31, 32, 64, 65), (257, 5, 0, 100), (300,), (129,) * 3, (1,) * 70, (0,) * 9 + (7,)]


@pytest.mark.parametrize("counts", COUNTS, ids=lambda c: f"{len(c)}e{sum(c)}")
@pytest.mark.parametrize("K,N", [(8, 8), (128, 128), (136, 264), (512, 72), (1160, 520), (2048, 256)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_product(counts, K, N, dtype):
    rows = sum(counts) + 3
    xq, xb, wq, wb = operands(counts, K, N, K + N, rows)
    y = torch.full((rows, N), -7.0, dtype=dtype, device="cuda")
    print(f"[gpu] product {counts[:6]} K={K} N={N} {dtype}", flush=True)
    B.moe_expert_product_fp8(rows, len(counts), K, N, xq, xb, starts(counts), wq, wb, y)
    torch.cuda.synchronize()
    want, off = exact_product(xq, xb, wq, wb, counts, N)
    n = sum(counts)
    close(y[:n], want[:n], off[:n])
    assert (y[n:] == -7.0).all()


@pytest.mark.parametrize("counts,K,N", [((700, 900, 300), 640, 776), ((4000,), 384, 256), ((40,) * 100, 256, 384), ((8,) * 256, 520, 128),
                                        ((2500, 100, 0, 1), 1024, 1032), ((4000,), 384, 4096), ((2500, 1200, 0, 700), 1160, 2056),
                                        ((257,) * 64, 136, 1048), ((30, 0, 70, 64) * 64, 120, 1032), ((33,) * 200, 384, 1160)])
def test_larger_products(counts, K, N):
    xq, xb, wq, wb = operands(counts, K, N, K + N)
    y = torch.empty((sum(counts), N), dtype=torch.bfloat16, device="cuda")
    print(f"[gpu] product {counts[:6]} K={K} N={N}", flush=True)
    B.moe_expert_product_fp8(sum(counts), len(counts), K, N, xq, xb, starts(counts), wq, wb, y)
    torch.cuda.synchronize()
    want, off = exact_product(xq, xb, wq, wb, counts, N)
    close(y, want, off)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_of_4096_bytes(dtype):
    """Many experts of few rows whose reductions begin at different places; data of any bytes, checked on the GPU."""
    counts, K, N = (5, 0, 33, 64, 1, 2, 70) * 4, 4096, 1032
    E, T, g = len(counts), sum(counts), torch.Generator(device="cuda").manual_seed(3)
    assert B.moe_fp8_kernels(B.make_fp8_shape(T, N, K, E, 1, B.BF16, B.GELU))[1] == 3

    def data(*shape):
        v = torch.randint(0, 255, shape, generator=g, dtype=U8, device="cuda")
        return torch.where((v & 0x7f) == 0x7f, 0, v).to(U8)

    xq, wq = data(T, K), data(E, B.fp8_padded(N), K)
    xb = torch.randint(118, 128, (T, K // 128), generator=g, dtype=U8, device="cuda")
    wb = torch.randint(118, 128, (E, B.fp8_padded(N) // 128, K // 128), generator=g, dtype=U8, device="cuda")
    y = torch.empty((T, N), dtype=dtype, device="cuda")
    B.moe_expert_product_fp8(T, E, K, N, xq, xb, starts(counts), wq, wb, y)
    torch.cuda.synchronize()
    unit, a = lambda b: torch.exp2(b.double() - 127).repeat_interleave(128, -1), 0
    for e, n in enumerate(counts):
        x, w = xq[a:a + n].view(F8).double() * unit(xb[a:a + n]), wq[e].view(F8).double() * unit(wb[e]).repeat_interleave(128, 0)
        w = w[:N].t().contiguous()
        off = 7 * 2.0 ** -13 * (x.abs().reshape(n, K // 8, 8).amax(2) @ w.abs().reshape(K // 8, 8, N).amax(1)) if n else 0
        off = off + K / 8 * 2.0 ** -23 * (x.abs() @ w.abs())
        if n:
            close(y[a:a + n], (x @ w).cpu(), off.cpu())
        a += n


def test_every_kernel_is_reached_above():
    kinds = lambda counts, d, f: B.moe_fp8_kernels(B.make_fp8_shape(sum(counts), d, f, len(counts), 1, B.BF16, B.GELU))
    assert kinds((2500, 1200, 0, 700), 264, 2056)[0] == 0 and kinds((900, 700, 800), 256, 512) == (1, 1)
    # as products: K is the reduction, which is d_ff for the second
    assert kinds((4000,), 4096, 384)[1] == kinds((2500, 1200, 0, 700), 2056, 1160)[1] == 0
    assert kinds((40,) * 100, 256, 384) == kinds((30, 0, 70, 64) * 64, 120, 1032) == kinds((33,) * 200, 384, 1160) == (3, 3)
    assert kinds((1,), 264, 2048)[1] == kinds((3, 0, 2, 3), 264, 1160)[1] == 2


def test_exponents_at_their_ends():
    """Blocks whose exponents are far apart, and far from 0."""
    counts, K, N = (20, 13), 384, 136
    xq, xb, wq, wb = operands(counts, K, N, 3)
    rng = np.random.default_rng(0)
    xb[:, :3] = torch.from_numpy(rng.integers(60, 190, (33, 3)).astype(np.uint8)).cuda()
    wb[:, :, :3] = torch.from_numpy(rng.integers(60, 190, (2, 2, 3)).astype(np.uint8)).cuda()
    y = torch.empty((33, N), dtype=torch.bfloat16, device="cuda")
    B.moe_expert_product_fp8(33, 2, K, N, xq, xb, starts(counts), wq, wb, y)
    torch.cuda.synchronize()
    want, off = exact_product(xq, xb, wq, wb, counts, N)
    close(y, want, off)


def test_a_value_that_is_not_finite_stays_in_its_row():
    counts, K, N = (40, 30), 256, 128
    xq, xb, wq, wb = operands(counts, K, N, 5)
    xq.view(U8)[17, 200] = 0x7f
    y = torch.empty((70, N), dtype=torch.bfloat16, device="cuda")
    B.moe_expert_product_fp8(70, 2, K, N, xq, xb, starts(counts), wq, wb, y)
    torch.cuda.synchronize()
    bad = torch.isnan(y).all(1).cpu()
    assert bad[17] and not torch.isnan(y[torch.arange(70) != 17]).any()


def test_starts_outside_of_the_rows_are_clamped():
    xq, xb, wq, wb = operands((20, 20), 128, 128, 6)
    y = torch.full((40, 128), -7.0, dtype=torch.bfloat16, device="cuda")
    start = torch.tensor([-5, 20, 1000], dtype=torch.int32, device="cuda")
    B.moe_expert_product_fp8(40, 2, 128, 128, xq, xb, start, wq, wb, y)
    torch.cuda.synchronize()
    want, off = exact_product(xq, xb, wq, wb, (20, 20), 128)
    close(y, want, off)


@pytest.mark.parametrize("act", [B.RELU, B.GELU])
@pytest.mark.parametrize("counts,d,f", [((1,), 8, 8), ((5, 0, 40), 136, 264), ((64, 70, 3, 1), 256, 1032), ((300, 20), 392, 640),
                                        ((20,) * 60, 128, 520), ((900, 700, 800), 256, 512), ((2500, 1200, 0, 700), 264, 2056)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_block(act, counts, d, f, dtype):
    T, E = sum(counts), len(counts)
    xq, xb, w1q, w1b = operands(counts, d, f, d + f, wstd=0.5 / d ** 0.5)
    _, _, w2q, w2b = operands(counts, f, d, f, rows=1)
    s = B.make_fp8_shape(T, d, f, E, 1, B.BF16, act)
    hq = torch.full((T, B.fp8_padded(f)), 0x55, dtype=U8, device="cuda")
    hb = torch.full((T, B.fp8_scale_bytes(f)), 0x55, dtype=U8, device="cuda")
    yd = torch.empty((T, d), dtype=dtype, device="cuda")
    print(f"[gpu] block {counts[:6]} d={d} f={f} act={act}", flush=True)
    B.moe_expert_ffn_fwd_fp8(s, xq, xb, starts(counts), w1q, w1b, w2q, w2b, hq, hb, yd)
    torch.cuda.synchronize()
    z, zoff = exact_product(xq, xb, w1q, w1b, counts, f)
    h = torch.zeros(T, B.fp8_padded(f), dtype=torch.float64)
    h[:, :f] = R.act(z, act == B.GELU)
    # of h in fp32: the sum's (|act'| < 1.13) and the activation's own (gelu's fit is 1.1e-6 off at most, computed in fp32)
    off = torch.zeros_like(h)
    off[:, :f] = 1.13 * zoff + 2.0 ** -21 * h[:, :f].abs() + 1.2e-6 * (act == B.GELU)
    nb = f // 128 + (f % 128 > 0)
    top, slack = h.abs().reshape(T, nb, 128).amax(2), off.reshape(T, nb, 128).amax(2)
    lo, hi = R.exponent((top - slack).clamp(min=0)), R.exponent(top + slack)
    e = hb.cpu()[:, :nb].long() - 127
    zero = top <= slack
    assert (zero | ((e >= lo) & (e <= hi))).all() and (hb.cpu()[:, nb:] == 127).all()
    got = R.wide_rows(hq.cpu().view(F8), hb.cpu())
    step = R.unit(e).repeat_interleave(128, 1) * 2.0 ** -10        # half of a subnormal step
    assert ((got - h).abs() <= torch.maximum(2.0 ** -4 * (h.abs() + off), step) + off).all()
    assert (got[:, f:] == 0).all()
    # the second product on the hidden activation as it is
    close(yd, *exact_product(hq.view(F8), hb, w2q, w2b, counts, d))


@pytest.mark.parametrize("counts,d,f", [((1,), 8, 136), ((33, 0, 48, 64), 136, 264), ((1, 2, 3) * 30, 1112, 376), ((40,) * 20, 2048, 520), ((9, 0, 40), 4096, 136)])
def test_hidden_of_few_rows_has_fp32_sums(counts, d, f):
    """Experts of few rows: the hidden activation is the 64-bit one rounded, but for what fp32 sums are off (an addition per
    16 products, those of a block of 128, and the 16 at once; each cut off at worst: 2^-23 of the sum of magnitudes)."""
    T, E = sum(counts), len(counts)
    xq, xb, w1q, w1b = operands(counts, d, f, d + f, wstd=0.5 / d ** 0.5)
    _, _, w2q, w2b = operands(counts, f, d, f, rows=1)
    s = B.make_fp8_shape(T, d, f, E, 1, B.BF16, B.RELU)
    assert B.moe_fp8_kernels(s)[0] == 3
    hq, hb = torch.empty((T, B.fp8_padded(f)), dtype=U8, device="cuda"), torch.empty((T, B.fp8_scale_bytes(f)), dtype=U8, device="cuda")
    yd = torch.empty((T, d), dtype=torch.float32, device="cuda")
    B.moe_expert_ffn_fwd_fp8(s, xq, xb, starts(counts), w1q, w1b, w2q, w2b, hq, hb, yd)
    torch.cuda.synchronize()
    x, w = R.wide_rows(xq.cpu(), xb.cpu()), R.wide_weights(w1q.cpu(), w1b.cpu())
    h, off, a = torch.zeros(T, B.fp8_padded(f), dtype=torch.float64), torch.zeros(T, B.fp8_padded(f), dtype=torch.float64), 0
    for e, n in enumerate(counts):
        h[a:a + n, :f] = torch.relu(x[a:a + n] @ w[e][:, :f])
        off[a:a + n, :f] = (d / 16 + d / 128 + 16) * 2.0 ** -23 * (x[a:a + n].abs() @ w[e][:, :f].abs())
        a += n
    got = R.wide_rows(hq.cpu().view(F8), hb.cpu())
    unit = R.unit(hb.cpu()[:, :h.shape[1] // 128].long() - 127).repeat_interleave(128, 1)
    _, e = torch.frexp(h / unit)
    half = R.unit((e - 5).clamp(min=-10)) * unit        # of a step at h
    assert ((got - h).abs() <= half + off).all()


def test_block_with_infinite_and_nan_rows():
    """relu and gelu keep NaN; other rows do not see it."""
    counts, d, f = (40,), 128, 256
    xq, xb, w1q, w1b = operands(counts, d, f, 9)
    _, _, w2q, w2b = operands(counts, f, d, 10, rows=1)
    xq.view(U8)[3, 7] = 0x7f
    for act in (B.RELU, B.GELU):
        s = B.make_fp8_shape(40, d, f, 1, 1, B.BF16, act)
        hq, hb = torch.empty(40, 256, dtype=U8, device="cuda"), torch.empty(40, 4, dtype=U8, device="cuda")
        yd = torch.empty((40, d), dtype=torch.bfloat16, device="cuda")
        B.moe_expert_ffn_fwd_fp8(s, xq, xb, starts(counts), w1q, w1b, w2q, w2b, hq, hb, yd)
        torch.cuda.synchronize()
        bad = torch.isnan(yd).all(1).cpu()
        assert bad[3] and not torch.isnan(yd[torch.arange(40) != 3]).any()


@pytest.mark.parametrize("T,k,d", [(1, 1, 8), (5, 8, 136), (70, 3, 520), (333, 2, 1024)])
@pytest.mark.parametrize("yd_dtype", [torch.bfloat16, torch.float32])
def test_dispatch_and_combine(T, k, d, yd_dtype):
    dtype = torch.bfloat16
    rng = np.random.default_rng(T)
    x = values((T, d), T + d, dtype)
    row = rng.permutation(T * k).astype(np.int32).reshape(T, k)
    row[rng.random((T, k)) < 0.2] = -1
    row[rng.random((T, k)) < 0.05] = T * k
    s = B.make_fp8_shape(T, d, 128, 4, k, B.BF16, B.RELU)
    q = torch.full((T * k, B.fp8_padded(d)), 0x55, dtype=U8, device="cuda")
    b = torch.full((T * k, B.fp8_scale_bytes(d)), 0x55, dtype=U8, device="cuda")
    rows = torch.from_numpy(row).cuda()
    print(f"[gpu] dispatch T={T} k={k} d={d}", flush=True)
    B.moe_dispatch_fp8(s, x.cuda(), rows, q, b)
    yd = values((T * k, d), 3, yd_dtype)
    ok = (row >= 0) & (row < T * k)
    unused = np.setdiff1d(np.arange(T * k), row[ok])
    yd[unused] = float("nan")
    w = torch.from_numpy(rng.random((T, k)).astype(np.float32))
    y = torch.empty((T, d), dtype=dtype, device="cuda")
    B.moe_combine_rows(s, yd.cuda(), rows, w.cuda(), y)
    torch.cuda.synchronize()
    wq, wb = R.quantise_rows(x)
    for t in range(T):
        want, mag = torch.zeros(d, dtype=torch.float64), torch.zeros(d, dtype=torch.float64)
        for j in range(k):
            if ok[t, j]:
                assert torch.equal(b[row[t, j]].cpu(), wb[t])
                same(q[row[t, j]], wq[t])
                want += float(w[t, j]) * yd[row[t, j]].double()
                mag += float(w[t, j]) * yd[row[t, j]].double().abs()
        tol = k * 2.0 ** -24 * mag + 2.0 ** -8 * want.abs()
        assert ((y[t].cpu().double() - want).abs() <= tol).all()
    assert (q[torch.from_numpy(unused).cuda()] == 0x55).all() and (b[torch.from_numpy(unused).cuda()] == 0x55).all()


def layer_inputs(T, d, f, E, seed, pad=0.2):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, d, generator=g).to(torch.bfloat16)
    W1 = (torch.randn(E, d, f, generator=g) / d ** 0.5).to(torch.bfloat16)
    W2 = (torch.randn(E, f, d, generator=g) / f ** 0.5).to(torch.bfloat16)
    Wg = torch.randn(d, E, generator=g) / d ** 0.5
    bias = torch.randn(E, generator=g) * 0.05
    mask = (torch.rand(T, generator=g) >= pad).to(U8)
    return [t.cuda() for t in (x, W1, W2, Wg, bias, mask)]


@pytest.mark.parametrize("T,d,f,E,k,groups,top,act", [(1, 128, 256, 8, 2, 1, 1, B.GELU), (37, 136, 264, 16, 4, 4, 2, B.RELU),
                                                      (400, 256, 512, 64, 8, 8, 3, B.GELU), (1500, 200, 392, 6, 2, 2, 1, B.GELU)])
def test_whole_pass(T, d, f, E, k, groups, top, act):
    """Router, sort, dispatch, experts and mixture together, twice with different tokens through the same buffers: against
    the layer in 64 bits on the same choices and 8-bit weights and tokens.  The hidden activation is rounded to 8 bits: by
    half a step, 2^-4 of a value or 2^-10 of the block's unit, after the first product's own error, |act'| < 1.13 of it."""
    x, W1, W2, Wg, bias, mask = layer_inputs(T, d, f, E, T)
    w1, w2 = Fp8MoELayer.quantise_weights(W1), Fp8MoELayer.quantise_weights(W2)
    layer = Fp8MoELayer(T, d, f, E, k, B.BF16, act, w1, w2, score=B.SIGMOID, n_groups=groups, top_groups=top, scale=1.5)
    for again in range(2):
        xi = x if again == 0 else torch.flip(x, (0,))
        print(f"[gpu] fp8 layer T={T} d={d} f={f} E={E} k={k}", flush=True)
        y = layer.forward(xi.contiguous(), Wg, select_bias=bias, token_mask=mask)
        torch.cuda.synchronize()
        logits = layer.logits.cpu()
        ref = xi.cpu().double() @ Wg.cpu().double()
        assert (logits - ref).abs().max() <= 1e-5 * ref.abs().max()
        idx, w = R.route(layer.router, logits, bias.cpu(), mask.cpu())
        assert torch.equal(layer.expert_idx.cpu(), idx)
        assert (layer.gate_w.cpu() - w).abs().max() <= 1.5 * 16 * 2.0 ** -24
        xw = R.wide_rows(*R.quantise_rows(xi.cpu()))[:, :d]
        m1, m2 = R.wide_weights(w1[0].cpu(), w1[1].cpu()), R.wide_weights(w2[0].cpu(), w2[1].cpu())
        for t in range(T):
            want, mag = torch.zeros(d, dtype=torch.float64), torch.zeros(d, dtype=torch.float64)
            for j in range(k):
                e = int(idx[t, j])
                if e >= 0:
                    z = xw[t] @ m1[e][:d, :f]
                    h, o = R.act(z, act == B.GELU), m2[e][:f, :d]
                    want += float(w[t, j]) * (h @ o)
                    zoff = 7 * 2.0 ** -13 * (xw[t].abs().reshape(-1, 8).amax(1) @ m1[e][:d, :f].abs().reshape(d // 8, 8, f).amax(1))
                    hoff = 1.13 * zoff + 2.0 ** -20 * z.abs() + 1.2e-6
                    # a block's unit is at most 2 / 448 of its largest value; the whole row's largest bounds it
                    hoff = hoff + torch.maximum(2.0 ** -4 * (h.abs() + hoff), 2.0 ** -9 / 448 * (h.abs() + hoff).max())
                    ho = (h.abs() + hoff).reshape(-1, 8).amax(1) @ o.abs().reshape(f // 8, 8, d).amax(1)
                    mag += float(w[t, j]) * (hoff @ o.abs() + 8 * 2.0 ** -13 * ho)
            tol = mag + 2.0 ** -8 * (want.abs() + mag)
            assert ((y[t].cpu().double() - want).abs() <= tol).all(), t
            if not mask[t]:
                assert not y[t].any()
        counts = torch.bincount(idx.reshape(-1)[idx.reshape(-1) >= 0].long(), minlength=E)
        before = bias.cpu().clone()
        mean = int(counts.sum())
        layer.update_select_bias(bias, 0.01)
        step = torch.where(counts * E < mean, 0.01, torch.where(counts * E > mean, -0.01, 0.0))
        assert torch.allclose(bias.cpu(), before + step, atol=1e-7)


def test_pass_captured_and_replayed():
    T, d, f, E, k = 130, 128, 256, 16, 4
    x, W1, W2, Wg, bias, mask = layer_inputs(T, d, f, E, 3)
    layer = Fp8MoELayer(T, d, f, E, k, B.BF16, B.GELU, Fp8MoELayer.quantise_weights(W1), Fp8MoELayer.quantise_weights(W2),
                        score=B.SIGMOID, n_groups=4, top_groups=2, group_best=2)
    run = lambda: layer.forward(x, Wg, select_bias=bias, token_mask=mask)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for seed in range(3):
        x.copy_(layer_inputs(T, d, f, E, 10 + seed)[0])
        run()
        torch.cuda.synchronize()
        want = [t.clone() for t in (layer.y, layer.expert_idx, layer.row_of)]
        layer.y.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((layer.y, layer.expert_idx, layer.row_of), want))


def test_layer_refuses_weights_of_another_layout():
    q, b = Fp8MoELayer.quantise_weights(torch.randn(4, 128, 256).cuda())
    with pytest.raises(B.MoeError):
        Fp8MoELayer(8, 128, 256, 4, 2, B.BF16, B.GELU, (q, b), (q, b))
    q2, b2 = Fp8MoELayer.quantise_weights(torch.randn(4, 256, 128).cuda())
    layer = Fp8MoELayer(8, 128, 256, 4, 2, B.BF16, B.GELU, (q, b), (q2, b2))
    x = torch.zeros(8, 128, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(B.MoeError):
        layer.forward(x)
    l, bias, mask = torch.zeros(8, 4, device="cuda"), torch.zeros(4, device="cuda"), torch.ones(8, dtype=torch.uint8, device="cuda")
    layer.forward(x, logits=l, select_bias=bias, token_mask=mask.bool())
    for bad in (dict(x=x[:7]), dict(x=x.float()), dict(x=x.cpu()), dict(x=x.t().contiguous().t()), dict(logits=l.double()),
                dict(logits=l[:, :3]), dict(select_bias=bias[:3]), dict(token_mask=mask.int())):
        with pytest.raises(B.MoeError):
            layer.forward(**{**dict(x=x, logits=l, select_bias=bias, token_mask=mask), **bad})
    with pytest.raises(B.MoeError):
        Fp8MoELayer(8, 128, 256, 4, 2, B.BF16, B.GELU, (q.cpu(), b), (q2, b2))
    with pytest.raises(B.MoeError):
        Fp8MoELayer.quantise_weights(torch.randn(4, 256, 128))


def test_mixture_of_more_tokens_than_a_grid_has():
    T = (1 << 25) + 5
    s = B.make_fp8_shape(T, 8, 8, 4, 1, B.BF16, B.RELU)
    g = torch.Generator(device="cuda").manual_seed(2)
    yd, w = torch.randn((T, 8), generator=g, device="cuda"), torch.rand((T, 1), generator=g, device="cuda")
    row_of = torch.arange(T - 1, -1, -1, dtype=torch.int32, device="cuda")
    y = torch.empty((T, 8), dtype=torch.bfloat16, device="cuda")
    B.moe_combine_rows(s, yd, row_of, w, y)
    torch.cuda.synchronize()
    assert torch.equal(y, (yd.flip(0) * w).bfloat16())      # one product, one rounding of it
