"""GeLU's left tail in the 8-bit experts' hidden activation: a block of 128 has an exponent of its own, so that a block of nothing
but small values is held as exactly as any other."""
import math

import pytest
import torch

from paper_2109_10465_amd import binding as B

import wide_ref as R

pytestmark = pytest.mark.gpu

F8, U8 = torch.float8_e4m3fn, torch.uint8
# pre-activations of a block, all e4m3 numbers; the last block's activations are below what fp32 holds
BLOCKS = [(-4.0, -4.5), (-4.5, -5.0), (-5.0, -5.5), (-5.5, -6.0), (-6.0, -7.0, -6.5), (-7.5, -8.0), (-9.0, -10.0), (-11.0, -12.0),
          (-0.0078125, -0.01), (-1.0, 0.5, -4.0), (-2.0, -3.0, 3.0), (-18.0, -20.0)]


@pytest.mark.parametrize("counts,d,f,kind", [((1,), 8, 1536, 3), ((40, 0, 33), 264, 1544, 3), ((900, 700, 800), 256, 1536, 1),
                                             ((2500, 1200, 0, 700), 264, 2056, 0)])
def test_blocks_of_small_values(counts, d, f, kind):
    T, E = sum(counts), len(counts)
    s = B.make_fp8_shape(T, d, f, E, 1, B.BF16, B.GELU)
    assert B.moe_fp8_kernels(s)[0] == kind
    # row r picks row r % 2 of its expert's matrix: the product of one entry, exact
    x, W = torch.zeros(T, d), torch.zeros(E, d, f)
    x[torch.arange(T), torch.arange(T) % 2] = 1.0
    for n in range(f):
        of = BLOCKS[n // 128 % len(BLOCKS)]
        for e in range(E):
            W[e, 0, n], W[e, 1, n] = of[(n + e) % len(of)], of[n // 3 % len(of)]
    xq, xb = R.quantise_rows(x)
    w1q, w1b = R.quantise_weights(W)
    w2q, w2b = R.quantise_weights(torch.ones(E, f, d))
    dev = [t.to(F8).cuda() if t.dtype == torch.float64 else t.cuda() for t in (xq, xb, w1q, w1b, w2q, w2b)]
    start = torch.tensor([sum(counts[:i]) for i in range(E + 1)], dtype=torch.int32, device="cuda")
    hq = torch.empty((T, B.fp8_padded(f)), dtype=U8, device="cuda")
    hb = torch.empty((T, B.fp8_scale_bytes(f)), dtype=U8, device="cuda")
    yd = torch.empty((T, d), dtype=torch.float32, device="cuda")
    print(f"[gpu] tail {counts} d={d} f={f}", flush=True)
    B.moe_expert_ffn_fwd_fp8(s, dev[0], dev[1], start, *dev[2:], hq, hb, yd)
    torch.cuda.synchronize()
    xw, ww = R.wide_rows(xq, xb), R.wide_weights(w1q, w1b)
    z, a = torch.zeros(T, B.fp8_padded(f), dtype=torch.float64), 0
    for e, n in enumerate(counts):
        z[a:a + n, :f] = xw[a:a + n, :2] @ ww[e][:2, :f]
        a += n
    h = 0.5 * z * torch.erfc(-z * math.sqrt(0.5))
    nb = h.shape[1] // 128
    # the activation in fp32: 1.6e-6 of its fit, the roundings of its exponent (z^2 / 2 of them, three, and a few more) and of z
    off = (1.6e-6 + (10 + 1.5 * z ** 2) * 2.0 ** -24) * h.abs()
    got, bytes_ = R.wide_rows(hq.cpu().view(F8), hb.cpu()), hb.cpu()[:, :nb].long()
    top = h.abs().reshape(T, nb, 128).amax(2)
    gone = top < 2.0 ** -130
    assert (bytes_[gone] == 127).all()
    slack = off.reshape(T, nb, 128).amax(2)
    lo, hi = R.exponent(top - slack) + 127, R.exponent(top + slack) + 127
    assert (gone | ((bytes_ >= lo) & (bytes_ <= hi))).all()
    unit = R.unit(bytes_ - 127).repeat_interleave(128, 1)
    _, e = torch.frexp(h / unit)
    half = R.unit((e - 5).clamp(min=-10)) * unit            # of a step of e4m3 at h
    assert ((got - h).abs() <= half + 2 * off)[~gone.repeat_interleave(128, 1)].all()
    assert (got[gone.repeat_interleave(128, 1)] == 0).all()
