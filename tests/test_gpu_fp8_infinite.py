"""Hidden activations that are not finite, on every kernel of the experts' first product: such an entry becomes NaN, the finite
ones of its block are rounded with an exponent of 120, and no other row sees any of it."""
import pytest
import torch

from paper_2109_10465_amd import binding as B

import wide_ref as R

pytestmark = pytest.mark.gpu

F8, U8 = torch.float8_e4m3fn, torch.uint8


@pytest.mark.parametrize("act", [B.RELU, B.GELU])
@pytest.mark.parametrize("counts,d,f,kind", [((7, 0, 40), 136, 520, 3), ((900, 700, 800), 256, 512, 1), ((2500, 1200, 0, 700), 264, 2056, 0)])
def test_infinite_hidden_values(act, counts, d, f, kind):
    T, E = sum(counts), len(counts)
    s = B.make_fp8_shape(T, d, f, E, 1, B.BF16, act)
    assert B.moe_fp8_kernels(s)[0] == kind
    # one entry of every row is 1, of the rows `odd` 2^120: products of 3584 2^120 are infinite.  Blocks of columns in turn: with
    # infinite ones and finite ones, with such below zero, without any
    x, W = torch.zeros(T, d), torch.zeros(E, d, f)
    x[:, 3] = 1.0
    n = torch.arange(f)
    W[:, 3] = torch.where(n % 2 == 0, 0.125 * (1 + n % 7), 0.5)
    big = (n // 128 % 3 < 2) & (n % 5 == 0)
    W[:, 3, big] = torch.where(n // 128 % 3 == 0, 3584.0, -3584.0)[big]
    xq, xb = R.quantise_rows(x)
    odd = torch.tensor(sorted({1, T // 2, T - 1}))
    xb[odd, 0] += 120
    w1q, w1b = R.quantise_weights(W)
    w2q, w2b = R.quantise_weights(torch.ones(E, f, d))
    dev = [t.to(F8).cuda() if t.dtype == torch.float64 else t.cuda() for t in (xq, xb, w1q, w1b, w2q, w2b)]
    start = torch.tensor([sum(counts[:i]) for i in range(E + 1)], dtype=torch.int32, device="cuda")
    hq, hb = torch.empty((T, B.fp8_padded(f)), dtype=U8, device="cuda"), torch.empty((T, B.fp8_scale_bytes(f)), dtype=U8, device="cuda")
    yd = torch.empty((T, d), dtype=torch.float32, device="cuda")
    print(f"[gpu] infinite {counts} d={d} f={f} act={act}", flush=True)
    B.moe_expert_ffn_fwd_fp8(s, dev[0], dev[1], start, *dev[2:], hq, hb, yd)
    torch.cuda.synchronize()
    # (x 2^120 W as fp32 holds it; gelu(z) = z or 0 at such sizes)
    z = R.wide_weights(w1q, w1b)[0][3, :f].float() * 2.0 ** 120
    h = torch.zeros(B.fp8_padded(f), dtype=torch.float64)
    h[:f] = torch.relu(z).double()
    assert torch.isinf(h[:f]).any() and (z == float("-inf")).any()
    want, byte = R.quantise_rows(h[None])
    got, bytes_ = hq.cpu().view(F8).double(), hb.cpu()
    for r in odd.tolist():
        assert torch.equal(bytes_[r], byte[0]), r
        assert torch.equal(torch.isnan(got[r]), torch.isnan(want[0])) and torch.equal(torch.nan_to_num(got[r]), torch.nan_to_num(want[0])), r
    assert byte[0, 0] == 247 and torch.isnan(want[0, :128]).sum() == 26 and (want[0, :128] > 0).any()
    others = torch.ones(T, dtype=torch.bool)
    others[odd] = False
    assert torch.isnan(yd[odd.cuda()]).all() and torch.isfinite(yd[others.cuda()]).all() and not torch.isnan(got[others]).any()
