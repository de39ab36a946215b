"""NaN logits count as -inf in the wide gate's choice, whatever the token's neighbours are."""
import numpy as np
import pytest
import torch

from paper_2109_10465_amd import binding as B

import route_ref as Q
import wide_ref as R

pytestmark = pytest.mark.gpu


def forward(r, l, b, mask=None):
    idx = torch.full((r.T, r.k), -7, dtype=torch.int32, device="cuda")
    w = torch.full((r.T, r.k), -7.0, device="cuda")
    B.moe_router_fwd(r, l.cuda(), None if b is None else b.cuda(), mask, idx, w)
    torch.cuda.synchronize()
    return idx.cpu(), w.cpu()


def inputs(T, E, seed, share):
    rng = np.random.default_rng(seed)
    l = rng.standard_normal((T, E)).astype(np.float32) * np.float32(1.5)
    l[rng.random((T, E)) < share] = np.nan
    l[::3, int(rng.integers(E))] = np.nan
    l[:, 5] = np.abs(l[:, 5])           # (never a whole row)
    l[np.isnan(l[:, 5]), 5] = 0.5
    return torch.from_numpy(l), torch.from_numpy(rng.standard_normal(E).astype(np.float32) * np.float32(0.05))


@pytest.mark.parametrize("score", [B.SOFTMAX, B.SIGMOID])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("E,groups,top,best", [(64, 1, 1, 1), (64, 8, 3, 1), (64, 8, 3, 2), (60, 1, 1, 1), (256, 8, 4, 2), (250, 10, 4, 2)])
@pytest.mark.parametrize("share", [0.01, 0.2])
def test_choice(score, bias, E, groups, top, best, share):
    T, k = 96, 6
    l, b = inputs(T, E, E + groups + best, share)
    b = b if bias else None
    for renorm in (True, False):
        r = B.make_router(T, E, k, score, groups, top, best, renorm, 1.5)
        idx, w = forward(r, l, b)
        ids, weights = Q.route(r, l, b)
        assert idx.tolist() == ids
        # NaN are chosen where a token's groups have nothing else: those weights are not defined
        ok = ~torch.isnan(l.gather(1, idx.long())).any(1)
        assert ok.sum() > T // 2
        # weights: the roundings of the fp32 formulas, as without NaN
        assert (w.double() - torch.tensor(weights, dtype=torch.float64))[ok].abs().max() <= 1.5 * 16 * 2.0 ** -24


def test_choice_beside_other_tokens():
    """The same tokens alone, and beside tokens whose two best are equal, which are decided in 64 bits."""
    T, E = 64, 64
    l, b = inputs(T, E, 1, 0.05)
    b[9] = b[8]
    tied = l.clone()
    tied[1::2] = 0.25
    tied[1::2, 8:10] = 4.0
    for score in (B.SOFTMAX, B.SIGMOID):
        one = [forward(B.make_router(1, E, 6, score), l[t:t + 1], b)[0].tolist()[0] for t in range(0, T, 2)]
        assert forward(B.make_router(T, E, 6, score), l, b)[0][::2].tolist() == one
        assert forward(B.make_router(T, E, 6, score), tied, b)[0][::2].tolist() == one


def test_rows_of_nothing_but_nan():
    l = torch.full((9, 24), float("nan"))
    for bias in (None, torch.linspace(-1, 1, 24)):
        for score in (B.SOFTMAX, B.SIGMOID):
            assert forward(B.make_router(9, 24, 4, score), l, bias)[0].tolist() == [[0, 1, 2, 3]] * 9


def test_gradient_beside_nan():
    """NaN that were not chosen leave the gradient of the softmax's weights as -inf do."""
    T, E = 40, 64
    l, b = inputs(T, E, 3, 0.1)
    r = B.make_router(T, E, 4, B.SOFTMAX, renormalise=False)
    idx, _ = forward(r, l, b)
    dw = torch.randn(T, 4, generator=torch.Generator().manual_seed(1))
    dl = torch.full((T, E), -7.0, device="cuda")
    B.moe_router_bwd(r, l.cuda(), idx.cuda(), dw.cuda(), dl)
    torch.cuda.synchronize()
    want = R.route_grad(r, Q.clean(l), idx, dw)
    # as for finite logits: 128 roundings of 2^-24 of 2 max |dw|
    assert (dl.cpu().double() - want).abs().max() <= 2 * float(dw.abs().max()) * 128 * 2.0 ** -24
