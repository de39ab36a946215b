"""What the wide gate, the 8-bit experts and clipping refuse, on the host and before any launch (no GPU: had a kernel
been issued, this process would get MOE_ERR_LAUNCH), and the sizes that they ask for."""
import ctypes

import pytest
import torch

from paper_2109_10465_amd import binding as B

P = 1 << 20         # "somewhere": a pointer that is never followed
REF = ctypes.byref


def router(**over):
    a = dict(T=64, E=32, k=4, score=B.SIGMOID, n_groups=8, top_groups=2, group_best=2, renormalise=True, scale=1.0)
    a.update(over)
    return B.make_router(**a)


def shape(**over):
    a = dict(T=64, d_model=128, d_ff=256, E=32, k=4, dtype=B.BF16, act=B.GELU)
    a.update(over)
    return B.make_fp8_shape(**a)


BAD_ROUTER = [(dict(T=0), -2), (dict(k=0), -2), (dict(k=9), -2), (dict(E=3, n_groups=1, top_groups=1), -2),
              (dict(E=264, n_groups=1, top_groups=1), -2), (dict(n_groups=5), -2), (dict(n_groups=0), -2),
              (dict(E=130, n_groups=65, group_best=1), -2), (dict(top_groups=0), -2), (dict(top_groups=9), -2),
              (dict(group_best=0), -2), (dict(group_best=3), -2), (dict(n_groups=32, top_groups=8), -2),
              (dict(top_groups=1, k=5), -2), (dict(scale=float("inf")), -2), (dict(scale=float("nan")), -2),
              (dict(score=2), -3), (dict(T=1 << 28), -2)]


@pytest.mark.parametrize("over,code", BAD_ROUTER)
def test_router(over, code):
    L, r = B.lib(), router(**over)
    assert L.moe_router_fwd(REF(r), P, None, None, P, P, None) == code
    assert L.moe_router_bwd(REF(r), P, P, P, P, None) == code
    assert L.moe_sort_choices(REF(r), P, P, P, P, 1 << 40, None) == code
    assert L.moe_router_bias_update(REF(r), P, 0.1, P, None) == code
    assert B.moe_sort_workspace_bytes(r) == 0


def test_router_pointers_and_workspace():
    L, r = B.lib(), router()
    for i in (0, 3, 4):
        a = [P, P, P, P, P]
        a[i] = None
        assert L.moe_router_fwd(REF(r), *a, None) == -1
    for i in range(4):
        a = [P] * 4
        a[i] = None
        assert L.moe_router_bwd(REF(r), *a, None) == -1
    for i in range(3):
        a = [P] * 3
        a[i] = None
        assert L.moe_sort_choices(REF(r), *a, P, 1 << 40, None) == -1
    n = B.moe_sort_workspace_bytes(r)
    assert n > 0 and n % 256 == 0
    for ws, b in ((None, n), (P, n - 1), (P + 16, n)):
        assert L.moe_sort_choices(REF(r), P, P, P, ws, b, None) == -4
    assert L.moe_router_bias_update(REF(r), None, 0.1, P, None) == -1
    assert L.moe_router_bias_update(REF(r), P, float("nan"), P, None) == -2
    assert L.moe_router_fwd(None, *[P] * 5, None) == -1


BAD_SHAPE = [(dict(T=0), -2), (dict(k=0), -2), (dict(k=9), -2), (dict(E=0), -2), (dict(E=257), -2), (dict(d_model=12), -2),
             (dict(d_ff=0), -2), (dict(d_model=(1 << 20) + 8), -2), (dict(d_model=1 << 16, d_ff=1 << 15), -2),
             (dict(T=1 << 28), -2), (dict(dtype=B.F32), -3), (dict(act=2), -3)]


@pytest.mark.parametrize("over,code", BAD_SHAPE)
def test_fp8_shape(over, code):
    L, s = B.lib(), shape(**over)
    assert L.moe_dispatch_fp8(REF(s), P, P, P, P, None) == code
    assert L.moe_expert_ffn_fwd_fp8(REF(s), *[P] * 9, 1, P, None) == code
    assert L.moe_combine_rows(REF(s), 1, *[P] * 4, None) == code


def test_fp8_pointers():
    L, s = B.lib(), shape()
    ffn = lambda s, *a: L.moe_expert_ffn_fwd_fp8(s, *a[:9], 0, *a[9:])
    combine = lambda s, *a: L.moe_combine_rows(s, 0, *a)
    for f, n in ((L.moe_dispatch_fp8, 4), (ffn, 10), (combine, 4)):
        assert f(None, *[P] * n, None) == -1
        for i in range(n):
            a = [P] * n
            a[i] = None
            assert f(REF(s), *a, None) == -1
    assert L.moe_expert_ffn_fwd_fp8(REF(s), *[P] * 9, 2, P, None) == -3
    assert L.moe_combine_rows(REF(s), 2, *[P] * 4, None) == -3
    for i in range(3):
        a = [P] * 3
        a[i] = None
        assert L.moe_quantise_rows_fp8(4, 128, 0, *a, None) == -1
        assert L.moe_quantise_weights_fp8(2, 128, 64, 0, *a, None) == -1
    for i in range(6):
        a = [P] * 6
        a[i] = None
        assert L.moe_expert_product_fp8(4, 2, 128, 64, *a[:5], 1, a[5], None) == -1


@pytest.mark.parametrize("rows,E,K,N,dtype,code", [(0, 1, 128, 128, 0, -2), (1 << 30, 1, 128, 128, 0, -2), (4, 1, 12, 128, 0, -2),
                                                   (4, 1, 128, 4, 0, -2), (4, 257, 128, 128, 0, -2), (4, 1, 128, 128, 2, -3),
                                                   (4, 1, 1 << 20, 1 << 12, 1, -2)])
def test_fp8_extents(rows, E, K, N, dtype, code):
    L = B.lib()
    assert L.moe_expert_product_fp8(rows, E, K, N, *[P] * 5, dtype, P, None) == code
    if rows == 4:
        assert L.moe_quantise_weights_fp8(E, K, N, dtype, P, P, P, None) == code
    if N == 128 and E == 1:
        assert L.moe_quantise_rows_fp8(rows, K, dtype, P, P, P, None) == code


def test_fp8_alignment():
    L, s = B.lib(), shape()
    ffn = lambda s, *a: L.moe_expert_ffn_fwd_fp8(s, *a[:9], 0, *a[9:])
    combine = lambda s, *a: L.moe_combine_rows(s, 1, *a)
    product = lambda *a: L.moe_expert_product_fp8(4, 2, 128, 64, *a[:5], 1, *a[5:])
    rows, weights = (lambda *a: L.moe_quantise_rows_fp8(4, 128, 0, *a)), (lambda *a: L.moe_quantise_weights_fp8(2, 128, 64, 0, *a))
    # per entry: the arguments that are values, and those that are exponents
    for f, n, values, exponents in ((lambda *a: L.moe_dispatch_fp8(REF(s), *a), 4, (0, 2), (3,)),
                                    (lambda *a: ffn(REF(s), *a), 10, (0, 3, 5, 7, 9), (1, 4, 6, 8)),
                                    (lambda *a: combine(REF(s), *a), 4, (0, 3), ()), (product, 6, (0, 3, 5), (1, 4)),
                                    (rows, 3, (0, 1), (2,)), (weights, 3, (0, 1), (2,))):
        for i in (*values, *exponents):
            a = [P] * n
            a[i] = P + (8 if i in values else 2)
            assert f(*a, None) == -2, (n, i)


def test_fp8_layer_reports_every_error_before_its_first_launch():
    L, r, s = B.lib(), router(), shape()

    def call(s=s, r=r, given=0, without=(), x=P, Wg=P, weights=(P,) * 4, ws=None):
        b = B.Fp8Buffers()
        for n, _ in B.Fp8Buffers._fields_:
            setattr(b, n, None if n in without else P)
        b.ws_bytes = B.moe_sort_workspace_bytes(r) if ws is None else ws
        return L.moe_layer_fwd_fp8(REF(s), REF(r), given, REF(b), x, Wg, None, None, *weights, None)

    for n in ("logits", "expert_idx", "gate_w", "row_of", "expert_start", "xq", "xb", "hq", "hb", "yd", "y"):
        assert call(without=(n,)) == -1, n
    assert call(without=("ws",)) == -4 and call(ws=16) == -4
    assert call(x=None) == -1 and call(Wg=None) == -1 and call(given=1, x=None) == -1
    for i in range(4):
        assert call(weights=[None if j == i else P for j in range(4)]) == -1
    for over in (dict(T=63), dict(E=64), dict(k=3)):
        assert call(r=router(**over)) == -2
    assert call(s=shape(act=5)) == -3
    assert call(s=shape(E=257), r=router()) == -2


def test_grads():
    L = B.lib()
    one = lambda **o: (B.MoeGrad * 1)(B.MoeGrad(**{**dict(grad=P, out=P, n=4, dtype=0), **o}))
    big = 1 << 20
    for f in (lambda g, n=1, ws=P, b=big: L.moe_grad_norm(g, n, P, ws, b, None),
              lambda g, n=1, ws=P, b=big: L.moe_clip_grads(g, n, 1.0, P, ws, b, None)):
        assert f(None) == -1
        assert f(one(), n=-1) == -2
        assert f(one(n=-1)) == -2
        assert f(one(grad=None)) == -1
        assert f(one(dtype=2)) == -3
        assert f(one(grad=P + 2)) == -2
        assert f(one(grad=P + 1, dtype=1)) == -2
        assert f(one(), ws=None) == -4 and f(one(), b=8) == -4 and f(one(), ws=P + 8) == -4
    clip = lambda g, m=1.0, norm=P: L.moe_clip_grads(g, 1, m, norm, P, big, None)
    assert clip(one(out=None)) == -1 and clip(one(out=P + 2)) == -2
    assert clip(one(), norm=None) == -1 and L.moe_grad_norm(one(), 1, None, P, big, None) == -1
    for m in (-1.0, float("inf"), float("nan")):
        assert clip(one(), m) == -2
    # the workspace covers the list: more for longer tensors, something for an empty list
    size = lambda n: L.moe_grad_workspace_bytes(one(n=n), 1)
    assert size(0) > 0 and size(1 << 30) > size(1 << 20) >= size(0) and L.moe_grad_workspace_bytes(None, 0) > 0
    assert L.moe_grad_workspace_bytes(one(n=-1), 1) == 0


def test_grads_of_tensors():
    a, b = torch.zeros(4, 4), torch.zeros(16, dtype=torch.bfloat16)
    g = B.make_grads([(a, a), (b, None), (torch.zeros(0), torch.zeros(0))])
    assert [(m.n, m.dtype) for m in g.list] == [(16, 0), (16, 1), (0, 0)]
    for pair in ((a.t()[:2], None), (a, b), (a, torch.zeros(15)), (a.half(), None)):
        with pytest.raises(B.MoeError):
            B.make_grads([pair])
    with pytest.raises(B.MoeError):                 # clipped twice
        B.make_grads([(a, a), (b, b), (a, a)])


def test_extents_of_the_8_bit_format():
    assert [B.fp8_padded(n) for n in (8, 128, 136)] == [128, 128, 256]
    assert [B.fp8_scale_bytes(n) for n in (8, 512, 520, 2048)] == [4, 4, 8, 16]

