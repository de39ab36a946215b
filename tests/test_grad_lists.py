"""Lists of gradients whose outputs would be written while others read or write them: refused, on the host."""
import pytest
import torch

from paper_2109_10465_amd import binding as B


def test_lists_that_share_memory():
    a, b = torch.zeros(100), torch.zeros(100)
    for pairs in ([(a, a), (a[99:], a[99:])], [(a[:50], a[:50]), (a[49:], a[49:])],     # two in place
                  [(a[:50], b[:50]), (a[50:], b[49:99])],                                # two outputs
                  [(a[:50], a[50:]), (a[60:], b[:40])], [(a[:50], a[1:51])],             # an output and a gradient, another's or its own
                  [(a[:50], b[:50]), (b[10:20], torch.zeros(10))], [(b[10:20], torch.zeros(10)), (a, b)]):
        with pytest.raises(B.MoeError):
            B.make_grads(pairs)
    # bytes of another type
    with pytest.raises(B.MoeError):
        B.make_grads([(a, a), (a.view(torch.bfloat16)[198:], a.view(torch.bfloat16)[198:])])


def test_lists_that_do_not():
    a, b = torch.zeros(100), torch.zeros(100)
    cut = [a[i:i + 7] for i in range(0, 98, 7)]
    for pairs in ([(t, t) for t in cut], [(t, t) for t in cut[::-1]], [(t, b[i * 7:i * 7 + 7]) for i, t in enumerate(cut)],
                  [(a[:50], a[50:])], [(a[:50], b[:50]), (a[:50], b[50:])],              # (a gradient may be read twice)
                  [(a, None), (a, None)], [(a, a), (b, None)], [(a[:0], a[:0]), (a, a), (a[50:50], a[50:50])]):
        assert len(B.make_grads(pairs).pairs) == len(pairs)
