"""What an 8-bit layer takes for its weights: e4m3 values or their bytes, and no other type of 8 bits."""
import pytest
import torch

from paper_2109_10465_amd import binding as B
from paper_2109_10465_amd.layer import Fp8MoELayer

pytestmark = pytest.mark.gpu


def test_types_of_the_weights():
    g = torch.Generator().manual_seed(1)
    w1, w2 = (Fp8MoELayer.quantise_weights(torch.randn(s, generator=g).cuda()) for s in ((4, 128, 256), (4, 256, 128)))
    x = torch.randn(8, 128, generator=g).to(torch.bfloat16).cuda()
    logits = torch.randn(8, 4, generator=g).cuda()

    def run(a, b):
        return Fp8MoELayer(8, 128, 256, 4, 2, B.BF16, B.GELU, a, b).forward(x, logits=logits).clone()

    view = lambda w, t: (w[0].view(t), w[1])
    assert torch.equal(run(w1, w2), run(view(w1, torch.uint8), view(w2, torch.uint8)))
    for other in (torch.float8_e5m2, torch.float8_e4m3fnuz, torch.int8):
        with pytest.raises(B.MoeError):
            run(view(w1, other), w2)
        with pytest.raises(B.MoeError):
            run(w1, view(w2, other))
    with pytest.raises(B.MoeError):
        run((w1[0], w1[1].view(torch.int8)), w2)
