"""Which kernels the rules of the 8-bit products choose, at shapes where both sides have been measured (host-only queries; the
times are microseconds on an MI355X)."""
import pytest

from paper_2109_10465_amd import binding as B


@pytest.mark.parametrize("T,k,d,f,E,kinds", [
    (65536, 2, 2048, 8192, 16, (0, 0)),     # large 2409, 1775; small 2792, 2226
    (5003, 2, 776, 3080, 6, (1, 0)),        # large 58, 43; small 52, 52
    (7375, 4, 1024, 4096, 64, (0, 0)),      # large 205, 140; small 229, 171
    (2048, 2, 1024, 4096, 16, (0, 1)),      # large 28, 51; small 28, 29
    (2048, 2, 1024, 4096, 32, (1, 1)),      # large 58, 36; small 41, 33
    (768, 2, 1024, 4096, 32, (3, 3)),       # narrow 34, 24; small 36, 27
    (61, 2, 1024, 4096, 32, (3, 3)),        # narrow 27, 23; small 34, 25; second thin 41
    (1, 8, 1024, 4096, 8, (3, 2)),          # first: narrow 12.1, small 13.5; second: small 23, thin 10
    (1, 8, 2048, 2048, 8, (3, 3)),          # narrow 14.2, 12.8; small 17, 13; second thin 16
])
def test_kernels_of_the_block(T, k, d, f, E, kinds):
    for act in (B.RELU, B.GELU):
        assert B.moe_fp8_kernels(B.make_fp8_shape(T, d, f, E, k, B.BF16, act)) == kinds


def test_query_refuses_what_the_block_refuses():
    with pytest.raises(B.MoeError):
        B.moe_fp8_kernels(B.make_fp8_shape(1, 12, 16, 1, 1, B.BF16, B.GELU))
