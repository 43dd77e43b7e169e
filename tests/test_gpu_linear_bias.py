"""dbias of fp32 layers over many rows: its error does not grow with them.

The terms of half a slice, 16, are added in fp32, by a unit that may cut (2^-23 of the magnitudes
for each addition); those sums are added in fp64 and rounded once for each part of the rows and
once at the end: within (16 + 2) 2^-23 of the sum of the magnitudes."""
import pytest

from gpu_util import say

pytestmark = pytest.mark.gpu


# whole (the tiles fill 256 CUs, in tiles of 64 and of 128) and in parts
@pytest.mark.parametrize("M,K,N", [(64000, 1024, 1024), (20000, 4100, 4100), (64000, 128, 160), (8000, 384, 512),
                                   (33, 1100, 1100), (100001, 3, 5)])
@pytest.mark.parametrize("want_weight", [True, False])
def test_sums_over_many_rows(M, K, N, want_weight):
    import torch
    from paper_2211_00484_amd import tbs
    g = torch.Generator(device="cuda").manual_seed(M)
    x, w = torch.randn((M, K), generator=g, device="cuda"), torch.zeros((N, K), device="cuda")
    dy = torch.randn((M, N), generator=g, device="cuda").abs()
    say(f"dbias {M} x {K} x {N}")
    for d in (dy, dy.where(torch.rand((M, 1), generator=g, device="cuda") < 0.5, -dy)):
        got = tbs.linear_backward(d, x, w, want_x=False, want_weight=want_weight).bias.double()
        want = d.double().sum(0)
        assert ((got - want).abs() <= 18 * 2.0 ** -23 * dy.double().sum(0)).all()
        assert torch.equal(tbs.linear_backward(d, x, w, want_x=False, want_weight=want_weight).bias.double(), got)
