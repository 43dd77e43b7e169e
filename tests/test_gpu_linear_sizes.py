"""Linear layers at the ends of what a launch takes."""
import pytest

from gpu_util import say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", [1, 20])
def test_few_rows_of_very_many_columns(M):
    """Columns beyond what one workgroup per 16 of them could be launched for (2^24 workgroups of
    256 threads)."""
    import torch
    from paper_2211_00484_amd import tbs
    N = 2 ** 28 + 5
    say(f"linear {M} x 1 x {N}")
    w = torch.randint(-8, 9, (N, 1), dtype=torch.int8, device="cuda").to(torch.bfloat16)
    x = torch.arange(1, M + 1, device="cuda").to(torch.bfloat16)[:, None]
    out = tbs.linear(x, w)
    for m in range(M):
        assert torch.equal(out[m], w[:, 0] * (m + 1))
