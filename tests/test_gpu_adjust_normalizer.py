"""Log-softmax of tbs_adjust_logits on rows far from 0.

Logits are multiples of 2^-6 up to 2^17, so that a row shifted by a constant is exact and so is its
distance to the row's largest: results do not depend on the shift.  Tolerance: the sum's
(V / 64 + 20) 2^-23 and 2e-6 for exponentials and logarithm, as in test_gpu_adjust, and three
roundings of the result; nothing that grows with the shift."""
import pytest

from gpu_util import say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [2, 50, 700, 6000, 8192, 40000])
@pytest.mark.parametrize("shift", [-65536.0, -1000.0, 1000.0, 65536.0])
def test_shifted_rows(V, shift):
    import torch
    from paper_2211_00484_amd import tbs
    say(f"log-softmax of {V} labels around {shift}")
    g = torch.Generator(device="cuda").manual_seed(V)
    z = torch.randint(-300, 300, (7, V), generator=g, device="cuda").float() / 64
    z[1, V // 2] += 25.0        # one label leads
    z[2] = 0.0                  # all alike
    z[3, 1:] -= 500.0           # one is left
    moved = z + shift
    assert torch.equal(moved - shift, z)
    got, want = tbs.adjust_logits(moved, normalize=True), torch.log_softmax(z.double(), 1)
    tol = (V / 64 + 20) * 2.0 ** -23 + 2e-6 + 3 * 2.0 ** -24 * want.abs()
    assert ((got.double() - want).abs() <= tol).all()
    assert (got <= 0).all()
    assert torch.equal(got, tbs.adjust_logits(z, normalize=True))
