"""Activations and their slopes where they are small.

gelu's distribution comes from a fit to within 5e-8 of its tail and some 16 roundings of 2^-24 (nine
steps of a polynomial, a reciprocal, an exponential, products): within 1.1e-6 of its value, however
small it is (what lies below fp32's normal range may be taken as 0); 2e-6 is allowed.  The slope's
second term, z e^(-z^2 / 2) / sqrt(2 pi), has 6 roundings: 1e-6."""
import math

import pytest

from test_gpu_linear import _half, _t, _tiny

pytestmark = pytest.mark.gpu

DTYPES = ["float32", "bfloat16", "float16"]


def _through(z, act):
    """act(z) and act'(z) for every value of z, as a layer with one input gives them."""
    import torch
    from paper_2211_00484_amd import tbs
    n = z.numel()
    zero = torch.zeros((1, 1), dtype=z.dtype, device="cuda")
    w = torch.zeros((n, 1), dtype=z.dtype, device="cuda")
    g = torch.ones((1, n), dtype=z.dtype, device="cuda")
    return (tbs.linear(zero, w, z, activation=act)[0],
            tbs.linear_backward(g, zero, w, pre=z[None], activation=act, want_x=False, want_weight=False,
                                want_bias=False, want_pre=True).pre[0])


@pytest.mark.parametrize("dtype", DTYPES)
def test_gelu_tails(dtype):
    import torch
    dt = _t(dtype)
    z = torch.cat([torch.linspace(-14, 14, 28001), torch.logspace(-30, 1, 500), -torch.logspace(-30, 1, 500)])
    z = z.to(dt).cuda()
    out, slope = _through(z, "gelu")
    d = z.double()
    cdf = 0.5 * torch.erfc(-d * math.sqrt(0.5))
    density = torch.exp(-0.5 * d * d) / math.sqrt(2 * math.pi)
    low = 2.0 ** -126 * (1 + d.abs()) + _tiny(dt)
    want = d * cdf
    e = 2e-6 * want.abs() + low
    over = (out.double() - want).abs() - e - _half(dt) * (want.abs() + e)
    i = over.argmax()
    assert over.max() <= 0, (z[i].item(), out[i].item(), want[i].item())
    want = cdf + d * density
    e = 2e-6 * cdf + 1e-6 * (d * density).abs() + 2.0 ** -23 * want.abs() + low
    over = (slope.double() - want).abs() - e - _half(dt) * (want.abs() + e)
    i = over.argmax()
    assert over.max() <= 0, (z[i].item(), slope[i].item(), want[i].item())
