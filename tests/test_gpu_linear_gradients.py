"""Gradients of 16-bit linear layers through an activation: dx, dw and dbias are those of the
unrounded gradient of the activation's argument, dz, and are rounded once.

Tolerances, with h = eps / 2 of the type: dz is within 2e-6 |grad_out| (the slope) and, held in
two parts of the type, within h^2 of itself and 2^-36 (half the smallest step of fp16's second
part, which is held times 2^11); a sum of 2 n products in fp32, in any order, is within
2 n 2^-23 of the sum of their magnitudes; the result is rounded once, by h of it.

That holds for each value.  For all of them together: a result whose sum is off by d is off by at
most 2 |d| more than the rounded exact one (the two are the same, or d has carried it over a tie,
from which both are then within |d| of half a step); and over terms of random signs the errors
before the rounding are those of independent terms, the root of the sum of e^2 and, for 2 n
additions to partial sums of the terms' own norm, sqrt(2 n) 2^-24 of that.  A dz rounded to the
type would be off by as much as the result's own rounding, 1.4 times in all."""
import ctypes

import pytest

from gpu_util import say
from test_gpu_linear import _half, _slope64, _t, _tiny, _within

pytestmark = pytest.mark.gpu

HALVES = ["bfloat16", "float16"]
SMOOTH = ["tanh", "silu", "gelu"]


def _inputs(M, K, N, dtype, seed, scale=1.0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    dt = _t(dtype)
    return (r(M, N) * scale).to(dt), r(M, K).to(dt), (r(N, K) * K ** -0.5).to(dt), r(M, N).to(dt)


def _check(g, x, w, pre, act, dx=None, dw=None, db=None, signs=True):
    import torch
    M, N = g.shape
    h, tiny = _half(x.dtype), _tiny(x.dtype)
    gd, xd, wd = g.double(), x.double(), w.double()
    dz = gd * _slope64(pre.double(), act)
    e = 2e-6 * gd.abs() + h * h * dz.abs() + 2.0 ** -36
    t = lambda m: m.t().contiguous()
    one = torch.ones((M, 1), dtype=torch.float64, device=g.device)
    for got, a, er, b, n, what in ((dx, dz, e, wd, N, "dx"), (dw, t(dz), t(e), xd, M, "dw"),
                                   (None if db is None else db[:, None], t(dz), t(e), one, M, "dbias")):
        if got is None:
            continue
        v, er1 = a @ b, er @ b.abs()
        tol = er1 + (2 * n + 2) * 2.0 ** -23 * (a.abs() @ b.abs() + er1)
        _within(got, v, tol + h * (v.abs() + tol) + tiny, what)
        if signs:
            d = (er ** 2 @ b ** 2).sqrt() + (2 * n) ** 0.5 * 2.0 ** -24 * (a ** 2 @ b ** 2).sqrt()
            off, rounding = (got.double() - v).norm().item(), (v.to(got.dtype).double() - v).norm().item()
            assert off <= rounding + 2 * d.norm().item(), (what, off, rounding, d.norm().item())


# single rows, odd sizes, one and several parts of the sums, each tile, slices that are not whole
@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("act", SMOOTH)
@pytest.mark.parametrize("M,K,N", [(1, 33, 7), (3, 512, 500), (40, 65, 129), (150, 70, 90), (1000, 256, 500),
                                   (5000, 64, 20), (6000, 130, 200), (2100, 320, 520), (300, 1500, 1700)])
def test_products_of_the_unrounded_gradient(M, K, N, act, dtype):
    from paper_2211_00484_amd import tbs
    g, x, w, pre = _inputs(M, K, N, dtype, M + K + N)
    say(f"linear_backward {M} x {K} x {N} {act} {dtype}")
    for want_pre in (False, True):
        got = tbs.linear_backward(g, x, w, pre=pre, activation=act, want_pre=want_pre)
        _check(g, x, w, pre, act, got.x, got.weight, got.bias)


# where 256 CUs take tiles of 256 x 256 (dx, then dw) and of 128 x 128 (the same, dw in parts), each
# with rows that are copied directly and (odd sizes) rows that are not; every shape has tiles that
# the edge of the result cuts and a slice that is not whole
@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("M,K,N", [(16300, 770, 70), (16300, 769, 71), (100, 4000, 3100), (101, 4001, 3101),
                                   (9000, 520, 400), (9000, 521, 401), (2100, 1000, 900), (2101, 1001, 901)])
def test_large_tiles(M, K, N, dtype):
    from paper_2211_00484_amd import tbs
    g, x, w, pre = _inputs(M, K, N, dtype, M + K + N)
    say(f"linear_backward {M} x {K} x {N} tanh {dtype}")
    got = tbs.linear_backward(g, x, w, pre=pre, activation="tanh")
    _check(g, x, w, pre, "tanh", got.x, got.weight, got.bias)


@pytest.mark.parametrize("act", SMOOTH)
def test_small_gradients_add_up(act):
    """fp16 gradients near and below the type's smallest step: the rows' sums keep them."""
    import torch
    from paper_2211_00484_amd import tbs
    M, K, N = 20000, 40, 60
    g, x, w, pre = _inputs(M, K, N, "float16", 3, 1e-6)
    x, pre = x.abs(), (pre.float() - 3).half()
    got = tbs.linear_backward(g.abs(), x, w, pre=pre, activation=act)
    _check(g.abs(), x, w, pre, act, got.x, got.weight, got.bias, signs=False)
    assert (got.bias != 0).all()


@pytest.mark.parametrize("dtype", HALVES)
def test_rows_of_their_own(dtype):
    """The C entry with rows further apart than their width; every choice of outputs."""
    import torch
    from paper_2211_00484_amd import tbs
    L, M, K, N, pad = tbs.lib(), 700, 90, 150, 5
    code = 1 if dtype == "bfloat16" else 2
    g, x, w, pre = _inputs(M, K, N, dtype, 4)
    for bits in range(1, 16):
        new = lambda rows, cols: torch.full((rows, cols + pad), -77.0, dtype=x.dtype, device="cuda")
        dx, dw, db, dz = new(M, K), new(N, K), torch.empty(N, dtype=x.dtype, device="cuda"), new(M, N)
        wants = [int(bits >> i & 1) for i in range(4)]
        n = L.tbs_linear_backward_workspace(code, 2, M, N, K, *wants)
        ws = torch.full((n + 64,), 0xA5, dtype=torch.uint8, device="cuda")
        p = lambda t, want=1: ctypes.c_void_p(t.data_ptr()) if want else None
        assert L.tbs_linear_backward(code, p(g), N, p(x), K, p(w), K, p(pre), N, 2, M, N, K, p(dx, wants[0]),
                                     K + pad, p(dw, wants[1]), K + pad, p(db, wants[2]), p(dz, wants[3]), N + pad,
                                     p(ws), n, tbs._stream_ptr()) == 0
        assert (ws[n:] == 0xA5).all()
        _check(g, x, w, pre, "tanh", dx[:, :K] if wants[0] else None, dw[:, :K] if wants[1] else None,
               db if wants[2] else None)
        for t, cols in ((dx, K), (dw, K), (dz, N)):
            assert (t[:, cols:] == -77.0).all()
        if wants[3]:
            s = _slope64(pre.double(), "tanh") * g.double()
            e = 2e-6 * g.double().abs()
            _within(dz[:, :N], s, e + _half(x.dtype) * (s.abs() + e) + _tiny(x.dtype), "dz")


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("act", SMOOTH)
@pytest.mark.parametrize("M,K,N", [(5, 100, 37), (130, 100, 70), (3000, 64, 66)])
def test_special_values(M, K, N, act, dtype):
    """Infinities and NaN in grad_out, w and x reach what the formula takes them to, with their
    signs, and nothing else."""
    import math
    import torch
    from paper_2211_00484_amd import tbs
    g, x, w, pre = _inputs(M, K, N, dtype, 3)
    run = lambda g, x, w: tbs.linear_backward(g, x, w, pre=pre, activation=act, want_pre=True)
    ref = run(g, x, w)
    assert (ref.pre != 0).all()
    sign = ref.pre.double().sign()

    g2 = g.clone()
    g2[2, N - 1], g2[1, 0] = math.nan, math.inf
    got = run(g2, x, w)
    keep = [m for m in range(M) if m not in (1, 2)]
    assert torch.equal(got.x[keep], ref.x[keep]) and torch.isnan(got.x[2]).all()
    up = _slope64(pre[1:2, :1].double(), act).sign().item()
    assert torch.equal(got.x[1].double(), math.inf * up * w[0].double().sign())
    assert torch.equal(got.weight[1:N - 1], ref.weight[1:N - 1]) and torch.isnan(got.weight[N - 1]).all()
    assert torch.equal(got.weight[0].double(), math.inf * up * x[1].double().sign())
    assert torch.equal(got.bias[1:N - 1], ref.bias[1:N - 1]) and torch.isnan(got.bias[N - 1])
    assert got.bias[0].item() == math.inf * up

    w2 = w.clone()
    w2[N - 1, K - 1], w2[N - 2, 0] = math.inf, math.nan
    got = run(g, x, w2)
    assert torch.equal(got.x[:, 1:K - 1], ref.x[:, 1:K - 1]) and torch.isnan(got.x[:, 0]).all()
    assert torch.equal(got.x[:, K - 1].double(), math.inf * sign[:, N - 1])
    assert torch.equal(got.weight, ref.weight) and torch.equal(got.bias, ref.bias)

    x2 = x.clone()
    x2[1, 0], x2[3, K - 1] = -math.inf, math.nan
    got = run(g, x2, w)
    assert torch.equal(got.weight[:, 1:K - 1], ref.weight[:, 1:K - 1]) and torch.isnan(got.weight[:, K - 1]).all()
    assert torch.equal(got.weight[:, 0].double(), -math.inf * sign[1])
    assert torch.equal(got.x, ref.x) and torch.equal(got.bias, ref.bias)
