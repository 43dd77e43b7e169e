"""Linear layers and their gradients (tbs_linear, tbs_linear_backward) against 64 bits.

Tolerances, from the inputs as they are given: a sum of n products in fp32, in any order,
is within n 2^-23 of the sum of their magnitudes (half a step per addition, and as much
again for a unit that cuts); an activation passes an error on with a factor of at most 1.13
(gelu's steepest slope) and adds 1e-6 of its value (exponentials and reciprocals of a few
steps of 2^-24); a result is rounded once, by eps / 2 of it."""
import ctypes
import math

import pytest

from gpu_util import say

pytestmark = pytest.mark.gpu

DTYPES = ["float32", "bfloat16", "float16"]
ACTS = ["none", "relu", "tanh", "silu", "gelu"]
# (M, K, N): single rows and columns, odd sizes, edges of chunks, slices and tiles
SHAPES = [(1, 1, 1), (1, 512, 500), (4, 512, 500), (3, 7, 5), (2, 9, 300), (16, 64, 16), (17, 33, 65),
          (31, 15, 33), (64, 32, 64), (65, 31, 63), (64, 2048, 48), (100, 100, 100), (129, 513, 127),
          (130, 384, 512), (257, 72, 258), (512, 512, 512), (700, 40, 1000), (1030, 257, 36),
          (5000, 64, 20), (333, 1111, 777), (2100, 320, 520)]


def _t(name):
    import torch
    return getattr(torch, name)


def _act64(z, act):
    import torch
    f = torch.nn.functional
    return {"none": lambda v: v, "relu": torch.relu, "tanh": torch.tanh, "silu": f.silu,
            "gelu": f.gelu}[act](z)


def _slope64(z, act):
    import torch
    if act == "none":
        return torch.ones_like(z)
    z = z.detach().clone().requires_grad_(True)
    g, = torch.autograd.grad(_act64(z, act).sum(), z)
    return g


def _inputs(M, K, N, dtype, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    dt = _t(dtype)
    return (r(M, K).to(dt), (r(N, K) * K ** -0.5).to(dt), r(N).to(dt), r(M, N).to(dt), r(M, N).to(dt))


def _within(got, want, tol, what):
    import torch
    got = got.double()
    assert torch.isfinite(got).all(), what
    over = (got - want).abs() - tol
    i = over.argmax()
    assert over.max() <= 0, (f"{what}: {got.flatten()[i].item()} for {want.flatten()[i].item()}, "
                             f"tolerance {tol.flatten()[i].item()}")


def _half(t):
    import torch
    return torch.finfo(t).eps / 2


def _tiny(t):
    """Half the smallest step of the type (for results below its normal range)."""
    import torch
    return torch.finfo(t).smallest_normal * torch.finfo(t).eps


def _check_forward(x, w, b, r, act, after, out, pre):
    import torch
    K, dt = x.shape[1], x.dtype
    xd, wd = x.double(), w.double()
    z = xd @ wd.t().contiguous()
    mag = xd.abs() @ wd.abs().t().contiguous()
    if b is not None:
        z, mag = z + b.double(), mag + b.double().abs()
    if r is not None and not after:
        z, mag = z + r.double(), mag + r.double().abs()
    err = (K + 2) * 2.0 ** -23 * mag
    y = _act64(z, act)
    e = 1.13 * err + (0 if act == "none" else 1e-6 * (y.abs() + 1e-6))
    if r is not None and after:
        y = y + r.double()
        e = e + 2.0 ** -24 * y.abs()
    _within(out, y, e + _half(dt) * (y.abs() + e) + _tiny(dt), "out")
    if pre is not None:
        _within(pre, z, err + _half(dt) * (z.abs() + err) + _tiny(dt), "pre")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_forward_shapes(M, K, N, dtype):
    from paper_2211_00484_amd import tbs
    x, w, b, r, _ = _inputs(M, K, N, dtype, M + K + N)
    say(f"linear {M} x {K} x {N} {dtype}")
    out = tbs.linear(x, w)
    _check_forward(x, w, None, None, "none", False, out, None)
    out, pre = tbs.linear(x, w, b, residual=r, activation="tanh", want_pre=True)
    _check_forward(x, w, b, r, "tanh", False, out, pre)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("res", ["none", "before", "after", "row"])
@pytest.mark.parametrize("M,K,N", [(6, 96, 50), (140, 96, 203)])
def test_epilogues(M, K, N, res, act, dtype):
    from paper_2211_00484_amd import tbs
    x, w, b, r, _ = _inputs(M, K, N, dtype, 5)
    r = None if res == "none" else r[0] if res == "row" else r
    out, pre = tbs.linear(x, w, b, residual=r, activation=act, residual_after=res == "after",
                          want_pre=True)
    _check_forward(x, w, b, r, act, res == "after", out, pre)
    same = tbs.linear(x, w, b, residual=r, activation=act, residual_after=res == "after")
    assert (same == out).all()


def _check_backward(g, x, w, pre, act, got):
    dt = x.dtype
    M, N = g.shape
    K = x.shape[1]
    h = _half(dt)
    gd, xd, wd = g.double(), x.double(), w.double()
    if act == "none":
        dz, e = gd, 0 * gd
    else:
        dz = gd * _slope64(pre.double(), act)
        e = 2e-6 * gd.abs()          # the slope, absolutely (at most 1.13)
        e = e + h * (dz.abs() + e) + _tiny(dt)
        _within(got.pre, dz, e, "dz")
    dx = dz @ wd
    tol = e @ wd.abs() + (N + 1) * 2.0 ** -23 * ((dz.abs() + e) @ wd.abs())
    _within(got.x, dx, tol + h * (dx.abs() + tol) + _tiny(dt), "dx")
    t = lambda m: m.t().contiguous()
    dw = t(dz) @ xd
    tol = t(e) @ xd.abs() + (M + 1) * 2.0 ** -23 * (t(dz.abs() + e) @ xd.abs())
    _within(got.weight, dw, tol + h * (dw.abs() + tol) + _tiny(dt), "dw")
    db = dz.sum(0)
    tol = e.sum(0) + (M + 1) * 2.0 ** -23 * (dz.abs() + e).sum(0)
    _within(got.bias, db, tol + h * (db.abs() + tol) + _tiny(dt), "dbias")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_backward_shapes(M, K, N, dtype):
    from paper_2211_00484_amd import tbs
    x, w, _, pre, g = _inputs(M, K, N, dtype, M * 3 + K + N)
    say(f"linear_backward {M} x {K} x {N} {dtype}")
    _check_backward(g, x, w, None, "none", tbs.linear_backward(g, x, w))
    got = tbs.linear_backward(g, x, w, pre=pre, activation="tanh", want_pre=True)
    _check_backward(g, x, w, pre, "tanh", got)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("act", ACTS)
def test_backward_wants(act, dtype):
    """Every choice of outputs gives the same bits as all of them."""
    from paper_2211_00484_amd import tbs
    x, w, _, pre, g = _inputs(150, 70, 90, dtype, 9)
    pre = None if act == "none" else pre * 4
    full = tbs.linear_backward(g, x, w, pre=pre, activation=act, want_pre=True)
    _check_backward(g, x, w, pre, act, full)
    for bits in range(16):
        wx, ww, wb, wp = (bool(bits >> i & 1) for i in range(4))
        got = tbs.linear_backward(g, x, w, pre=pre, activation=act, want_x=wx, want_weight=ww,
                                  want_bias=wb, want_pre=wp)
        for name, want in (("x", wx), ("weight", ww), ("bias", wb), ("pre", wp)):
            v = getattr(got, name)
            assert (v is not None) == want
            assert v is None or (v == getattr(full, name)).all(), (bits, name)


def _ints(shape, dtype, seed, lim=4):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-lim, lim + 1, shape, generator=g, device="cuda").to(_t(dtype))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K,N", SHAPES + [(3000, 700, 600), (20000, 48, 500), (300, 2048, 4999)])
def test_integers_are_exact(M, K, N, dtype):
    """Small integers: every partial sum is exact in fp32 (below 2^24), so the results are
    the exact ones rounded once, bit for bit, whatever the order of the sums."""
    import torch
    from paper_2211_00484_amd import tbs
    dt = _t(dtype)
    x, w, g = _ints((M, K), dtype, 1), _ints((N, K), dtype, 2), _ints((M, N), dtype, 3)
    r = _ints((M, N), dtype, 4)
    say(f"integers {M} x {K} x {N} {dtype}")
    z = x.double() @ w.double().t().contiguous()
    assert torch.equal(tbs.linear(x, w), z.to(dt))
    assert torch.equal(tbs.linear(x, w, residual=r, activation="relu", residual_after=True),
                       (torch.relu(z) + r.double()).to(dt))
    got = tbs.linear_backward(g, x, w)
    gt = g.double().t().contiguous()
    assert torch.equal(got.x, (g.double() @ w.double()).to(dt))
    assert torch.equal(got.weight, (gt @ x.double()).to(dt))
    assert torch.equal(got.bias, gt.sum(1).to(dt))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (3, 1), (8, 0), (6, 2)])
def test_strides_and_alignment(dtype, pad, offset):
    """Rows further apart than their width, starting at any element; what lies between the
    rows (NaN here) is not used."""
    import torch
    from paper_2211_00484_amd import tbs
    dt = _t(dtype)

    def spread(t):
        rows, cols = t.shape
        buf = torch.full((rows * (cols + pad) + offset,), math.nan, dtype=dt, device="cuda")
        v = buf[offset:].view(rows, cols + pad)[:, :cols]
        v.copy_(t)
        return v

    for M, K, N in ((70, 96, 130), (5, 130, 40), (300, 75, 66)):
        x, w, g, r = (_ints(s, dtype, i) for i, s in enumerate(((M, K), (N, K), (M, N), (M, N))))
        xs, ws, gs, rs = (spread(t) for t in (x, w, g, r))
        want = tbs.linear(x, w, residual=r)
        assert torch.equal(want, (x.double() @ w.double().t().contiguous() + r.double()).to(dt))
        assert torch.equal(tbs.linear(xs, ws, residual=rs), want)
        a, b = tbs.linear_backward(g, x, w), tbs.linear_backward(gs, xs, ws)
        p = tbs.linear_backward(gs, xs, ws, pre=rs, activation="relu", want_pre=True)
        q = tbs.linear_backward(g, x, w, pre=r, activation="relu", want_pre=True)
        for name in ("x", "weight", "bias"):
            assert torch.equal(getattr(a, name), getattr(b, name)), name
            assert torch.equal(getattr(p, name), getattr(q, name)), name
        # columns as rows: copied
        assert torch.equal(tbs.linear(x.t().contiguous().t(), ws), tbs.linear(x, w))


@pytest.mark.parametrize("dtype", DTYPES)
def test_output_rows(dtype):
    """The C entry writes its rows and nothing between or behind them."""
    import torch
    from paper_2211_00484_amd import tbs
    L, dt = tbs.lib(), _t(dtype)
    code = {"float32": 0, "bfloat16": 1, "float16": 2}[dtype]
    for M, K, N, ld in ((70, 40, 61, 67), (9, 100, 33, 40), (200, 520, 130, 131)):
        x, w, g = _ints((M, K), dtype, 1), _ints((N, K), dtype, 2), _ints((M, N), dtype, 3)
        p = lambda t: ctypes.c_void_p(t.data_ptr())
        new = lambda rows, l: torch.full((rows + 2, l), -77.0, dtype=dt, device="cuda")
        out, pre, dx, dw = new(M, ld), new(M, ld), new(M, K + 3), new(N, K + 3)
        n = L.tbs_linear_workspace(code, M, N, K)
        n2 = L.tbs_linear_backward_workspace(code, 0, M, N, K, 1, 1, 0, 0)
        ws = torch.full((max(n, n2, 16) + 64,), 0xA5, dtype=torch.uint8, device="cuda")
        st = tbs._stream_ptr()
        assert L.tbs_linear(code, p(x), K, p(w), K, None, None, 0, 0, 0, M, N, K, p(out), ld,
                            p(pre), ld, p(ws), n, st) == 0
        assert (ws[n:] == 0xA5).all()
        assert L.tbs_linear_backward(code, p(g), N, p(x), K, p(w), K, None, 0, 0, M, N, K, p(dx),
                                     K + 3, p(dw), K + 3, None, None, 0, p(ws), n2, st) == 0
        assert (ws[max(n, n2):] == 0xA5).all()
        z = x.double() @ w.double().t().contiguous()
        for o, want, cols in ((out, z, N), (pre, z, N), (dx, g.double() @ w.double(), K),
                              (dw, g.double().t().contiguous() @ x.double(), K)):
            rows = want.shape[0]
            assert torch.equal(o[:rows, :cols], want.to(dt))
            assert (o[rows:] == -77.0).all() and (o[:, cols:] == -77.0).all()


def test_leading_dimensions_and_empty_batches():
    import torch
    from paper_2211_00484_amd import tbs
    x, w, b, _, _ = _inputs(60, 24, 10, "float32", 1)
    out = tbs.linear(x.view(3, 4, 5, 24), w, b)
    assert out.shape == (3, 4, 5, 10) and torch.equal(out.view(60, 10), tbs.linear(x, w, b))
    assert torch.equal(tbs.linear(x[0], w, b), tbs.linear(x[:1], w, b)[0])
    e = x[:0]
    assert tbs.linear(e, w, b).shape == (0, 10)
    got = tbs.linear_backward(torch.zeros((0, 10), device="cuda"), e, w)
    assert got.x.shape == (0, 24) and (got.weight == 0).all() and (got.bias == 0).all()
    got = tbs.linear_backward(torch.zeros((0, 10), device="cuda"), e, w, activation="tanh",
                              pre=torch.zeros((0, 10), device="cuda"), want_pre=True)
    assert (got.weight == 0).all() and (got.bias == 0).all() and got.pre.shape == (0, 10)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K,N", [(5, 100, 37), (130, 100, 70)])
def test_special_values_stay_in_their_rows(dtype, M, K, N):
    """An infinity or NaN in a row of x, w or dz reaches that row's (column's) results."""
    import torch
    from paper_2211_00484_amd import tbs
    x, w, _, _, g = _inputs(M, K, N, dtype, 3)
    clean = tbs.linear(x, w)
    x2 = x.clone()
    x2[1, K - 1] = math.nan
    x2[3, 0] = math.inf
    out = tbs.linear(x2, w)
    assert torch.isnan(out[1]).all()
    want = (x2[3:4].double() @ w.double().t().contiguous())[0]
    assert torch.equal(out[3].double(), want)
    keep = [m for m in range(M) if m not in (1, 3)]
    assert torch.equal(out[keep], clean[keep])
    w2 = w.clone()
    w2[N - 1, K - 1] = math.nan
    out = tbs.linear(x, w2)
    assert torch.isnan(out[:, N - 1]).all() and torch.equal(out[:, :N - 1], clean[:, :N - 1])
    ref = tbs.linear_backward(g, x, w)
    g2 = g.clone()
    g2[2, N - 1] = math.nan
    got = tbs.linear_backward(g2, x, w)
    keep = [m for m in range(M) if m != 2]
    assert torch.isnan(got.x[2]).all() and torch.equal(got.x[keep], ref.x[keep])
    assert torch.isnan(got.weight[N - 1]).all() and torch.isnan(got.bias[N - 1])
    assert torch.equal(got.weight[:N - 1], ref.weight[:N - 1])
    assert torch.equal(got.bias[:N - 1], ref.bias[:N - 1])


def test_activations_at_the_ends():
    """Values of any size through each activation and its slope (x = 1, w = 1: z = bias)."""
    import torch
    from paper_2211_00484_amd import tbs
    v = [0.0, -0.0, 1e-30, -1e-30, 1e-4, -1e-4, 0.2, 0.2499, 0.25, 0.2501, 0.5, -0.7, 1.0, 3.0, -4.0, 8.0,
         -9.5, 20.0, -30.0, 87.0, -87.0, 89.0, -89.0, 200.0, -200.0, 1e10, -1e10, math.inf]
    z = torch.tensor(v, device="cuda")
    one = torch.zeros((1, 1), device="cuda")
    w = torch.zeros((len(v), 1), device="cuda")
    for act in ACTS:
        out = tbs.linear(one, w, z, activation=act)[0].double()
        want = _act64(z.double(), act)
        fin = torch.isfinite(want)
        assert torch.equal(out[~fin], want[~fin]), act
        # silu: a sigmoid below 2^-126 (z < -87.3) may be taken as 0, which costs 2^-126 |z|;
        # from z = -104 on its value is below fp32's smallest
        under = 2.0 ** -126 * z[fin].double().abs().clamp(max=104.0)
        assert ((out - want).abs()[fin] <= 1e-6 * want[fin].abs() + under).all() or act == "gelu", act
        if act == "gelu":  # (1 + erf loses its small part for z well below 0)
            assert ((out - want).abs()[fin] <= 1e-6 * want[fin].abs() + 2e-7 * z[fin].abs()).all()
        if act == "none":
            continue
        zz = z[:-1]
        g = torch.ones((1, len(v) - 1), device="cuda")
        got = tbs.linear_backward(g, one, w[:-1], pre=zz[None], activation=act, want_pre=True).pre[0]
        s = _slope64(zz.double(), act)
        if act == "relu":
            s = (zz > 0).double()
        assert ((got.double() - s).abs() <= 2e-6).all(), act


def test_far_rows():
    """Rows whose offsets pass 32 bits (in elements and in bytes)."""
    import torch
    from paper_2211_00484_amd import tbs
    M, K, N, ld = 40000, 64, 48, 65544
    buf = torch.empty(M * ld, dtype=torch.bfloat16, device="cuda")
    x = buf.view(M, ld)[:, :K]
    x.copy_(_ints((M, K), "bfloat16", 1, 2))
    w = _ints((N, K), "bfloat16", 2, 2)
    xd = x.contiguous()
    assert torch.equal(tbs.linear(x, w), tbs.linear(xd, w))
    g = buf.view(M, ld)[:, 128:128 + N]
    g.copy_(_ints((M, N), "bfloat16", 3, 2))
    a, b = tbs.linear_backward(g, x, w), tbs.linear_backward(g.contiguous(), xd, w)
    want = xd[-100:].double() @ w.double().t().contiguous()
    assert torch.equal(tbs.linear(x, w)[-100:], want.to(torch.bfloat16))
    for name in ("x", "weight", "bias"):
        assert torch.equal(getattr(a, name), getattr(b, name))


def test_in_place_residual():
    import torch
    from paper_2211_00484_amd import tbs
    L = tbs.lib()
    for M, K, N in ((7, 64, 50), (300, 64, 200), (64, 2048, 64)):
        x, w, b, r, _ = _inputs(M, K, N, "bfloat16", 2)
        want = tbs.linear(x, w, b, residual=r, activation="silu", residual_after=True)
        n = L.tbs_linear_workspace(1, M, N, K)
        ws = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
        p = lambda t: ctypes.c_void_p(t.data_ptr())
        assert L.tbs_linear(1, p(x), K, p(w), K, p(b), p(r), N, 1, 3, M, N, K, p(r), N, None, 0,
                            p(ws), n, tbs._stream_ptr()) == 0
        assert torch.equal(r, want)


@pytest.mark.parametrize("dtype", DTYPES)
def test_gradients_against_differences(dtype):
    """Along random directions, the change of sum(out * g) in 64 bits over a step each way;
    its own error is of the third order in the step."""
    import torch
    from paper_2211_00484_amd import tbs
    M, K, N, h = 40, 30, 21, 1e-4
    x, w, b, r, g = _inputs(M, K, N, dtype, 77)
    for act in ACTS:
        if act == "relu":
            continue  # (its kink is met by some of the steps)
        out, pre = tbs.linear(x, w, b, residual=r, activation=act, want_pre=True)
        got = tbs.linear_backward(g, x, w, pre=None if act == "none" else pre, activation=act,
                                  want_pre=True)
        f = lambda x, w, b, r: (_act64(x @ w.t() + b + r, act) * g.double()).sum()
        at = [t.double() for t in (x, w, b, r)]
        for i, name in enumerate(("x", "weight", "bias", "pre")):
            d = torch.randn(at[i].shape, dtype=torch.float64, device="cuda")
            up = [t + h * d if j == i else t for j, t in enumerate(at)]
            dn = [t - h * d if j == i else t for j, t in enumerate(at)]
            want = ((f(*up) - f(*dn)) / (2 * h)).item()
            have = (getattr(got, name).double() * d).sum().item()
            # every term of the sum is off by the roundings of its gradient and of the
            # pre-activation (whose slope changes by at most 1.1 of it)
            size = (getattr(got, name).double().abs() * d.abs()).sum().item()
            spread = (g.double().abs().sum() * d.abs().max()).item() * (3 if i < 2 else 1)
            assert abs(have - want) <= 8 * _half(x.dtype) * (size + 0.2 * spread) + 1e-5 * spread, (act, name)
