"""Linear layers and their gradients in each of the large tiles, not split (256 CUs: 16-bit 256 x 256
from 192 such tiles on, 16-bit 128 x 128 from 256, fp32 128 x 128 from 1,024), with operands that
are copied directly and operands that are not (odd rows of 16-bit values, fp32 rows 2^20 apart).

Small integers: every sum is exact in fp32, so results are the exact ones rounded once.  Every
shape has tiles inside the result and cut by its edge, and a last slice that is not whole."""
import pytest

from gpu_util import say
from test_gpu_linear import _check_forward, _inputs, _ints, _t

pytestmark = pytest.mark.gpu

CODES = {"float32": 0, "bfloat16": 1, "float16": 2}
# (rows, columns of the result, terms): tiles of 256, 128, and fp32 of 128
SHAPES = [(16200, 1000, 200, "bfloat16"), (16200, 1000, 201, "float16"), (16200, 1001, 201, "bfloat16"),
          (4000, 1100, 500, "float16"), (4000, 1101, 499, "bfloat16"), (16500, 1030, 70, "float32"),
          (16500, 1031, 69, "float32")]


def _spread(t, ld):
    """t in rows of ld elements."""
    import torch
    v = torch.empty((t.shape[0] - 1) * ld + t.shape[1], dtype=t.dtype, device="cuda").as_strided(t.shape, (ld, 1))
    v.copy_(t)
    return v


def _mm(a, b):
    """a b of integers in fp64, in blocks of rows (and b contiguous)."""
    import torch
    b = b.double().contiguous()
    return torch.cat([r.double() @ b for r in a.split(4096)])


@pytest.mark.parametrize("M,N,K,dtype", SHAPES)
def test_forward(M, N, K, dtype):
    import torch
    from paper_2211_00484_amd import tbs
    dt = _t(dtype)
    assert tbs.lib().tbs_linear_workspace(CODES[dtype], M, N, K) == 0
    x, w, b, r = (_ints(s, dtype, i) for i, s in enumerate(((M, K), (N, K), (1, N), (M, N))))
    b = b[0]
    z = _mm(x, w.t())
    ws = _spread(w, 1 << 20) if dtype == "float32" else _spread(w, K + 2)
    for wi in (w, ws):
        say(f"linear {M} x {K} x {N} {dtype}, rows of {wi.stride(0)}")
        assert torch.equal(tbs.linear(x, wi), z.to(dt))
        for res, after in ((None, False), (r, False), (r, True), (r[0], False), (r[0], True)):
            add = 0 if res is None else res.double()
            pre = z + b.double() + (0 if after else add)
            for act, y in (("none", pre), ("relu", torch.relu(pre))):
                out, p = tbs.linear(x, wi, b, residual=res, activation=act, residual_after=after, want_pre=True)
                assert torch.equal(out, (y + (add if after else 0)).to(dt)), (act, after)
                assert torch.equal(p, pre.to(dt)), (act, after)
                assert torch.equal(out, tbs.linear(x, wi, b, residual=res, activation=act, residual_after=after))


@pytest.mark.parametrize("M,N,K,dtype", SHAPES)
@pytest.mark.parametrize("act", ["tanh", "silu", "gelu"])
def test_activations(M, N, K, dtype, act):
    from paper_2211_00484_amd import tbs
    x, w, b, r, _ = _inputs(M, K, N, dtype, M + N)
    out, pre = tbs.linear(x, w, b, residual=r, activation=act, want_pre=True)
    _check_forward(x, w, b, r, act, False, out, pre)
    out = tbs.linear(x, w, b, residual=r, activation=act, residual_after=True)
    _check_forward(x, w, b, r, act, True, out, None)


@pytest.mark.parametrize("M,K,N,dtype", SHAPES)
def test_gradient_of_the_input(M, K, N, dtype):
    import torch
    from paper_2211_00484_amd import tbs
    assert tbs.lib().tbs_linear_backward_workspace(CODES[dtype], 0, M, N, K, 1, 0, 0, 0) == 0
    x, w, g = (_ints(s, dtype, i) for i, s in enumerate(((M, K), (N, K), (M, N))))
    want = _mm(g, w).to(_t(dtype))
    for wi in (w, _spread(w, 1 << 20) if dtype == "float32" else _spread(w, K + 2)):
        say(f"dx {M} x {K} x {N} {dtype}, rows of {wi.stride(0)}")
        got = tbs.linear_backward(g, x, wi, want_weight=False, want_bias=False)
        assert torch.equal(got.x, want)
        got = tbs.linear_backward(g, x, wi, pre=g, activation="relu", want_weight=False, want_bias=False)
        assert torch.equal(got.x, _mm(torch.relu(g), w).to(_t(dtype)))


@pytest.mark.parametrize("N,K,M,dtype", [(4000, 4000, 200, "bfloat16"), (4000, 4001, 201, "float16"),
                                         (4001, 4000, 201, "bfloat16"), (4000, 1100, 500, "float16"),
                                         (4001, 1101, 499, "bfloat16"), (4100, 4100, 70, "float32"),
                                         (4101, 4103, 69, "float32")])
def test_gradients_of_weight_and_bias(N, K, M, dtype):
    import torch
    from paper_2211_00484_amd import tbs
    assert tbs.lib().tbs_linear_backward_workspace(CODES[dtype], 0, M, N, K, 0, 1, 1, 0) == 0
    x, w, g = (_ints(s, dtype, i) for i, s in enumerate(((M, K), (N, K), (M, N))))
    gt = g.t().contiguous()
    want, bias = _mm(gt, x).to(_t(dtype)), gt.double().sum(1).to(_t(dtype))
    for xi in (x, _spread(x, 1 << 20) if dtype == "float32" else _spread(x, K + 2)):
        say(f"dw {N} x {K} x {M} {dtype}, rows of {xi.stride(0)}")
        got = tbs.linear_backward(g, xi, w, want_x=False)
        assert torch.equal(got.weight, want) and torch.equal(got.bias, bias)
