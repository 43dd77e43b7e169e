"""Gradient of the transducer log-likelihoods (tbs_transducer_gradient) against automatic
differentiation of the recursions in 64 bits, and against differences of tbs_transducer_forward.

Tolerance: a share is a product of four fp32 mantissas and an exponential, each within two
steps of 2^-24, in four products and a rounding: 16 2^-24 = 1e-6 of it; what an unlikely cell
loses to a likely one in the recursions (2^-50 of the whole) is nothing in fp32."""
import math

import numpy as np
import pytest

from gpu_util import say

pytestmark = pytest.mark.gpu

KINDS = ["standard", "modified", "constrained"]
REL = 1e-6


def reference(kind, blank, label, frames, labels):
    """total [B] and the derivatives of their sum, in 64 bits on the CPU."""
    import torch
    bl = torch.from_numpy(np.asarray(blank, np.float64)).requires_grad_(True)
    lb = torch.from_numpy(np.asarray(label, np.float64)).requires_grad_(True)
    low = -1e30
    total = []
    for b in range(bl.shape[0]):
        T, U = int(frames[b]), int(labels[b])
        # where an input is -inf the path is impossible: a large negative number keeps
        # differences of infinities out, and carries no weight
        x = bl[b, :T, :U + 1].clamp(min=low)
        y = lb[b, :T, :U].clamp(min=low)
        wall = torch.full((1,), low, dtype=torch.float64)
        a = torch.cat([torch.zeros(1, dtype=torch.float64), wall.expand(U)])
        if kind == "standard":
            for t in range(T):
                come = a if t == 0 else a + x[t - 1]
                row = [come[0]]
                for u in range(1, U + 1):
                    v = row[-1] + y[t, u - 1]
                    row.append(v if t == 0 else torch.logaddexp(come[u], v))
                a = torch.stack(row)
            total.append(a[U] + x[T - 1, U])
        else:
            for t in range(T):
                up = torch.cat([wall, a[:U] + y[t]])
                if kind == "constrained":
                    up = up + x[t]
                a = torch.logaddexp(a + x[t], up)
            total.append(a[U])
    total = torch.stack(total)
    gb, gl = torch.autograd.grad(total.sum(), [bl, lb], allow_unused=True)
    gl = torch.zeros_like(lb) if gl is None else gl
    total = total.detach().numpy().copy()
    gb, gl = gb.numpy().copy(), gl.numpy().copy()
    none = total < 0.5 * low
    total[none], gb[none], gl[none] = -math.inf, 0.0, 0.0
    return total, gb, gl


def _inputs(seed, B, T, U, lo=0.01):
    rng = np.random.default_rng(seed)
    blank = np.log(rng.uniform(lo, 1.0, size=(B, T, U + 1))).astype(np.float32)
    label = np.log(rng.uniform(lo, 1.0, size=(B, T, U))).astype(np.float32)
    frames = rng.integers(1, T + 1, size=B).astype(np.int32)
    labels = rng.integers(0, U + 1, size=B).astype(np.int32)
    frames[0], labels[0] = T, U
    return blank, label, frames, labels


def _run(kind, blank, label, frames, labels, weights=None):
    import torch
    from paper_2211_00484_amd import tbs
    w = None if weights is None else torch.tensor(weights, dtype=torch.float64, device="cuda")
    out = tbs.transducer_gradient(kind, torch.from_numpy(blank).cuda(), torch.from_numpy(label).cuda(),
                                  np.stack([frames, labels], 1), weights=w)
    return [o.cpu().numpy() for o in out]


def _close(got, want, what):
    err = np.abs(got.astype(np.float64) - want) - (REL * np.abs(want) + 1e-30)
    assert np.isfinite(got).all(), what
    if err.size:
        i = np.unravel_index(err.argmax(), err.shape)
        assert err[i] <= 0, (what, i, got[i], want[i])


def _check(kind, blank, label, frames, labels, weights=None):
    B, T, U1 = blank.shape
    say(f"transducer gradient {kind} B={B} T={T} U={U1 - 1}")
    total, gb, gl, status = _run(kind, blank, label, frames, labels, weights)
    t, wb, wl = reference(kind, blank, label, frames, labels)
    assert (status == 0).all()
    w = np.ones(B) if weights is None else np.asarray(weights)
    fin = np.isfinite(t)
    assert np.array_equal(total[~fin], t[~fin])
    assert np.allclose(total[fin], t[fin], rtol=1e-9, atol=1e-9)
    _close(gb, wb * w[:, None, None], "blank")
    _close(gl, wl * w[:, None, None], "label")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("B,T,U", [
    (3, 1, 0), (3, 1, 1), (4, 2, 1), (4, 2, 2), (5, 7, 3), (4, 16, 12), (4, 17, 16), (3, 33, 31), (2, 20, 63),
    (2, 66, 64), (2, 40, 130), (1, 5, 300)])
def test_against_differentiation(kind, B, T, U):
    """Ragged utterances; for (2) and (3) some with more labels than frames (no path)."""
    blank, label, frames, labels = _inputs(B + T + U, B, T, U)
    _check(kind, blank, label, frames, labels)
    _check(kind, blank, label, frames, np.minimum(labels, frames))


@pytest.mark.parametrize("kind", ["modified", "constrained"])
@pytest.mark.parametrize("B,T,U", [(2, 260, 255), (1, 300, 256), (1, 1030, 1023), (300, 20, 18), (520, 9, 7)])
def test_wide_and_many(kind, B, T, U):
    blank, label, frames, labels = _inputs(T, B, T, U)
    _check(kind, blank, label, frames, np.minimum(labels, frames))


@pytest.mark.parametrize("B,T,U", [(300, 12, 9), (520, 6, 5), (1, 12, 400), (1, 3, 1023)])
def test_wide_and_many_standard(B, T, U):
    blank, label, frames, labels = _inputs(T, B, T, U)
    _check("standard", blank, label, frames, labels)


@pytest.mark.parametrize("kind", ["modified", "constrained"])
@pytest.mark.parametrize("T,U", [(70, 64), (90, 65), (130, 127), (129, 128), (210, 190), (230, 192), (250, 200),
                                 (260, 206), (270, 207), (300, 255), (500, 470), (530, 511), (520, 512)])
def test_chain_splits(kind, T, U):
    """Few utterances: one to four waves side by side, one to sixteen cells a lane; ragged ones
    whose labels end inside any wave, and inputs that the linear domain does not take."""
    blank, label, frames, labels = _inputs(T + U, 4, T, U)
    labels = np.minimum(labels, frames)
    labels[1] = min(63, frames[1])
    blank[2, frames[2] // 2, labels[2] // 2] = -np.inf
    label[3, :, labels[3] // 2] = -400.0
    _check(kind, blank, label, frames, labels)


@pytest.mark.parametrize("kind", KINDS)
def test_likely_paths_and_weights(kind):
    """Inputs as a trained model gives them (a few cells carry the path, the rest are steep),
    with an upstream gradient per utterance."""
    rng = np.random.default_rng(3)
    B, T, U = 6, 70, 24
    t, u = np.arange(T)[None, :, None], np.arange(U + 1)[None, None, :]
    s = 6.0 - 1.5 * np.abs(t - (u + 0.5) * T / (U + 1)) + rng.normal(size=(B, T, U + 1))
    blank = (-np.logaddexp(0, s)).astype(np.float32)
    label = (-np.logaddexp(0, -s))[:, :, :U].astype(np.float32)
    frames, labels = np.array([70, 60, 70, 33, 50, 24], np.int32), np.array([24, 20, 0, 24, 1, 24], np.int32)
    _check(kind, blank, label, frames, labels, weights=[-1.0, 0.5, 2.0, 0.0, -1e-3, 1e4])


@pytest.mark.parametrize("kind", KINDS)
def test_long_utterances(kind):
    """Scores of tens of thousands: shares keep their digits."""
    blank, label, frames, labels = _inputs(9, 2, 900, 12, lo=1e-30)
    _check(kind, blank, label, frames, labels)


@pytest.mark.parametrize("kind", KINDS)
def test_impossible_and_steep_inputs(kind):
    blank, label, frames, labels = _inputs(5, 9, 40, 12)
    frames[:], labels[:] = 40, 12
    blank[0] -= 290.0
    label[1] = -299.0
    label[2, :, 3] = -np.inf             # no path
    blank[3, 7, 2] = -np.inf
    label[4, 5, 5] = 100.0
    blank[5, :, 1:] = -np.inf
    label[6, 3:9] = -np.inf
    blank[7] = -5000.0
    label[8, :, 4] = -1e6
    _check(kind, blank, label, frames, labels)


@pytest.mark.parametrize("kind", KINDS)
def test_nan_and_padding(kind):
    """A NaN that is read makes its utterance's gradients NaN and no other's; cells outside the
    lengths are not read, and their gradients are 0."""
    blank, label, frames, labels = _inputs(6, 4, 30, 10)
    frames[:], labels[:] = [30, 20, 25, 30], [10, 7, 10, 10]
    clean = _run(kind, blank, label, frames, labels)
    blank[2, 11, 4] = np.nan
    for b in range(4):
        blank[b, frames[b]:], blank[b, :, labels[b] + 1:] = np.nan, np.nan
        label[b, frames[b]:], label[b, :, labels[b]:] = np.nan, np.nan
    got = _run(kind, blank, label, frames, labels)
    for b in range(4):
        ins = np.s_[b, :frames[b], :labels[b] + 1], np.s_[b, :frames[b], :labels[b]]
        for g, c, i in zip(got[1:3], clean[1:3], ins):
            if b == 2:
                assert np.isnan(g[i]).all()
                g[i] = 0.0
                assert (g[b] == 0).all()
            else:
                assert np.array_equal(g[b], c[b])
    assert np.isnan(got[0][2]) and np.isfinite(np.delete(got[0], 2)).all()


@pytest.mark.parametrize("kind", KINDS)
def test_bad_lengths(kind):
    blank, label, _, _ = _inputs(7, 5, 9, 4)
    total, gb, gl, status = _run(kind, blank, label, np.array([9, 0, 10, 9, 9], np.int32),
                                 np.array([4, 1, 2, -1, 5], np.int32))
    assert status.tolist() == [0, 1, 1, 1, 1] and np.isnan(total[1:]).all()
    assert (gb[1:] == 0).all() and (gl[1:] == 0).all() and (gb[0] != 0).any()


@pytest.mark.parametrize("kind", KINDS)
def test_against_differences(kind):
    """Totals are within 1e-9; inputs move by h (as fp32 holds it), whose third order is h^2."""
    import torch
    from paper_2211_00484_amd import tbs
    blank, label, frames, labels = _inputs(12, 3, 25, 9)
    labels = np.minimum(labels, frames)
    _, gb, gl, _ = _run(kind, blank, label, frames, labels)
    lens = np.stack([frames, labels], 1)
    f = lambda b, l: tbs.transducer_forward(kind, torch.from_numpy(b).cuda(), torch.from_numpy(l).cuda(),
                                            lens)[0].cpu().numpy()
    rng = np.random.default_rng(1)
    h = 2.0 ** -7
    for x, g, which in ((blank, gb, 0), (label, gl, 1)):
        for _ in range(12):
            i = tuple(rng.integers(0, n) for n in x.shape)
            up, dn = x.copy(), x.copy()
            up[i] += h
            dn[i] -= h
            a, b = ((up, label), (dn, label)) if which == 0 else ((blank, up), (blank, dn))
            step = float(up[i]) - float(dn[i])
            d = (f(*a)[i[0]] - f(*b)[i[0]]) / step
            assert abs(d - g[i]) <= h * h + 1e-6, (i, d, g[i])


def test_same_bits_and_other_stream():
    import torch
    from paper_2211_00484_amd import tbs
    blank, label, frames, labels = _inputs(4, 40, 90, 30)
    labels = np.minimum(labels, frames)
    bl, lb = torch.from_numpy(blank).cuda(), torch.from_numpy(label).cuda()
    lens = torch.from_numpy(np.stack([frames, labels], 1)).cuda()
    s = torch.cuda.Stream()
    for kind in KINDS:
        a = tbs.transducer_gradient(kind, bl, lb, lens)
        torch.cuda.synchronize()
        b = tbs.transducer_gradient(kind, bl, lb, lens, stream=s)
        s.synchronize()
        c = tbs.transducer_forward(kind, bl, lb, lens)
        for x, y in zip(a, b):
            assert torch.equal(x, y)
        assert torch.allclose(a[0], c[0], rtol=1e-12, atol=1e-9)
        # rows that are not contiguous are copied
        t = lambda v: v.transpose(0, 1).contiguous().transpose(0, 1)
        for x, y in zip(a, tbs.transducer_gradient(kind, t(bl), t(lb), lens)):
            assert torch.equal(x, y)
