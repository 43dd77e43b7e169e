"""Gradients of transducer log-likelihoods: where the values that stand for no share, 0 and NaN, are
written, and totals far from 0: 0 below -1e8, NaN above 1e8, and between
them those of the definition, whether one input or a sum of many leads there.

Tolerance as in test_gpu_transducer_gradient (16 2^-24 of a share), and for the reference, which
takes exponentials of differences of numbers of up to 1.8e8 in 64 bits, 2^-53 of that for each of
its 3 (T + U) roundings."""
import numpy as np
import pytest

from gpu_util import say
from test_gpu_transducer_gradient import KINDS, REL, _inputs, _run, reference

pytestmark = pytest.mark.gpu

LIMIT = 1e8


def _expect(kind, blank, label, frames, labels):
    """Checks every utterance and returns how many have each outcome (0, share, NaN)."""
    B, T, U1 = blank.shape
    total, gb, gl, status = _run(kind, blank, label, frames, labels)
    t, wb, wl = reference(kind, blank, label, frames, labels)
    say(f"transducer range {kind} T={T} U={U1 - 1}: totals {[float('%.4g' % v) for v in t]}")
    assert (status == 0).all()
    rel = REL + 3 * (T + U1) * 1.8e8 * 2.0 ** -53
    seen = [0, 0, 0]
    for b in range(B):
        assert total[b] == t[b] or abs(total[b] - t[b]) <= 1e-9 * abs(t[b]) + 1e-9
        ins = np.s_[:frames[b], :labels[b] + 1], np.s_[:frames[b], :labels[b]]
        for g, w, i in ((gb[b], wb[b], ins[0]), (gl[b], wl[b], ins[1])):
            if t[b] < -LIMIT:
                assert (g == 0).all(), (b, t[b])
            elif t[b] > LIMIT:
                assert np.isnan(g[i]).all(), (b, t[b])
                g[i] = 0.0
                assert (g == 0).all()
            else:
                assert np.isfinite(g).all(), (b, t[b])
                assert (np.abs(g - w) <= rel * np.abs(w) + 1e-30).all(), (b, t[b], g, w)
        seen[0 if t[b] < -LIMIT else 2 if t[b] > LIMIT else 1] += 1
    return seen


VALUES = [0.4e8, 0.9e8, 0.99e8, 1.2e8, 1.5e8, 1.7e8, 1.9e8, 3e8, 1e12]


@pytest.mark.parametrize("kind", KINDS)
def test_one_cell(kind):
    """A single frame without labels: the input is the total and its share 1."""
    v = np.array(VALUES + [-x for x in VALUES] + [1e8, -1e8, -100000024.0, 100000024.0, -1e-3], np.float32)
    blank = v[:, None, None].copy()
    n = len(v)
    seen = _expect(kind, blank, np.zeros((n, 1, 0), np.float32), np.ones(n, np.int32), np.zeros(n, np.int32))
    assert seen == [7, 9, 7]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,U", [(6, 2), (40, 12), (3, 130)])
def test_one_frame_and_many(kind, T, U):
    """Totals near and beyond the limits from one frame whose inputs are all far off, and from
    all frames a little."""
    blank, label, frames, labels = _inputs(T + U, 2 * len(VALUES) * 2, T, U)
    frames[:], labels[:] = T, min(T, U)
    if kind == "standard":
        labels[:] = U
    for i, v in enumerate(VALUES + [-x for x in VALUES]):
        for x in (blank, label):
            x[2 * i, T // 2] += v
            x[2 * i + 1] += v / T
    assert all(_expect(kind, blank, label, frames, labels))


@pytest.mark.parametrize("kind", ["standard", "modified"])
def test_far_and_back(kind):
    """Inputs and scores beyond the limits whose total is not: one frame far off, a later one
    back (no label is taken in either, so that every path has both)."""
    T, U = 9, 3
    pairs = [(-1.5e8, 0.8e8), (-1.7e8, 1.6e8), (1.5e8, -1.2e8), (1.7e8, -1.7e8), (0.9e8, -1.8e8)]
    blank, label, frames, labels = _inputs(4, len(pairs), T, U)
    frames[:], labels[:] = T, U
    for b, (x, y) in enumerate(pairs):
        for t, v in ((2, x), (5, y)):
            blank[b, t] += np.float32(v)
            label[b, t] = -np.inf
    seen = _expect(kind, blank, label, frames, labels)
    assert seen == [0, len(pairs), 0]


@pytest.mark.parametrize("kind", KINDS)
def test_far_inputs_keep_their_digits(kind):
    """Shares of inputs of up to 9e7 are as exact as others (in eq. (2) blank and label are alike,
    so that neither is certain)."""
    B, T, U = 6, 5, 2
    blank, label, frames, labels = _inputs(8, B, T, U)
    frames[:], labels[:] = T, U
    for b, v in enumerate([2e4, 1e6, 1.2e7, 3e7, -4e7, -9e7]):
        for x in (blank, label):
            x[b, 1] = np.float32(v) + np.float32(8.0) * np.arange(x.shape[2], dtype=np.float32)
    _expect(kind, blank, label, frames, labels)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,U", [(8, 5), (30, 140)])
def test_nan_inside_the_lengths_only(kind, T, U):
    """An utterance of fewer frames and labels than the batch has, with a total of NaN: NaN in all
    of its cells, 0 in all others."""
    blank, label, frames, labels = _inputs(T, 3, T, U)
    frames[:], labels[:] = [T, T - 2, 1], [min(T, U), 3, 0]
    blank[1:, 0, 0] = np.nan
    total, gb, gl, status = _run(kind, blank, label, frames, labels)
    assert np.isfinite(total[0]) and np.isnan(total[1:]).all() and (status == 0).all()
    assert np.isfinite(gb[0]).all() and np.isfinite(gl[0]).all()
    for b in (1, 2):
        inside = np.zeros(gb[b].shape, bool), np.zeros(gl[b].shape, bool)
        inside[0][:frames[b], :labels[b] + 1] = True
        inside[1][:frames[b], :labels[b]] = True
        for g, i in zip((gb[b], gl[b]), inside):
            assert np.isnan(g[i]).all() and (g[~i] == 0).all()
