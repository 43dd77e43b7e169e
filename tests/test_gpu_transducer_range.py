"""Gradients of transducer log-likelihoods: where the values that stand for no share, 0 and NaN, are
written."""
import numpy as np
import pytest

from test_gpu_transducer_gradient import KINDS, _inputs, _run

pytestmark = pytest.mark.gpu


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
