"""Refusals of the joiner's operators, all made on the host before any device work: the C
entries with NULL or made-up pointers (never used), and the binding's own checks."""
import ctypes
import math

import numpy as np
import pytest

from paper_2211_00484_amd import tbs

EINVAL, ECAPACITY = -1, -4
P = ctypes.c_void_p(4096)       # stands for a device pointer; no call here gets as far as using it


def _message():
    return tbs.lib().tbs_last_error().decode()


LINEAR = dict(dtype=0, x=P, ldx=8, w=P, ldw=8, bias=None, residual=None, ldr=0, after=0, act=0, M=4, N=6,
              K=8, out=P, ldo=6, pre=None, ldp=0, ws=None, nbytes=0)


@pytest.mark.parametrize("change,status,fragment", [
    (dict(dtype=3), EINVAL, "dtype"), (dict(dtype=-1), EINVAL, "dtype"),
    (dict(act=5), EINVAL, "activation"), (dict(act=-1), EINVAL, "activation"),
    (dict(M=-1), EINVAL, "M >= 0"), (dict(N=0), EINVAL, "N >= 1"), (dict(K=0), EINVAL, "K >= 1"),
    (dict(x=None), EINVAL, "NULL"), (dict(w=None), EINVAL, "NULL"), (dict(out=None), EINVAL, "NULL"),
    (dict(ldx=7), EINVAL, "row length"), (dict(ldw=7), EINVAL, "row length"),
    (dict(ldo=5), EINVAL, "row length"), (dict(residual=P, ldr=5), EINVAL, "row length"),
    (dict(pre=P, ldp=5), EINVAL, "row length"), (dict(ldx=-8), EINVAL, "row length"),
    (dict(M=2 ** 31 - 1, N=2 ** 20, ldo=2 ** 20), ECAPACITY, "too large"),
])
def test_linear_refusals(change, status, fragment):
    a = dict(LINEAR, **change)
    assert tbs.lib().tbs_linear(*a.values(), None) == status
    assert fragment in _message()


def test_linear_empty_batch_needs_no_pointers():
    assert tbs.lib().tbs_linear(*dict(LINEAR, M=0, x=None, w=None, out=None).values(), None) == 0


BACKWARD = dict(dtype=0, g=P, ldg=6, x=P, ldx=8, w=P, ldw=8, pre=P, ldp=6, act=2, M=4, N=6, K=8, dx=P, lddx=8,
                dw=P, lddw=8, db=P, dz=P, lddz=6, ws=P, nbytes=1 << 30)


@pytest.mark.parametrize("change,status,fragment", [
    (dict(dtype=7), EINVAL, "dtype"), (dict(act=9), EINVAL, "activation"), (dict(M=-3), EINVAL, "M >= 0"),
    (dict(N=0), EINVAL, "N >= 1"), (dict(K=0), EINVAL, "K >= 1"),
    (dict(g=None), EINVAL, "NULL"), (dict(x=None), EINVAL, "NULL"), (dict(w=None), EINVAL, "NULL"),
    (dict(pre=None), EINVAL, "NULL"), (dict(ldg=5), EINVAL, "row length"), (dict(ldx=7), EINVAL, "row length"),
    (dict(ldw=7), EINVAL, "row length"), (dict(ldp=5), EINVAL, "row length"),
    (dict(lddx=7), EINVAL, "row length"), (dict(lddw=7), EINVAL, "row length"),
    (dict(lddz=5), EINVAL, "row length"),
    (dict(dz=None, nbytes=8), EINVAL, "workspace"), (dict(dz=None, ws=None), EINVAL, "workspace"),
    (dict(dz=None, ws=ctypes.c_void_p(4104)), EINVAL, "aligned"),
    (dict(M=2 ** 31 - 1, K=2 ** 20, ldx=2 ** 20, ldw=2 ** 20, lddx=2 ** 20, lddw=2 ** 20), ECAPACITY, "too large"),
])
def test_linear_backward_refusals(change, status, fragment):
    a = dict(BACKWARD, **change)
    assert tbs.lib().tbs_linear_backward(*a.values(), None) == status, _message()
    assert fragment in _message()


def test_linear_backward_without_outputs():
    a = dict(BACKWARD, dx=None, dw=None, db=None, dz=None, g=None, ws=None, nbytes=0)
    assert tbs.lib().tbs_linear_backward(*a.values(), None) == 0


def test_workspaces_cover_the_wanted_outputs():
    L = tbs.lib()
    assert L.tbs_linear_workspace(9, 4, 4, 4) == 0 and L.tbs_linear_workspace(0, 0, 4, 4) == 0
    full = L.tbs_linear_backward_workspace(1, 2, 5000, 300, 200, 1, 1, 1, 0)
    assert full >= L.tbs_linear_backward_workspace(1, 2, 5000, 300, 200, 1, 1, 1, 1) + 2 * 5000 * 300
    assert L.tbs_linear_backward_workspace(1, 0, 5000, 300, 200, 0, 0, 0, 0) == 0
    assert L.tbs_transducer_gradient_workspace(0, 4, 4) == 0
    assert L.tbs_transducer_gradient_workspace(3, 100, 20) >= 2 * 3 * 100 * 21 * 8


def _adjust(dtype=0, logits=P, ldz=10, R=3, V=10, out=P, ldo=10, ws=None, nbytes=0, adjustments=True, **a):
    adj = tbs.Adjustments(**dict(dict(repetition=1.0), **a))
    return tbs.lib().tbs_adjust_logits(dtype, logits, ldz, R, V, ctypes.byref(adj) if adjustments else None,
                                       out, ldo, ws, nbytes, None)


@pytest.mark.parametrize("change,fragment", [
    (dict(dtype=4), "dtype"), (dict(R=-1), "R >= 0"), (dict(V=0), "V >= 1"), (dict(adjustments=False), "NULL"),
    (dict(logits=None), "NULL"), (dict(out=None), "NULL"), (dict(ldz=9), "row length"),
    (dict(ldo=9), "row length"), (dict(repetition=0.0), "penalties"), (dict(repetition=-1.0), "penalties"),
    (dict(repetition=math.nan), "penalties"), (dict(repetition=math.inf), "penalties"),
    (dict(presence=math.nan), "penalties"), (dict(frequency=math.inf), "penalties"),
    (dict(history=4096, history_cols=5, ld_history=4), "history_cols"),
    (dict(history=4096, history_cols=-1, ld_history=4), "history_cols"),
    (dict(bias=4096, ld_bias=9), "row length"), (dict(allowed=4096, ld_allowed=-1), "row length"),
    (dict(states=4096), "go together"),
])
def test_adjust_refusals(change, fragment):
    assert _adjust(**change) == EINVAL, _message()
    assert fragment in _message()


def test_sizes_beyond_the_limits():
    assert _adjust(V=2 ** 30 + 1, ldz=2 ** 31, ldo=2 ** 31) == ECAPACITY and "limit" in _message()
    assert _adjust(R=2 ** 31 - 1, V=2 ** 20, ldz=2 ** 20, ldo=2 ** 20) == ECAPACITY
    L = tbs.lib()
    assert L.tbs_transducer_gradient(0, P, P, P, None, 1, 2 ** 30 + 1, 1, P, P, P, None, P, 1 << 62,
                                     None) == ECAPACITY
    assert L.tbs_transducer_gradient(0, P, P, P, None, 2 ** 21 + 1, 2, 1, P, P, P, None, P, 1 << 62,
                                     None) == ECAPACITY
    big = dict(LINEAR, K=2 ** 30 + 1, ldx=2 ** 31, ldw=2 ** 31)
    assert L.tbs_linear(*big.values(), None) == ECAPACITY


def test_adjust_empty_batch():
    assert _adjust(R=0, logits=None, out=None) == 0


@pytest.mark.parametrize("a,status,fragment", [
    ((5, P, P, P, None, 1, 2, 2, P, P, P, None, P, 1 << 20), EINVAL, "kind"),
    ((0, P, P, P, None, -1, 2, 2, P, P, P, None, P, 1 << 20), EINVAL, "B >= 0"),
    ((0, P, P, P, None, 1, 0, 2, P, P, P, None, P, 1 << 20), EINVAL, "T >= 1"),
    ((0, P, P, P, None, 1, 2, -1, P, P, P, None, P, 1 << 20), EINVAL, "U >= 0"),
    ((0, P, P, P, None, 1, 2, 1024, P, P, P, None, P, 1 << 20), ECAPACITY, "1023"),
    ((0, None, P, P, None, 1, 2, 2, P, P, P, None, P, 1 << 20), EINVAL, "NULL"),
    ((0, P, None, P, None, 1, 2, 2, P, P, P, None, P, 1 << 20), EINVAL, "NULL"),
    ((0, P, P, None, None, 1, 2, 2, P, P, P, None, P, 1 << 20), EINVAL, "NULL"),
    ((0, P, P, P, None, 1, 2, 2, None, P, P, None, P, 1 << 20), EINVAL, "NULL"),
    ((0, P, P, P, None, 1, 2, 2, P, None, P, None, P, 1 << 20), EINVAL, "NULL"),
    ((0, P, P, P, None, 1, 2, 2, P, P, None, None, P, 1 << 20), EINVAL, "NULL"),
    ((0, P, P, P, None, 1, 2, 2, P, P, P, None, None, 1 << 20), EINVAL, "workspace"),
    ((0, P, P, P, None, 1, 2, 2, P, P, P, None, P, 15), EINVAL, "workspace"),
    ((0, P, P, P, None, 1, 2, 2, P, P, P, None, ctypes.c_void_p(4100), 1 << 20), EINVAL, "aligned"),
])
def test_transducer_gradient_refusals(a, status, fragment):
    assert tbs.lib().tbs_transducer_gradient(*a, None) == status
    assert fragment in _message()


def test_transducer_gradient_empty_batch():
    assert tbs.lib().tbs_transducer_gradient(1, None, None, None, None, 0, 2, 2, None, None, None, None, None, 0,
                                             None) == 0


def test_binding_refuses_host_tensors():
    import torch
    x = torch.zeros((2, 3))
    with pytest.raises(ValueError, match="device tensor"):
        tbs.linear(x, torch.zeros((4, 3)))
    with pytest.raises(ValueError, match="device tensor"):
        tbs.linear_backward(x, x, x)
    with pytest.raises(ValueError, match="device tensor"):
        tbs.adjust_logits(x)
    with pytest.raises(ValueError, match="device tensor"):
        tbs.transducer_gradient("standard", torch.zeros((1, 2, 2)), torch.zeros((1, 2, 1)), [[2, 1]])


@pytest.mark.gpu
def test_binding_checks():
    import torch
    z = lambda *s, **k: torch.zeros(s, device="cuda", **k)
    i32 = dict(dtype=torch.int32)
    x, w = z(4, 8), z(6, 8)
    bad = [
        lambda: tbs.linear(x, z(6, 9)), lambda: tbs.linear(x, w.half()), lambda: tbs.linear(x.double(), w.double()),
        lambda: tbs.linear(x, w, z(5)), lambda: tbs.linear(x, w, z(6).half()),
        lambda: tbs.linear(x, w, residual=z(4, 5)), lambda: tbs.linear(x, w, residual=z(3, 6)),
        lambda: tbs.linear(x, w.cpu()), lambda: tbs.linear(x, w[0]),
        lambda: tbs.linear_backward(z(4, 6), x, w, activation="tanh"),
        lambda: tbs.linear_backward(z(4, 6), x, w, pre=z(4, 6)),
        lambda: tbs.linear_backward(z(5, 6), x, w), lambda: tbs.linear_backward(z(4, 5), x, w),
        lambda: tbs.linear_backward(z(4, 6), x, w, pre=z(3, 6), activation="relu"),
        lambda: tbs.adjust_logits(z(3, 9), history=z(2, 4, **i32)), lambda: tbs.adjust_logits(z(3, 9), history=z(3, 4)),
        lambda: tbs.adjust_logits(z(3, 9), history=z(4, **i32)),
        lambda: tbs.adjust_logits(z(3, 9), history=z(3, 4, **i32), history_lengths=z(2, **i32)),
        lambda: tbs.adjust_logits(z(3, 9), history_lengths=z(3, **i32)),
        lambda: tbs.adjust_logits(z(3, 9), history=z(3, 4, **i32), row_penalties=z(3, 2)),
        lambda: tbs.adjust_logits(z(3, 9), bias=z(8)), lambda: tbs.adjust_logits(z(3, 9), bias=z(2, 9)),
        lambda: tbs.adjust_logits(z(3, 9), allowed=z(3, 2, **i32)), lambda: tbs.adjust_logits(z(3, 9), allowed=z(1)),
        lambda: tbs.adjust_logits(z(3, 9), states=z(3, **i32)),
        lambda: tbs.adjust_logits(z(3, 9), graph=tbs.Graph.trivial(9)),
        lambda: tbs.adjust_logits(z(3, 9), out=z(3, 8)), lambda: tbs.adjust_logits(z(3, 9), out=z(9, 3).t()),
        lambda: tbs.adjust_logits(z(3, 9, **i32)),
        lambda: tbs.transducer_gradient("standard", z(1, 3, 3), z(1, 3, 3), [[3, 2]]),
        lambda: tbs.transducer_gradient("standard", z(1, 3, 3).half(), z(1, 3, 2).half(), [[3, 2]]),
        lambda: tbs.transducer_gradient("standard", z(1, 3, 3), z(1, 3, 2), [[3, 2]], weights=[1.0, 2.0]),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"call {i} was accepted")
    with pytest.raises(tbs.TbsError, match="vocab_size"):
        tbs.adjust_logits(z(3, 9), graph=tbs.Graph.trivial(8), states=z(3, **i32))
    with pytest.raises(tbs.TbsError, match="penalties"):
        tbs.adjust_logits(z(3, 9), repetition=0.0)
    with pytest.raises(tbs.TbsError, match="K >= 1"):
        tbs.linear(z(3, 0), z(4, 0))
    with pytest.raises(tbs.TbsError, match="1023"):
        tbs.transducer_gradient("standard", z(1, 2, 1025), z(1, 2, 1024), [[2, 3]])
    with pytest.raises(KeyError):
        tbs.linear(x, w, activation="swish")


@pytest.mark.gpu
def test_binding_refuses_sizes_beyond_int32():
    """Each would be a small size in its low 32 bits (nothing here takes memory)."""
    import torch
    n = 2 ** 32 + 1
    wide = lambda *s, **k: torch.zeros((1,), device="cuda", **k).expand(s)
    i32 = dict(dtype=torch.int32)
    for f in (lambda: tbs.linear(wide(1, n), wide(2, n)), lambda: tbs.linear(wide(1, 2), wide(n, 2)),
              lambda: tbs.linear_backward(wide(1, 2), wide(1, n), wide(2, n)),
              lambda: tbs.adjust_logits(wide(1, n)),
              lambda: tbs.adjust_logits(wide(1, 9), history=wide(1, n, **i32)),
              lambda: tbs.transducer_gradient("modified", wide(1, n, 2), wide(1, n, 1), [[1, 1]]),
              lambda: tbs.transducer_gradient("modified", wide(1, 2, n + 1), wide(1, 2, n), [[1, 1]])):
        with pytest.raises(ValueError, match="a dimension of"):
            f()
