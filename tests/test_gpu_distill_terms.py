"""Distillation with one of its two terms switched off: a term of weight 0 takes no part, whatever its inputs hold."""
import numpy as np
import pytest

from test_gpu_distill import check, gpu, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("tau", [1.0, 2.0, 4.0, 1.5])
@pytest.mark.parametrize("V", [603, 9001])
def test_no_weight_on_the_teacher(V, tau, dtype):
    """kd = 0: the labels' cross-entropy alone, also where the teacher names masked words or holds NaN and infinities"""
    T, k = 7, 5
    z, ids, top, labels, w = inputs(T, V, k, 3, dtype)
    z[1, ids[1, 0]] = -np.inf
    labels[1] = ids[1, 1]
    top[2], top[3, 2], top[4, 1] = np.nan, np.inf, -np.inf
    ids[5] = ids[5, 0]
    labels[6] = ids[6, 3]
    none = np.full_like(ids, -1)
    got = gpu(z, ids, top, tau, 0.0, labels, 0.7, w, dtype)
    assert all(np.isfinite(x).all() for x in got)
    want = gpu(z, none, top, 1.0, 0.0, labels, 0.7, w, dtype)
    assert all(np.array_equal(a, b) for a, b in zip(got, want))
    check(z, none, top, 1.0, 0.0, labels, 0.7, w, dtype, "labels alone")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_no_weight_on_either(dtype):
    z, ids, top, labels, w = inputs(4, 603, 5, 4, dtype)
    top[0] = np.nan
    for lab, ce in ((labels, 0.0), (None, 0.5)):
        lt, loss, dz = gpu(z, ids, top, 2.0, 0.0, lab, ce, w, dtype)
        assert loss == 0 and not lt.any() and not dz.any()


def test_no_weight_on_the_labels():
    """ce = 0: labels of masked words do not matter"""
    z, ids, top, labels, w = inputs(4, 603, 5, 5, "fp32")
    word = np.setdiff1d(np.arange(603), ids[2])[0]
    z[2, word], labels[2] = -np.inf, word
    for tau in (1.0, 2.0):
        a = gpu(z, ids, top, tau, 1.0, labels, 0.0, w)
        b = gpu(z, ids, top, tau, 1.0, None, 0.0, w)
        assert all(np.array_equal(x, y) for x, y in zip(a, b)) and np.isfinite(a[1])
