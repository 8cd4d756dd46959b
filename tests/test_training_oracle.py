"""The definitions of the operators around a training step's layers, on the CPU: their gradients against differences, the
generator against its published vectors, and the library's refusals, which need no GPU."""
import ctypes

import numpy as np
import pytest

from oracle import training as ot
from paper_2605_08527_b200 import binding as B


def slope(f, x, u, h=1e-6):
    return (f(x + h * u) - f(x - h * u)) / (2 * h)


@pytest.mark.parametrize("rms", [False, True])
def test_layer_norm_gradients(rms):
    r = np.random.RandomState(0)
    T, d, n, eps = 6, 16, 2, 1e-3
    x, w = r.randn(T, d), r.randn(T, d)
    gain, bias, rows = r.randn(n + 1, d), r.randn(n + 1, d), np.array([0, 2, 2, 0, 1, 0])
    f = lambda x_, g_, b_: float((w * ot.layer_norm(x_, rows, g_, b_, eps, rms)[0]).sum())      # noqa: E731
    _, mean, rstd = ot.layer_norm(x, rows, gain, bias, eps, rms)
    dx, dg, db = ot.layer_norm_backward(x, w, rows, gain, mean, rstd, rms)
    for _ in range(4):
        u, v = r.randn(T, d), r.randn(n + 1, d)
        assert abs(slope(lambda a: f(a, gain, bias), x, u) - (dx * u).sum()) < 1e-6
        assert abs(slope(lambda a: f(x, a, bias), gain, v) - (dg * v).sum()) < 1e-6
        assert abs(slope(lambda a: f(x, gain, a), bias, v) - (db * v).sum()) < 1e-6


def test_dropout_gradients():
    r = np.random.RandomState(1)
    T, K, N = 7, 10, 6
    tok, rates, scale = [0, 1, -1, 0, 2, 1, 0], [0.3, 0.5, 0.0], [2.0, 0.5, 1.0]
    x, W, w = r.randn(T, K), r.randn(K, N), r.randn(T, N)
    A, Bm = [r.randn(K, 3), r.randn(K, 2), None], [r.randn(3, N), r.randn(2, N), None]
    keep = ot.dropout_keep(tok, K, rates, 99, 3)
    assert keep[2].all() and keep[4].all() and not keep[[0, 1, 3, 5, 6]].all()
    f = lambda x_, A_, B_: float((w * ot.dropout_forward(x_, W, tok, A_, B_, scale, rates, keep)[0]).sum())      # noqa: E731
    dx, dA, dB = ot.dropout_backward(x, W, w, tok, A, Bm, scale, rates, keep)
    for _ in range(4):
        u = r.randn(T, K)
        assert abs(slope(lambda a: f(a, A, Bm), x, u) - (dx * u).sum()) < 1e-6
        for t in (0, 1):
            u, v = r.randn(*A[t].shape), r.randn(*Bm[t].shape)
            assert abs(slope(lambda a: f(x, [a if i == t else q for i, q in enumerate(A)], Bm), A[t], u) - (dA[t] * u).sum()) < 1e-6
            assert abs(slope(lambda a: f(x, A, [a if i == t else q for i, q in enumerate(Bm)]), Bm[t], v) - (dB[t] * v).sum()) < 1e-6


def test_generator():
    # published vectors of the generator's authors, for seven and for ten rounds
    assert ot.philox((0, 0, 0, 0), (0, 0)) == [0x5F6FB709, 0x0D893F64, 0x4F121F81, 0x4F730A48]
    assert ot.philox((0, 0, 0, 0), (0, 0), 10) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    # the share that is dropped: 65536 elements, five standard deviations
    for rate in (0.05, 0.5, 0.9):
        keep = ot.dropout_keep([0] * 64, 1024, [rate], 7, 1)
        assert abs(1 - keep.mean() - rate) < 5 * (rate * (1 - rate) / 65536) ** 0.5 + 1 / 65536
    assert ot.threshold(float("nan")) == 0 and ot.threshold(-1.0) == 0 and ot.threshold(3.0) == 65536 and ot.dropout_factor(1.0, 1.0) == 0


def test_head_gradient():
    r = np.random.RandomState(2)
    T, d, V, k = 5, 6, 9, 1.3
    x, W, w = r.randn(T, d), r.randn(d, V), np.array([1.0, -0.5, 0.0, 2.0, 1.0])
    tgt, tok = [3, 8, 1, -1, 0], [0, 1, 1, 0, -1]
    logp, stats, dx = ot.head_cross_entropy(x, W, tgt, w, tok, 2, k)
    f = lambda a: ot.head_cross_entropy(a, W, tgt, w, tok, 2, k)[1][:, 0].sum()      # noqa: E731
    for _ in range(4):
        u = r.randn(T, d)
        assert abs(slope(f, x, u) - (dx * u).sum()) < 1e-6
    assert logp[2] == logp[3] == 0 and not dx[2].any() and stats[:, 3].tolist() == [1.0, 1.0, 1.0]


@pytest.fixture(scope="module")
def lib():
    from paper_2605_08527_b200 import build
    build.build()
    return B.load_library()


def test_refusals_without_a_pool(lib):
    assert lib.marlaas_layer_norm_workspace_bytes(None, 1, 8, 1, 1) == 0
    assert lib.marlaas_head_cross_entropy_workspace_bytes(None, 1, 8, 8, 1, 1) == 0
    assert lib.marlaas_lora_dropout_workspace_bytes(None, 1) == 0
    bad = B.MARLAAS_ERR_INVALID_ARG
    assert lib.marlaas_layer_norm(None, 1, 8, None, 8, None, None, None, 1e-5, None, 8, None, None, None, 0, 0, None) == bad
    assert lib.marlaas_layer_norm_backward(None, 1, 8, None, 8, None, 8, None, None, None, None, None, 8, None, None, None, 0, 0, None) == bad
    assert lib.marlaas_head_cross_entropy(None, 1, 8, 8, None, 8, None, 8, None, None, None, 1.0, 1.0, None, 8, None, None, None, 0, 0, None) == bad
    drop = B.marlaas_dropout_t(None, 0, 0)
    assert lib.marlaas_lora_forward_dropout(None, 1, None, 8, None, 8, None, 8, None, ctypes.byref(drop), None, None, 0, 0, None) == bad
    assert lib.marlaas_lora_backward_dropout(None, 1, None, 8, None, 8, None, 8, None, 8, None, None, None, ctypes.byref(drop), None, None, 0, 0, None) == bad
    assert "NULL" in B.marlaas_last_error()
