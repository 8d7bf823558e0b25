"""The oracle of the separate products: its gradients against central
differences of its own forward functions, its codes against their definition."""
import numpy as np
import pytest

from oracle import layer_oracle as L


def _difference(f, a, eps=1e-6):
    g = np.zeros_like(a)
    for i in np.ndindex(a.shape):
        keep = a[i]
        a[i] = keep + eps
        hi = f()
        a[i] = keep - eps
        lo = f()
        a[i] = keep
        g[i] = (hi - lo) / (2 * eps)
    return g


OFFSETS = np.array([0, 2, 2, 5, 6])  # one empty group, one of a single row


@pytest.mark.parametrize("gather", [False, True])
def test_product_gradients_are_those_of_the_product(gather):
    rng = np.random.default_rng(1)
    R, N, K, k = 6, 3, 4, 2
    src = L.source_rows(R, rng.permutation(R), k) if gather else L.source_rows(R)
    x = rng.normal(size=(R // k if gather else R, K))
    w = rng.normal(size=(4, N, K))
    dy = rng.normal(size=(R, N))
    loss = lambda: (L.grouped_matmul(x, OFFSETS, w, src)[0] * dy).sum()  # noqa: E731
    dw, _ = L.grouped_matmul_dw(dy, x, OFFSETS, src)
    assert np.allclose(dw, _difference(loss, w), atol=1e-8)
    assert (dw[1] == 0).all()
    dx, _ = L.grouped_matmul_dx(dy, OFFSETS, w)
    tokens = np.zeros_like(x)
    np.add.at(tokens, src, dx)
    assert np.allclose(tokens, _difference(loss, x), atol=1e-8)


def test_swiglu_gradient():
    rng = np.random.default_rng(2)
    gu = rng.normal(size=(3, 10)) * 3
    dh = rng.normal(size=(3, 5))
    got = L.swiglu_backward(gu, dh)
    assert np.allclose(got, _difference(lambda: (L.swiglu(gu) * dh).sum(), gu), atol=1e-7)


def test_combine_gradient():
    rng = np.random.default_rng(3)
    T, k, H = 3, 2, 4
    inv = np.array([4, 0, -1, 2, 1, 3])  # one slot elsewhere
    y, w, dout = rng.normal(size=(6, H)), rng.normal(size=(T, k)), rng.normal(size=(T, H))
    dy, dw, _ = L.combine_backward(dout, y, inv, w)
    loss = lambda: (L.combine(y, inv, w) * dout).sum()  # noqa: E731
    assert np.allclose(dw, _difference(loss, w), atol=1e-8) and dw[1, 0] == 0
    named = np.array([0, 1, 2, 3, 4])
    assert np.allclose(dy[named], _difference(loss, y)[named], atol=1e-8)
    assert np.isnan(dy[5]).all()


def test_int8_rows():
    x = np.array([[0, 0, 0], [127, 63.5, -0.5], [np.inf, 1, 2], [1, np.nan, 0]], np.float32)
    q, s = L.quantize_rows_int8(x)
    assert s[0] == 1 and s[1] == 1 and np.isnan(s[2:]).all()
    assert q.tolist() == [[0, 0, 0], [127, 64, 0], [0, 0, 0], [0, 0, 0]]  # ties to even


def test_int8_product_of_small_whole_numbers_is_exact():
    rng = np.random.default_rng(4)
    xq = rng.integers(-127, 128, (6, 9)).astype(np.int8)
    wq = rng.integers(-127, 128, (4, 5, 9)).astype(np.int8)
    one = np.ones(6, np.float32)
    y = L.grouped_matmul_int8(xq, one, OFFSETS, wq, np.ones((4, 5), np.float32), np.arange(6))
    ref, _ = L.grouped_matmul(xq.astype(float), OFFSETS, wq.astype(float), np.arange(6))
    assert (y == ref).all()
