"""Pins of the oracle of block-scaled e4m3 products and of the gated product: the format
against torch's cast, the scales by closed forms, gradients against differences."""
import numpy as np
import pytest
import torch

from oracle import layer_oracle as L


def test_values_and_codes_are_those_of_the_format():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(L.e4m3_values(), want)
    finite = np.array([c for c in range(256) if c & 127 != 127])
    np.testing.assert_array_equal(L.e4m3_codes(L.e4m3_values()[finite]), finite)
    v = np.unique(L.e4m3_values()[:127])
    rng = np.random.default_rng(0)
    x = np.concatenate([(v[1:] + v[:-1]) / 2, -(v[1:] + v[:-1]) / 2, rng.normal(size=20000) * 100,
                        rng.normal(size=20000) * 0.01]).astype(np.float32)
    x = x[np.abs(x) <= 448]
    cast = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(L.e4m3_codes(x), cast)
    assert L.e4m3_codes(np.array([449.0, 1e30, -500.0])).tolist() == [0x7E, 0x7E, 0xFE]


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("n,K", [(1, 1), (3, 127), (130, 129), (128, 256), (257, 300)])
def test_blocks(n, K, block_rows):
    rng = np.random.default_rng([n, K])
    x = (rng.normal(size=(n, K)) * np.exp(rng.normal(size=(n, 1)) * 3)).astype(np.float32)
    x[0, 0] = 0
    q, s = L.quantize_blocks(x, block_rows)
    assert s.shape == (-(-n // block_rows), -(-K // 128))
    d = L.dequantized(q, s, block_rows)
    full = np.repeat(np.repeat(s, block_rows, 0), 128, 1)[:n, :K].astype(np.float64)
    # half a step: 2^-4 of the value, or 2^-10 of the scale below the format's normal range
    assert (np.abs(d - x) <= np.maximum(np.abs(x) * 2.0 ** -4, full * 2.0 ** -10) * 1.0001).all()
    for i in range(s.shape[0]):
        b = np.abs(x[i * block_rows: (i + 1) * block_rows, :128]).max()
        assert s[i, 0] == (np.float32(b) * np.float32(1 / 448) if b else 1)


def test_blocks_of_zeros_and_of_no_numbers():
    x = np.zeros((3, 256), np.float32)
    x[1, 5], x[2, 130] = np.inf, np.nan
    q, s = L.quantize_blocks(x)
    assert (q == 0).all() and s[0].tolist() == [1, 1]
    assert np.isnan(s[1, 0]) and s[1, 1] == 1 and s[2, 0] == 1 and np.isnan(s[2, 1])


def test_product_and_its_gradient_on_transposed_weights():
    rng = np.random.default_rng(2)
    E, N, K, off = 2, 200, 300, np.array([0, 3, 7])
    w = rng.normal(size=(E, N, K)).astype(np.float32)
    wq, ws = (np.stack(t) for t in zip(*[L.quantize_blocks(m, 128) for m in w]))
    x = L.quantize_blocks(rng.normal(size=(7, K)).astype(np.float32))
    y, mag = L.grouped_matmul_fp8(*x, off, wq, ws, np.arange(7))
    v = L.e4m3_values()
    r, n = 4, 150  # one result by hand
    want = sum(float(x[1][r, b]) * float(ws[1, n // 128, b]) *
               sum(v[x[0][r, k]] * v[wq[1, n, k]] for k in range(128 * b, min(K, 128 * b + 128)))
               for b in range(3))
    assert abs(y[r, n] - want) < 1e-12 * mag[r, n]
    # 128 x 128 blocks transpose exactly: the gradient in the rows is the product with them
    dy = L.quantize_blocks(rng.normal(size=(7, N)).astype(np.float32))
    dx, _ = L.grouped_matmul_fp8(*dy, off, wq.transpose(0, 2, 1), ws.transpose(0, 2, 1),
                                 np.arange(7))
    full = np.stack([L.dequantized(wq[e], ws[e], 128) for e in range(E)])
    want, _ = L.grouped_matmul_dx(L.dequantized(*dy), off, full)
    np.testing.assert_allclose(dx, want, rtol=1e-12, atol=1e-12)


def test_gated_product_and_differences():
    """dL/dx, dL/dW of the gated half and the down projection, by central differences."""
    rng = np.random.default_rng(3)
    E, H, I, R = 2, 5, 4, 6
    off, src = np.array([0, 2, 6]), np.arange(R)
    x, wgu = rng.normal(size=(R, H)), rng.normal(size=(E, 2 * I, H))
    wd, dy = rng.normal(size=(E, H, I)), rng.normal(size=(R, H))

    def loss(x, wgu, wd):
        h, _, _ = L.grouped_swiglu(x, off, wgu, src)
        return (L.grouped_matmul(h, off, wd, src)[0] * dy).sum()

    h, gu, _ = L.grouped_swiglu(x, off, wgu, src)
    dgu, again, _, _ = L.grouped_swiglu_backward(dy, off, wd, gu)
    np.testing.assert_array_equal(again, h)
    grads = (L.grouped_matmul_dx(dgu, off, wgu)[0], L.grouped_matmul_dw(dgu, x, off, src)[0],
             L.grouped_matmul_dw(dy, h, off, src)[0])
    at = [x, wgu, wd]
    for n, g in enumerate(grads):
        for _ in range(8):
            i = tuple(rng.integers(0, m) for m in at[n].shape)
            d = []
            for step in (1e-5, -1e-5):
                moved = [a.copy() for a in at]
                moved[n][i] += step
                d.append(loss(*moved))
            assert abs((d[0] - d[1]) / 2e-5 - g[i]) < 1e-7 * max(1, abs(g[i]))
