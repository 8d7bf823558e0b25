"""CPU oracle of the separate products of an expert layer: the definitions in
64 bits, written as plainly as they read (numpy, one group at a time)."""
from __future__ import annotations

import numpy as np


def _groups(offsets):
    for e in range(len(offsets) - 1):
        yield e, int(offsets[e]), int(offsets[e + 1])


def source_rows(R, perm=None, k=1):
    return np.arange(R) if perm is None else np.asarray(perm)[:R] // k


def grouped_matmul(x, offsets, w, src):
    """(y, sum of the magnitudes of its terms) for x [*, K], w [E, N, K]."""
    n = int(offsets[-1])
    y = np.zeros((len(src), w.shape[1]))
    mag = np.zeros_like(y)
    for e, a, b in _groups(offsets):
        if b > a:
            y[a:b] = x[src[a:b]] @ w[e].T
            mag[a:b] = np.abs(x[src[a:b]]) @ np.abs(w[e]).T
    return y[:n], mag[:n]


def grouped_matmul_dx(dy, offsets, w):
    n = int(offsets[-1])
    dx = np.zeros((len(dy), w.shape[2]))
    mag = np.zeros_like(dx)
    for e, a, b in _groups(offsets):
        if b > a:
            dx[a:b] = dy[a:b] @ w[e]
            mag[a:b] = np.abs(dy[a:b]) @ np.abs(w[e])
    return dx[:n], mag[:n]


def grouped_matmul_dw(dy, x, offsets, src):
    dw = np.zeros((len(offsets) - 1, dy.shape[1], x.shape[1]))
    mag = np.zeros_like(dw)
    for e, a, b in _groups(offsets):
        if b > a:
            dw[e] = dy[a:b].T @ x[src[a:b]]
            mag[e] = np.abs(dy[a:b]).T @ np.abs(x[src[a:b]])
    return dw, mag


def quantize_rows_int8(x):
    """(codes, scales) of fp32 rows: scale amax * fp32(1/127), 1 where that is zero, and
    quotients in fp32, codes to the nearest integer, ties to even; a row that is not
    finite gets a NaN scale and zero codes."""
    x = np.asarray(x, np.float32)
    q = np.zeros(x.shape, np.int8)
    s = np.zeros(x.shape[0], np.float32)
    for r in range(x.shape[0]):
        if not np.isfinite(x[r]).all():
            s[r] = np.nan
            continue
        step = np.float32(np.abs(x[r]).max() * np.float32(1 / 127))
        s[r] = np.float32(1) if step == 0 else step
        q[r] = np.clip(np.rint(x[r] / s[r]), -127, 127).astype(np.int8)
    return q, s


def grouped_matmul_int8(xq, xs, offsets, wq, wscale, src):
    """fp32 results: the int32 sum rounded to fp32, times the row's scale, times
    the channel's, each product rounded."""
    n = int(offsets[-1])
    y = np.zeros((len(src), wq.shape[1]), np.float32)
    for e, a, b in _groups(offsets):
        if b > a:
            s = xq[src[a:b]].astype(np.int64) @ wq[e].astype(np.int64).T
            y[a:b] = s.astype(np.float32) * xs[src[a:b]][:, None] * wscale[e][None, :]
    return y[:n]


def sigmoid(g):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-g))


def swiglu(gu):
    I = gu.shape[1] // 2
    g, u = gu[:, :I], gu[:, I:]
    return g * sigmoid(g) * u


def swiglu_backward(gu, dh):
    I = gu.shape[1] // 2
    g, u = gu[:, :I], gu[:, I:]
    t = sigmoid(g)
    return np.concatenate([dh * u * t * (1 + g * (1 - t)), dh * g * t], axis=1)


def combine(y, inv, weights):
    """out[t] = sum over the valid slots of weights[t,j] * y[inv[t*k+j]]."""
    T, k = weights.shape
    out = np.zeros((T, y.shape[1]))
    for t in range(T):
        for j in range(k):
            r = inv[t * k + j]
            if r >= 0:
                out[t] += weights[t, j] * y[r]
    return out


def combine_backward(dout, y, inv, weights):
    """(dy, dweights, sum of the magnitudes of dweights' terms); rows of dy that
    no slot names are NaN here."""
    T, k = weights.shape
    dy = np.full(y.shape, np.nan)
    dw, mag = np.zeros((T, k)), np.zeros((T, k))
    for t in range(T):
        for j in range(k):
            r = inv[t * k + j]
            if r >= 0:
                dy[r] = weights[t, j] * dout[t]
                dw[t, j] = (dout[t] * y[r]).sum()
                mag[t, j] = np.abs(dout[t] * y[r]).sum()
    return dy, dw, mag
