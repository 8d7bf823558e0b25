"""Operands and results cut out of one wider array, on the host: rows side by side
do not overlap, rows that share an element do.  (The shape splits its sum, so a call
whose arguments are accepted ends at the missing workspace and enqueues nothing.)"""
import ctypes

import pytest

from paper_2509_17863_amd import eaas

INVALID, WORKSPACE = -1, -3
A, B, C = (i << 32 for i in range(1, 4))
R, N, K = 32, 64, 8192


def forward(x, ldx, y, ldy, n=N, dt=0):
    s = eaas._GroupShape(R, 1, n, K)
    assert eaas.lib().eaas_grouped_workspace_bytes(ctypes.byref(s)) > 256
    return eaas.lib().eaas_grouped_matmul(ctypes.byref(s), x, ldx, None, 1, B, C, y, ldy, dt, None,
                                          0, None)


def rows(dy, lddy, dx, lddx):  # the sum is N here
    s = eaas._GroupShape(R, 1, K, N)
    return eaas.lib().eaas_grouped_matmul_dx(ctypes.byref(s), dy, lddy, B, C, dx, lddx, 0, None, 0,
                                             None)


@pytest.mark.parametrize("call", [forward, rows])
def test_rows_of_one_array(call):
    ld = K + N + 16
    assert call(A, ld, A + 2 * K, ld) == WORKSPACE              # the result after the operand
    assert call(A, ld, A + 2 * (K + 16), ld) == WORKSPACE       # up to the end of the row
    assert call(A + 2 * N, ld, A, ld) == WORKSPACE              # before it
    assert call(A, ld, A + 2 * (3 * ld + K), ld) == WORKSPACE   # some rows further down
    assert call(A + 2 * (3 * ld + N), ld, A, ld) == WORKSPACE
    assert call(A, ld, A + 2 * (K - 1), ld) == INVALID          # one element shared
    assert call(A, ld, A + 2 * (K + 17), ld) == INVALID         # with the next row
    assert call(A + 2 * (N - 1), ld, A, ld) == INVALID
    assert call(A, ld, A, ld) == INVALID
    assert call(A, ld, A + 2 * (3 * ld + 5), ld) == INVALID
    assert call(A, ld, A + 2 * K, ld + 8) == INVALID            # rows drift into each other
    assert call(A, ld, A + 2 * ((R - 1) * ld + K), ld) == WORKSPACE  # past the last row


def test_fp32_results_in_an_array_of_bf16_rows():
    """The distance of rows counts in bytes."""
    ld = K + 2 * N
    assert forward(A, ld, A + 2 * K, ld // 2, dt=2) == WORKSPACE
    assert forward(A, ld, A + 2 * K - 4, ld // 2, dt=2) == INVALID
    assert forward(A, ld, A + 2 * K, ld, dt=2) == INVALID
