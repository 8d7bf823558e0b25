"""eaas_swiglu_int8 where its values leave the normal range of fp32 or come close.

Tolerances.  A value takes at most six roundings (the exponential, once or twice,
counts one unit in the last place each time): 6 * 2^-23 of itself, and below the
normal range 6 * 2^-149 more.  A scale adds one rounding to its row's largest value.
A code is then within half a step, and those errors in steps, of the value.
"""
import numpy as np
import pytest
import torch

from oracle import layer_oracle as L
from paper_2509_17863_amd import eaas

pytestmark = pytest.mark.gpu
TINY = 2.0 ** -149


def swiglu_int8(gu):
    rows, I = gu.shape[0], gu.shape[1] // 2
    q = torch.full((rows, I), 99, dtype=torch.int8, device="cuda")
    s = torch.full((rows,), 99.0, device="cuda")
    eaas.eaas_swiglu_int8(gu.cuda(), q, s)
    return q.cpu().numpy(), s.double().cpu().numpy()


@pytest.mark.parametrize("rows,I", [(5, 16), (5, 2064), (2050, 16)])
@pytest.mark.parametrize("up", [1.0, 1e20, 3e38, 0.75])
@pytest.mark.parametrize("gates", [(-85.5, -86.0, -86.5, -87.0), (-87.5, -88.0, -88.5),
                                   (-88.5, -89.0, -90.0, -95.0), (-100.0, -102.0),
                                   (-20.0, -87.5, -103.0)], ids=str)
def test_gates_far_below_zero(gpu, gates, up, rows, I):
    g = torch.tensor(gates)[torch.arange(rows * I) % len(gates)].view(rows, I)
    u = torch.full((rows, I), up) * (1 - torch.arange(I) % 7 / 16)
    gu = torch.cat([g, u], dim=1).to(torch.bfloat16)
    q, s = swiglu_int8(gu)
    h = L.swiglu(gu.double().numpy())
    err = 6 * 2.0 ** -23 * np.abs(h) + 6 * TINY
    step = np.abs(h).max(axis=1) / 127
    assert (np.abs(s - step) <= step * 7 * 2.0 ** -23 + 7 * TINY).all(), (s[0], step[0])
    codes = np.clip(h / s[:, None], -127, 127)
    off = np.abs(q - codes) - 0.5 - err / s[:, None]
    assert (off <= 2.0 ** -16).all(), off.max()  # (2^-16: the quotient's own rounding)


@pytest.mark.parametrize("rows,I", [(4, 24), (2050, 24), (3, 2056), (2, 20000)])
def test_a_scale_below_the_smallest_number_counts_as_zero(gpu, rows, I):
    """33 * 2^-149 at the most, a 127th of which rounds to zero."""
    gu = torch.zeros((rows, 2 * I))
    gu[:, :I] = -0.001
    gu[:, I::2] = 2.0 ** -133
    gu = gu.to(torch.bfloat16)
    h = L.swiglu(gu.double().numpy())
    assert 0 < np.abs(h).max() < 63 * TINY
    q, s = swiglu_int8(gu)
    assert (s == 1).all() and (q == 0).all()
    qr, sr = L.quantize_rows_int8(h[:2])
    assert (sr == 1).all() and (qr == 0).all()


def test_other_extremes(gpu):
    """Gates of any size next to a gate of 1."""
    g = torch.tensor([[-3e38, -1000.0, -104.0, -86.0, 0.0, 1.0, 87.0, 1000.0]] * 3)
    u = torch.tensor([[1.0] * 8, [0.5] * 8, [-1.0, 1.0] * 4])
    gu = torch.cat([g, u], dim=1).to(torch.bfloat16)
    q, s = swiglu_int8(gu)
    h = L.swiglu(gu.double().numpy())
    step = np.abs(h).max(axis=1) / 127
    assert (np.abs(s - step) <= step * 7 * 2.0 ** -23).all()
    err = np.abs(q - h / s[:, None])
    assert (err <= 0.5 + 127 * 7 * 2.0 ** -23 + 2.0 ** -16).all()
