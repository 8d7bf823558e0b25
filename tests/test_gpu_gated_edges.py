"""The gated product and the h of its way back where the gate's sigmoid, or the gate times it,
is below fp32's normal range and the product with up is not.

Tolerances: exponential, sum, reciprocal and products err by (|g| + 8) 2^-23 of the result,
bf16 adds 2^-8 of it, or half its least step of 2^-133.
"""
import numpy as np
import pytest
import torch

from oracle import layer_oracle as L
from paper_2509_17863_amd import eaas

pytestmark = pytest.mark.gpu
GATES = [-170.0, -150.0, -127.0, -110.0, -104.0, -103.0, -100.0, -95.0, -88.5, -87.5, -60.0, -3.0, 0.0, 2.0, 90.0]
UPS = [3e38, -1e30, 1e20, 1e10, -3e5, 1.0, 0.0, 1e-20, -1e-38, 1e-40]


def near(got, g, u):
    want = L.swiglu(np.concatenate([g, u], 1))
    fits = np.abs(want) < 2.0 ** 127
    tol = ((np.abs(g) + 8) * 2.0 ** -23 + 2.0 ** -8) * np.abs(want) * 1.001 + 2.0 ** -134
    err = np.abs(got.double().cpu().numpy() - want)
    assert (err <= tol)[fits].all(), [(g[i], u[i], got[i], want[i]) for i in map(tuple, np.argwhere((err > tol) & fits)[:4])]


# any alignment, few rows, large tiles, and a sum in parts
@pytest.mark.parametrize("R,E,I,K", [(200, 3, 96, 160), (300, 6, 33, 47), (12, 3, 64, 256), (1200, 3, 3104, 264),
                                     (3, 1, 40, 70000)])
def test_gates_far_below_zero(gpu, R, E, I, K):
    n = torch.arange(E * I)
    gate = torch.tensor(GATES)[n % len(GATES)].view(E, I).to(torch.bfloat16)
    up = torch.tensor(UPS)[n // len(GATES) % len(UPS)].view(E, I).to(torch.bfloat16)
    off = torch.tensor([R * e // E for e in range(E + 1)], dtype=torch.int32)
    group = torch.repeat_interleave(torch.arange(E), off.diff())
    g, u = gate[group].double().numpy(), up[group].double().numpy()
    bf = dict(dtype=torch.bfloat16, device="cuda")
    # the sums are one product with 1
    x, w = torch.zeros((R, K), **bf), torch.zeros((E, 2 * I, K), **bf)
    x[:, 0] = 1
    w[:, :, 0] = torch.cat([gate, up], 1).cuda()
    h, gu = torch.empty((R, I), **bf), torch.empty((R, 2 * I), **bf)
    eaas.eaas_grouped_swiglu(x, off.cuda(), w, h, eaas.alloc_grouped_workspace(R, E, 2 * I, K), gu=gu)
    assert np.array_equal(gu.double().cpu().numpy(), np.concatenate([g, u], 1))
    near(h, g, u)
    h.zero_()
    dy, wd, dgu = torch.zeros((R, K), **bf), torch.zeros((E, K, I), **bf), torch.empty((R, 2 * I), **bf)
    eaas.eaas_grouped_swiglu_backward(dy, off.cuda(), wd, gu, dgu, eaas.alloc_grouped_workspace(R, E, K, I), h=h)
    near(h, g, u)
    assert (dgu == 0).all()
