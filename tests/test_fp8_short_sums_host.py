"""Sums of fewer bits than fp32, on the host: only the e4m3 product takes them, only for bf16
results and only where the caller asks; refusals before anything reaches a device."""
import ctypes

import pytest
import torch
from test_fused_products_host import A, B, C, D, F, G, fp8, ref, shape

from paper_2509_17863_amd import eaas

SHORT = eaas.EAAS_BF16_SHORT_SUMS


def test_refusals_are_those_of_bf16_results():
    for bad in (dict(x=None), dict(y=None), dict(y=D + 1), dict(ldy=127), dict(y=A + 8), dict(y=C),
                dict(y=F + 64), dict(y=G + 4)):
        assert fp8(dt=SHORT, **bad) == -1, bad
    assert fp8(dt=SHORT + 1) == -1 and fp8(dt=SHORT | eaas.EAAS_FP32) == -1
    assert fp8(dt=SHORT, s=shape(R=0), x=None, xs=None, off=None, w=None, wsc=None, y=None, ws=None, n=0) == 0
    large = shape(R=1500, E=3, N=6208, K=784)  # the table of row tiles
    assert fp8(dt=SHORT, s=large, ldy=6208, ws=None) == -3 and fp8(dt=SHORT, s=large, ldy=6208, n=16) == -3


def test_other_products_refuse_it():
    lib, s, ws = eaas.lib(), ref(shape()), 1 << 40
    assert lib.eaas_grouped_matmul(s, A, 256, None, 1, B, C, D, 128, SHORT, ws, ws, None) == -1
    assert lib.eaas_grouped_matmul_int8(s, A, F, None, 1, B, C, G, D, 128, SHORT, ws, ws, None) == -1
    assert lib.eaas_grouped_matmul_dx(s, A, 128, B, C, D, 256, SHORT, ws, ws, None) == -1
    assert lib.eaas_grouped_matmul_dw(s, A, 128, F, 256, None, 1, B, D, SHORT, 0, ws, ws, None) == -1
    assert lib.eaas_quantize_blocks_fp8(A, SHORT, 200, 2, 130, 200, 128, B, C, None) == -1


@pytest.mark.parametrize("R,E,N,K", [(1500, 3, 6208, 784), (32768, 32, 4096, 7168), (64, 8, 256, 272), (5, 1, 40, 70000)])
def test_sums_in_fp32_are_the_default_and_one_workspace_serves_both(R, E, N, K):
    exact, short = eaas._grouped_plan("fp8_fp32", R, E, N, K, True), eaas._grouped_plan("fp8", R, E, N, K, True)
    assert exact[0] != "large" and (short == exact or short[0] == "large")
    need = max(p * R * N * 4 for _, _, p in (exact, short) if p > 1) if exact[2] > 1 else 0
    if short[0] == "large":
        need = max(need, 16 * (1 + R // 256 + min(R, E)))
    assert eaas.lib().eaas_grouped_fp8_workspace_bytes(ctypes.byref(eaas._group_shape(R, E, N, K))) >= need


def test_binding():
    u8 = torch.uint8
    a = (torch.zeros((4, 130), dtype=u8), torch.zeros((4, 2)), torch.zeros(3, dtype=torch.int32),
         torch.zeros((2, 8, 130), dtype=u8), torch.zeros((2, 1, 2)))
    with pytest.raises(ValueError):
        eaas.eaas_grouped_matmul_fp8(*a, torch.zeros((4, 8)), torch.zeros(256, dtype=u8), short_sums=True)
