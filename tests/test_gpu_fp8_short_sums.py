"""Block-scaled e4m3 products that may sum in fewer bits than fp32: the same tests as of the
products with sums in fp32 (test_gpu_fp8_blocks.py has the tolerances), and every variant of
the kernel for large tiles: rows gathered or not, rows of scales in multiples of 16 bytes or
not, sums of one to twelve fours of blocks, several tiles to a workgroup.
"""
import numpy as np
import pytest
import torch
import test_gpu_fp8_blocks as exact
from paper_2509_17863_amd import eaas
from test_gpu_fp8_blocks import (Case, blocks,  # noqa: F401
                                 test_equal_calls_other_streams_and_graphs,
                                 test_no_numbers_stay_in_their_rows,
                                 test_offsets_that_do_not_ascend_stay_in_bounds,
                                 test_result_past_32_bit_offsets, test_results_from_any_element,
                                 test_two_calls_at_once)

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(autouse=True)
def short_sums(monkeypatch):
    """Every product here with bf16 results may take them."""
    product = eaas.eaas_grouped_matmul_fp8

    def call(xq, xs, offsets, wq, wscale, y, ws, **kw):
        product(xq, xs, offsets, wq, wscale, y, ws, short_sums=y.dtype == BF16, **kw)

    monkeypatch.setattr(eaas, "eaas_grouped_matmul_fp8", call)


LARGE = [(3000, 5, 6200, 528, "ragged", 0), (3000, 4, 6201, 1040, "some", 4),
         (26638, 23, 416, 352, "even", 2), (1030, 63, 672, 512, "even", 0), (1500, 3, 6201, 784, "some", 0),
         # rows of scales in fours: one, two, three and twelve, and gathered
         (1030, 63, 672, 512, "ragged", 5), (1030, 63, 672, 1024, "even", 0), (1040, 60, 700, 1024, "even", 2),
         (1030, 63, 672, 1536, "ragged", 0), (1500, 3, 6208, 1536, "some", 4), (1200, 40, 1296, 6144, "even", 3),
         # the last block of a row part empty; two and three tiles of results to a workgroup
         (2060, 63, 1200, 1488, "even", 0), (4120, 63, 1808, 688, "ragged", 4), (3000, 5, 12304, 2032, "even", 2)]


def test_every_variant_is_among_these():
    seen = set()
    for R, E, N, K, _, k in LARGE:
        assert eaas._grouped_plan("fp8", R, E, N, K, True)[0] == "large"
        seen.add((k > 0, blocks(K) % 4 == 0, blocks(K) > 4, blocks(K) > 8))
    for gather in (False, True):
        for fours in (False, True):
            assert (gather, fours, True, False) in seen and (gather, True, True, True) in seen
        assert (gather, True, False, False) in seen
    assert (True, False, False, False) in seen


@pytest.mark.parametrize("shape", LARGE + exact.EXACT[:4], ids=str)
def test_whole_numbers(gpu, shape):
    """Every product is a multiple of what the instructions keep: nothing is rounded."""
    c = Case(*shape, whole=True)
    want = torch.from_numpy(c.want()[0]).float().to(BF16)
    assert torch.equal(c.run(BF16).cpu(), want)


@pytest.mark.parametrize("shape", LARGE + [s[:-1] for s in exact.SHAPES], ids=str)
def test_product(gpu, shape):
    c = Case(*shape)
    c.check(c.run(BF16, pad=shape[0] % 9))


@pytest.mark.parametrize("shape", [(1030, 63, 672, 1024, "even", 0), (1500, 3, 6208, 1536, "some", 4)], ids=str)
@pytest.mark.parametrize("lead", [1, 2])
def test_rows_of_scales_from_any_element(gpu, shape, lead):
    c = Case(*shape, whole=True)
    want = torch.from_numpy(c.want()[0]).float().to(BF16)
    xq, xs, *rest = c.d
    flat = torch.full((xs.numel() + 8,), float("nan"), device="cuda")
    flat[lead: lead + xs.numel()] = xs.reshape(-1)
    c.d = (xq, flat[lead: lead + xs.numel()].view(xs.shape), *rest)
    assert torch.equal(c.run(BF16).cpu(), want)


def test_what_is_lost_on_normal_data(gpu):
    """2^-16 of the results' norm before they are rounded.  A value that is moved by d ends
    in another place of its 8 bits, a step of at most 2^-7 of it away, with probability d
    over that step; so the results differ from the rounded exact ones by the root of 2^-7 *
    2^-16 of their norm."""
    R, E, N, K = 1500, 3, 6208, 2048
    g = torch.Generator(device="cuda").manual_seed(7)
    x, w = torch.randn((R, K), device="cuda", generator=g), torch.randn((E, N, K), device="cuda", generator=g)
    xq, xs = torch.empty((R, K), dtype=torch.uint8, device="cuda"), torch.empty((R, blocks(K)), device="cuda")
    wq = torch.empty((E, N, K), dtype=torch.uint8, device="cuda")
    ws = torch.empty((E, blocks(N), blocks(K)), device="cuda")
    eaas.eaas_quantize_blocks_fp8(x, xq, xs)
    eaas.eaas_quantize_blocks_fp8(w, wq, ws)
    off = torch.tensor([0, 500, 1000, 1500], dtype=torch.int32, device="cuda")
    assert eaas._grouped_plan("fp8", R, E, N, K, True)[0] == "large"
    y = torch.empty((R, N), dtype=BF16, device="cuda")
    eaas.eaas_grouped_matmul_fp8(xq, xs, off, wq, ws, y, eaas.alloc_grouped_fp8_workspace(R, E, N, K))
    err = norm = 0.0
    full = xs.double().repeat_interleave(128, 1) * xq.view(torch.float8_e4m3fn).double()
    for e in range(E):
        v = wq[e].view(torch.float8_e4m3fn).double() * ws[e].double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)
        want = (full[500 * e: 500 * e + 500] @ v.t()).to(BF16).double()
        err += ((y[500 * e: 500 * e + 500].double() - want) ** 2).sum().item()
        norm += (want ** 2).sum().item()
    assert 0 < (err / norm) ** 0.5 < 2.0 ** -11.5


def test_whole_sums_are_the_default(gpu, monkeypatch):
    """The same call that does not ask for them, on the same rows."""
    monkeypatch.undo()
    c = Case(1500, 3, 6208, 784, "even")
    want, mag = c.want()
    y = c.run(BF16).double().cpu().numpy()
    tol = (128 + blocks(c.K) + 6) * 2.0 ** -23 * mag
    assert (np.abs(y - want) <= tol + 2.0 ** -8 * (np.abs(want) + tol)).all()
    with pytest.raises(ValueError):
        eaas.eaas_grouped_matmul_fp8(*c.d, torch.empty((c.R, c.N), device="cuda"), c.scratch, short_sums=True)
