"""Block-scaled e4m3 products whose scales' product leaves fp32's range, or its normal range,
while the result does not.

Tolerances are those of test_gpu_fp8_blocks.py, plus half the spacing below the normal
range, 2^-150, for each of B + 4 P + 2 roundings in fp32, and 2^-134 for one to bf16.
"""
import numpy as np
import pytest
import torch

from test_gpu_fp8_blocks import Case, blocks

pytestmark = pytest.mark.gpu
DTYPES = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])

# few rows of 16, 32 and 64 to a tile, in one part and in several; any alignment; 128 x 128
KERNELS = [(5, 1, 40, 4096, "one", 0), (24, 3, 300, 320, "even", 0), (200, 3, 300, 160, "even", 2),
           (200, 3, 301, 163, "even", 0), (9, 2, 33, 3001, "even", 3), (839, 1, 2048, 2592, "one", 0),
           (1500, 3, 6208, 528, "some", 4), (64, 1, 64, 4096, "even", 0), (512, 16, 1024, 512, "ragged", 2),
           (32, 1, 12256, 528, "one", 4)]


def scaled(shape, rows, cols, seed=0):
    """A case with scales of each row near two to the power of one of `rows`, and of each block
    of a matrix of `cols`."""
    c = Case(*shape)
    rng = np.random.default_rng(seed)
    c.xs = np.exp2(rng.choice(rows, (len(c.xs), 1)) + rng.random(c.xs.shape)).astype(np.float32)
    c.ws = np.exp2(rng.choice(cols, c.ws.shape) + rng.random(c.ws.shape)).astype(np.float32)
    unread = torch.isnan(c.d[1]).all(1)
    c.d[1].copy_(torch.from_numpy(c.xs))
    c.d[1][unread] = float("nan")
    c.d[4].copy_(torch.from_numpy(c.ws))
    return c


def check(c, y):
    want, mag = c.want()
    parts = c.plan(torch.float32)[2]
    ends = (blocks(c.K) + 4 * parts + 2) * 2.0 ** -150
    tol = (128 + blocks(c.K) + 4 * parts + 2) * 2.0 ** -23 * mag + ends
    if y.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol) + 2.0 ** -134
    err = np.abs(y.double().cpu().numpy() - want)
    assert (err <= tol).all(), (err.max(), np.argwhere(~(err <= tol))[:4])


@DTYPES
@pytest.mark.parametrize("shape", KERNELS, ids=str)
@pytest.mark.parametrize("row,col", [(-100, -40), (-40, -100), (-146, 100), (-30, -130)])
def test_small_scales(gpu, shape, row, col, dtype):
    """Products of scales of about 2^-140, and of a scale with few bits left."""
    c = scaled(shape, (row, row, 0), (col, col, 0))
    check(c, c.run(dtype))


@DTYPES
@pytest.mark.parametrize("shape", KERNELS, ids=str)
def test_rows_beside_others_of_small_scales(gpu, shape, dtype):
    """Scales whose product is in range, but not the larger one's with a sum."""
    c = scaled(shape, (-120, 0, 115), (-100, -40))
    check(c, c.run(dtype))


@DTYPES
@pytest.mark.parametrize("shape", KERNELS, ids=str)
def test_large_scales(gpu, shape, dtype):
    """Products of scales past fp32's largest number, on codes that bring them back."""
    c = scaled(shape, (88, 88, 0), (40, 40, 0))
    # values of at most 7 * 2^-9: the magnitudes of a result's terms stay below 2^127 in all
    for n, codes in ((0, c.xq), (3, c.wq)):
        codes &= 0x87
        c.d[n].copy_(torch.where(c.d[n] == 0x7F, c.d[n], torch.from_numpy(codes).cuda()))
    assert c.want()[1].max() < 2.0 ** 127
    check(c, c.run(dtype))


@DTYPES
@pytest.mark.parametrize("shape", KERNELS, ids=str)
def test_blocks_of_zeros_under_large_scales(gpu, shape, dtype):
    c = scaled(shape, (100, 0), (100, 0))
    c.wq[:] = 0
    c.d[3].zero_()
    assert (c.run(dtype) == 0).all()
