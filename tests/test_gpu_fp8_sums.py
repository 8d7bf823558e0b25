"""What block-scaled e4m3 products keep: sums in fp32 for either type of result, whatever
the batch.

Tolerances.  Where every product and every sum is a whole number below 2^24, nothing is
rounded but the result.
"""
import numpy as np
import pytest
import torch

from oracle import layer_oracle as L
from test_gpu_fp8_blocks import NAN_CODE, SHAPES, Case

pytestmark = pytest.mark.gpu
DTYPES = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])


def set_codes(c, xq, wq):
    """Other codes in place of a case's (rows that no group reads stay as they are)."""
    unread = (c.d[0] == NAN_CODE).all(1).cpu().numpy()
    c.xq, c.wq = xq, wq
    c.d[0].copy_(torch.from_numpy(np.where(unread[:, None], np.uint8(NAN_CODE), xq)))
    c.d[3].copy_(torch.from_numpy(wq))


def cancelling(*shape):
    """Of every eight products two are +-448^2 and cancel; the others are whole numbers of
    at most 16, and all that is left of the sum.  (A block's magnitudes are below 2^23.)"""
    c = Case(*shape, whole=True)
    big = L.e4m3_codes(np.array([448.0, -448.0]))
    xq, wq = c.xq.copy(), c.wq.copy()
    for n in (0, 1):
        xq[:, n::8] = big[0]
        wq[:, :, n::8] = big[n]
    set_codes(c, xq, wq)
    return c


# few rows of 16, 32 and 64 to a tile, in one part and in several; any alignment; 128 x 128
# and groups that were summed on large tiles
CANCEL = [(5, 1, 40, 4096, "one", 0), (24, 3, 300, 320, "even", 0), (200, 3, 300, 160, "even", 2),
          (200, 3, 301, 163, "even", 0), (9, 2, 33, 3001, "even", 3), (839, 1, 2048, 2592, "one", 0),
          (3000, 3, 6188, 528, "even", 0), (1500, 3, 6208, 1536, "some", 4),
          (26638, 23, 416, 352, "even", 2)]


@DTYPES
@pytest.mark.parametrize("shape", CANCEL, ids=str)
def test_terms_that_cancel(gpu, shape, dtype):
    c = cancelling(*shape)
    want = torch.from_numpy(c.want()[0]).float().to(dtype)
    assert torch.equal(c.run(dtype).cpu(), want)


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_bf16_results_are_the_fp32_ones_rounded(gpu, shape):
    c = Case(*shape[:-1])
    assert torch.equal(c.run(torch.bfloat16), c.run(torch.float32).to(torch.bfloat16))
