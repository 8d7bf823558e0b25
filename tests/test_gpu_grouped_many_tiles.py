"""Results of more tiles than one dimension of a grid holds (2^32 threads).  The
operands are small whole numbers, so every result is exact."""
import pytest
import torch

from paper_2509_17863_amd import eaas

pytestmark = pytest.mark.gpu
E, WIDE = 1024, 1 << 21  # 1024 x 2^14 tiles of 128 columns and 256 threads


def whole(shape):
    t = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    for part in t.view(-1).split(1 << 28):
        part.copy_(torch.randint(-4, 5, part.shape, dtype=torch.int8, device="cuda"))
    return t


@pytest.fixture(autouse=True)
def free_memory():
    yield
    torch.cuda.empty_cache()


def test_forward(gpu):
    x, w = whole((E, 1)), whole((E, WIDE, 1))
    off = torch.arange(E + 1, dtype=torch.int32, device="cuda")
    y = torch.empty((E, WIDE), dtype=torch.bfloat16, device="cuda")
    eaas.eaas_grouped_matmul(x, off, w, y, eaas.alloc_grouped_workspace(E, E, WIDE, 1))
    for r in range(0, E, 64):
        assert torch.equal(y[r: r + 64], w[r: r + 64, :, 0] * x[r: r + 64])


def test_gradient_in_the_rows(gpu):
    dy, w = whole((E, 1)), whole((E, 1, WIDE))
    off = torch.arange(E + 1, dtype=torch.int32, device="cuda")
    dx = torch.empty((E, WIDE), dtype=torch.bfloat16, device="cuda")
    eaas.eaas_grouped_matmul_dx(dy, off, w, dx, eaas.alloc_grouped_workspace(E, E, 1, WIDE))
    for r in range(0, E, 64):
        assert torch.equal(dx[r: r + 64], w[r: r + 64, 0] * dy[r: r + 64])


def test_gradient_in_the_weights(gpu):
    rows = {0: 1, 5: 2, 511: 1, E - 1: 2}  # of the groups that have any
    n = torch.tensor([rows.get(e, 0) for e in range(E)])
    off = torch.zeros(E + 1, dtype=torch.int32)
    off[1:] = n.cumsum(0)
    R = int(off[E])
    dy, x = whole((R, 1)), whole((R, WIDE))
    dw = torch.full((E, 1, WIDE), 7.0, dtype=torch.bfloat16, device="cuda")
    eaas.eaas_grouped_matmul_dw(dy, x, off.cuda(), dw, eaas.alloc_grouped_workspace(R, E, 1, WIDE))
    for e in range(E):
        want = (dy[off[e]: off[e + 1]].float() * x[off[e]: off[e + 1]].float()).sum(0)
        assert torch.equal(dw[e, 0].float(), want), e
