"""Results of more tiles than one dimension of a grid holds (2^32 threads), with sums of one
product, which are exact: the gated product, its way back and block-scaled e4m3."""
import pytest
import torch

from paper_2509_17863_amd import eaas

pytestmark = pytest.mark.gpu
E, WIDE = 1024, 1 << 21  # 1024 x 2^14 tiles of 128 columns (64 of h) and 256 threads


def whole(shape, top=4):
    t = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    for part in t.view(-1).split(1 << 28):
        part.copy_(torch.randint(-top, top + 1, part.shape, dtype=torch.int8, device="cuda"))
    return t


@pytest.fixture(autouse=True)
def free_memory():
    yield
    torch.cuda.empty_cache()


def offsets():
    return torch.arange(E + 1, dtype=torch.int32, device="cuda")


def test_gated(gpu):
    x, w = whole((E, 1)), whole((E, WIDE, 1))
    h = torch.empty((E, WIDE // 2), dtype=torch.bfloat16, device="cuda")
    gu = torch.empty((E, WIDE), dtype=torch.bfloat16, device="cuda")
    eaas.eaas_grouped_swiglu(x, offsets(), w, h, eaas.alloc_grouped_workspace(E, E, WIDE, 1), gu=gu)
    for r in range(0, E, 64):
        assert torch.equal(gu[r: r + 64], w[r: r + 64, :, 0] * x[r: r + 64])
        g, u = gu[r: r + 64].double().split(WIDE // 2, dim=1)
        want = g * torch.sigmoid(g) * u
        # (|g| <= 16: the activation errs by 24 * 2^-23 of itself)
        assert ((h[r: r + 64].double() - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -18)).all()


def test_way_back(gpu):
    dy, w, gu = whole((E, 1)), whole((E, 1, WIDE)), whole((E, 2 * WIDE))
    keep = gu[::64].clone()
    eaas.eaas_grouped_swiglu_backward(dy, offsets(), w, gu, gu, eaas.alloc_grouped_workspace(E, E, 1, WIDE))
    for n, r in enumerate(range(0, E, 64)):
        dh = w[r, 0].double() * dy[r].double()
        g, u = keep[n].double().split(WIDE)
        t = torch.sigmoid(g)
        want = torch.cat([dh * u * t * (1 + g * (1 - t)), dh * g * t])
        # (no gate here lies next to the zero of 1 + g (1 - t), at -1.28: 24 * 5 * 2^-22)
        assert ((gu[r].double() - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -14)).all()


def test_e4m3(gpu):
    value = torch.arange(-4, 5, device="cuda").to(torch.float8_e4m3fn).view(torch.uint8)
    x = value[torch.randint(0, 9, (E, 1), device="cuda")]
    w = torch.empty((E, WIDE, 1), dtype=torch.uint8, device="cuda")
    for part in w.view(-1).split(1 << 27):
        part.copy_(value[torch.randint(0, 9, part.shape, device="cuda")])
    xs, ws = torch.full((E, 1), 2.0, device="cuda"), torch.empty((E, WIDE // 128, 1), device="cuda")
    ws.copy_(2.0 ** torch.randint(-1, 2, ws.shape, device="cuda"))
    y = torch.empty((E, WIDE), dtype=torch.bfloat16, device="cuda")
    eaas.eaas_grouped_matmul_fp8(x, xs, offsets(), w, ws, y, eaas.alloc_grouped_fp8_workspace(E, E, WIDE, 1))
    for r in range(0, E, 64):
        want = w[r: r + 64, :, 0].view(torch.float8_e4m3fn).float() * x[r: r + 64].view(torch.float8_e4m3fn).float()
        want = want * 2 * ws[r: r + 64, :, 0].repeat_interleave(128, 1)
        assert torch.equal(y[r: r + 64].float(), want)
