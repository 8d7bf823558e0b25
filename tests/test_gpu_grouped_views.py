"""Grouped products of operands and results that start at any element and lie side by
side in one array.  Whole numbers small enough for every order of summation to be
exact: results are equal bit for bit, to one rounding in bf16, and nothing around
them changes."""
import pytest
import torch

from paper_2509_17863_amd import eaas

pytestmark = pytest.mark.gpu
CANARY = 99.0


def whole(shape, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-4, 5, shape, generator=g).to(torch.bfloat16)


class View:
    """`rows` x `cols` on the device, `lead` elements into its buffer, `pad` between rows."""

    def __init__(self, rows, cols, lead, pad, dtype=torch.bfloat16, data=None):
        fill = CANARY if data is None else float("nan")
        self.flat = torch.full((lead + rows * (cols + pad),), fill, dtype=dtype, device="cuda")
        self.wide = self.flat[lead:].view(rows, cols + pad)
        self.t = self.wide[:, :cols]
        if data is not None:
            self.t.copy_(data)

    def check(self, want, live):
        assert torch.equal(self.t[:live].cpu().double(), want[:live].to(self.flat.dtype).double())
        rest = self.flat.clone()
        lead = self.flat.numel() - self.wide.numel()
        rest[lead:].view(self.wide.shape)[:live, : self.t.shape[1]] = CANARY
        assert (rest == CANARY).all()


def offsets_of(R, E, seed):
    g = torch.Generator().manual_seed(seed)
    n = torch.bincount(torch.randint(0, max(E // 2, 1), (R,), generator=g) * 2 % E, minlength=E)
    return torch.cat([torch.zeros(1, dtype=torch.long), n.cumsum(0)])


# few rows, many rows on large tiles (some of whose results leave element by element),
# and the kernel for any alignment, whose sums are in one part or several
SHAPES = [(96, 8, 256, 512), (1500, 3, 6208, 264), (1040, 2, 264, 6208), (300, 3, 136, 200),
          (7, 2, 24, 8200), (1030, 3, 1800, 1544)]
# (elements ahead of an operand, of a result, between rows)
PLACES = [(1, 0, 0), (0, 1, 0), (1, 1, 3), (3, 2, 8), (8, 4, 8), (0, 0, 5)]


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("place", PLACES, ids=str)
@pytest.mark.parametrize("R,E,N,K", SHAPES)
def test_bases_of_any_element(gpu, R, E, N, K, place, out):
    lead, lead_out, pad = place
    off = offsets_of(R, E, R)
    x, dy, w = whole((R, K), 1), whole((R, N), 2), whole((E, N, K), 3)
    dx_, ddy = View(R, K, lead, pad, data=x), View(R, N, lead, pad, data=dy)
    doff, dw = off.to(torch.int32).cuda(), w.cuda()
    ws = eaas.alloc_grouped_workspace(R, E, N, K)
    y, dx = View(R, N, lead_out, pad, out), View(R, K, lead_out, pad, out)
    eaas.eaas_grouped_matmul(dx_.t, doff, dw, y.t, ws)
    eaas.eaas_grouped_matmul_dx(ddy.t, doff, dw, dx.t, ws)
    gw = torch.full((E, N, K), CANARY, dtype=out, device="cuda")
    eaas.eaas_grouped_matmul_dw(ddy.t, dx_.t, doff, gw, ws)
    want_y, want_dx = torch.zeros((R, N)), torch.zeros((R, K))
    for e in range(E):
        s = slice(off[e], off[e + 1])
        want_y[s] = x[s].float() @ w[e].float().t()
        want_dx[s] = dy[s].float() @ w[e].float()
        assert torch.equal(gw[e].cpu(), (dy[s].float().t() @ x[s].float()).to(out))
    y.check(want_y, R)
    dx.check(want_dx, R)


@pytest.mark.parametrize("lead", [1, 3, 16])
@pytest.mark.parametrize("R,E,N,K", [(96, 8, 256, 512), (1500, 3, 6208, 272), (300, 3, 133, 209)])
def test_8_bit_rows_of_any_byte(gpu, R, E, N, K, lead):
    g = torch.Generator().manual_seed(lead)
    off = offsets_of(R, E, R)
    x, w = (torch.randint(-127, 128, s, generator=g, dtype=torch.int8) for s in ((R, K), (E, N, K)))
    flat = torch.full((lead + R * K,), 77, dtype=torch.int8, device="cuda")
    dx = flat[lead:].view(R, K)
    dx.copy_(x)
    y = View(R, N, lead, 3, torch.float32)
    eaas.eaas_grouped_matmul_int8(dx, torch.ones(R, device="cuda"), off.to(torch.int32).cuda(),
                                  w.cuda(), torch.ones((E, N), device="cuda"), y.t,
                                  eaas.alloc_grouped_workspace(R, E, N, K))
    want = torch.zeros((R, N))
    for e in range(E):
        s = slice(off[e], off[e + 1])
        want[s] = (x[s].double() @ w[e].double().t()).float()
    y.check(want, R)


@pytest.mark.parametrize("R,E,N,K", [(96, 8, 256, 512), (1500, 3, 6208, 264), (300, 3, 133, 209)])
def test_results_beside_their_operands(gpu, R, E, N, K):
    off = offsets_of(R, E, R)
    x, dy, w = whole((R, K), 4), whole((R, N), 5), whole((E, N, K), 6)
    doff, dw = off.to(torch.int32).cuda(), w.cuda()
    ws = eaas.alloc_grouped_workspace(R, E, N, K)
    both = View(R, K + N, 0, 0)
    both.t[:, :K] = x.cuda()
    eaas.eaas_grouped_matmul(both.t[:, :K], doff, dw, both.t[:, K:], ws)
    back = View(R, K + N, 0, 0)
    back.t[:, K:] = dy.cuda()
    eaas.eaas_grouped_matmul_dx(back.t[:, K:], doff, dw, back.t[:, :K], ws)
    want_y, want_dx = torch.zeros((R, N)), torch.zeros((R, K))
    for e in range(E):
        s = slice(off[e], off[e + 1])
        want_y[s] = x[s].float() @ w[e].float().t()
        want_dx[s] = dy[s].float() @ w[e].float()
    both.check(torch.cat([x.float(), want_y], 1), R)
    back.check(torch.cat([want_dx, dy.float()], 1), R)
