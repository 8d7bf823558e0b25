"""Grouped products of an expert layer (forward, both gradients, 8-bit integers)
against the 64-bit oracle.

Tolerances, from the arithmetic.  Products of bf16 values are exact in fp32; a sum
of S of them errs by at most S * 2^-23 of the sum of their magnitudes (each of S
additions by one unit in the last place at most, whatever their order), and a bf16
result by 2^-8 of itself more.  8-bit sums are exact and their two fp32 products
are defined one after the other, so those results are equal bit for bit.
"""
import numpy as np
import pytest
import torch

from oracle import layer_oracle as L
from paper_2509_17863_amd import eaas

pytestmark = pytest.mark.gpu
CANARY = 12345.0


def bf16(a):
    return torch.from_numpy(np.asarray(a, np.float32)).to(torch.bfloat16)


def sizes_of(kind, E, R, rng):
    """Rows of each group, R in all or (kind 'some') fewer."""
    if kind == "even":
        n = np.full(E, R // E)
        n[: R - n.sum()] += 1
    elif kind == "one":                      # every row in one group, the rest empty
        n = np.zeros(E, int)
        n[rng.integers(E)] = R
    elif kind == "some":                     # rows of other servers' experts at the end
        n = np.bincount(rng.integers(0, 2 * E, R), minlength=2 * E)[:E]
    else:                                    # ragged, some empty
        n = np.bincount(rng.integers(0, max(E // 2, 1), R) * 2 % E, minlength=E)
    return n


class Case:
    """Seeded inputs on the host (64 bits) and the device; whatever no result may
    depend on (pads between rows, rows of no group) is NaN on the device."""

    def __init__(self, R, E, N, K, kind="ragged", k=0, pad=0, seed=0, i8=False):
        rng = np.random.default_rng([R, E, N, K, seed])
        self.R, self.E, self.N, self.K, self.k, self.pad = R, E, N, K, k, pad
        n = sizes_of(kind, E, R, rng)
        self.offsets = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        self.live = int(self.offsets[-1])
        self.perm = rng.permutation(R).astype(np.int32) if k else None
        self.src = L.source_rows(R, self.perm, max(k, 1))
        self.take = {}
        if k:
            self.take = dict(perm=torch.from_numpy(self.perm).cuda(), k=k)
        self.off = torch.from_numpy(self.offsets).cuda()
        xr = R // k if k else R
        used = np.zeros(xr, bool)
        used[self.src[: self.live]] = True
        if i8:
            self.xq = rng.integers(-127, 128, (xr, K)).astype(np.int8)
            self.xs = (rng.random(xr) + 0.5).astype(np.float32)
            self.wq = rng.integers(-127, 128, (E, N, K)).astype(np.int8)
            self.wscale = (rng.random((E, N)) + 0.5).astype(np.float32) * 1e-3
        else:
            self.x = bf16(rng.normal(size=(xr, K)))
            self.w = bf16(rng.normal(size=(E, N, K)) / np.sqrt(K))
            self.dy = bf16(rng.normal(size=(R, N)))
            self.dx_ = self.rows(self.x, used)
            self.dw_ = self.w.cuda()
            rows = np.zeros(R, bool)
            rows[: self.live] = True
            self.ddy = self.rows(self.dy, rows)
        self.ws = eaas.alloc_grouped_workspace(R, E, N, K)
        self.ws.fill_(0xFF)

    def rows(self, t, used):
        """On the device, `pad` elements between the rows, NaN where unused."""
        d = torch.full((t.shape[0], t.shape[1] + self.pad), float("nan"), dtype=t.dtype)
        d[:, : t.shape[1]] = t
        d[~torch.from_numpy(used)] = float("nan")
        return d.cuda()[:, : t.shape[1]]

    def out(self, rows, cols, dtype):
        return torch.full((rows, cols + self.pad), CANARY, dtype=dtype, device="cuda")[:, :cols]

    def check(self, got, want, mag, terms):
        """Rows of the groups within the tolerance, everything else untouched."""
        g = got.double().cpu().numpy()
        tol = terms * 2.0 ** -23 * mag
        if got.dtype == torch.bfloat16:
            tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
        err = np.abs(g[: len(want)] - want)
        assert (err <= tol).all(), (err.max(), np.argwhere(~(err <= tol))[:4])
        whole = got._base if got._base is not None else got
        c = torch.tensor(CANARY, dtype=got.dtype).item()
        assert (whole[len(want):] == c).all()
        assert (whole[:, got.shape[1]:] == c).all()


# (R, E, N, K, kind, k, pad): one row, one group, many groups, edges of the tiles
# on either side, sizes below a chunk, odd sizes, long sums that are split
SHAPES = [
    (1, 1, 1, 1, "even", 0, 0),
    (1, 5, 128, 256, "one", 0, 0),
    (8, 128, 192, 128, "ragged", 8, 0),
    (64, 8, 256, 256, "even", 2, 0),
    (130, 3, 129, 65, "ragged", 0, 3),
    (257, 4, 127, 191, "some", 0, 0),
    (256, 2, 128, 64, "even", 0, 8),
    (300, 7, 136, 200, "some", 3, 8),
    (96, 1024, 40, 72, "ragged", 4, 0),
    (33, 6, 7, 5, "ragged", 0, 1),
    (48, 2, 64, 4096, "even", 0, 0),
    (40, 1, 4096, 96, "one", 4, 0),
    (5000, 2, 72, 88, "ragged", 2, 0),
    (3001, 3, 33, 47, "some", 0, 5),
    (700, 2, 520, 264, "even", 0, 0),
    (1111, 5, 384, 640, "ragged", 0, 0),
    (0, 3, 32, 32, "even", 0, 0),
]


# groups of many rows, rows and columns that end inside a 256 x 256 tile, sums that end
# inside a step: the gradient in the weights takes those tiles here, the gradient in
# the rows in one case, other products the other kernels (test_gpu_grouped_plans.py has
# shapes for each kernel by name, and results of more tiles than CUs)
LARGE = [
    (1500, 3, 6200, 72, "ragged", 0, 0),
    (1040, 2, 9000, 136, "even", 4, 8),
    (1024, 4, 200, 9224, "some", 0, 0),
    (1030, 5, 1800, 1544, "even", 0, 0),
    (1290, 3, 2568, 2056, "ragged", 6, 8),
]


# sums of some steps, which take the large tiles in every direction (8-bit included),
# with empty groups; and sums of one to many parts (whose tolerance grows with the
# length of the sum; test_gpu_grouped_plans.py has exact ones)
LONGER = [
    (1200, 4, 8200, 464, "some", 0, 0),
    (1040, 2, 9000, 528, "even", 4, 8),
    (1024, 4, 264, 9224, "ragged", 0, 0),
    (5, 1, 40, 70000, "one", 0, 0),
    (9, 2, 33, 30001, "even", 3, 1),
    (3, 2, 30000, 48, "some", 0, 0),
    (30000, 1, 24, 40, "even", 2, 0),
    (200, 2, 264, 9000, "one", 4, 8),
]


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES + LARGE + LONGER, ids=str)
def test_forward(gpu, shape, out):
    c = Case(*shape)
    y = c.out(c.R, c.N, out)
    eaas.eaas_grouped_matmul(c.dx_, c.off, c.dw_, y, c.ws, **c.take)
    want, mag = L.grouped_matmul(c.x.double().numpy(), c.offsets, c.w.double().numpy(), c.src)
    c.check(y, want, mag, c.K)


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES + LARGE + LONGER, ids=str)
def test_gradient_in_the_rows(gpu, shape, out):
    c = Case(*shape)
    dx = c.out(c.R, c.K, out)
    eaas.eaas_grouped_matmul_dx(c.ddy, c.off, c.dw_, dx, c.ws)
    want, mag = L.grouped_matmul_dx(c.dy.double().numpy(), c.offsets, c.w.double().numpy())
    c.check(dx, want, mag, c.N)


@pytest.mark.parametrize("mode", ["bf16", "fp32", "accumulate"])
@pytest.mark.parametrize("shape", SHAPES + LARGE + LONGER, ids=str)
def test_gradient_in_the_weights(gpu, shape, mode):
    c = Case(*shape)
    dt = torch.bfloat16 if mode == "bf16" else torch.float32
    dw = torch.full((c.E, c.N, c.K), 3.0 if mode == "accumulate" else float("nan"), dtype=dt,
                    device="cuda")
    eaas.eaas_grouped_matmul_dw(c.ddy, c.dx_, c.off, dw, c.ws, accumulate=mode == "accumulate",
                                **c.take)
    want, mag = L.grouped_matmul_dw(c.dy.double().numpy(), c.x.double().numpy(), c.offsets, c.src)
    terms = max(c.R, 1)
    if mode == "accumulate":  # one more term
        want, mag, terms = want + 3.0, mag + 3.0, terms + 1
    g = dw.double().cpu().numpy()
    tol = terms * 2.0 ** -23 * mag
    if mode == "bf16":
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
    assert (np.abs(g - want) <= tol).all()


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES + LARGE + LONGER, ids=str)
def test_int8(gpu, shape, out):
    c = Case(*shape, i8=True)
    y = c.out(c.R, c.N, out)
    d = [torch.from_numpy(a).cuda() for a in (c.xq, c.xs, c.wq, c.wscale)]
    eaas.eaas_grouped_matmul_int8(d[0], d[1], c.off, d[2], d[3], y, c.ws, **c.take)
    want = torch.from_numpy(L.grouped_matmul_int8(c.xq, c.xs, c.offsets, c.wq, c.wscale, c.src))
    assert torch.equal(y[: c.live].cpu(), want.to(out))
    c.check(y, want.to(out).double().numpy(), np.zeros(want.shape), 0)


def test_int8_largest_sums(gpu):
    """K just below its limit, every product at its largest."""
    K = (1 << 17) - 1
    x = torch.full((3, K), -128, dtype=torch.int8, device="cuda")
    w = torch.full((1, 5, K), -128, dtype=torch.int8, device="cuda")
    one = torch.ones(3, device="cuda")
    y = torch.empty((3, 5), device="cuda")
    off = torch.tensor([0, 3], dtype=torch.int32, device="cuda")
    eaas.eaas_grouped_matmul_int8(x, one, off, w, torch.ones((1, 5), device="cuda"), y,
                                  eaas.alloc_grouped_workspace(3, 1, 5, K))
    assert (y == float(np.float32(K * 16384))).all()


def test_infinities_and_nan_stay_in_their_rows(gpu):
    c = Case(200, 3, 96, 160, "even")
    x = c.x.clone()
    x[5, 7], x[100, 0] = float("inf"), float("nan")
    y = c.out(c.R, c.N, torch.float32)
    eaas.eaas_grouped_matmul(x.cuda(), c.off, c.dw_, y, c.ws)
    bad = ~torch.isfinite(y).all(dim=1).cpu()
    assert bad.nonzero().reshape(-1).tolist() == [5, 100]
    assert not torch.isfinite(y[5]).any() and torch.isnan(y[100]).all()
    # and in the weights' gradient, in their group and column
    dw = torch.empty((c.E, c.N, c.K), device="cuda")
    eaas.eaas_grouped_matmul_dw(c.ddy, x.cuda(), c.off, dw, c.ws)
    bad = (~torch.isfinite(dw)).any(dim=1).cpu().nonzero().tolist()
    e5, e100 = [int(np.searchsorted(c.offsets, r, "right") - 1) for r in (5, 100)]
    assert sorted(bad) == sorted([[e5, 7], [e100, 0]])


def test_equal_calls_give_equal_bits(gpu):
    c = Case(900, 4, 200, 2048, "ragged")
    outs = []
    for _ in range(3):
        y, dx = c.out(c.R, c.N, torch.float32), c.out(c.R, c.K, torch.float32)
        dw = torch.empty((c.E, c.N, c.K), device="cuda")
        eaas.eaas_grouped_matmul(c.dx_, c.off, c.dw_, y, c.ws)
        eaas.eaas_grouped_matmul_dx(c.ddy, c.off, c.dw_, dx, c.ws)
        eaas.eaas_grouped_matmul_dw(c.ddy, c.dx_, c.off, dw, c.ws)
        outs.append((y.clone(), dx.clone(), dw.clone()))
    for o in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o, outs[0]))


def test_offsets_outside_the_rows_are_clamped(gpu):
    c = Case(64, 4, 32, 32, "even")
    y = c.out(c.R, c.N, torch.float32)
    wild = torch.tensor([-5, 16, 32, 48, 1 << 30], dtype=torch.int32, device="cuda")
    eaas.eaas_grouped_matmul(c.dx_, wild, c.dw_, y, c.ws)
    want, mag = L.grouped_matmul(c.x.double().numpy(), c.offsets, c.w.double().numpy(), c.src)
    c.check(y, want, mag, c.K)


@pytest.mark.parametrize("R,E,N,K", [(1024, 8, 6200, 72), (64, 8, 64, 2048), (300, 6, 33, 47)])
def test_offsets_that_do_not_ascend_stay_in_bounds(gpu, R, E, N, K):
    """Results are then undefined, but nothing outside the result is written."""
    c = Case(R, E, N, K, "even")
    wild = torch.tensor([0, R] * (E // 2) + [0], dtype=torch.int32, device="cuda")
    guard = torch.zeros(c.ws.numel() + 4096, dtype=torch.uint8, device="cuda")
    ws = guard[: c.ws.numel()]
    y, dx = c.out(R + 8, N, torch.float32), c.out(R + 8, K, torch.float32)
    dw = torch.full((E + 1, N, K), CANARY, device="cuda")
    eaas.eaas_grouped_matmul(c.dx_, wild, c.dw_, y[:R], ws)
    eaas.eaas_grouped_matmul_dx(c.ddy, wild, c.dw_, dx[:R], ws)
    eaas.eaas_grouped_matmul_dw(c.ddy, c.dx_, wild, dw[:E], ws)
    torch.cuda.synchronize()
    assert (y[R:] == CANARY).all() and (dx[R:] == CANARY).all() and (dw[E] == CANARY).all()
    assert (guard[c.ws.numel():] == 0).all()


def test_another_stream_and_a_graph(gpu):
    c = Case(512, 4, 128, 256, "even", k=2)
    y = c.out(c.R, c.N, torch.float32)
    dw = torch.empty((c.E, c.N, c.K), device="cuda")

    def step(stream):
        eaas.eaas_grouped_matmul(c.dx_, c.off, c.dw_, y, c.ws, stream=stream, **c.take)
        eaas.eaas_grouped_matmul_dw(c.ddy, c.dx_, c.off, dw, c.ws, stream=stream, **c.take)

    step(None)
    torch.cuda.synchronize()
    want = y.clone(), dw.clone()
    side = torch.cuda.Stream()
    y.fill_(0)
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    assert torch.equal(y, want[0]) and torch.equal(dw, want[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(torch.cuda.current_stream())
    for _ in range(3):
        y.fill_(0)
        dw.fill_(0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[0]) and torch.equal(dw, want[1])
        (y.sum() + dw.sum()).item()


def test_result_past_32_bit_offsets(gpu):
    """More than 2^32 bytes and 2^31 elements of y and dW."""
    R, N, K = 70000, 32768, 32
    x = torch.randn((R, K), device="cuda").to(torch.bfloat16)
    w = torch.randn((1, N, K), device="cuda").to(torch.bfloat16)
    off = torch.tensor([0, R], dtype=torch.int32, device="cuda")
    y = torch.empty((R, N), dtype=torch.bfloat16, device="cuda")
    ws = eaas.alloc_grouped_workspace(R, 1, N, K)
    eaas.eaas_grouped_matmul(x, off, w, y, ws)
    for r in (0, 65535, 65536, 69999):
        want = w[0].double() @ x[r].double()
        assert ((y[r].double() - want).abs() <= 2.0 ** -7 * want.abs() + 1e-4).all()
    dx = torch.empty((R, K), dtype=torch.float32, device="cuda")
    eaas.eaas_grouped_matmul_dx(y, off, w, dx, ws)
    for r in (0, 69999):
        t = y[r].double()[:, None] * w[0].double()
        assert ((dx[r].double() - t.sum(0)).abs() <= N * 2.0 ** -23 * t.abs().sum(0)).all()
    del y, dx
    E, n = 5, 21000
    dy = torch.randn((8, n), device="cuda").to(torch.bfloat16)
    xx = torch.randn((8, n), device="cuda").to(torch.bfloat16)
    off = torch.tensor([0, 1, 2, 3, 4, 8], dtype=torch.int32, device="cuda")
    dw = torch.empty((E, n, n), dtype=torch.bfloat16, device="cuda")
    eaas.eaas_grouped_matmul_dw(dy, xx, off, dw, eaas.alloc_grouped_workspace(8, E, n, n))
    for row in (0, n - 1):
        want = (dy[4:, row].double()[:, None] * xx[4:].double()).sum(0)
        mag = (dy[4:, row].double()[:, None] * xx[4:].double()).abs().sum(0)
        assert ((dw[4, row].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -20 * mag).all()
