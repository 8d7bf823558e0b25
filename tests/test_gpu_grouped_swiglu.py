"""The gated product and its way back against the 64-bit oracle.

Tolerances, from the arithmetic.  A sum of S products that are exact in fp32 errs by at
most S * 2^-23 of its terms' magnitudes (S + parts roundings at most).  |silu'| < 1.1, so h
moves by 1.1 dg |u| + (|silu(g)| + 1.1 dg) du where the sums move by dg and du; exponential,
sum, reciprocal and products err by (|g| + 8) 2^-23 of the result.  In the way back
|t (1 + g (1 - t))| < 1.1 as well, and that factor's error is (|g| + 8) (1 + |g|) 2^-22, in
units of dh u t, since 1 + g (1 - t) may cancel.  A bf16 result adds 2^-8 of itself.
"""
import numpy as np
import pytest
import torch

from oracle import layer_oracle as L
from paper_2509_17863_amd import eaas

pytestmark = pytest.mark.gpu
CANARY = 12345.0
TINY = 2.0 ** -133  # bf16's least step


def sizes_of(kind, E, R, rng):
    if kind == "even":
        n = np.full(E, R // E)
        n[: R - n.sum()] += 1
    elif kind == "one":
        n = np.zeros(E, int)
        n[rng.integers(E)] = R
    elif kind == "some":                     # rows of no group at the end
        n = np.bincount(rng.integers(0, 2 * E, R), minlength=2 * E)[:E]
    else:                                    # ragged, some empty
        n = np.bincount(rng.integers(0, max(E // 2, 1), R) * 2 % E, minlength=E)
    return n


def rounded(a):
    return torch.from_numpy(np.asarray(a, np.float32)).to(torch.bfloat16)


class Place:
    """rows x cols bf16 on the device, `lead` elements into its buffer and `pad` between
    rows, all of it NaN (operands) or CANARY (results) beside the rows that exist."""

    def __init__(self, rows, cols, lead=0, pad=0, data=None, used=None):
        fill = float("nan") if data is not None else CANARY
        self.flat = torch.full((lead + rows * (cols + pad) + 8,), fill, dtype=torch.bfloat16, device="cuda")
        self.t = self.flat[lead: lead + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
        if data is not None:
            d = data.clone()
            if used is not None:
                d[~torch.from_numpy(used)] = float("nan")
            self.t.copy_(d)

    def values(self, live):
        """The first rows' values; everything else has to be untouched."""
        v = self.t[:live].double().cpu().numpy()
        rest = self.flat.clone()
        rows, cols = self.t.shape
        lead = self.t.storage_offset()
        if rows:
            view = torch.as_strided(rest, (live, cols), (self.t.stride(0), 1), lead)
            view.fill_(CANARY)
        assert (rest == torch.tensor(CANARY, dtype=torch.bfloat16)).all()
        return v


class Case:
    """wide: columns of W (K) in the forward product, its outputs (N) in the way back."""

    def __init__(self, R, E, I, wide, kind="ragged", k=0, pad=0, lead=0, whole=False):
        rng = np.random.default_rng([R, E, I, wide])
        self.R, self.E, self.I, self.wide, self.k, self.pad, self.lead = R, E, I, wide, k, pad, lead
        self.offsets = np.concatenate([[0], np.cumsum(sizes_of(kind, E, R, rng))]).astype(np.int32)
        self.live = int(self.offsets[-1])
        self.off = torch.from_numpy(self.offsets).cuda()
        self.rng = rng

        def make(*shape, scale=1.0):
            if whole:
                return rounded(rng.integers(-2, 3, shape))
            return rounded(rng.normal(size=shape) * scale)

        self.make = make

    def forward(self, keep=True, **kw):
        c, k = self, self.k
        perm = c.rng.permutation(c.R).astype(np.int32) if k else None
        src = L.source_rows(c.R, perm, max(k, 1))
        x = c.make(c.R // k if k else c.R, c.wide)
        w = c.make(c.E, 2 * c.I, c.wide, scale=1.5 / np.sqrt(c.wide))
        used = np.zeros(len(x), bool)
        used[src[: c.live]] = True
        ws = eaas.alloc_grouped_workspace(c.R, c.E, 2 * c.I, c.wide)
        ws.fill_(0xFF)
        wd = w.cuda()
        h = Place(c.R, c.I, c.lead, c.pad)
        gu = Place(c.R, 2 * c.I, c.lead, c.pad) if keep else None
        take = dict(perm=torch.from_numpy(perm).cuda(), k=k) if k else {}
        self.call = lambda **more: eaas.eaas_grouped_swiglu(  # noqa: E731
            xd.t, c.off, wd, h.t, ws, gu=gu.t if keep else None, **{**take, **more})
        xd = Place(len(x), c.wide, c.lead, c.pad, x, used)
        self.call(**kw)
        want = L.grouped_swiglu(x.double().numpy(), c.offsets, w.double().numpy(), src)
        return h, gu, want

    def backward(self, with_h=True, in_place=False, spread=1.0):
        c = self
        dy = c.make(c.R, c.wide)
        w = c.make(c.E, c.wide, c.I, scale=1 / np.sqrt(c.wide))
        gu = rounded(c.rng.normal(size=(c.R, 2 * c.I)) * 2 * spread)
        live = np.arange(c.R) < c.live
        ws = eaas.alloc_grouped_workspace(c.R, c.E, c.wide, c.I)
        ws.fill_(0xFF)
        wd = w.cuda()
        h = Place(c.R, c.I, c.lead, c.pad) if with_h else None
        if in_place:
            dgu = Place(c.R, 2 * c.I, c.lead, c.pad)
            dgu.t[: c.live] = gu[: c.live].cuda()
            gud = dgu
        else:
            dgu = Place(c.R, 2 * c.I, c.lead, c.pad)
            gud = Place(c.R, 2 * c.I, c.lead, c.pad, gu, live)
        dyd = Place(c.R, c.wide, c.lead, c.pad, dy, live)
        self.call = lambda **more: eaas.eaas_grouped_swiglu_backward(  # noqa: E731
            dyd.t, c.off, wd, gud.t, dgu.t, ws, h=h.t if with_h else None, **more)
        self.call()
        a = gu[: c.live].double().numpy()
        want = L.grouped_swiglu_backward(dy.double().numpy(), c.offsets, w.double().numpy(), a)
        return dgu, h, a, want


def near(got, want, tol):
    tol = (tol + 2.0 ** -8 * (np.abs(want) + tol)) * 1.001 + TINY
    err = np.abs(got - want)
    assert (err <= tol).all(), (err.max(), np.argwhere(~(err <= tol))[:4])


def check_forward(c, h, gu, want):
    wh, wgu, mag = want
    I = c.I
    d = (c.wide + 600) * 2.0 ** -23 * mag
    g, u, dg, du = wgu[:, :I], wgu[:, I:], d[:, :I], d[:, I:]
    s = np.abs(g * L.sigmoid(g))
    near(h.values(c.live), wh, 1.1 * dg * np.abs(u) + (s + 1.1 * dg) * du +
         (np.abs(g) + 8) * 2.0 ** -23 * np.abs(wh))
    if gu is not None:
        near(gu.values(c.live), wgu, d)


def check_backward(c, dgu, h, gu, want):
    wdgu, wh, dh, mag = want
    I = c.I
    d = (c.wide + 600) * 2.0 ** -23 * mag
    g, u, t = gu[:, :I], gu[:, I:], L.sigmoid(gu[:, :I])
    rel = (np.abs(g) + 8) * 2.0 ** -23
    tol = np.concatenate([1.1 * d * np.abs(u) + np.abs(dh * u) * t * rel * 2 * (1 + np.abs(g)),
                          (d + np.abs(dh) * rel) * np.abs(g) * t], axis=1)
    near(dgu.values(c.live), wdgu, tol)
    if h is not None:
        near(h.values(c.live), wh, np.abs(wh) * rel)


SHAPES = [
    # (R, E, I, K or N, kind, k, pad, lead)
    (1, 1, 1, 1, "even", 0, 0, 0),
    (1, 5, 64, 256, "one", 0, 0, 0),
    (8, 128, 96, 128, "ragged", 8, 0, 0),
    (64, 8, 128, 256, "even", 2, 0, 0),
    (130, 3, 65, 65, "ragged", 0, 3, 1),
    (257, 4, 63, 191, "some", 0, 0, 0),
    (300, 7, 136, 200, "some", 3, 8, 8),
    (33, 6, 7, 5, "ragged", 0, 1, 3),
    (96, 512, 40, 72, "ragged", 4, 0, 0),
    (20, 2, 64, 4096, "even", 0, 0, 0),
    (9, 2, 33, 30001, "even", 3, 1, 0),
    (3, 1, 40, 70000, "one", 0, 0, 0),
    (300, 2, 72, 2048, "one", 0, 0, 0),
    (700, 2, 520, 264, "even", 0, 0, 0),
    (1040, 2, 3208, 328, "even", 4, 8, 0),
    (1500, 3, 3100, 264, "some", 0, 0, 0),
    (1300, 4, 6200, 272, "ragged", 0, 0, 0),
    (0, 3, 32, 32, "even", 0, 0, 0),
]


@pytest.mark.parametrize("keep", [False, True], ids=["h", "h_and_gu"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward(gpu, shape, keep):
    c = Case(*shape)
    check_forward(c, *c.forward(keep))


@pytest.mark.parametrize("mode", ["dgu", "dgu_and_h", "in_place"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_backward(gpu, shape, mode):
    c = Case(*shape)
    check_backward(c, *c.backward(with_h=mode != "dgu", in_place=mode == "in_place"))


WHOLE = [(5, 1, 40, 9000, "one", 0), (20, 2, 96, 1024, "some", 4), (64, 1, 64, 2048, "even", 0),
         (9, 2, 33, 3001, "even", 3), (512, 16, 512, 512, "ragged", 2), (3000, 5, 3500, 264, "ragged", 0),
         (3000, 4, 3501, 264, "some", 4), (2600, 5, 3080, 392, "ragged", 0),
         (13, 1, 16, 2992, "even", 0), (263, 1, 160, 5232, "one", 0), (18, 1, 40, 176, "even", 3),
         (2981, 1, 496, 1808, "even", 0), (17, 1, 16, 3328, "even", 0), (362, 1, 272, 4320, "one", 0),
         (2002, 1, 1632, 1760, "even", 0), (130, 3, 65, 65, "ragged", 0),
         # large tiles whose sums are three and four steps
         (24506, 31, 240, 144, "even", 0), (28561, 14, 400, 160, "even", 0), (34026, 63, 16, 224, "even", 3)]


def test_every_kernel_is_among_these():
    """On the host: every way of computing either, in one part and in several."""
    for way in ("swiglu", "swiglu_backward"):
        seen = set()
        for R, E, I, wide, *_ in WHOLE:
            N, K = (2 * I, wide) if way == "swiglu" else (wide, I)
            in16 = K % 8 == 0 and (way == "swiglu" or N % 8 == 0)
            kernel, rows, parts = eaas._grouped_plan(way, R, E, N, K, in16)
            seen.add((in16, kernel, rows if kernel == "few" else 0, parts > 1))
        for want in [(True, "large", 0, False), (True, "any", 0, True), (False, "any", 0, False),
                     (False, "any", 0, True), (True, "few", 16, False), (True, "few", 16, True),
                     (True, "few", 32, False), (True, "few", 32, True), (True, "few", 64, False),
                     (True, "few", 64, True)]:
            assert want in seen, (way, want, seen)



@pytest.mark.parametrize("shape", WHOLE, ids=str)
def test_sums_that_are_exact_in_any_order(gpu, shape):
    """Parts, columns or tiles that are lost, doubled or misplaced show: whole numbers, in
    bf16 to the one rounding."""
    c = Case(*shape, whole=True)
    h, gu, want = c.forward()
    assert np.array_equal(gu.values(c.live), rounded(want[1]).double().numpy())
    check_forward(c, h, gu, want)
    check_backward(c, *c.backward())


@pytest.mark.parametrize("shape", [(64, 1, 64, 2048, "even", 0), (3000, 5, 6200, 264, "ragged", 0),
                                   (9, 2, 33, 3001, "even", 0)], ids=str)
def test_gates_of_any_size(gpu, shape):
    c = Case(*shape)
    check_backward(c, *c.backward(spread=20.0))


def test_projections_of_any_size(gpu):
    """Sums of hundreds: no infinity where h is finite, zero where the gate is far below."""
    x = torch.full((2, 64), 8.0, dtype=torch.bfloat16, device="cuda")
    w = torch.zeros((1, 4, 64), dtype=torch.bfloat16, device="cuda")
    w[0, 0], w[0, 1], w[0, 2], w[0, 3] = 8.0, -8.0, 2.0, 2.0  # gates +-4096, ups 1024
    h = torch.empty((2, 2), dtype=torch.bfloat16, device="cuda")
    eaas.eaas_grouped_swiglu(x, torch.tensor([0, 2], dtype=torch.int32, device="cuda"), w, h,
                             eaas.alloc_grouped_workspace(2, 1, 4, 64))
    assert (h[:, 0] == 4096.0 * 1024).all() and (h[:, 1] == 0).all()


@pytest.mark.parametrize("R,E,I,K", [(200, 3, 96, 160), (1200, 3, 3104, 264), (12, 3, 64, 256)])
def test_no_numbers_stay_in_their_rows(gpu, R, E, I, K):
    g = torch.Generator().manual_seed(0)
    x = torch.randn((R, K), generator=g).to(torch.bfloat16)
    x[5, 7], x[R - 3, 0] = float("inf"), float("nan")
    w = torch.randn((E, 2 * I, K), generator=g).to(torch.bfloat16).cuda()
    off = torch.tensor([R * e // E for e in range(E + 1)], dtype=torch.int32, device="cuda")
    h, gu = (torch.empty((R, n), dtype=torch.bfloat16, device="cuda") for n in (I, 2 * I))
    eaas.eaas_grouped_swiglu(x.cuda(), off, w, h, eaas.alloc_grouped_workspace(R, E, 2 * I, K), gu=gu)
    bad = (~torch.isfinite(gu)).any(1).nonzero().reshape(-1).tolist()
    assert bad == [5, R - 3] and torch.isnan(h[R - 3]).all()
    assert torch.isfinite(h[torch.arange(R) != 5][: R - 4]).all()


@pytest.mark.parametrize("shape", [(900, 4, 200, 2048, "ragged", 0), (1500, 3, 3104, 264, "even", 0),
                                   (16, 8, 256, 1024, "even", 2)], ids=str)
def test_equal_calls_other_streams_and_graphs(gpu, shape):
    for way in ("forward", "backward"):
        c = Case(*shape)
        first = c.forward() if way == "forward" else c.backward()
        outs = [p.t for p in first[:2]]
        want = [t.clone() for t in outs]
        side = torch.cuda.Stream()
        for stream in (None, side):
            for t in outs:
                t.zero_()
            side.wait_stream(torch.cuda.current_stream())
            c.call(stream=stream)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs, want))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.call()
        for _ in range(3):
            for t in outs:
                t.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs, want))
            outs[0].float().sum().item()


@pytest.mark.parametrize("R,E,N,K", [(1024, 8, 6200, 264), (64, 8, 64, 2048), (300, 6, 34, 47)])
def test_offsets_that_do_not_ascend_stay_in_bounds(gpu, R, E, N, K):
    """Results are then undefined, but nothing outside the results is written."""
    wild = torch.tensor([0, R] * (E // 2) + [0], dtype=torch.int32, device="cuda")
    bf = dict(dtype=torch.bfloat16, device="cuda")
    x, w = torch.randn((R, K), **bf), torch.randn((E, N, K), **bf)
    n = eaas.eaas_grouped_workspace_bytes(R, E, N, K)
    guard = torch.zeros(n + 4096, dtype=torch.uint8, device="cuda")
    h, gu = torch.full((R + 8, N // 2), CANARY, **bf), torch.full((R + 8, N), CANARY, **bf)
    eaas.eaas_grouped_swiglu(x, wild, w, h[:R], guard[:n], gu=gu[:R])
    c = torch.tensor(CANARY, dtype=torch.bfloat16).item()
    assert (h[R:] == c).all() and (gu[R:] == c).all()
    dy = torch.randn((R, N), **bf)
    dgu, h, gu = torch.full((R + 8, 2 * K), CANARY, **bf), torch.full((R + 8, K), CANARY, **bf), torch.randn((R, 2 * K), **bf)
    eaas.eaas_grouped_swiglu_backward(dy, wild, w, gu, dgu[:R], guard[:n], h=h[:R])
    assert (h[R:] == c).all() and (dgu[R:] == c).all() and (guard[n:] == 0).all()


def test_results_beside_one_another(gpu):
    """h and the projections in one array, and in place of them their gradients."""
    R, E, I, K = 300, 3, 136, 200
    c = Case(R, E, I, K, "some")
    x, w = c.make(R, K), c.make(E, 2 * I, K, scale=0.1)
    both = Place(R, 3 * I)
    ws = eaas.alloc_grouped_workspace(R, E, 2 * I, K)
    eaas.eaas_grouped_swiglu(x.cuda(), c.off, w.cuda(), both.t[:, :I], ws, gu=both.t[:, I:])
    want = L.grouped_swiglu(x.double().numpy(), c.offsets, w.double().numpy(), np.arange(R))
    v = both.values(c.live)
    near(v[:, I:], want[1], (K + 600) * 2.0 ** -23 * want[2])
    h, gu = (torch.empty((R, n), dtype=torch.bfloat16, device="cuda") for n in (I, 2 * I))
    eaas.eaas_grouped_swiglu(x.cuda(), c.off, w.cuda(), h, ws, gu=gu)
    assert np.array_equal(v[:, :I], h[: c.live].double().cpu().numpy())


@pytest.mark.parametrize("R,E,I,wide", [(1500, 3, 3104, 264), (1300, 4, 6200, 272), (64, 8, 128, 256),
                                        (300, 2, 72, 2048)])
def test_results_from_any_element(gpu, R, E, I, wide):
    """Aligned operands (the kernels for those), results and projections from odd elements."""
    for lead, pad in ((0, 0), (1, 3), (3, 0)):
        c = Case(R, E, I, wide, "some")
        x, w = c.make(R, wide), c.make(E, 2 * I, wide, scale=0.1)
        h, gu = Place(R, I, lead, pad), Place(R, 2 * I, lead, pad)
        eaas.eaas_grouped_swiglu(x.cuda(), c.off, w.cuda(), h.t,
                                 eaas.alloc_grouped_workspace(R, E, 2 * I, wide), gu=gu.t)
        check_forward(c, h, gu, L.grouped_swiglu(x.double().numpy(), c.offsets, w.double().numpy(), np.arange(R)))
        dy, wd = c.make(R, wide), c.make(E, wide, I, scale=0.1)
        proj = rounded(c.rng.normal(size=(R, 2 * I)))
        gud, dgu, h = Place(R, 2 * I, lead, pad, proj), Place(R, 2 * I, lead, pad), Place(R, I, lead, pad)
        eaas.eaas_grouped_swiglu_backward(dy.cuda(), c.off, wd.cuda(), gud.t, dgu.t,
                                          eaas.alloc_grouped_workspace(R, E, wide, I), h=h.t)
        a = proj[: c.live].double().numpy()
        check_backward(c, dgu, h, a, L.grouped_swiglu_backward(dy.double().numpy(), c.offsets,
                                                               wd.double().numpy(), a))


def test_rows_past_32_bit_offsets(gpu):
    """More than 2^31 elements of the projections, of dgu and h."""
    R, I, K = 70000, 16384, 32
    bf = dict(dtype=torch.bfloat16, device="cuda")
    x, w = torch.randn((R, K), **bf), torch.randn((1, 2 * I, K), **bf)
    off = torch.tensor([0, R], dtype=torch.int32, device="cuda")
    h, gu = torch.empty((R, I), **bf), torch.empty((R, 2 * I), **bf)
    eaas.eaas_grouped_swiglu(x, off, w, h, eaas.alloc_grouped_workspace(R, 1, 2 * I, K), gu=gu)
    for r in (0, 65535, 65536, 69999):
        p = w[0].double() @ x[r].double()
        assert ((gu[r].double() - p).abs() <= 2.0 ** -8 * p.abs() + 1e-4).all()
        want = torch.sigmoid(p[:I]) * p[:I] * p[I:]
        assert ((h[r].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-3).all()
    dy, wd = torch.randn((R, 8), **bf), torch.randn((1, 8, I), **bf)
    keep = gu[[0, 65536, 69999]].double()
    eaas.eaas_grouped_swiglu_backward(dy, off, wd, gu, gu, eaas.alloc_grouped_workspace(R, 1, 8, I), h=h)
    for n, r in enumerate((0, 65536, 69999)):
        dh = dy[r].double() @ wd[0].double()
        g, u = keep[n, :I], keep[n, I:]
        t = torch.sigmoid(g)
        want = torch.cat([dh * u * t * (1 + g * (1 - t)), dh * g * t])
        assert ((gu[r].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-3).all()
        assert ((h[r].double() - g * t * u).abs() <= 2.0 ** -8 * (g * t * u).abs() + 1e-6).all()
