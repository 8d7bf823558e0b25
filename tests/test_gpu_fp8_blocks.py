"""Block-scaled e4m3: codes and scales bit for bit, products against the 64-bit oracle.

Tolerances, from the arithmetic.  Codes hold whole multiples of 2^-9, products of them
are exact in fp32; a sum of a block's 128 errs by at most 128 * 2^-23 of its terms'
magnitudes, the scales' product by 2^-24, and joining B blocks in P parts by B + P + 1
roundings: (128 + B + P + 2) * 2^-23 of the magnitudes in all.  On large tiles with bf16
results the matrix instruction rounds each of eight products that it adds at a time to
2^-13 of the power of two under the largest, that is by at most 2^-14 of it: 7 * 2^-14 of
the magnitudes.  A bf16 result adds 2^-8 of itself.
"""
import numpy as np
import pytest
import torch

from oracle import layer_oracle as L
from paper_2509_17863_amd import eaas

pytestmark = pytest.mark.gpu
CANARY = 12345.0
NAN_CODE = 0x7F


def blocks(n):
    return -(-n // 128)


def values(shape, seed, dtype=torch.bfloat16, spread=2.0):
    """Values of very different sizes, some zero, on the host."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * torch.exp(spread * torch.randn(shape, generator=g))
    x[torch.rand(shape, generator=g) < 0.05] = 0.0
    return x.to(dtype)


# ------------------------------------------------------------------ quantizers
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("rows,K,pad", [(1, 1, 0), (1, 128, 0), (5, 127, 1), (3, 129, 2), (70, 200, 8),
                                        (9, 2048, 0), (300, 1000, 3), (2, 20011, 0), (40000, 16, 0)])
def test_rows(gpu, rows, K, pad, dtype):
    x = values((rows, K), rows + K, dtype)
    wide = torch.full((rows, K + pad), float("nan"), dtype=dtype)
    wide[:, :K] = x
    flat = torch.full((rows * K + 16,), 77, dtype=torch.uint8, device="cuda")
    q, s = flat[: rows * K].view(rows, K), torch.empty((rows, blocks(K)), device="cuda")
    eaas.eaas_quantize_blocks_fp8(wide.cuda()[:, :K], q, s)
    wq, ws = L.quantize_blocks(x.float().numpy())
    assert np.array_equal(s.cpu().numpy(), ws)
    assert np.array_equal(q.cpu().numpy(), wq)
    assert (flat[rows * K:] == 77).all()


def test_rows_beside_the_step_s_own_quantizer(gpu):
    """That one divides by 448: scales a unit in the last place apart at most, codes one."""
    x = values((333, 1024), 3).cuda()
    q, s = torch.empty((333, 1024), dtype=torch.uint8, device="cuda"), torch.empty((333, 8), device="cuda")
    q2, s2 = torch.empty_like(q).view(torch.float8_e4m3fn), torch.empty_like(s)
    eaas.eaas_quantize_rows_fp8(x, q, s)
    eaas.eaas_quantize_blocks_fp8(x, q2, s2)
    assert ((s - s2).abs() <= 2.0 ** -23 * s).all()
    same = (s == s2).repeat_interleave(128, 1)
    q2 = q2.view(torch.uint8)
    assert torch.equal(q[same], q2[same]) and ((q.int() - q2.int()).abs() <= 1).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("E,N,K", [(1, 1, 1), (2, 128, 128), (3, 129, 127), (2, 300, 513), (5, 7, 40)])
def test_weights(gpu, E, N, K, dtype):
    w = values((E, N, K), N + K, dtype)
    q = torch.empty((E, N, K), dtype=torch.uint8, device="cuda")
    s = torch.empty((E, blocks(N), blocks(K)), device="cuda")
    eaas.eaas_quantize_blocks_fp8(w.cuda(), q, s)
    for e in range(E):
        wq, ws = L.quantize_blocks(w[e].float().numpy(), 128)
        assert np.array_equal(s[e].cpu().numpy(), ws)
        assert np.array_equal(q[e].cpu().numpy(), wq)


@pytest.mark.parametrize("per_block", [False, True], ids=["rows", "blocks"])
def test_scales_of_extremes(gpu, per_block):
    """Zeros, the ends of fp32's range, infinities and NaN; other blocks stay as they were."""
    x = torch.zeros((6, 4 * 128))
    x[0, 0], x[1, 130], x[2, 3] = 1e-45, 3e38, 6e-44   # (below 448 times the least: scale 1)
    x[2, 200], x[3, 300], x[4, 400] = 1e-40, float("inf"), float("nan")
    x[5, 0], x[5, 511] = -0.0, -float("inf")
    q = torch.empty((6, 512), dtype=torch.uint8, device="cuda")
    if per_block:
        s = torch.empty((1, 1, 4), device="cuda")
        eaas.eaas_quantize_blocks_fp8(x[None].cuda(), q[None], s)
    else:
        s = torch.empty((6, 4), device="cuda")
        eaas.eaas_quantize_blocks_fp8(x.cuda(), q, s)
    wq, ws = L.quantize_blocks(x.numpy(), 128 if per_block else 1)
    assert np.array_equal(s.reshape(ws.shape).cpu().numpy(), ws, equal_nan=True)
    assert np.array_equal(q.cpu().numpy(), wq)


def silu_up(gu):
    """The definition: 64 bits, rounded once to fp32."""
    I = gu.shape[1] // 2
    g, u = gu[:, :I].double(), gu[:, I:].double()
    return (g / (1 + torch.exp(-g)) * u).float().numpy()


@pytest.mark.parametrize("rows,I", [(1, 1), (1, 7), (3, 128), (5, 129), (64, 512), (17, 768), (2, 9001),
                                    (2000, 200)])
def test_swiglu_rows(gpu, rows, I):
    gu = values((rows, 2 * I), rows + I, spread=1.0) * 2
    q = torch.empty((rows, I), dtype=torch.uint8, device="cuda")
    s = torch.empty((rows, blocks(I)), device="cuda")
    eaas.eaas_swiglu_fp8(gu.cuda(), q, s)
    wq, ws = L.quantize_blocks(silu_up(gu))
    assert np.array_equal(s.cpu().numpy(), ws)
    assert np.array_equal(q.cpu().numpy(), wq)


def test_swiglu_rows_on_millions_of_values(gpu):
    """Values next to the middle between two codes come up about once in 10^6."""
    gu = torch.randn((8192, 1536), generator=torch.Generator().manual_seed(5)).to(torch.bfloat16)
    q = torch.empty((8192, 768), dtype=torch.float8_e4m3fn, device="cuda")
    s = torch.empty((8192, 6), device="cuda")
    eaas.eaas_swiglu_fp8(gu.cuda(), q, s)
    h = torch.from_numpy(silu_up(gu)).view(8192, 6, 128)
    ws = h.abs().amax(2) * torch.tensor(1 / 448, dtype=torch.float32)
    assert torch.equal(s.cpu(), ws)
    want = (h / ws[:, :, None]).to(torch.float8_e4m3fn).view(8192, 768)
    assert torch.equal(q.cpu().view(torch.uint8), want.view(torch.uint8))


def test_swiglu_rows_of_extremes(gpu):
    """Gates far below zero, products near either end of fp32's range, no numbers, and rows
    past the count, which stay as they were."""
    gates = torch.tensor([0.0, -0.0, -1e4, -86.0, -87.5, -88.8, -100.0, -103.0, 3e38, 50.0])
    ups = torch.tensor([1.0, -3.0, 1e30, 1e-30, 3e38, 1e-38, 1e10])
    gu = torch.zeros((80, 2 * 128), dtype=torch.bfloat16)
    n = 0
    for g in gates:
        for u in ups:
            gu[n, 3], gu[n, 128 + 3] = g, u
            gu[n, 9], gu[n, 128 + 9] = g / 2, u / 4
            n += 1
    gu[n, 0], gu[n, 128] = float("inf"), 1.0
    gu[n + 1, 5], gu[n + 2, 128 + 7] = float("nan"), float("nan")
    gu[n + 3, 5], gu[n + 3, 128 + 5] = -float("inf"), 1.0
    live = n + 5
    q = torch.full((80, 128), 99, dtype=torch.uint8, device="cuda")
    s = torch.full((80, 1), CANARY, device="cuda")
    eaas.eaas_swiglu_fp8(gu.cuda(), q, s, n_rows=torch.tensor([live], dtype=torch.int32, device="cuda"))
    wq, ws = L.quantize_blocks(silu_up(gu[:live]))
    assert np.array_equal(s[:live].cpu().numpy(), ws, equal_nan=True)
    assert np.array_equal(q[:live].cpu().numpy(), wq)
    assert (q[live:] == 99).all() and (s[live:] == CANARY).all()
    for count in (-5, 0):
        q.fill_(99)
        eaas.eaas_swiglu_fp8(gu.cuda(), q, s, n_rows=torch.tensor([count], dtype=torch.int32, device="cuda"))
        assert (q == 99).all()


# ------------------------------------------------------------------ the product
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


class Case:
    """Codes and scales on the host and the device.  `whole`: small whole numbers and
    scales that are powers of two, whose sums are exact in any order."""

    def __init__(self, R, E, N, K, kind="ragged", k=0, whole=False, lead=0, seed=0):
        rng = np.random.default_rng([R, E, N, K, seed])
        self.R, self.E, self.N, self.K, self.k = R, E, N, K, k
        self.offsets = np.concatenate([[0], np.cumsum(sizes_of(kind, E, R, rng))]).astype(np.int32)
        self.live = int(self.offsets[-1])
        self.perm = rng.permutation(R).astype(np.int32) if k else None
        self.src = L.source_rows(R, self.perm, max(k, 1))
        xr = R // k if k else R
        if whole:
            self.xq = L.e4m3_codes(rng.integers(-4, 5, (xr, K)).astype(float))
            self.wq = L.e4m3_codes(rng.integers(-4, 5, (E, N, K)).astype(float))
            self.xs = (2.0 ** rng.integers(-1, 2, (xr, blocks(K)))).astype(np.float32)
            self.ws = (2.0 ** rng.integers(-1, 2, (E, blocks(N), blocks(K)))).astype(np.float32)
        else:
            # every code that stands for a number
            self.xq, self.wq = (np.where((c & 127) == 127, 0x31, c) for c in (
                rng.integers(0, 256, (xr, K)).astype(np.uint8),
                rng.integers(0, 256, (E, N, K)).astype(np.uint8)))
            self.xs = np.exp(rng.normal(size=(xr, blocks(K)))).astype(np.float32)
            self.ws = np.exp(rng.normal(size=(E, blocks(N), blocks(K)))).astype(np.float32)
        used = np.zeros(xr, bool)
        used[self.src[: self.live]] = True
        xq, xs = self.xq.copy(), self.xs.copy()
        xq[~used], xs[~used] = NAN_CODE, np.nan      # no result may depend on these
        flat = torch.full((lead + xr * K + 64,), NAN_CODE, dtype=torch.uint8)
        flat[lead: lead + xr * K] = torch.from_numpy(xq.reshape(-1))
        self.d = (flat.cuda()[lead: lead + xr * K].view(xr, K), torch.from_numpy(xs).cuda(),
                  torch.from_numpy(self.offsets).cuda(), torch.from_numpy(self.wq).cuda(),
                  torch.from_numpy(self.ws).cuda())
        self.take = dict(perm=torch.from_numpy(self.perm).cuda(), k=k) if k else {}
        # partial sums that nothing wrote are NaN
        self.scratch = eaas.alloc_grouped_fp8_workspace(R, E, N, K)
        self.scratch.fill_(0xFF)

    def plan(self, dtype, in16=None):
        return eaas._grouped_plan("fp8" if dtype == torch.bfloat16 else "fp8_fp32", self.R, self.E,
                                  self.N, self.K, self.K % 16 == 0 if in16 is None else in16)

    def run(self, dtype, pad=0, **kw):
        wide = torch.full((self.R, self.N + pad), CANARY, dtype=dtype, device="cuda")
        y = wide[:, : self.N]
        eaas.eaas_grouped_matmul_fp8(*self.d, y, self.scratch, **self.take, **kw)
        c = torch.tensor(CANARY, dtype=dtype).item()
        assert (wide[self.live:] == c).all() and (wide[:, self.N:] == c).all()
        return y[: self.live]

    def want(self):
        return L.grouped_matmul_fp8(self.xq, self.xs, self.offsets, self.wq, self.ws, self.src)

    def check(self, y, in16=None):
        want, mag = self.want()
        kernel, _, parts = self.plan(y.dtype, in16)
        rel = (128 + blocks(self.K) + parts * 4 + 2) * 2.0 ** -23
        if kernel == "large" and y.dtype == torch.bfloat16:
            rel += 7 * 2.0 ** -14
        tol = rel * mag
        if y.dtype == torch.bfloat16:
            tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
        err = np.abs(y.double().cpu().numpy() - want)
        assert (err <= tol).all(), (err.max(), np.argwhere(~(err <= tol))[:4])


SHAPES = [
    # (R, E, N, K, kind, k, pad of y): edges of tiles and blocks on either side, odd sizes
    (1, 1, 1, 1, "even", 0, 0),
    (1, 5, 128, 256, "one", 0, 0),
    (8, 128, 192, 128, "ragged", 8, 0),
    (64, 8, 256, 272, "even", 2, 0),
    (130, 3, 129, 65, "ragged", 0, 3),
    (257, 4, 127, 191, "some", 0, 0),
    (256, 2, 130, 144, "even", 0, 8),
    (300, 7, 136, 200, "some", 3, 1),
    (33, 6, 7, 5, "ragged", 0, 1),
    (96, 512, 40, 80, "ragged", 4, 0),
    (48, 2, 64, 4096, "even", 0, 0),
    (9, 2, 33, 30001, "even", 3, 1),
    (5, 1, 40, 70000, "one", 0, 0),
    (700, 2, 520, 1040, "even", 0, 0),
    (1111, 5, 384, 640, "ragged", 0, 0),
    (1040, 2, 6200, 528, "even", 4, 8),
    (1500, 3, 6201, 784, "some", 0, 0),
    (0, 3, 32, 32, "even", 0, 0),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_product(gpu, shape, dtype):
    c = Case(*shape[:-1])
    c.check(c.run(dtype, pad=shape[-1]))


# (R, E, N, K, kind, k, pad, lead): rows of codes that start on any byte
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("shape", [(64, 8, 256, 272, "even", 2, 3, 1), (1200, 2, 6200, 528, "even", 0, 0, 8),
                                   (40, 2, 64, 1024, "some", 0, 5, 3)], ids=str)
def test_codes_from_any_byte(gpu, shape, dtype):
    c = Case(*shape[:-2], lead=shape[-1])
    c.check(c.run(dtype, pad=shape[-2]), in16=False)


EXACT = [(5, 1, 40, 70000, "one", 0), (20, 2, 96, 4096, "some", 4), (64, 1, 64, 8192, "even", 0),
         (200, 2, 264, 9008, "one", 4), (9, 2, 33, 30001, "even", 3), (512, 16, 1024, 2048, "ragged", 2),
         (3000, 5, 6200, 528, "ragged", 0), (3000, 4, 6201, 1040, "some", 4),
         (2600, 5, 6144, 1300, "ragged", 0), (13, 1, 32, 448, "even", 0), (19, 1, 224, 6080, "even", 0),
         (32, 1, 12256, 2192, "one", 4), (300, 7, 136, 64, "some", 3), (839, 1, 2048, 2592, "one", 0),
         # large tiles whose sums are three and four blocks
         (26638, 23, 416, 352, "even", 2), (1030, 63, 672, 512, "even", 0)]


def test_every_kernel_is_among_these():
    """On the host: every way of computing the product, in one part and in several."""
    seen = set()
    for R, E, N, K, *_ in EXACT:
        for product in ("fp8", "fp8_fp32"):
            kernel, rows, parts = eaas._grouped_plan(product, R, E, N, K, K % 16 == 0)
            seen.add((product, K % 16 == 0, kernel, rows if kernel == "few" else 0, parts > 1))
    for want in [("fp8", True, "large", 0, False), ("fp8", True, "any", 0, False),
                 ("fp8", True, "any", 0, True), ("fp8", False, "any", 0, False),
                 ("fp8", False, "any", 0, True), ("fp8", True, "few", 16, False),
                 ("fp8", True, "few", 16, True), ("fp8", True, "few", 32, False),
                 ("fp8", True, "few", 32, True), ("fp8", True, "few", 64, False)]:
        assert want in seen, (want, seen)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("shape", EXACT, ids=str)
def test_sums_that_are_exact_in_any_order(gpu, shape, dtype):
    """Parts, blocks or tiles that are lost, doubled or misplaced show."""
    c = Case(*shape, whole=True)
    want = torch.from_numpy(c.want()[0]).float().to(dtype)
    assert torch.equal(c.run(dtype).cpu(), want)


# (few rows, any alignment, 128 x 128 tiles in fp32 and large tiles in bf16)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("R,N,K", [(200, 300, 160), (24, 300, 320), (200, 301, 163), (3000, 6188, 528)])
def test_no_numbers_stay_in_their_rows(gpu, R, N, K, dtype):
    c = Case(R, 3, N, K, "even", whole=True)
    xq, xs = c.d[0], c.d[1]
    xq[5, 7], xs[R // 2, 1], xs[R - 3, 0] = NAN_CODE, float("nan"), float("inf")
    y = c.run(dtype)
    bad = (~torch.isfinite(y)).any(1).nonzero().reshape(-1).tolist()
    assert bad == [5, R // 2, R - 3] and torch.isnan(y[[5, R // 2]]).all()
    c = Case(R, 3, N, K, "even", whole=True)
    c.d[4][1, 2, 0] = float("nan")  # columns 256.. 383 of expert 1
    y = torch.isnan(c.run(dtype))
    a, b, end = int(c.offsets[1]), int(c.offsets[2]), min(N, 384)
    assert y[a:b, 256:end].all() and int(y.sum()) == (b - a) * (end - 256)


@pytest.mark.parametrize("shape", [(900, 4, 200, 2048, "ragged", 0), (1500, 3, 6208, 784, "even", 0),
                                   (16, 8, 256, 1024, "even", 2)], ids=str)
def test_equal_calls_other_streams_and_graphs(gpu, shape):
    c = Case(*shape)
    want = c.run(torch.bfloat16).clone()
    assert torch.equal(c.run(torch.bfloat16), want)
    side = torch.cuda.Stream()
    y = torch.empty((c.R, c.N), dtype=torch.bfloat16, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    eaas.eaas_grouped_matmul_fp8(*c.d, y, c.scratch, stream=side, **c.take)
    side.synchronize()
    assert torch.equal(y[: c.live], want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        eaas.eaas_grouped_matmul_fp8(*c.d, y, c.scratch, **c.take)
    for _ in range(3):
        y.zero_()
        c.scratch.fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y[: c.live], want)
        y.float().sum().item()


@pytest.mark.parametrize("R,E,N,K", [(1024, 8, 6200, 528), (64, 8, 64, 2048), (300, 6, 33, 47)])
def test_offsets_that_do_not_ascend_stay_in_bounds(gpu, R, E, N, K):
    """Results are then undefined, but nothing outside the result is written."""
    c = Case(R, E, N, K, "even")
    wild = torch.tensor([0, R] * (E // 2) + [0], dtype=torch.int32, device="cuda")
    guard = torch.zeros(c.scratch.numel() + 4096, dtype=torch.uint8, device="cuda")
    for dtype in (torch.bfloat16, torch.float32):
        y = torch.full((R + 8, N), CANARY, dtype=dtype, device="cuda")
        eaas.eaas_grouped_matmul_fp8(c.d[0], c.d[1], wild, *c.d[3:], y[:R], guard[: c.scratch.numel()])
        assert (y[R:] == torch.tensor(CANARY, dtype=dtype).item()).all()
    assert (guard[c.scratch.numel():] == 0).all()
    # and offsets past the rows are clamped to them
    off = c.offsets.copy()
    off[0], off[-1] = -5, 1 << 30
    y = torch.empty((R, N), device="cuda")
    eaas.eaas_grouped_matmul_fp8(c.d[0], c.d[1], torch.from_numpy(off).cuda(), *c.d[3:], y, c.scratch)
    assert torch.equal(y, c.run(torch.float32))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("shape", [(1500, 3, 6208, 784, "some", 0), (64, 8, 256, 272, "even", 2),
                                   (300, 3, 136, 2000, "even", 0)], ids=str)
def test_results_from_any_element(gpu, shape, dtype):
    c = Case(*shape, whole=True)
    want = torch.from_numpy(c.want()[0]).float().to(dtype)
    for lead, pad in ((1, 0), (3, 5), (2, 1)):
        flat = torch.full((lead + c.R * (c.N + pad) + 8,), CANARY, dtype=dtype, device="cuda")
        y = flat[lead: lead + c.R * (c.N + pad)].view(c.R, c.N + pad)[:, : c.N]
        eaas.eaas_grouped_matmul_fp8(*c.d, y, c.scratch, **c.take)
        assert torch.equal(y[: c.live].cpu(), want)
        y[: c.live] = CANARY
        assert (flat == torch.tensor(CANARY, dtype=dtype)).all()


def test_two_calls_at_once(gpu):
    """On two streams, each with its workspace: large tiles beside a sum in parts."""
    a, b = Case(1500, 3, 6208, 784, "even", whole=True), Case(20, 2, 96, 4096, "some", 4, whole=True)
    want = [torch.from_numpy(c.want()[0]).float().to(torch.bfloat16) for c in (a, b)]
    ys = [torch.empty((c.R, c.N), dtype=torch.bfloat16, device="cuda") for c in (a, b)]
    streams = [torch.cuda.Stream() for _ in ys]
    torch.cuda.synchronize()
    for _ in range(8):
        for c, y, s in zip((a, b), ys, streams):
            eaas.eaas_grouped_matmul_fp8(*c.d, y, c.scratch, stream=s, **c.take)
    torch.cuda.synchronize()
    assert all(torch.equal(y[: c.live].cpu(), w) for c, y, w in zip((a, b), ys, want))


def test_gradient_in_the_rows_by_transposed_weights(gpu):
    """From quantized weights and their transposed codes and scales, through the calls."""
    R, E, N, K = 90, 3, 300, 200
    g = torch.Generator().manual_seed(1)
    w = torch.randn((E, N, K), generator=g).cuda()
    dy = torch.randn((R, N), generator=g).to(torch.bfloat16)
    wq = torch.empty((E, N, K), dtype=torch.uint8, device="cuda")
    ws = torch.empty((E, 3, 2), device="cuda")
    eaas.eaas_quantize_blocks_fp8(w, wq, ws)
    q, s = torch.empty((R, N), dtype=torch.uint8, device="cuda"), torch.empty((R, 3), device="cuda")
    eaas.eaas_quantize_blocks_fp8(dy.cuda(), q, s)
    off = torch.tensor([0, 30, 31, 90], dtype=torch.int32, device="cuda")
    dx = torch.empty((R, K), device="cuda")
    eaas.eaas_grouped_matmul_fp8(q, s, off, wq.transpose(1, 2).contiguous(),
                                 ws.transpose(1, 2).contiguous(), dx,
                                 eaas.alloc_grouped_fp8_workspace(R, E, K, N))
    full = np.stack([L.dequantized(wq[e].cpu().numpy(), ws[e].cpu().numpy(), 128) for e in range(E)])
    want, mag = L.grouped_matmul_dx(L.dequantized(q.cpu().numpy(), s.cpu().numpy()), off.cpu().numpy(), full)
    assert (np.abs(dx.double().cpu().numpy() - want) <= (128 + 3 + 6) * 2.0 ** -23 * mag).all()


def test_result_past_32_bit_offsets(gpu):
    """More than 2^32 bytes of results."""
    R, N, K = 70000, 32768, 32
    c = torch.randint(0, 100, (R, K), dtype=torch.uint8, device="cuda")
    w = torch.randint(0, 100, (1, N, K), dtype=torch.uint8, device="cuda")
    off = torch.tensor([0, R], dtype=torch.int32, device="cuda")
    xs, ws = torch.rand((R, 1), device="cuda") + 0.5, torch.rand((1, N // 128, 1), device="cuda") + 0.5
    y = torch.empty((R, N), dtype=torch.bfloat16, device="cuda")
    eaas.eaas_grouped_matmul_fp8(c, xs, off, w, ws, y, eaas.alloc_grouped_fp8_workspace(R, 1, N, K))
    wv = w[0].view(torch.float8_e4m3fn).double() * ws[0].double().repeat_interleave(128, 0)
    for r in (0, 65535, 65536, 69999):
        want = wv @ (c[r].view(torch.float8_e4m3fn).double() * xs[r].double())
        assert ((y[r].double() - want).abs() <= (7 * 2.0 ** -14 + 160 * 2.0 ** -23 + 2.0 ** -8) * want).all()
