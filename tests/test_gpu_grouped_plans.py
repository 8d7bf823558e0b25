"""The ways in which the grouped products are computed, each named and checked by the
library's own choice: sums in many parts, and large tiles of which a workgroup takes
several.  Operands are small whole numbers and scales powers of two, so every order
of summation is exact: results are equal bit for bit (in bf16 to the one rounding),
and a part or a tile that is lost, doubled or misplaced shows."""
import pytest
import torch

from paper_2509_17863_amd import eaas

CANARY = 99.0
CUS = 256  # workgroups of the large tiles' launch, at most


def offsets_of(sizes):
    return torch.cat([torch.zeros(1, dtype=torch.long), torch.tensor(sizes).cumsum(0)])


def sizes_even(R, E):
    return [R // E + (e < R % E) for e in range(E)]


class Product:
    """One product's operands on the host, its result by groups, and its call."""

    def __init__(self, product, R, sizes, N, K, k=0, pad=0):
        self.product, self.R, self.N, self.K, self.k, self.pad = product, R, N, K, k, pad
        self.E, self.off = len(sizes), offsets_of(sizes)
        g = torch.Generator().manual_seed(R + N + K)
        top = 127 if product == "int8" else 4
        dt = torch.int8 if product == "int8" else torch.bfloat16

        def whole(*shape):
            return torch.randint(-top, top + 1, shape, generator=g, dtype=torch.int16).to(dt)

        def powers(*shape):
            return 2.0 ** torch.randint(-2, 3, shape, generator=g)

        tokens = R // k if k else R
        self.perm = torch.randperm(R, generator=g) if k else None
        self.src = self.perm // k if k else torch.arange(R)
        if product in ("forward", "int8", "dw"):
            self.x = whole(tokens, K)
        if product in ("dx", "dw"):
            self.dy = whole(R, N)
        if product != "dw":
            self.w = whole(self.E, N, K)
        if product == "int8":
            self.xs, self.ws = powers(tokens), powers(self.E, N)

    def plan(self):
        m = 16 if self.product == "int8" else 8
        cols = [self.K] if self.product in ("forward", "int8") else [self.N, self.K]
        in16 = all(c % m == 0 for c in cols) and (self.pad % 8 == 0 or self.product == "int8")
        return eaas._grouped_plan(self.product, self.R, self.E, self.N, self.K, in16)

    def tiles(self, bi):
        """Tiles of the result that exist, `bi` high and wide."""
        up = lambda n: -(-int(n) // bi)  # noqa: E731
        if self.product == "dw":
            return self.E * up(self.N) * up(self.K)
        return sum(map(up, self.off.diff())) * up(self.K if self.product == "dx" else self.N)

    def want(self):
        """Whole numbers below 2^24 (8-bit: in 64 bits, rounded to fp32 once)."""
        if self.product == "dw":
            out = torch.zeros((self.E, self.N, self.K))
        else:
            out = torch.zeros((self.R, self.K if self.product == "dx" else self.N))
        for e in range(self.E):
            s = slice(self.off[e], self.off[e + 1])
            if self.product == "forward":
                out[s] = self.x[self.src[s]].float() @ self.w[e].float().t()
            elif self.product == "dx":
                out[s] = self.dy[s].float() @ self.w[e].float()
            elif self.product == "dw":
                out[e] = self.dy[s].float().t() @ self.x[self.src[s]].float()
            else:
                p = (self.x[self.src[s]].double() @ self.w[e].double().t()).float()
                out[s] = p * self.xs[self.src[s]][:, None] * self.ws[e][None, :]
        return out

    def rows(self, t, used=None):
        """On the device, `pad` elements between rows; NaN there and in unused rows."""
        d = torch.full((t.shape[0], t.shape[1] + self.pad), float("nan"), dtype=t.dtype)
        d[:, : t.shape[1]] = t
        if used is not None:
            d[~used] = float("nan")
        return d.cuda()[:, : t.shape[1]]

    def check(self, out, accumulate=False):
        live = int(self.off[-1])
        in_group = torch.arange(self.R) < live
        off, ws = self.off.to(torch.int32).cuda(), eaas.alloc_grouped_workspace(
            self.R, self.E, self.N, self.K)
        ws.fill_(0xFF)  # (NaN in every partial sum)
        take = dict(perm=self.perm.to(torch.int32).cuda(), k=self.k) if self.k else {}
        used = torch.zeros(self.R // self.k if self.k else self.R, dtype=torch.bool)
        used[self.src[:live]] = True
        want = self.want()
        if self.product == "dw":
            got = torch.full(want.shape, 3.0 if accumulate else float("nan"), dtype=out,
                             device="cuda")
            eaas.eaas_grouped_matmul_dw(self.rows(self.dy, in_group), self.rows(self.x, used), off,
                                        got, ws, accumulate=accumulate, **take)
            assert torch.equal(got.cpu(), (want + (3.0 if accumulate else 0.0)).to(out))
            return
        wide = torch.full((self.R, want.shape[1] + self.pad), CANARY, dtype=out, device="cuda")
        got = wide[:, : want.shape[1]]
        if self.product == "forward":
            eaas.eaas_grouped_matmul(self.rows(self.x, used), off, self.w.cuda(), got, ws, **take)
        elif self.product == "dx":
            eaas.eaas_grouped_matmul_dx(self.rows(self.dy, in_group), off, self.w.cuda(), got, ws)
        else:
            eaas.eaas_grouped_matmul_int8(self.x.cuda(), self.xs.cuda(), off, self.w.cuda(),
                                          self.ws.cuda(), got, ws, **take)
        assert torch.equal(got[:live].cpu(), want[:live].to(out))
        assert (wide[live:] == CANARY).all() and (wide[:, want.shape[1]:] == CANARY).all()


# (product, R, sizes, N, K, k, kernel): sums in parts, with and without whole quads
# of columns, gathered, with an empty group and rows of no group
PARTS = [
    ("forward", 5, [5], 40, 70000, 0, "few"),
    ("forward", 9, [4, 5], 33, 30001, 3, "any"),
    ("forward", 20, [12, 0, 8], 96, 4096, 4, "few"),
    ("forward", 64, [50], 64, 8192, 0, "few"),
    ("forward", 200, [0, 200], 264, 9000, 4, "few"),
    ("int8", 5, [5], 40, 70000, 0, "few"),
    ("int8", 9, [4, 5], 33, 30001, 3, "any"),
    ("int8", 64, [0, 50], 64, 8192, 2, "few"),
    ("int8", 200, [150, 0], 264, 9000, 4, "any"),
    ("dx", 5, [5], 70000, 40, 0, "few"),
    ("dx", 9, [4, 5], 30001, 33, 0, "any"),
    ("dx", 300, [299], 8192, 64, 0, "few"),
    ("dw", 30000, [30000], 24, 40, 2, "any"),
    ("dw", 66000, [66000], 23, 39, 0, "any"),
    ("dw", 9001, [0, 4000, 5000], 72, 136, 0, "any"),
]


def ident(case):
    return "-".join(map(str, case))


@pytest.mark.parametrize("case", PARTS, ids=ident)
def test_every_part_of_these_sums_shows(case):
    """On the host: each part (and each wave's share of it) changes some result."""
    product, R, sizes, N, K, k, kernel = case
    p = Product(product, R, sizes, N, K, k)
    got, _, parts = p.plan()
    assert got == kernel and parts > 1
    if product == "dw":
        for e, n in enumerate(sizes):
            s, steps = int(p.off[e]), -(-n // 64)
            for i in range(min(parts, steps)):
                a, b = (s + min(64 * (steps * (i + j) // parts), n) for j in (0, 1))
                assert a == b or (p.dy[a:b].float().t() @ p.x[p.src[a:b]].float()).any()
        return
    e = max(range(len(sizes)), key=lambda i: sizes[i])
    rows = slice(int(p.off[e]), int(p.off[e + 1]))
    a = (p.dy[rows] if product == "dx" else p.x[p.src[rows]]).float()
    b = (p.w[e] if product == "dx" else p.w[e].t()).float()
    step, parts = 128 if product == "int8" else 64, parts * (4 if kernel == "few" else 1)
    steps = -(-a.shape[1] // step)
    for i in range(parts):
        s = slice(step * (steps * i // parts), step * (steps * (i + 1) // parts))
        assert a[:, s].shape[1] == 0 or (a[:, s] @ b[s]).any()


@pytest.mark.gpu
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("case", PARTS, ids=ident)
def test_sums_in_parts(gpu, case, out):
    p = Product(*case[:-1])
    assert p.plan()[0] == case[-1] and p.plan()[2] > 1
    p.check(out)
    if case[0] == "dw" and out == torch.float32:
        p.check(out, accumulate=True)


# Large tiles, more than CUs and no multiple of them, so that workgroups go on to a
# second or third; groups that are empty, of one row, of whole tiles and not; sums that
# end inside a step; columns that end inside a tile, in whole 16 bytes or not
UNEVEN = [0, 1, 256, 257, 1100, 1386]           # 3000 rows
ELSEWHERE = [700, 0, 513, 1, 1030, 512]         # 244 rows of no group
OTHER = [0, 1, 64, 65, 200, 0, 700, 1300, 1670]  # 4000 rows; sums of 0 to 27 steps in dW
LARGE = [
    # (product, R, sizes, N, K, k, pad)
    ("forward", 3000, UNEVEN, 7000, 200, 0, 0),
    ("forward", 3000, UNEVEN, 7001, 264, 0, 0),
    ("forward", 3000, ELSEWHERE, 7000, 520, 4, 8),
    ("forward", 3000, UNEVEN, 6998, 1096, 3, 0),
    ("forward", 4000, OTHER, 6200, 264, 0, 8),
    ("int8", 3000, UNEVEN, 6200, 512, 0, 0),
    ("int8", 3000, ELSEWHERE, 6201, 528, 4, 0),
    ("int8", 4000, OTHER, 6200, 1040, 2, 3),
    ("dx", 3000, UNEVEN, 264, 7000, 0, 0),
    ("dx", 3000, ELSEWHERE, 520, 7000, 0, 8),
    ("dx", 4000, OTHER, 1096, 6200, 0, 0),
    ("dw", 4000, OTHER, 1288, 1544, 0, 0),
    ("dw", 4000, OTHER, 1288, 1544, 4, 8),
    ("dw", 3000, ELSEWHERE, 2056, 1800, 2, 0),
]


def several_each(p):
    kernel, bi, parts = p.plan()
    n = p.tiles(bi)
    return kernel == "large" and parts == 1 and n > CUS and n % CUS


@pytest.mark.parametrize("case", LARGE, ids=ident)
def test_these_shapes_take_large_tiles_several_to_a_workgroup(case):
    assert several_each(Product(*case))


@pytest.mark.gpu
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("case", LARGE, ids=ident)
def test_large_tiles_several_to_a_workgroup(gpu, case, out):
    p = Product(*case)
    assert several_each(p)
    p.check(out)
    if case[0] == "dw" and out == torch.float32:
        p.check(out, accumulate=True)


@pytest.mark.gpu
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("pad", [3, 4])
def test_large_tiles_into_rows_that_are_not_16_bytes_apart(gpu, pad, out):
    """The operands are in multiples of 16 bytes, the result's rows are not."""
    p = Product("dx", 3000, UNEVEN, 264, 7000)
    assert several_each(p)
    live, off = int(p.off[-1]), p.off.to(torch.int32).cuda()
    wide = torch.full((3000, 7000 + pad), CANARY, dtype=out, device="cuda")
    eaas.eaas_grouped_matmul_dx(p.dy.cuda(), off, p.w.cuda(), wide[:, :7000],
                                eaas.alloc_grouped_workspace(3000, p.E, 264, 7000))
    assert torch.equal(wide[:live, :7000].cpu(), p.want()[:live].to(out))
    assert (wide[:, 7000:] == CANARY).all()
