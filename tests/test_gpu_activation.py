"""Activation, its gradient, 8-bit rows and the combine's gradient against the
64-bit oracle.

Tolerances.  1/(1 + exp(-g)) in fp32: the exponential's argument is rounded, which
moves it by |g| * 2^-23 of itself at most, and exponential, sum and reciprocal each
err by a unit in the last place or so: (|g| + 8) * 2^-23 of the result.  A bf16
result adds 2^-8 of itself.  In the gradient 1 + g (1 - t) may cancel: its error is
(|g| + 8) (1 + |g|) * 2^-23, in units of dh * up * t.
"""
import numpy as np
import pytest
import torch

from oracle import layer_oracle as L
from paper_2509_17863_amd import eaas

pytestmark = pytest.mark.gpu

ROWS = [(1, 1), (1, 7), (3, 8), (5, 129), (64, 512), (17, 768), (9, 2048), (4, 2056), (3, 8192),
        (2, 9001), (2, 20000), (600, 96)]


def host(shape, seed, scale=2.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(torch.bfloat16)


def within(got, want, tol):
    got = got.double().cpu().numpy()
    assert (np.abs(got - want) <= tol + 1e-37).all(), np.abs(got - want).max()


@pytest.mark.parametrize("rows,I", ROWS)
def test_swiglu(gpu, rows, I):
    gu = host((rows, 2 * I), 1, 4.0)
    h = torch.empty((rows, I), dtype=torch.bfloat16, device="cuda")
    eaas.eaas_swiglu(gu.cuda(), h)
    a = gu.double().numpy()
    want = L.swiglu(a)
    within(h, want, np.abs(want) * ((np.abs(a[:, :I]) + 8) * 2.0 ** -23 + 2.0 ** -8) * 1.01)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("rows,I", ROWS)
def test_swiglu_backward(gpu, rows, I, in_place):
    gu, dh = host((rows, 2 * I), 2, 4.0), host((rows, I), 3)
    d = gu.cuda()
    dgu = d if in_place else torch.empty_like(d)
    eaas.eaas_swiglu_backward(d, dh.cuda(), dgu)
    a, b = gu.double().numpy(), dh.double().numpy()
    want = L.swiglu_backward(a, b)
    g, u = np.abs(a[:, :I]), np.abs(a[:, I:])
    rel = (g + 8) * 2.0 ** -23
    t = L.sigmoid(a[:, :I])
    tol = np.concatenate([np.abs(b) * u * t * rel * (1 + g) * 2, np.abs(b) * g * t * rel], axis=1)
    within(dgu, want, tol + 2.0 ** -8 * (np.abs(want) + tol))


def test_swiglu_extremes(gpu):
    """Gates of any size: no infinity where the value is finite."""
    g = torch.tensor([[-3e38, -1000.0, -88.8, -87.0, 0.0, 87.0, 1000.0, 3e38]])
    gu = torch.cat([g, torch.full_like(g, 0.5)], dim=1).to(torch.bfloat16)
    h = torch.empty((1, 8), dtype=torch.bfloat16, device="cuda")
    eaas.eaas_swiglu(gu.cuda(), h)
    want = L.swiglu(gu.double().numpy())
    got = h.double().cpu().numpy()
    assert np.isfinite(got).all()
    # below the normal range the result may be flushed
    assert (np.abs(got - want) <= 2.0 ** -7 * np.abs(want) + 1.2e-38).all()
    dgu = torch.empty((1, 16), dtype=torch.bfloat16, device="cuda")
    eaas.eaas_swiglu_backward(gu.cuda(), torch.ones((1, 8), dtype=torch.bfloat16).cuda(), dgu)
    assert torch.isfinite(dgu).all()
    want = L.swiglu_backward(gu.double().numpy(), np.ones((1, 8)))
    assert (np.abs(dgu.double().cpu().numpy() - want) <= 2.0 ** -7 * np.abs(want) + 1e-36).all()


@pytest.mark.parametrize("pad", [0, 3, 8])
@pytest.mark.parametrize("rows,K", ROWS)
def test_quantize_rows(gpu, rows, K, pad):
    x = host((rows, K), 4)
    if rows > 2:
        x[1] = 0
        x[2] = (torch.arange(K) % 255 - 127).to(torch.bfloat16)
        x[2, 0] = 127  # a scale of exactly 1
    wide = torch.full((rows, K + pad), float("nan"), dtype=torch.bfloat16)
    wide[:, :K] = x
    q = torch.full((rows, K), 99, dtype=torch.int8, device="cuda")
    s = torch.empty(rows, device="cuda")
    eaas.eaas_quantize_rows_int8(wide.cuda()[:, :K], q, s)
    qr, sr = L.quantize_rows_int8(x.float().numpy())
    assert np.array_equal(s.cpu().numpy(), sr)
    assert np.array_equal(q.cpu().numpy(), qr)


@pytest.mark.parametrize("K", [96, 2048, 9001])
def test_quantize_rows_that_are_not_finite_or_tiny(gpu, K):
    x = host((5, K), 5)
    x[1, K // 2] = float("inf")
    x[2, 0] = float("nan")
    x[3, K - 1] = -float("inf")
    x[4] = 1e-39                      # below the normal range
    x[4, 1] = -9.2e-41
    q = torch.full((5, K), 99, dtype=torch.int8, device="cuda")
    s = torch.empty(5, device="cuda")
    eaas.eaas_quantize_rows_int8(x.cuda(), q, s)
    qr, sr = L.quantize_rows_int8(x.float().numpy())
    assert np.array_equal(s.cpu().numpy(), sr, equal_nan=True)
    assert np.array_equal(q.cpu().numpy(), qr)


@pytest.mark.parametrize("rows,I", ROWS)
def test_swiglu_int8(gpu, rows, I):
    """The scale within the error of h, and every code within one (half a code of
    rounding, and half a code more at the most from that error) of h over it."""
    gu = host((rows, 2 * I), 6)
    q = torch.empty((rows, I), dtype=torch.int8, device="cuda")
    s = torch.empty(rows, device="cuda")
    eaas.eaas_swiglu_int8(gu.cuda(), q, s)
    a = gu.double().numpy()
    h = L.swiglu(a)
    rel = (np.abs(a[:, :I]).max() + 8) * 2.0 ** -23
    amax = np.abs(h).max(axis=1)
    sc = s.double().cpu().numpy()
    assert (np.abs(sc - amax / 127) <= amax / 127 * (rel + 2.0 ** -23)).all()
    ratio = h / sc[:, None]
    err = np.abs(q.double().cpu().numpy() - ratio)
    assert (err <= 0.5 + 127 * (rel + 2.0 ** -22)).all(), err.max()
    # almost all are the code of the 64-bit value itself
    assert (q.cpu().numpy() != np.rint(ratio)).sum() <= 1 + q.numel() // 500


@pytest.mark.parametrize("bound", [-4, 0, 3, 64, 1000])
def test_rows_bounded_on_the_device(gpu, bound):
    rows, I = 64, 40
    gu, dh = host((rows, 2 * I), 7).cuda(), host((rows, I), 8).cuda()
    n = torch.tensor([bound], dtype=torch.int32, device="cuda")
    live = min(rows, max(bound, 0))
    h = torch.full((rows, I), 7.0, dtype=torch.bfloat16, device="cuda")
    dgu = torch.full((rows, 2 * I), 7.0, dtype=torch.bfloat16, device="cuda")
    q = torch.full((rows, I), 7, dtype=torch.int8, device="cuda")
    s = torch.full((rows,), 7.0, device="cuda")
    eaas.eaas_swiglu(gu, h, n_rows=n)
    eaas.eaas_swiglu_backward(gu, dh, dgu, n_rows=n)
    eaas.eaas_swiglu_int8(gu, q, s, n_rows=n)
    h1, dgu1 = torch.empty_like(h), torch.empty_like(dgu)
    q1, s1 = torch.empty_like(q), torch.empty_like(s)
    eaas.eaas_swiglu(gu, h1)
    eaas.eaas_swiglu_backward(gu, dh, dgu1)
    eaas.eaas_swiglu_int8(gu, q1, s1)
    for part, whole in ((h, h1), (dgu, dgu1), (q, q1), (s, s1)):
        assert torch.equal(part[:live], whole[:live])
        assert (part[live:] == 7).all()


@pytest.mark.parametrize("dout", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("T,k,E,H", [(1, 1, 1, 128), (5, 3, 4, 256), (64, 8, 32, 1152),
                                     (700, 7, 9, 384), (33, 2, 64, 7168)])
def test_combine_backward(gpu, T, k, E, H, dout):
    """dy is one product, rounded: equal bit for bit.  dweights: a sum of H."""
    R = T * k
    g = torch.Generator().manual_seed(T + H)
    ids = torch.randint(-2, E + 2, (T, k), generator=g, dtype=torch.int32)
    r = eaas.alloc_routing(T, k, E)
    ws = eaas.alloc_workspace(T, H, 128, E, k)
    eaas.eaas_route_permute(ids.cuda(), E, r, ws, H=H)
    d = torch.randn((T, H), generator=g).to(dout)
    y = torch.randn((R, H), generator=g)
    w = torch.rand((T, k), generator=g)
    inv = r["inv"].cpu().numpy()[:R]
    live = int(r["offsets"][E])
    yd = y.clone()
    yd[live:] = float("nan")
    dy = torch.full((R, H), 7.0, dtype=torch.bfloat16, device="cuda")
    dw = torch.full((T, k), float("nan"), device="cuda")
    eaas.eaas_unpermute_combine_backward(d.cuda(), yd.cuda(), r, w.cuda(), dy, dw, E)
    perm = r["perm"].cpu().long()[:live]
    want = (w.reshape(-1)[perm][:, None] * d.float()[perm // k]).to(torch.bfloat16)
    assert torch.equal(dy[:live].cpu(), want)
    assert (dy[live:] == 7).all()
    dy64, dw64, mag = L.combine_backward(d.double().numpy(), y.double().numpy(), inv,
                                         w.double().numpy())
    within(dw, dw64, H * 2.0 ** -23 * mag)
    assert (dw.cpu().numpy().reshape(-1)[inv < 0] == 0).all()
    named = dy64[:live]
    within(dy[:live], named, 2.0 ** -7 * np.abs(named))
