"""The gated product, its way back and the block-scaled e4m3 product on the host: what
they refuse, and with which status, before anything reaches a device; and the binding's
own checks."""
import ctypes

import pytest
import torch

from paper_2509_17863_amd import eaas

A, B, C, D, F, G = (i << 30 for i in range(1, 7))  # stand-ins for device pointers, far apart
BIG = 1 << 40


def shape(R=64, E=4, N=128, K=256):
    return eaas._GroupShape(R, E, N, K)


def ref(s):
    return ctypes.byref(s) if s is not None else None


def fp8(s=shape(), x=A, xs=F, perm=None, k=1, off=B, w=C, wsc=G, y=D, ldy=128, dt=0, ws=BIG,
        n=1 << 40):
    return eaas.lib().eaas_grouped_matmul_fp8(ref(s), x, xs, perm, k, off, w, wsc, y, ldy, dt, ws,
                                              n, None)


def gated(s=shape(), x=A, ldx=256, perm=None, k=1, off=B, w=C, h=D, ldh=64, gu=F, ldgu=128, ws=BIG,
          n=1 << 40):
    return eaas.lib().eaas_grouped_swiglu(ref(s), x, ldx, perm, k, off, w, h, ldh, gu, ldgu, ws, n,
                                          None)


def back(s=shape(), dy=A, lddy=128, off=B, w=C, gu=D, ldgu=512, dgu=F, lddgu=512, h=G, ldh=256,
         ws=BIG, n=1 << 40):
    return eaas.lib().eaas_grouped_swiglu_backward(ref(s), dy, lddy, off, w, gu, ldgu, dgu, lddgu, h,
                                                   ldh, ws, n, None)


@pytest.mark.parametrize("call", [fp8, gated, back])
def test_shapes(call):
    assert call(s=None) == -1
    for bad in (dict(R=-1), dict(E=0), dict(N=0), dict(K=-3)):
        assert call(s=shape(**bad)) == -1
    assert call(s=shape(E=1025)) == -2
    assert call(s=shape(N=1 << 16, K=1 << 16)) == -2
    assert call(off=None) == -1 and call(off=B + 2) == -1
    assert call(w=None) == -1 and call(w=C + 8) == -1


@pytest.mark.parametrize("call", [fp8, gated])
def test_gather(call):
    assert call(perm=B, k=0) == -1
    assert call(perm=B, k=3) == -1          # 64 rows are not 3 a token
    assert call(perm=B + 2, k=2) == -1
    assert call(s=shape(R=1 << 26), perm=B, k=1) == -2


def test_fp8():
    for bad in (dict(x=None), dict(xs=None), dict(wsc=None), dict(y=None), dict(xs=F + 2),
                dict(wsc=G + 1), dict(ldy=127), dict(dt=1), dict(dt=3), dict(y=D + 1),
                dict(y=D + 2, dt=2), dict(y=A + 8), dict(y=C), dict(y=F + 64), dict(y=G + 4),
                dict(xs=D + 1000), dict(wsc=D)):
        assert fp8(**bad) == -1, bad
    assert fp8(ldy=(1 << 22) + 1) == -2
    s = shape(R=0)
    assert fp8(s=s, x=None, xs=None, off=None, w=None, wsc=None, y=None, ws=None, n=0) == 0
    assert eaas.lib().eaas_grouped_fp8_workspace_bytes(None) == 0
    for kw, ok in ((dict(), True), (dict(R=0), True), (dict(N=1, K=1), True), (dict(E=1025), False),
                   (dict(N=46341, K=46341), False)):
        n = eaas.lib().eaas_grouped_fp8_workspace_bytes(ref(shape(**kw)))
        assert (n > 0) == ok and n % 256 == 0
    long = shape(R=32, E=1, N=64, K=8192)   # a sum that is split needs its parts' memory
    assert fp8(s=long, ws=None) == -3 and fp8(s=long, ws=BIG + 8) == -3 and fp8(s=long, n=256) == -3


def test_gated():
    assert gated(s=shape(N=127)) == -1      # no two halves
    for bad in (dict(x=None), dict(h=None), dict(ldx=255), dict(ldh=63), dict(ldgu=127),
                dict(x=A + 1), dict(h=D + 1), dict(gu=F + 1), dict(h=A), dict(h=C + 64),
                dict(gu=A + 2), dict(gu=C), dict(gu=D), dict(h=F + 64),
                dict(h=F + 128, ldh=128)):
        assert gated(**bad) == -1, bad
    for bad in ("ldx", "ldh", "ldgu"):
        assert gated(**{bad: (1 << 22) + 1}) == -2
    assert gated(s=shape(R=0), x=None, off=None, w=None, h=None, gu=None, ws=None, n=0) == 0
    assert gated(s=shape(R=0), gu=None, ldgu=0, x=None, h=None) == 0
    long = shape(R=32, E=1, N=64, K=8192)
    assert eaas.lib().eaas_grouped_workspace_bytes(ref(long)) > 256
    assert gated(s=long, ldx=8192, ws=None) == -3 and gated(s=long, ldx=8192, n=256) == -3


def test_backward():
    for bad in (dict(dy=None), dict(gu=None), dict(dgu=None), dict(lddy=127), dict(ldgu=511),
                dict(lddgu=511), dict(ldh=255), dict(dy=A + 1), dict(gu=D + 1), dict(dgu=F + 1),
                dict(h=G + 1), dict(dgu=A), dict(dgu=C), dict(h=A), dict(h=C), dict(h=F + 512),
                dict(h=D), dict(dgu=D, lddgu=520), dict(dgu=D + 2), dict(dgu=D + 512)):
        assert back(**bad) == -1, bad
    for bad in ("lddy", "ldgu", "lddgu", "ldh"):
        assert back(**{bad: (1 << 22) + 1}) == -2
    assert back(s=shape(R=0), dy=None, off=None, w=None, gu=None, dgu=None, h=None, ws=None) == 0
    long = shape(R=32, E=1, N=8192, K=64)
    assert back(s=long, lddy=8192, ws=None) == -3 and back(s=long, lddy=8192, n=256) == -3


def test_quantizers():
    L = eaas.lib()

    def q(x=A, dt=0, ld=200, mats=2, rows=130, K=200, per=128, q=B, s=C):
        return L.eaas_quantize_blocks_fp8(x, dt, ld, mats, rows, K, per, q, s, None)

    for bad in (dict(x=None), dict(q=None), dict(s=None), dict(mats=-1), dict(rows=-1), dict(K=0),
                dict(ld=199), dict(dt=1), dict(dt=5), dict(per=0), dict(per=64), dict(x=A + 1),
                dict(x=A + 2, dt=2), dict(s=C + 2), dict(q=A + 100), dict(s=A), dict(s=B + 4)):
        assert q(**bad) == -1, bad
    assert q(K=1 << 23, ld=1 << 23) == -2 and q(rows=1 << 31) == -2
    assert q(mats=1 << 16, rows=1 << 16) == -2 and q(ld=(1 << 22) + 1) == -2
    assert q(rows=0, x=None, q=None, s=None) == 0 and q(mats=0, x=None) == 0

    def f(gu=A, rows=8, I=64, n=None, q=B, s=C):
        return L.eaas_swiglu_fp8(gu, rows, I, n, q, s, None)

    for bad in (dict(gu=None), dict(q=None), dict(s=None), dict(rows=-1), dict(I=0),
                dict(gu=A + 1), dict(s=C + 2), dict(n=D + 2), dict(q=A), dict(s=A + 4), dict(s=B)):
        assert f(**bad) == -1, bad
    assert f(I=(1 << 21) + 1) == -2 and f(rows=0, gu=None, q=None, s=None) == 0


def test_binding_checks():
    """Shapes and types that the C ABI cannot see."""
    bf, f32, i32, u8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
    off, ws = torch.zeros(3, dtype=i32), torch.zeros(256, dtype=u8)
    xq, xs = torch.zeros((4, 130), dtype=u8), torch.zeros((4, 2))
    wq, sc, y = torch.zeros((2, 8, 130), dtype=u8), torch.zeros((2, 1, 2)), torch.zeros((4, 8))
    for a in ((xq[:, :128], xs, off, wq, sc, y), (xq.to(torch.int8), xs, off, wq, sc, y),
              (xq, xs[:, :1], off, wq, sc, y), (xq, xs, off[:2], wq, sc, y),
              (xq, xs, off, wq.to(torch.int8), sc, y), (xq, xs, off, wq, sc[:, :, :1], y),
              (xq, xs.double(), off, wq, sc, y), (xq, xs, off, wq, sc, y.half()),
              (xq[:2], xs[:2], off, wq, sc, y), (xq, xs, off, wq, sc, y[:, :4])):
        with pytest.raises(ValueError):
            eaas.eaas_grouped_matmul_fp8(*a, ws)
    x, w, h = torch.zeros((4, 16), dtype=bf), torch.zeros((2, 8, 16), dtype=bf), torch.zeros((4, 4), dtype=bf)
    for a, kw in (((x.float(), off, w, h), {}), ((x, off, w[:, :7], h), {}), ((x, off, w, h[:, :3]), {}),
                  ((x, off, w, h.float()), {}), ((x[:2], off, w, h), {}), ((x, off.long(), w, h), {}),
                  ((x, off, w, h), dict(gu=h)), ((x, off, w, h), dict(gu=torch.zeros((3, 8), dtype=bf))),
                  ((x, off, w, h), dict(perm=torch.zeros(4, dtype=i32), k=2))):
        with pytest.raises(ValueError):
            eaas.eaas_grouped_swiglu(*a, ws, **kw)
    dy, wd, gu = torch.zeros((4, 6), dtype=bf), torch.zeros((2, 6, 5), dtype=bf), torch.zeros((4, 10), dtype=bf)
    for a, kw in (((dy[:3], off, wd, gu, gu), {}), ((dy, off, wd, gu[:3], gu), {}),
                  ((dy, off, wd, gu[:, :9], gu), {}), ((dy, off, wd, gu, gu.float()), {}),
                  ((dy, off, wd, gu, gu), dict(h=gu)), ((dy, off, wd, gu, gu), dict(h=gu[:3, :5])),
                  ((dy, off, wd.float(), gu, gu), {})):
        with pytest.raises(ValueError):
            eaas.eaas_grouped_swiglu_backward(*a, ws, **kw)
    q = eaas.eaas_quantize_blocks_fp8
    for a in ((x.half(), torch.zeros((4, 16), dtype=u8), torch.zeros((4, 1))),
              (x, torch.zeros((4, 16), dtype=torch.int8), torch.zeros((4, 1))),
              (x, torch.zeros((4, 16), dtype=u8), torch.zeros((4, 2))),
              (w, torch.zeros((2, 8, 16), dtype=u8), torch.zeros((2, 8, 1))),
              (w.transpose(1, 2), torch.zeros((2, 16, 8), dtype=u8), torch.zeros((2, 1, 1))),
              (x[0], torch.zeros(16, dtype=u8), torch.zeros(1))):
        with pytest.raises(ValueError):
            q(*a)
    with pytest.raises(ValueError):
        eaas.eaas_swiglu_fp8(torch.zeros((2, 7), dtype=bf), xq, xs)
    with pytest.raises(ValueError):
        eaas.eaas_swiglu_fp8(gu, torch.zeros((4, 5), dtype=u8), torch.zeros((4, 2)))
