"""The separate products' C ABI on the host: what they refuse, and with which
status, before anything reaches a device; and the binding's own checks."""
import ctypes

import pytest
import torch

from paper_2509_17863_amd import eaas

A, B, C, D = (i << 30 for i in range(1, 5))  # stand-ins for device pointers, far apart
BIG = 1 << 40


def shape(R=64, E=4, N=128, K=256):
    return eaas._GroupShape(R, E, N, K)


def ref(s):
    return ctypes.byref(s) if s is not None else None


@pytest.mark.parametrize("kw,ok", [
    (dict(), True), (dict(R=0), True), (dict(N=1, K=1), True), (dict(E=1024), True),
    (dict(R=-1), False), (dict(E=0), False), (dict(E=1025), False), (dict(N=0), False),
    (dict(K=0), False), (dict(N=46341, K=46341), False), (dict(N=46340, K=46340), True),
])
def test_workspace_bytes(kw, ok):
    n = eaas.lib().eaas_grouped_workspace_bytes(ref(shape(**kw)))
    assert (n > 0) == ok and n % 256 == 0


def test_workspace_bytes_of_null():
    assert eaas.lib().eaas_grouped_workspace_bytes(None) == 0


def forward(s=shape(), x=A, ldx=256, perm=None, k=1, off=B, w=C, y=D, ldy=128, dt=0, ws=BIG,
            n=1 << 40):
    return eaas.lib().eaas_grouped_matmul(ref(s), x, ldx, perm, k, off, w, y, ldy, dt, ws, n, None)


def int8(s=shape(), x=A, xs=B, perm=None, k=1, off=B, w=C, wsc=B, y=D, ldy=128, dt=0, ws=BIG,
         n=1 << 40):
    return eaas.lib().eaas_grouped_matmul_int8(ref(s), x, xs, perm, k, off, w, wsc, y, ldy, dt, ws,
                                               n, None)


def rows(s=shape(), dy=A, lddy=128, off=B, w=C, dx=D, lddx=256, dt=0, ws=BIG, n=1 << 40):
    return eaas.lib().eaas_grouped_matmul_dx(ref(s), dy, lddy, off, w, dx, lddx, dt, ws, n, None)


def weights(s=shape(), dy=A, lddy=128, x=C, ldx=256, perm=None, k=1, off=B, dw=D, dt=2, acc=0,
            ws=BIG, n=1 << 40):
    return eaas.lib().eaas_grouped_matmul_dw(ref(s), dy, lddy, x, ldx, perm, k, off, dw, dt, acc,
                                             ws, n, None)


@pytest.mark.parametrize("call", [forward, int8, rows, weights])
def test_shapes(call):
    assert call(s=None) == -1
    assert call(s=shape(R=-1)) == -1
    assert call(s=shape(E=1025)) == -2
    assert call(s=shape(N=1 << 16, K=1 << 16)) == -2
    assert call(off=None) == -1
    assert call(off=B + 2) == -1
    assert call(dt=1) == -1


@pytest.mark.parametrize("call", [forward, int8, weights])
def test_gather(call):
    assert call(perm=B, k=0) == -1
    assert call(perm=B, k=3) == -1          # 64 rows are not 3 a token
    assert call(perm=B + 2, k=2) == -1
    assert call(s=shape(R=1 << 26), perm=B, k=1) == -2


def test_forward():
    for bad in (dict(x=None), dict(w=None), dict(y=None), dict(ldx=255), dict(ldy=127),
                dict(x=A + 1), dict(w=C + 8), dict(y=D + 1), dict(y=D + 2, dt=2), dict(y=A),
                dict(y=C + 64), dict(y=A + 63 * 512 + 511)):
        assert forward(**bad) == -1, bad
    assert forward(ldx=(1 << 22) + 1) == -2 and forward(ldy=(1 << 22) + 1) == -2
    empty = shape(R=0)
    assert forward(s=empty, x=None, off=None, w=None, y=None, ws=None, n=0) == 0


def test_int8():
    for bad in (dict(x=None), dict(xs=None), dict(wsc=None), dict(w=None), dict(y=None),
                dict(xs=B + 2), dict(wsc=B + 1), dict(w=C + 4), dict(y=A + 8)):
        assert int8(**bad) == -1, bad
    assert int8(s=shape(K=1 << 17)) == -2
    assert int8(s=shape(R=0), x=None, xs=None, off=None, w=None, y=None) == 0


def test_gradients():
    for bad in (dict(dy=None), dict(w=None), dict(dx=None), dict(lddy=127), dict(lddx=255),
                dict(dx=A + 2), dict(dx=C), dict(w=C + 2), dict(dx=D + 2, dt=2)):
        assert rows(**bad) == -1, bad
    assert rows(s=shape(R=0), dy=None, off=None, w=None, dx=None) == 0
    for bad in (dict(dy=None), dict(x=None), dict(dw=None), dict(dw=D + 8), dict(dw=A), dict(dw=C),
                dict(acc=1, dt=0), dict(ldx=255), dict(lddy=100), dict(x=C + 1)):
        assert weights(**bad) == -1, bad
    assert weights(s=shape(R=0), dy=None, x=None, dw=None, acc=1) == 0
    assert weights(s=shape(R=0), dy=None, x=None, dw=None) == -1


def test_workspace_refusals():
    """A shape whose long sum is split needs its partial sums' memory."""
    s = shape(R=32, E=1, N=64, K=8192)
    assert eaas.lib().eaas_grouped_workspace_bytes(ref(s)) > 256
    assert forward(s=s, ldx=8192, ws=None) == -3
    assert forward(s=s, ldx=8192, n=256) == -3
    assert forward(s=s, ldx=8192, ws=BIG + 8) == -3


def test_activation_refusals():
    L = eaas.lib()
    q = lambda x=A, ld=64, rows=8, K=64, q=B, s=C: L.eaas_quantize_rows_int8(  # noqa: E731
        x, ld, rows, K, q, s, None)
    for bad in (dict(x=None), dict(q=None), dict(s=None), dict(rows=-1), dict(K=0), dict(ld=63),
                dict(x=A + 1), dict(s=C + 2), dict(q=A + 100), dict(s=A)):
        assert q(**bad) == -1, bad
    assert q(K=1 << 23, ld=1 << 23) == -2 and q(rows=1 << 31) == -2
    assert q(rows=0, x=None, q=None, s=None) == 0
    f = lambda gu=A, rows=8, I=64, n=None, h=B: L.eaas_swiglu(gu, rows, I, n, h, None)  # noqa: E731
    for bad in (dict(gu=None), dict(h=None), dict(rows=-1), dict(I=0), dict(gu=A + 1), dict(h=A),
                dict(h=A + 2 * 8 * 128 - 2), dict(n=C + 2)):
        assert f(**bad) == -1, bad
    assert f(I=(1 << 21) + 1) == -2 and f(rows=0, gu=None, h=None) == 0
    i = lambda gu=A, rows=8, I=64, n=None, q=B, s=C: L.eaas_swiglu_int8(  # noqa: E731
        gu, rows, I, n, q, s, None)
    for bad in (dict(gu=None), dict(q=None), dict(s=None), dict(q=A), dict(s=A + 4)):
        assert i(**bad) == -1, bad
    b = lambda gu=A, dh=B, rows=8, I=64, n=None, o=C: L.eaas_swiglu_backward(  # noqa: E731
        gu, dh, rows, I, n, o, None)
    for bad in (dict(gu=None), dict(dh=None), dict(o=None), dict(o=A + 2), dict(o=B), dict(dh=B + 1)):
        assert b(**bad) == -1, bad


def test_combine_backward_refusals():
    L = eaas.lib()
    r = eaas._Routing(A, A, A, A, A)

    def f(s=eaas._Shape(64, 256, 128, 8, 2), d=B, dt=0, y=C, r=r, w=A, dy=D, dw=5 << 30):
        return L.eaas_unpermute_combine_backward(ctypes.byref(s) if s else None, d, dt, y,
                                                 ctypes.byref(r) if r else None, w, dy, dw, None)

    for bad in (dict(s=None), dict(d=None), dict(y=None), dict(r=None), dict(w=None),
                dict(dy=None), dict(dw=None), dict(dt=1), dict(d=B + 8), dict(dy=C), dict(dw=D),
                dict(dw=B + 16), dict(s=eaas._Shape(-1, 256, 128, 8, 2))):
        assert f(**bad) == -1, bad
    assert f(s=eaas._Shape(64, 200, 128, 8, 2)) == -2
    assert f(s=eaas._Shape(0, 256, 128, 8, 2), d=None, y=None, r=None) == 0


def test_binding_checks():
    """Shapes and types that the C ABI cannot see."""
    w, off = torch.zeros((2, 8, 16), dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    ws = torch.zeros(256, dtype=torch.uint8)
    x, y = torch.zeros((4, 16), dtype=torch.bfloat16), torch.zeros((4, 8))
    call = eaas.eaas_grouped_matmul
    for a in ((x[:, :8], off, w, y), (x.float(), off, w, y), (x, off[:2], w, y),
              (x, off.long(), w, y), (x, off, w.float(), y), (x[:2], off, w, y),
              (x, off, w, y.half()), (x.t().contiguous().t(), off, w, y),
              (x, off, w.transpose(1, 2).contiguous().transpose(1, 2), y)):
        with pytest.raises(ValueError):
            call(*a, ws)
    with pytest.raises(ValueError):
        call(x, off, w, y, ws, perm=torch.zeros(4, dtype=torch.int32), k=2)
    with pytest.raises(ValueError):
        eaas.eaas_swiglu(torch.zeros((2, 7), dtype=torch.bfloat16), x)
    with pytest.raises(ValueError):
        eaas.eaas_quantize_rows_int8(x, torch.zeros((4, 16), dtype=torch.int8), torch.zeros(3))
