"""The expert layer of examples/expert_layer.py: the separate products run
together, forward, backward and in 8-bit integers.

Tolerances.  The forward pass rounds gate/up and h to bf16, the backward pass dy, dh
and dgate_up too, and dx; each rounding moves a value by 2^-8 of itself at most, and
a chain of n of them the whole array by n * 2^-8 of its norm at most (in the norm the
independent roundings of many elements average far below that).  8-bit integers:
codes are half a step from the values, a step is amax/127 of a row, and the rows
here have amax below 5 times their rms: 5/127/2 of the norm per operand at most,
four operands.
"""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import layer_oracle as L
from paper_2509_17863_amd import eaas

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    path = os.path.join(ROOT, "examples", "expert_layer.py")
    spec = importlib.util.spec_from_file_location("expert_layer_example", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def forward64(x, off, perm, inv, k, scores, wgu, wd):
    src = L.source_rows(len(perm), perm, k)
    gu = np.zeros((len(perm), wgu.shape[1]))
    live = int(off[-1])
    gu[:live] = L.grouped_matmul(x, off, wgu, src)[0]
    h = L.swiglu(gu)
    y = np.zeros((len(perm), wd.shape[1]))
    y[:live] = L.grouped_matmul(h, off, wd, np.arange(len(perm)))[0]
    return gu, h, y, L.combine(y, inv, scores)


def backward64(dout, x, off, perm, inv, k, scores, wgu, wd, gu, h, y):
    src = L.source_rows(len(perm), perm, k)
    live = int(off[-1])
    dy, dscores, _ = L.combine_backward(dout, y, inv, scores)
    dy = np.nan_to_num(dy)
    dwd, _ = L.grouped_matmul_dw(dy, h, off, np.arange(len(perm)))
    dh = np.zeros_like(h)
    dh[:live] = L.grouped_matmul_dx(dy, off, wd)[0]
    dgu = L.swiglu_backward(gu, dh)
    dwgu, _ = L.grouped_matmul_dw(dgu, x, off, src)
    rows = np.zeros((len(perm), x.shape[1]))
    rows[:live] = L.grouped_matmul_dx(dgu, off, wgu)[0]
    dx = L.combine(rows, inv, np.ones_like(scores))
    return dx, dscores, dwgu, dwd


def rel(got, want):
    got = got.double().cpu().numpy()
    return np.linalg.norm(got - want) / np.linalg.norm(want)


def setup(example, T, H, I, E, k, elsewhere, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x, ids, scores = example.batch(T, H, E + elsewhere, k, gen)
    w = [v.to(torch.bfloat16) for v in example.weights(E, H, I, gen)]
    layer = example.ExpertLayer(T, H, I, E, k)
    out = torch.empty((T, H), device="cuda")
    layer.forward(x, ids, scores, *w, out)
    r = layer.routing
    host = dict(x=x.double().cpu().numpy(), off=r["offsets"].cpu().numpy(),
                perm=r["perm"].cpu().numpy()[: T * k], inv=r["inv"].cpu().numpy()[: T * k], k=k,
                scores=scores.double().cpu().numpy(), wgu=w[0].double().cpu().numpy(),
                wd=w[1].double().cpu().numpy())
    return layer, x, ids, scores, w, out, host


SHAPES = [(64, 256, 128, 8, 2, 0), (7, 128, 256, 5, 3, 4), (300, 384, 128, 16, 4, 16),
          (2048, 256, 128, 4, 2, 0)]


@pytest.mark.parametrize("T,H,I,E,k,elsewhere", SHAPES)
def test_layer(gpu, example, T, H, I, E, k, elsewhere):
    layer, x, ids, scores, w, out, host = setup(example, T, H, I, E, k, elsewhere, 1)
    gu, h, y, want = forward64(**host)
    assert rel(out, want) < 2 * 2.0 ** -8
    # the fused step computes the same layer
    fused = torch.empty_like(out)
    eaas.eaas_expert_forward(x, ids, scores, *w, fused, eaas.alloc_workspace(T, H, I, E, k))
    assert rel(fused, want) < 2 * 2.0 ** -8
    dout = torch.randn((T, H), device="cuda").to(torch.bfloat16)
    dx, dscores = torch.empty((T, H), device="cuda"), torch.empty((T, k), device="cuda")
    grads = [torch.full(v.shape, float("nan"), device="cuda") for v in w]
    layer.backward(dout, dx, dscores, *grads)
    ref = backward64(dout.double().cpu().numpy(), **host, gu=gu, h=h, y=y)
    for got, exact in zip((dx, dscores, *grads), ref):
        assert rel(got, exact) < 5 * 2.0 ** -8
    # a second pass adds up
    first = [g.clone() for g in grads]
    layer.backward(dout, dx, dscores, *grads, accumulate=True)
    for g, f in zip(grads, first):
        assert torch.allclose(g, 2 * f, rtol=1e-6, atol=0)


def test_gradients_against_differences(gpu, example):
    """Directional derivatives of the 64-bit loss <out, dout>."""
    T, H, I, E, k = 96, 128, 128, 4, 2
    layer, x, ids, scores, w, out, host = setup(example, T, H, I, E, k, 2, 2)
    dout = torch.randn((T, H), device="cuda").to(torch.bfloat16)
    dx, dscores = torch.empty((T, H), device="cuda"), torch.empty((T, k), device="cuda")
    grads = [torch.empty(v.shape, device="cuda") for v in w]
    layer.backward(dout, dx, dscores, *grads)
    d64 = dout.double().cpu().numpy()
    rng = np.random.default_rng(0)
    for name, g in (("x", dx), ("scores", dscores), ("wgu", grads[0]), ("wd", grads[1])):
        g = g.double().cpu().numpy()
        # along the gradient, where the derivative is its norm, and a random direction
        for step in (g / np.linalg.norm(g), rng.normal(size=g.shape) / np.sqrt(g.size)):
            eps = 1e-4
            loss = [(forward64(**{**host, name: host[name] + s * eps * step})[3] * d64).sum()
                    for s in (1, -1)]
            slope = (loss[0] - loss[1]) / (2 * eps)
            # (differences add eps^2 and 1e-16/eps of the loss: far below the roundings)
            assert abs(slope - (g * step).sum()) < 5 * 2.0 ** -8 * np.linalg.norm(g)


@pytest.mark.parametrize("T,H,I,E,k,elsewhere", SHAPES)
def test_int8(gpu, example, T, H, I, E, k, elsewhere):
    layer, x, ids, scores, w, out, host = setup(example, T, H, I, E, k, elsewhere, 3)
    served = torch.empty_like(out)
    example.Int8Experts(T, k, *w).forward(x, ids, scores, served)
    want = forward64(**host)[3]
    assert rel(served, want) < 4 * 5 / 127 / 2


def test_training_lowers_the_loss(gpu, example):
    losses, w, b, layer = example.train(steps=12)
    assert np.isfinite(losses).all() and losses[-1] < 0.7 * losses[0], losses
