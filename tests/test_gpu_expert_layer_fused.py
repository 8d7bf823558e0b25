"""The expert layer of examples/expert_layer.py with the activation inside its products,
forward and backward, and in e4m3: the calls run together.

Tolerances.  The forward pass rounds h to bf16 (gate and up reach the activation
unrounded), the backward pass dy, dgate and dup, from gate and up rounded, and dx: a
rounding moves a value by 2^-8 of itself at most, and a chain of n of them the whole array
by n * 2^-8 of its norm at most.  e4m3: a code is 2^-4 of its value away at most, for both
operands of both products (below the format's normal range 2^-10 of the scale, 448 of
which are the block's largest: far less of the norm), and gate and up are rounded to bf16.
"""
import pytest
import torch
from test_gpu_expert_layer import (SHAPES, backward64, example, forward64, rel,  # noqa: F401
                                   setup)

from paper_2509_17863_amd import eaas

pytestmark = pytest.mark.gpu


def fused(example, shape, seed):  # noqa: F811
    """The layer's inputs and its 64-bit reference, with the fused layer's outputs."""
    _, x, ids, scores, w, _, host = setup(example, *shape, seed)
    T, H, I, E, k, _ = shape
    layer = example.FusedExpertLayer(T, H, I, E, k)
    for t in (layer.h, layer.gate_up, layer.y, layer.dgate_up):
        t.fill_(float("nan"))
    out = torch.empty((T, H), device="cuda")
    layer.forward(x, ids, scores, *w, out)
    return layer, x, ids, scores, w, out, host


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_layer(gpu, example, shape):  # noqa: F811
    T, H, I, E, k, _ = shape
    layer, x, ids, scores, w, out, host = fused(example, shape, 1)
    gu, h, y, want = forward64(**host)
    assert rel(out, want) < 2.0 ** -8
    # the step computes the same layer
    step = torch.empty_like(out)
    eaas.eaas_expert_forward(x, ids, scores, *w, step, eaas.alloc_workspace(T, H, I, E, k))
    assert rel(step, want) < 2 * 2.0 ** -8
    dout = torch.randn((T, H), device="cuda").to(torch.bfloat16)
    dx, dscores = torch.empty((T, H), device="cuda"), torch.empty((T, k), device="cuda")
    grads = [torch.full(v.shape, float("nan"), device="cuda") for v in w]
    layer.h.fill_(float("nan"))  # computed again on the way back
    layer.backward(dout, dx, dscores, *grads)
    ref = backward64(dout.double().cpu().numpy(), **host, gu=gu, h=h, y=y)
    for got, exact in zip((dx, dscores, *grads), ref):
        assert rel(got, exact) < 4 * 2.0 ** -8
    first = [g.clone() for g in grads]
    layer.backward(dout, dx, dscores, *grads, accumulate=True)
    for g, f in zip(grads, first):
        assert torch.allclose(g, 2 * f, rtol=1e-6, atol=0)


def test_replayed_step(gpu, example):  # noqa: F811
    """Forward and backward in a captured graph, replayed on new tokens between eager work."""
    shape = (300, 384, 128, 16, 4, 16)
    layer, x, ids, scores, w, out, host = fused(example, shape, 4)
    T, H, I, E, k, _ = shape
    dout = torch.randn((T, H), device="cuda").to(torch.bfloat16)
    dx, dscores = torch.empty((T, H), device="cuda"), torch.empty((T, k), device="cuda")
    grads = [torch.empty(v.shape, device="cuda") for v in w]

    def step(l):
        l.forward(x, ids, scores, *w, out)
        l.backward(dout, dx, dscores, *grads)

    step(layer)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(layer)
    eager = example.FusedExpertLayer(T, H, I, E, k)
    gen = torch.Generator(device="cuda").manual_seed(9)
    for _ in range(3):
        for t, v in zip((x, ids, scores), example.batch(T, H, E + 16, k, gen)):
            t.copy_(v)
        step(eager)
        want = [t.clone() for t in (out, dx, dscores, *grads)]
        for t in (out, dx, dscores, *grads):
            t.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out, dx, dscores, *grads), want))


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_e4m3(gpu, example, shape):  # noqa: F811
    _, x, ids, scores, w, out, host = setup(example, *shape, 3)
    served = torch.empty_like(out)
    example.Fp8Experts(shape[0], shape[4], *w).forward(x, ids, scores, served)
    assert rel(served, forward64(**host)[3]) < 4 * 2.0 ** -4 + 2.0 ** -8


def test_training_runs(gpu, example):  # noqa: F811
    losses, w, b, layer = example.train(steps=3, make=example.FusedExpertLayer)
    assert all(v == v and v < float("inf") for v in losses)
    assert all(torch.isfinite(t).all() for t in w)
