"""The expert layer of examples/expert_layer.py on batches that give no expert a row."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    path = os.path.join(ROOT, "examples", "expert_layer.py")
    spec = importlib.util.spec_from_file_location("expert_layer_example_empty", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("T", [0, 1, 37])
def test_no_row_for_any_expert(gpu, example, T):
    """No tokens, or tokens whose every expert lives elsewhere."""
    H, I, E, k = 256, 128, 8, 2
    gen = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn((T, H), device="cuda", generator=gen).to(torch.bfloat16)
    ids = torch.full((T, k), -1, dtype=torch.int32, device="cuda")
    ids[:, 1:] = E + 3
    scores = torch.rand((T, k), device="cuda", generator=gen)
    w = [v.to(torch.bfloat16) for v in example.weights(E, H, I, gen)]
    layer = example.ExpertLayer(T, H, I, E, k)
    out, dx = (torch.full((T, H), 7.0, device="cuda") for _ in range(2))
    layer.forward(x, ids, scores, *w, out)
    assert (out == 0).all()
    dscores = torch.full((T, k), 7.0, device="cuda")
    grads = [torch.full(v.shape, float("nan"), device="cuda") for v in w]
    layer.backward(torch.randn((T, H), device="cuda", generator=gen), dx, dscores, *grads)
    assert (dx == 0).all() and (dscores == 0).all()
    assert all((g == 0).all() for g in grads)
    for g in grads:
        g.fill_(3.0)
    layer.backward(out, dx, dscores, *grads, accumulate=True)
    assert all((g == 3).all() for g in grads)
    served = torch.full((T, H), 7.0, device="cuda")
    example.Int8Experts(T, k, *w).forward(x, ids, scores, served)
    assert (served == 0).all()
