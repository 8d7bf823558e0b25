"""The expert layers of examples/expert_layer.py on batches whose products take large tiles and
the tiles of few rows, and the e4m3 layer stage by stage: each one's outputs against the
64-bit oracle of what the stage before it wrote.

Tolerances.  Codes and scales are equal (e4m3 rows of the activation come from the kept bf16
projections, which the oracle starts from).  Sums in fp32 as in test_gpu_fp8_blocks.py:
(128 + B + 4 P + 2) 2^-23 of the terms' magnitudes, 7 * 2^-14 more where short sums are
allowed, and 2^-8 of a bf16 result.  The weighted sum of k rows adds (k + 1) 2^-23 of its
terms.
"""
import numpy as np
import pytest
import torch
from test_gpu_expert_layer import example, setup  # noqa: F401
from test_gpu_expert_layer_fused import test_layer as fused_layer
from test_gpu_fp8_blocks import blocks, silu_up

from oracle import layer_oracle as L
from paper_2509_17863_amd import eaas

pytestmark = pytest.mark.gpu
# T, H, I, E, k, experts elsewhere: large tiles (gated product, way back; e4m3 with short
# sums), few rows (all products)
LARGE, FEW = (2048, 512, 1536, 8, 4, 0), (12, 512, 640, 6, 2, 2)


def plans(T, H, I, E, k, _):
    R = T * k
    return {p: eaas._grouped_plan(p, R, E, *d, True)[0] for p, d in (
        ("swiglu", (2 * I, H)), ("swiglu_backward", (H, I)), ("fp8", (2 * I, H)), ("fp8_fp32", (H, I)))}


def test_plans():
    assert {p for p, kernel in plans(*LARGE).items() if kernel == "large"} == {"swiglu", "swiglu_backward", "fp8"}
    assert set(plans(*FEW).values()) == {"few"}


@pytest.mark.parametrize("shape", [LARGE, FEW], ids=str)
def test_fused_layer(gpu, example, shape):  # noqa: F811
    fused_layer(gpu, example, shape)


def near(got, want, tol, bf16=False):
    if bf16:
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
    err = np.abs(got - want)
    assert (err <= tol).all(), (err.max(), np.argwhere(~(err <= tol))[:4])


@pytest.mark.parametrize("short_sums", [False, True])
@pytest.mark.parametrize("shape", [LARGE, FEW, (7, 128, 256, 5, 3, 4), (300, 384, 128, 16, 4, 16)], ids=str)
def test_e4m3_stages(gpu, example, shape, short_sums):  # noqa: F811
    T, H, I, E, k, _ = shape
    R = T * k
    _, x, ids, scores, w, _, _ = setup(example, *shape, 3)
    layer = example.Fp8Experts(T, k, *w, short_sums=short_sums)
    for t in (layer.gate_up, layer.y):
        t.fill_(float("nan"))
    out = torch.empty((T, H), device="cuda")
    layer.forward(x, ids, scores, out)
    host = lambda t: t.cpu().numpy()  # noqa: E731
    off, perm, inv = (host(layer.routing[n]) for n in ("offsets", "perm", "inv"))
    live = int(off[-1])

    def codes(q, s, a, block_rows=1):
        wq, ws = L.quantize_blocks(a, block_rows)
        assert np.array_equal(host(q.view(torch.uint8)), wq) and np.array_equal(host(s), ws)
        return wq, ws

    # weights and tokens
    gu_w = [codes(layer.gate_up_q[e], layer.gate_up_s[e], w[0][e].float().cpu().numpy(), 128) for e in range(E)]
    dn_w = [codes(layer.down_q[e], layer.down_s[e], w[1][e].float().cpu().numpy(), 128) for e in range(E)]
    xq = codes(layer.xq, layer.xs, x.float().cpu().numpy())
    # gate and up
    want, mag = L.grouped_matmul_fp8(*xq, off, *map(np.stack, zip(*gu_w)), L.source_rows(R, perm, k))
    parts = eaas._grouped_plan("fp8_fp32", R, E, 2 * I, H, H % 16 == 0)[2]
    tol = ((128 + blocks(H) + 4 * parts + 2) * 2.0 ** -23 + (7 * 2.0 ** -14 if short_sums else 0)) * mag
    near(host(layer.gate_up[:live].double()), want, tol, bf16=True)
    # the activation's codes
    hq = codes(layer.hq[:live], layer.hs[:live], silu_up(layer.gate_up[:live].cpu()))
    # the down projection
    want, mag = L.grouped_matmul_fp8(*hq, off, *map(np.stack, zip(*dn_w)), np.arange(live))
    parts = eaas._grouped_plan("fp8_fp32", R, E, H, I, I % 16 == 0)[2]
    y = host(layer.y.double())
    near(y[:live], want, (128 + blocks(I) + 4 * parts + 2) * 2.0 ** -23 * mag)
    # the weighted sum
    sc = host(scores.double())
    near(host(out.double()), L.combine(y, inv, sc), (k + 1) * 2.0 ** -23 * L.combine(np.abs(y), inv, sc))
