"""An expert layer trained and then served in 8-bit integers, on the library's
separate products.

    python examples/expert_layer.py

fits the experts of a small layer to another layer's outputs (fp32 master weights,
gradients of two micro-batches added up), then quantizes the trained experts and
serves the same tokens with 8-bit products.

The layer is the one of eaas_expert_forward: a token's k slots name experts (ids of
experts that live elsewhere are skipped), every expert is the SwiGLU form without
bias, and the token gets the sum of its experts' outputs weighted by the router's
scores.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2509_17863_amd import eaas  # noqa: E402


def _buf(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="cuda")


class ExpertLayer:
    """Forward and backward pass of E experts [H -> I -> H] for batches of T tokens
    with k slots each.  Activations that the backward pass reads stay in the
    object until the next forward pass."""

    def __init__(self, T, H, I, E, k):
        self.T, self.H, self.I, self.E, self.k = T, H, I, E, k
        R = T * k
        self.routing = eaas.alloc_routing(T, k, E)
        self.route_ws = eaas.alloc_workspace(T, H, I, E, k)
        n = max(eaas.eaas_grouped_workspace_bytes(R, E, 2 * I, H),
                eaas.eaas_grouped_workspace_bytes(R, E, H, I))
        self.ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        self.gate_up, self.h = _buf(R, 2 * I), _buf(R, I)
        self.y, self.dy = _buf(R, H, dtype=torch.float32), _buf(R, H)
        self.dh, self.dgate_up = _buf(R, I), _buf(R, 2 * I)
        self.dx_rows = _buf(R, H, dtype=torch.float32)
        self.ones = torch.ones((T, k), device="cuda")

    def forward(self, x, ids, scores, w_gate_up, w_down, out):
        """x [T,H] bf16, ids [T,k] int32, scores [T,k] fp32, w_gate_up [E,2I,H] and
        w_down [E,H,I] bf16 -> out [T,H] (bf16 or fp32)."""
        r = self.routing
        eaas.eaas_route_permute(ids, self.E, r, self.route_ws, H=self.H, I=self.I)
        self.off = r["offsets"]
        self.rows = r["offsets"][self.E:]  # rows that belong to an expert here
        self.x, self.scores, self.w_gate_up, self.w_down = x, scores, w_gate_up, w_down
        eaas.eaas_grouped_matmul(x, self.off, w_gate_up, self.gate_up, self.ws, perm=r["perm"],
                                 k=self.k)
        eaas.eaas_swiglu(self.gate_up, self.h, n_rows=self.rows)
        eaas.eaas_grouped_matmul(self.h, self.off, w_down, self.y, self.ws)
        eaas.eaas_unpermute_combine(self.y, r, scores, out, self.E, I=self.I)

    def backward(self, dout, dx, dscores, dw_gate_up, dw_down, accumulate=False):
        """dout [T,H] bf16 or fp32 -> dx [T,H], dscores [T,k] fp32, and the weights'
        gradients (accumulate: added to fp32 ones)."""
        r = self.routing
        eaas.eaas_unpermute_combine_backward(dout, self.y, r, self.scores, self.dy, dscores,
                                             self.E, I=self.I)
        eaas.eaas_grouped_matmul_dw(self.dy, self.h, self.off, dw_down, self.ws,
                                    accumulate=accumulate)
        eaas.eaas_grouped_matmul_dx(self.dy, self.off, self.w_down, self.dh, self.ws)
        eaas.eaas_swiglu_backward(self.gate_up, self.dh, self.dgate_up, n_rows=self.rows)
        eaas.eaas_grouped_matmul_dw(self.dgate_up, self.x, self.off, dw_gate_up, self.ws,
                                    perm=r["perm"], k=self.k, accumulate=accumulate)
        eaas.eaas_grouped_matmul_dx(self.dgate_up, self.off, self.w_gate_up, self.dx_rows, self.ws)
        # a token's gradient is the sum of its slots' rows
        eaas.eaas_unpermute_combine(self.dx_rows, r, self.ones, dx, self.E, I=self.I)


class Int8Experts:
    """The experts in 8-bit integers: weights with a scale per output channel,
    quantized once; activations with a scale per row, quantized on the way."""

    def __init__(self, T, k, w_gate_up, w_down):
        self.E, two_i, self.H = w_gate_up.shape
        self.T, self.k, self.I = T, k, two_i // 2
        R = T * k
        self.gate_up_q, self.gate_up_s = self._weights(w_gate_up)
        self.down_q, self.down_s = self._weights(w_down)
        self.routing = eaas.alloc_routing(T, k, self.E)
        self.route_ws = eaas.alloc_workspace(T, self.H, self.I, self.E, k)
        n = max(eaas.eaas_grouped_workspace_bytes(R, self.E, two_i, self.H),
                eaas.eaas_grouped_workspace_bytes(R, self.E, self.H, self.I))
        self.ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        self.xq, self.xs = _buf(T, self.H, dtype=torch.int8), _buf(T, dtype=torch.float32)
        self.gate_up = _buf(R, two_i)
        self.hq, self.hs = _buf(R, self.I, dtype=torch.int8), _buf(R, dtype=torch.float32)
        self.y = _buf(R, self.H, dtype=torch.float32)

    @staticmethod
    def _weights(w):
        E, N, K = w.shape
        q, s = _buf(E * N, K, dtype=torch.int8), _buf(E * N, dtype=torch.float32)
        eaas.eaas_quantize_rows_int8(w.view(E * N, K), q, s)
        return q.view(E, N, K), s.view(E, N)

    def forward(self, x, ids, scores, out):
        r = self.routing
        eaas.eaas_route_permute(ids, self.E, r, self.route_ws, H=self.H, I=self.I)
        off = r["offsets"]
        eaas.eaas_quantize_rows_int8(x, self.xq, self.xs)
        eaas.eaas_grouped_matmul_int8(self.xq, self.xs, off, self.gate_up_q, self.gate_up_s,
                                      self.gate_up, self.ws, perm=r["perm"], k=self.k)
        eaas.eaas_swiglu_int8(self.gate_up, self.hq, self.hs, n_rows=off[self.E:])
        eaas.eaas_grouped_matmul_int8(self.hq, self.hs, off, self.down_q, self.down_s, self.y,
                                      self.ws)
        eaas.eaas_unpermute_combine(self.y, r, scores, out, self.E, I=self.I)


def batch(T, H, E, k, gen):
    x = torch.randn((T, H), device="cuda", generator=gen).to(torch.bfloat16)
    val, ids = torch.topk(torch.randn((T, E), device="cuda", generator=gen), k, dim=1)
    return x, ids.to(torch.int32), torch.softmax(val, dim=1).contiguous()


def weights(E, H, I, gen):
    def make(*shape):
        return torch.randn(shape, device="cuda", generator=gen) / shape[-1] ** 0.5

    return make(E, 2 * I, H), make(E, H, I)


def train(steps=30, T=512, H=256, I=128, E=8, k=2, lr=64.0, seed=0):
    """Losses of the steps, and the trained experts (bf16) with a batch."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    layer = ExpertLayer(T, H, I, E, k)
    target = [w.to(torch.bfloat16) for w in weights(E, H, I, gen)]
    master = [t.float() + 0.5 * w for t, w in zip(target, weights(E, H, I, gen))]
    grads = [torch.empty_like(m) for m in master]
    out, want = _buf(T, H, dtype=torch.float32), _buf(T, H, dtype=torch.float32)
    dx, dscores = _buf(T, H), _buf(T, k, dtype=torch.float32)
    losses = []
    for _ in range(steps):
        loss = torch.zeros((), device="cuda")
        w = [m.to(torch.bfloat16) for m in master]
        for micro in range(2):
            b = batch(T, H, E, k, gen)
            layer.forward(*b, *target, want)
            layer.forward(*b, *w, out)
            err = out - want
            loss += (err * err).mean() / 2
            layer.backward(err / err.numel(), dx, dscores, *grads, accumulate=micro > 0)
        for m, g in zip(master, grads):
            m.sub_(g, alpha=lr)
        losses.append(loss)
    return [float(v) for v in losses], [m.to(torch.bfloat16) for m in master], b, layer


def main():
    losses, w, b, layer = train()
    print("loss", " ".join(f"{v:.4f}" for v in losses[::5] + losses[-1:]))
    T, H = b[0].shape
    out, served = _buf(T, H, dtype=torch.float32), _buf(T, H, dtype=torch.float32)
    layer.forward(*b, *w, out)
    Int8Experts(T, layer.k, *w).forward(*b, served)
    rel = ((served - out).norm() / out.norm()).item()
    print(f"8-bit experts: {rel:.4f} of the outputs' norm from the bf16 layer")


if __name__ == "__main__":
    main()
