"""The products of an expert layer on their own, as measurable cases: what a
user needs to train the experts that a server holds, and to serve them in 8-bit
integers.

A case is one pass through one operator:
  matmul   y[r] = W[e(r)] x[r] over rows grouped by expert (eaas_grouped_matmul)
  grads    its gradients dx[r] = W[e(r)]^T dy[r] and dW[e] = sum over the rows
           of e of dy[r] x[r]^T (eaas_grouped_matmul_dx, eaas_grouped_matmul_dw)
  int8     the product with weights in 8-bit integers, one scale per output
           channel, and rows quantized to 8 bits, one scale per row: from bf16
           rows (eaas_quantize_rows_int8) or, `gated`, from the gate and up
           projections (eaas_swiglu_int8); then eaas_grouped_matmul_int8
  swiglu   h = silu(gate) * up (eaas_swiglu), or `backward` its gradient
           (eaas_swiglu_backward)
  combine  the gradient of the weighted sum over a token's experts
           (eaas_unpermute_combine_backward)

Keys of a case: T tokens, k slots per token, E experts (a product's rows are the
T*k slots in the order that the routing gives them), N outputs and K inputs of an
expert's matrix (swiglu and combine: K is the width of a row).
  gather   the product reads token rows x[perm[r] / k] instead of rows x[r]
  pad      elements between the end of a row and the next one, x and dy
  out      type of y, dx and dW
  zipf     exponent of the experts' popularity, 0 for none
The sizes are those of this repository's shapes (paper_2509_17863_amd/synth.py,
perf/cases.py) and generic ones.
"""
from __future__ import annotations

import math

import torch

own = False


def _case(name, op, T, k, E, N, K, gather=False, pad=0, out="bf16", zipf=0.0, gated=False,
          backward=False):
    return dict(name=name, op=op, T=T, k=k, E=E, N=N, K=K, gather=gather, pad=pad, out=out,
                zipf=zipf, gated=gated, backward=backward)


def listed():
    return [
        # eight users on a many-expert model: about one row for each expert
        _case("matmul_decode_8", "matmul", 8, 8, 128, 1536, 2048, gather=True),
        # sizes that are no multiple of anything, rows cut out of a wider array
        _case("matmul_odd_777", "matmul", 777, 6, 24, 1283, 1921, pad=7, out="fp32", zipf=1.1),
        # gate and up projections of a prefill, unevenly used experts
        _case("matmul_prefill_4096", "matmul", 4096, 8, 32, 4096, 7168, gather=True, zipf=1.2),
        # a training micro-batch that gives each of many experts a few rows
        _case("grads_few_rows", "grads", 64, 8, 128, 2048, 768),
        # small matrices and many rows: the sum over the rows is the long axis
        _case("grads_long_axis", "grads", 16384, 2, 8, 256, 136, gather=True, out="fp32"),
        # a training step's down projection with few large experts
        _case("grads_train_4096", "grads", 4096, 2, 8, 4096, 14336, out="fp32"),
        # one user, one token, 8-bit weights
        _case("int8_decode_1", "int8", 1, 8, 32, 4096, 7168, gather=True),
        # the down projection of a prefill in 8 bits
        _case("int8_gated_4096", "int8", 4096, 8, 32, 7168, 2048, out="fp32", gated=True,
              zipf=1.2),
        # a decode batch's activation between the products
        _case("swiglu_decode_16", "swiglu", 16, 8, 128, 0, 768),
        # the activation's gradient in a training step
        _case("swiglu_backward_4096", "swiglu", 4096, 8, 32, 0, 2048, backward=True),
        # a small micro-batch's way back into the expert rows
        _case("combine_16", "combine", 16, 8, 128, 0, 2048),
        # a training step's
        _case("combine_4096", "combine", 4096, 8, 32, 0, 7168, zipf=1.2),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi):
    """A matrix dimension: two of three are multiples of 128, 16 or 8."""
    v, m = _log_int(rng, lo, hi), rng.choice([1, 1, 8, 16, 128, 128])
    return max(m, v // m * m)


_MAX_FLOPS = {"matmul": 2.0 * 32768 * 4096 * 7168, "grads": 4.0 * 8192 * 4096 * 14336,
              "int8": 2.0 * 32768 * 7168 * 2048, "swiglu": 1e12, "combine": 1e12}
_MAX_BYTES = {"matmul": 2.2e9, "grads": 3.0e9, "int8": 1.4e9, "swiglu": 6.7e8, "combine": 1.4e9}


def draw(rng):
    while True:
        op = rng.choice(["matmul", "matmul", "grads", "grads", "int8", "int8", "swiglu", "combine"])
        k = rng.randint(1, 8)
        E = _log_int(rng, max(k, 1), 160)
        T = _log_int(rng, 1, 16384)
        N, K = _size(rng, 24, 14336), _size(rng, 24, 14336)
        out, zipf = rng.choice(["bf16", "fp32"]), rng.choice([0.0, 0.0, 1.1])
        gather, pad = rng.random() < 0.5, rng.choice([0, 0, 8, 3])
        if op == "swiglu":
            c = _case(None, op, T, k, E, 0, K, backward=rng.random() < 0.5)
        elif op == "combine":
            # hidden sizes are multiples of 128 throughout
            c = _case(None, op, T, k, E, 0, max(128, K // 128 * 128), zipf=zipf)
        elif op == "int8" and rng.random() < 0.4:
            c = _case(None, op, T, k, E, N, K, out=out, zipf=zipf, gated=True)
        else:
            c = _case(None, op, T, k, E, N, K, gather=gather, pad=pad, out=out, zipf=zipf)
        w = work(c)
        # weights of every expert are in memory, used or not
        if w["flops"] > _MAX_FLOPS[op] or w["bytes"] > _MAX_BYTES[op] or E * N * K > 1.2e9:
            continue
        return c


# ------------------------------------------------------------------ inputs
def _popularity(case):
    p = [1.0 / (1 + i) ** case["zipf"] for i in range(case["E"])]
    return [v / sum(p) for v in p]


def _route(case, gen):
    """Top-k of random scores; the slots in stable order of their experts."""
    T, k, E = case["T"], case["k"], case["E"]
    score = torch.randn((T, E), device="cuda", generator=gen)
    if case["zipf"]:
        rank = torch.randperm(E, device="cuda", generator=gen).float() + 1.0
        score = score - case["zipf"] * torch.log(rank)
    val, ids = torch.topk(score, k, dim=1)
    flat = ids.reshape(-1)
    perm = torch.argsort(flat, stable=True)
    inv = torch.empty_like(perm)
    inv[perm] = torch.arange(T * k, device="cuda")
    counts = torch.bincount(flat, minlength=E)
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = torch.cumsum(counts, 0)
    active = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    used = counts.nonzero().reshape(-1)
    active[0] = used.numel()
    active[1: 1 + used.numel()] = used
    i32 = torch.int32
    routing = dict(counts=counts.to(i32), offsets=offsets, perm=perm.to(i32), inv=inv.to(i32),
                   active=active)
    return dict(routing, routing=routing, sizes=counts.tolist(),
                weights=torch.softmax(val, dim=1).contiguous())


def _rows(n, width, pad, gen, scale=1.0):
    """bf16 [n, width] ~ N(0, scale), `pad` elements between the rows."""
    a = torch.empty((n, width + pad), dtype=torch.bfloat16, device="cuda")
    step = max(1, (1 << 27) // (width + pad))
    for i in range(0, n, step):
        m = min(step, n - i)
        a[i: i + m] = torch.randn((m, width + pad), device="cuda", generator=gen).mul_(scale)
    return a[:, :width]


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + 17)
    op, T, k, E, N, K = (case[n] for n in ("op", "T", "k", "E", "N", "K"))
    R = T * k
    d = _route(case, gen)
    if op == "swiglu":
        d["gu"] = _rows(R, 2 * K, 0, gen)
        if case["backward"]:
            d["dh"] = _rows(R, K, 0, gen, 0.05)
        return d
    if op == "combine":
        d["dout"] = _rows(T, K, 0, gen, 0.05)
        d["y"] = torch.randn((R, K), device="cuda", generator=gen)
        return d
    if case["gated"] and op == "int8":
        d["gu"] = _rows(R, 2 * K, 0, gen)
    else:
        d["x"] = _rows(T if case["gather"] else R, K, case["pad"], gen)
    w = _rows(E * N, K, 0, gen, 1.0 / math.sqrt(K)).view(E, N, K)
    if op == "int8":
        # one scale per output channel, as a server quantizes its weights at load
        d["w"] = torch.empty((E, N, K), dtype=torch.int8, device="cuda")
        d["ws"] = torch.empty((E, N), device="cuda")
        for e in range(E):
            q, s = _quantize(w[e].float())
            d["w"][e], d["ws"][e] = q.to(torch.int8), s
    else:
        d["w"] = w
    if op == "grads":
        d["dy"] = _rows(R, N, case["pad"], gen, 0.05)
    return d


def prepare(case, seed):
    d = _inputs(case, seed)
    d["case"] = case
    if not own:
        return d
    from paper_2509_17863_amd import eaas

    op, T, k, E, N, K = (case[n] for n in ("op", "T", "k", "E", "N", "K"))
    R = T * k
    dt = torch.float32 if case["out"] == "fp32" else torch.bfloat16

    def buf(*shape, dtype=dt):
        return torch.empty(shape, dtype=dtype, device="cuda")

    if op in ("matmul", "int8"):
        d["out"] = buf(R, N)
    if op == "grads":
        d["dx"], d["dw"] = buf(R, K), buf(E, N, K)
    if op == "int8":
        n = R if case["gated"] or not case["gather"] else T
        d["q"], d["s"] = buf(n, K, dtype=torch.int8), buf(n, dtype=torch.float32)
    if op in ("matmul", "grads", "int8"):
        d["scratch"] = eaas.alloc_grouped_workspace(R, E, N, K)
    if op == "swiglu":
        d["out"] = buf(R, 2 * K if case["backward"] else K, dtype=torch.bfloat16)
    if op == "combine":
        d["dy"], d["dweights"] = buf(R, K, dtype=torch.bfloat16), buf(T, k, dtype=torch.float32)
    return d


# ------------------------------------------------------------------ one pass
def run(d):
    return _run_own(d) if own else _run_plain(d)


def _run_own(d):
    from paper_2509_17863_amd import eaas

    c = d["case"]
    op = c["op"]
    take = dict(perm=d["perm"], k=c["k"]) if c["gather"] else {}
    if op == "matmul":
        eaas.eaas_grouped_matmul(d["x"], d["offsets"], d["w"], d["out"], d["scratch"], **take)
        return d["out"]
    if op == "grads":
        eaas.eaas_grouped_matmul_dx(d["dy"], d["offsets"], d["w"], d["dx"], d["scratch"])
        eaas.eaas_grouped_matmul_dw(d["dy"], d["x"], d["offsets"], d["dw"], d["scratch"], **take)
        return {"dx": d["dx"], "dw": d["dw"]}
    if op == "int8":
        if c["gated"]:
            eaas.eaas_swiglu_int8(d["gu"], d["q"], d["s"])
        else:
            eaas.eaas_quantize_rows_int8(d["x"], d["q"], d["s"])
        eaas.eaas_grouped_matmul_int8(d["q"], d["s"], d["offsets"], d["w"], d["ws"], d["out"],
                                      d["scratch"], **take)
        return d["out"]
    if op == "swiglu":
        if c["backward"]:
            eaas.eaas_swiglu_backward(d["gu"], d["dh"], d["out"])
        else:
            eaas.eaas_swiglu(d["gu"], d["out"])
        return d["out"]
    eaas.eaas_unpermute_combine_backward(d["dout"], d["y"], d["routing"], d["weights"],
                                         d["dy"], d["dweights"], c["E"])
    return {"dy": d["dy"], "dweights": d["dweights"]}


def _quantize(a):
    """fp32 [n, K] -> whole numbers in [-127, 127] (as fp32) and a scale per row."""
    amax = a.abs().amax(dim=1)
    s = torch.where(amax > 0, amax / 127.0, torch.ones_like(amax))
    return torch.round(a / s[:, None]), s


def _groups(d):
    r = 0
    for e, n in enumerate(d["sizes"]):
        yield e, slice(r, r + n)
        r += n


def _token_rows(d, x):
    if d["case"]["gather"]:
        return x[(d["perm"] // d["case"]["k"]).long()]
    return x


def _run_plain(d):
    c = d["case"]
    op, R, E, N, K = c["op"], c["T"] * c["k"], c["E"], c["N"], c["K"]
    dt = torch.float32 if c["out"] == "fp32" else torch.bfloat16
    if op == "matmul":
        x = _token_rows(d, d["x"]).float()
        y = torch.empty((R, N), dtype=dt, device=x.device)
        for e, r in _groups(d):
            if r.stop > r.start:
                y[r] = (x[r] @ d["w"][e].float().t()).to(dt)
        return y
    if op == "grads":
        x, dy = _token_rows(d, d["x"]).float(), d["dy"].float()
        dx = torch.empty((R, K), dtype=dt, device=x.device)
        dw = torch.zeros((E, N, K), dtype=dt, device=x.device)
        for e, r in _groups(d):
            if r.stop > r.start:
                dx[r] = (dy[r] @ d["w"][e].float()).to(dt)
                dw[e] = (dy[r].t() @ x[r]).to(dt)
        return {"dx": dx, "dw": dw}
    if op == "int8":
        if c["gated"]:
            g, u = d["gu"].float().split(K, dim=1)
            q, s = _quantize(g / (1.0 + torch.exp(-g)) * u)
        else:
            q, s = _quantize(d["x"].float())
            q, s = _token_rows(d, q), _token_rows(d, s)
        y = torch.empty((R, N), dtype=dt, device=q.device)
        for e, r in _groups(d):
            if r.stop > r.start:
                p = q[r] @ d["w"][e].float().t()
                y[r] = (p * s[r][:, None] * d["ws"][e][None, :]).to(dt)
        return y
    if op == "swiglu":
        g, u = d["gu"].float().split(K, dim=1)
        sg = 1.0 / (1.0 + torch.exp(-g))
        if not c["backward"]:
            return (g * sg * u).to(torch.bfloat16)
        dh = d["dh"].float()
        dg = dh * u * sg * (1.0 + g * (1.0 - sg))
        return torch.cat([dg, dh * g * sg], dim=1).to(torch.bfloat16)
    k = c["k"]
    perm = d["perm"].long()
    do = d["dout"].float()
    dy = (do[perm // k] * d["weights"].reshape(-1)[perm][:, None]).to(torch.bfloat16)
    by_slot = d["y"][d["inv"].long()].view(c["T"], k, K)
    return {"dy": dy, "dweights": (by_slot * do[:, None, :]).sum(dim=2)}


# ------------------------------------------------------------------ measures
def work(case):
    """Each input read once (weights of the experts that get a row, token rows
    that are gathered once), each output written once; the products' and the
    sums' operations."""
    op, T, k, E, N, K = (case[n] for n in ("op", "T", "k", "E", "N", "K"))
    R = T * k
    used = sum(1.0 - (1.0 - min(1.0, k * p)) ** T for p in _popularity(case))
    out = 4 if case["out"] == "fp32" else 2
    rows = T if case["gather"] else R
    ids = 4.0 * R if case["gather"] else 0.0
    if op == "matmul":
        return {"bytes": 2.0 * rows * K + used * 2.0 * N * K + R * N * out + ids,
                "flops": 2.0 * R * N * K}
    if op == "grads":
        return {"bytes": (2.0 * rows * K + 2.0 * R * N + used * 2.0 * N * K + R * K * out
                          + E * N * K * float(out) + ids), "flops": 4.0 * R * N * K}
    if op == "int8":
        a = 4.0 * R * K if case["gated"] else 2.0 * rows * K
        return {"bytes": a + used * (N * K + 4.0 * N) + R * N * out + ids,
                "flops": 2.0 * R * N * K}
    if op == "swiglu":
        return {"bytes": R * K * (10.0 if case["backward"] else 6.0), "flops": R * K * 10.0}
    return {"bytes": 2.0 * T * K + 4.0 * R * K + 2.0 * R * K + 12.0 * R, "flops": 3.0 * R * K}


# ------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """The definitions in 64 bits.  (The 8-bit codes are those of the definition:
    quotient and scale of a row rounded to 32 bits, then to the nearest code.)"""
    d = _inputs(case, seed)
    op, T, k, E, N, K = (case[n] for n in ("op", "T", "k", "E", "N", "K"))
    R, f64 = T * k, torch.float64
    if op == "swiglu":
        a = d["gu"].double()
        g, u = a[:, :K], a[:, K:]
        sig = torch.sigmoid(g)
        if not case["backward"]:
            return sig * g * u
        dh = d["dh"].double()
        return torch.cat([dh * u * (sig + g * sig * (1 - sig)), dh * sig * g], dim=1)
    start = d["offsets"].tolist()
    if op == "combine":
        dy = torch.empty((R, K), dtype=f64, device="cuda")
        dweights = torch.empty((T, k), dtype=f64, device="cuda")
        do = d["dout"].double()
        for j in range(k):
            row = d["inv"].view(T, k)[:, j].long()
            dy[row] = d["weights"][:, j].double()[:, None] * do
            dweights[:, j] = (d["y"][row].double() * do).sum(dim=1)
        return {"dy": dy, "dweights": dweights}
    src = torch.div(d["perm"].long(), k, rounding_mode="floor") if case["gather"] else (
        torch.arange(R, device="cuda"))
    if op == "matmul":
        y = torch.zeros((R, N), dtype=f64, device="cuda")
        for e in range(E):
            a, b = start[e], start[e + 1]
            y[a:b] = torch.mm(d["x"][src[a:b]].double(), d["w"][e].double().t())
        return y
    if op == "grads":
        dx = torch.zeros((R, K), dtype=f64, device="cuda")
        dw = torch.zeros((E, N, K), dtype=f64, device="cuda")
        for e in range(E):
            a, b = start[e], start[e + 1]
            g = d["dy"][a:b].double()
            dx[a:b] = torch.mm(g, d["w"][e].double())
            dw[e] = torch.mm(g.t(), d["x"][src[a:b]].double())
        return {"dx": dx, "dw": dw}
    y = torch.zeros((R, N), dtype=f64, device="cuda")
    for e in range(E):
        a, b = start[e], start[e + 1]
        if case["gated"]:
            gu = d["gu"][a:b].double()
            v = (gu[:, :K] * torch.sigmoid(gu[:, :K]) * gu[:, K:]).float()
        else:
            v = d["x"][src[a:b]].float()
        top = v.abs().max(dim=1, keepdim=True).values if b > a else v[:, :1]
        scale = torch.where(top > 0, top / 127, torch.ones_like(top))
        codes = (v / scale).round().double()
        y[a:b] = torch.mm(codes, d["w"][e].double().t()) * scale.double() * d["ws"][e].double()
    return y
