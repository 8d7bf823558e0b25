"""An expert layer's product in 8-bit floating point and its gated half as one
kernel, as measurable cases.

A case is one pass through one operator:
  fp8       y[r] = W[e(r)] x[r] with e4m3 codes on both sides and fp32 scales, one for
            each 128 columns of a row and one for each 128 x 128 block of a matrix:
            from bf16 rows (eaas_quantize_blocks_fp8) or, `gated`, from the gate and
            up projections (eaas_swiglu_fp8); then eaas_grouped_matmul_fp8
  swiglu    h[r] = silu(Wgate x[r]) * (Wup x[r]): both projections, the activation
            and the product (eaas_grouped_swiglu); `keep`: the projections are
            written too, for the backward pass
  backward  its way back from the gradient of the down projection's result:
            dh = Wdown^T dy, then dgate, dup and h from the kept projections
            (eaas_grouped_swiglu_backward)

Keys of a case: T tokens, k slots per token, E experts (a product's rows are the
T*k slots in the order that the routing gives them), N and K:
  fp8       outputs and inputs of an expert's matrix
  swiglu    N gate columns (as many up columns), K inputs
  backward  N outputs of the down projection, K its inputs (gate columns)
  gather    the product reads token rows x[perm[r] / k] instead of rows x[r]
  pad       elements between the end of a row and the next one, bf16 x and dy
  out       type of y
  zipf      exponent of the experts' popularity, 0 for none
The sizes are those of this repository's shapes (paper_2509_17863_amd/synth.py,
perf/cases.py, perf/operators.py) and generic ones.
"""
from __future__ import annotations

import math

import torch

own = False


def _case(name, op, T, k, E, N, K, gather=False, pad=0, out="bf16", zipf=0.0, gated=False,
          keep=False):
    return dict(name=name, op=op, T=T, k=k, E=E, N=N, K=K, gather=gather, pad=pad, out=out,
                zipf=zipf, gated=gated, keep=keep)


def listed():
    return [
        # one user, one token: the weights of its eight experts
        _case("fp8_decode_1", "fp8", 1, 8, 32, 4096, 7168, gather=True),
        # eight users on a many-expert model: about one row for each expert
        _case("fp8_decode_8", "fp8", 8, 8, 128, 1536, 2048, gather=True),
        # sizes that are no multiple of a block or of 16 bytes
        _case("fp8_odd_777", "fp8", 777, 6, 24, 1283, 1921, pad=7, out="fp32", zipf=1.1),
        # gate and up projections of a prefill, unevenly used experts
        _case("fp8_prefill_4096", "fp8", 4096, 8, 32, 4096, 7168, gather=True, zipf=1.2),
        # the down projection of a prefill, from the gate and up projections
        _case("fp8_gated_4096", "fp8", 4096, 8, 32, 7168, 2048, out="fp32", gated=True, zipf=1.2),
        # one token through a layer of many small experts
        _case("swiglu_decode_1", "swiglu", 1, 8, 128, 768, 2048, gather=True),
        # a small decode batch on large experts
        _case("swiglu_decode_16", "swiglu", 16, 2, 8, 14336, 4096, gather=True),
        # odd sizes, rows cut out of a wider array
        _case("swiglu_odd_333", "swiglu", 333, 5, 20, 707, 1001, pad=3, keep=True, zipf=1.1),
        # a training step's forward pass
        _case("swiglu_train_4096", "swiglu", 4096, 8, 32, 2048, 7168, gather=True, keep=True,
              zipf=1.2),
        # a training micro-batch that gives each of many experts a few rows
        _case("backward_few_rows", "backward", 64, 8, 128, 2048, 768),
        # odd sizes
        _case("backward_odd_500", "backward", 500, 3, 6, 1003, 1411, pad=5, zipf=1.1),
        # a training step with few large experts
        _case("backward_train_4096", "backward", 4096, 2, 8, 4096, 14336),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi):
    """A matrix dimension: two of three are multiples of 128, 16 or 8."""
    v, m = _log_int(rng, lo, hi), rng.choice([1, 1, 8, 16, 128, 128])
    return max(m, v // m * m)


_MAX_FLOPS = {"fp8": 2.0 * 32768 * 4096 * 7168, "swiglu": 4.0 * 32768 * 2048 * 7168,
              "backward": 2.0 * 8192 * 4096 * 14336}
_MAX_BYTES = {"fp8": 1.6e9, "swiglu": 2.2e9, "backward": 1.9e9}


def draw(rng):
    while True:
        op = rng.choice(["fp8", "fp8", "fp8", "swiglu", "swiglu", "backward", "backward"])
        k = rng.randint(1, 8)
        E = _log_int(rng, max(k, 1), 160)
        T = _log_int(rng, 1, 16384)
        N, K = _size(rng, 24, 14336), _size(rng, 24, 14336)
        out, zipf = rng.choice(["bf16", "fp32"]), rng.choice([0.0, 0.0, 1.1])
        gather, pad = rng.random() < 0.5, rng.choice([0, 0, 8, 3])
        keep = rng.random() < 0.5
        if op == "fp8" and rng.random() < 0.4:
            c = _case(None, op, T, k, E, N, K, out=out, zipf=zipf, gated=True)
        elif op == "fp8":
            c = _case(None, op, T, k, E, N, K, gather=gather, pad=pad, out=out, zipf=zipf)
        elif op == "swiglu":
            c = _case(None, op, T, k, E, N, K, gather=gather, pad=pad, zipf=zipf, keep=keep)
        else:
            c = _case(None, op, T, k, E, N, K, pad=pad, zipf=zipf)
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
    ids = torch.topk(score, k, dim=1).indices
    flat = ids.reshape(-1)
    perm = torch.argsort(flat, stable=True)
    counts = torch.bincount(flat, minlength=E)
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = torch.cumsum(counts, 0)
    return dict(offsets=offsets, perm=perm.to(torch.int32), sizes=counts.tolist())


def _rows(n, width, pad, gen, scale=1.0):
    """bf16 [n, width] ~ N(0, scale), `pad` elements between the rows."""
    a = torch.empty((n, width + pad), dtype=torch.bfloat16, device="cuda")
    step = max(1, (1 << 27) // (width + pad))
    for i in range(0, n, step):
        m = min(step, n - i)
        a[i: i + m] = torch.randn((m, width + pad), device="cuda", generator=gen).mul_(scale)
    return a[:, :width]


def _blocks(n):
    return (n + 127) // 128


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + 29)
    op, T, k, E, N, K = (case[n] for n in ("op", "T", "k", "E", "N", "K"))
    R = T * k
    d = _route(case, gen)
    if op == "backward":
        d["dy"] = _rows(R, N, case["pad"], gen, 0.05)
        d["gu"] = _rows(R, 2 * K, 0, gen)
    elif case["gated"]:
        d["gu"] = _rows(R, 2 * K, 0, gen)
    else:
        d["x"] = _rows(T if case["gather"] else R, K, case["pad"], gen)
    wide = 2 * N if op == "swiglu" else N
    w = _rows(E * wide, K, 0, gen, 1.0 / math.sqrt(K)).view(E, wide, K)
    if op == "fp8":
        # a scale for each block of 128 x 128, as a server quantizes its weights at load
        d["w"] = torch.empty((E, N, K), dtype=torch.uint8, device="cuda")
        d["ws"] = torch.empty((E, _blocks(N), _blocks(K)), device="cuda")
        for e in range(E):
            a = w[e].float()
            s = _scale(_by_block(a, _blocks(N) * 128).abs().amax(dim=(1, 3)))
            d["ws"][e] = s
            full = s.repeat_interleave(128, 0).repeat_interleave(128, 1)[:N, :K]
            d["w"][e] = (a / full).to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        d["w"] = w
    return d


def _by_block(a, rows):
    """[n, K] -> [rows / 128, 128, K / 128, 128], zeros past the edges."""
    p = torch.zeros((rows, _blocks(a.shape[1]) * 128), dtype=a.dtype, device=a.device)
    p[: a.shape[0], : a.shape[1]] = a
    return p.view(rows // 128, 128, -1, 128)


def prepare(case, seed):
    d = _inputs(case, seed)
    d["case"] = case
    if not own:
        return d
    from paper_2509_17863_amd import eaas

    op, T, k, E, N, K = (case[n] for n in ("op", "T", "k", "E", "N", "K"))
    R = T * k

    def buf(*shape, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device="cuda")

    if op == "fp8":
        n = R if case["gated"] or not case["gather"] else T
        d["q"], d["s"] = buf(n, K, dtype=torch.uint8), buf(n, _blocks(K), dtype=torch.float32)
        d["out"] = buf(R, N, dtype=torch.float32 if case["out"] == "fp32" else torch.bfloat16)
        d["scratch"] = eaas.alloc_grouped_fp8_workspace(R, E, N, K)
    elif op == "swiglu":
        d["h"] = buf(R, N)
        d["gu"] = buf(R, 2 * N) if case["keep"] else None
        d["scratch"] = eaas.alloc_grouped_workspace(R, E, 2 * N, K)
    else:
        d["dgu"], d["h"] = buf(R, 2 * K), buf(R, K)
        d["scratch"] = eaas.alloc_grouped_workspace(R, E, N, K)
    return d


# ------------------------------------------------------------------ one pass
def run(d):
    return _run_own(d) if own else _run_plain(d)


def _run_own(d):
    from paper_2509_17863_amd import eaas

    c = d["case"]
    take = dict(perm=d["perm"], k=c["k"]) if c["gather"] else {}
    if c["op"] == "fp8":
        if c["gated"]:
            eaas.eaas_swiglu_fp8(d["gu"], d["q"], d["s"])
        else:
            eaas.eaas_quantize_blocks_fp8(d["x"], d["q"], d["s"])
        eaas.eaas_grouped_matmul_fp8(d["q"], d["s"], d["offsets"], d["w"], d["ws"], d["out"],
                                     d["scratch"], **take)
        return d["out"]
    if c["op"] == "swiglu":
        eaas.eaas_grouped_swiglu(d["x"], d["offsets"], d["w"], d["h"], d["scratch"], gu=d["gu"],
                                 **take)
        return {"h": d["h"], "gu": d["gu"]} if c["keep"] else d["h"]
    eaas.eaas_grouped_swiglu_backward(d["dy"], d["offsets"], d["w"], d["gu"], d["dgu"],
                                      d["scratch"], h=d["h"])
    return {"dgu": d["dgu"], "h": d["h"]}


def _scale(amax):
    s = amax / 448.0
    return torch.where(s > 0, s, torch.ones_like(s))


def _dequantized(a):
    """fp32 [n, K] -> the values that its e4m3 codes stand for, a scale for each 128
    columns of a row."""
    n, K = a.shape
    p = torch.zeros((n, _blocks(K) * 128), device=a.device)
    p[:, :K] = a
    p = p.view(n, -1, 128)
    s = _scale(p.abs().amax(dim=2, keepdim=True))
    return ((p / s).to(torch.float8_e4m3fn).float() * s).view(n, -1)[:, :K]


def _groups(d):
    r = 0
    for e, n in enumerate(d["sizes"]):
        if n:
            yield e, slice(r, r + n)
        r += n


def _token_rows(d, x):
    if d["case"]["gather"]:
        return x[(d["perm"] // d["case"]["k"]).long()]
    return x


def _run_plain(d):
    c = d["case"]
    op, R, N, K = c["op"], c["T"] * c["k"], c["N"], c["K"]
    bf16 = torch.bfloat16
    if op == "fp8":
        if c["gated"]:
            # (in 64 bits until it is rounded to 32: next to the middle between two codes
            # an error in the last place costs a whole step)
            g, u = d["gu"].double().split(K, dim=1)
            x = _dequantized((g / (1.0 + torch.exp(-g)) * u).float())
        else:
            x = _token_rows(d, _dequantized(d["x"].float()))
        y = torch.empty((R, N), dtype=torch.float32 if c["out"] == "fp32" else bf16,
                        device=x.device)
        for e, r in _groups(d):
            s = d["ws"][e].repeat_interleave(128, 0).repeat_interleave(128, 1)[:N, :K]
            w = d["w"][e].view(torch.float8_e4m3fn).float() * s
            y[r] = (x[r] @ w.t()).to(y.dtype)
        return y
    if op == "swiglu":
        x = _token_rows(d, d["x"]).float()
        h = torch.empty((R, N), dtype=bf16, device=x.device)
        gu = torch.empty((R, 2 * N), dtype=bf16, device=x.device) if c["keep"] else None
        for e, r in _groups(d):
            p = x[r] @ d["w"][e].float().t()
            g, u = p.split(N, dim=1)
            h[r] = (g / (1.0 + torch.exp(-g)) * u).to(bf16)
            if c["keep"]:
                gu[r] = p.to(bf16)
        return {"h": h, "gu": gu} if c["keep"] else h
    dy = d["dy"].float()
    dgu = torch.empty((R, 2 * K), dtype=bf16, device=dy.device)
    h = torch.empty((R, K), dtype=bf16, device=dy.device)
    for e, r in _groups(d):
        dh = dy[r] @ d["w"][e].float()
        g, u = d["gu"][r].float().split(K, dim=1)
        t = 1.0 / (1.0 + torch.exp(-g))
        dgu[r, :K] = (dh * u * t * (1.0 + g * (1.0 - t))).to(bf16)
        dgu[r, K:] = (dh * g * t).to(bf16)
        h[r] = (g * t * u).to(bf16)
    return {"dgu": dgu, "h": h}


# ------------------------------------------------------------------ measures
def work(case):
    """Each input read once (weights of the experts that get a row, token rows that
    are gathered once), each output written once; the products' operations."""
    op, T, k, E, N, K = (case[n] for n in ("op", "T", "k", "E", "N", "K"))
    R = T * k
    used = sum(1.0 - (1.0 - min(1.0, k * p)) ** T for p in _popularity(case))
    rows = T if case["gather"] else R
    ids = 4.0 * R if case["gather"] else 0.0
    if op == "fp8":
        a = 4.0 * R * K if case["gated"] else 2.0 * rows * K
        out = 4 if case["out"] == "fp32" else 2
        return {"bytes": a + used * (N * K + 4.0 * _blocks(N) * _blocks(K)) + R * N * out + ids,
                "flops": 2.0 * R * N * K}
    if op == "swiglu":
        return {"bytes": (2.0 * rows * K + used * 4.0 * N * K + (6.0 if case["keep"] else 2.0) * R * N
                          + ids), "flops": 4.0 * R * N * K}
    return {"bytes": 2.0 * R * N + used * 2.0 * N * K + 10.0 * R * K, "flops": 2.0 * R * N * K}


# ------------------------------------------------------------------ 64 bits
def _e4m3(t):
    """The nearest of the values +-m 2^(e-3), m in 8..15, e in -6..8 (m in 0..7 at
    e = -6), ties to even m, at most 448."""
    exponent = torch.frexp(t).exponent.double() - 1.0
    step = torch.exp2(exponent.clamp(min=-6.0) - 3.0)
    return ((t / step).round() * step).clamp(-448.0, 448.0)


def _exact_fp8(d, case):
    N, K, E, k = (case[n] for n in ("N", "K", "E", "k"))
    start = d["offsets"].tolist()
    R = case["T"] * k
    src = torch.div(d["perm"].long(), k, rounding_mode="floor") if case["gather"] else (
        torch.arange(R, device="cuda"))
    code = torch.arange(256, device="cuda")
    m, ex = (code & 7).double(), ((code >> 3) & 15).double()
    value = torch.where(ex > 0, (8.0 + m) * torch.exp2(ex - 10.0), m * 2.0 ** -9)
    value = torch.where(code >= 128, -value, value)
    y = torch.zeros((R, N), dtype=torch.float64, device="cuda")
    for e in range(E):
        a, b = start[e], start[e + 1]
        if a == b:
            continue
        if case["gated"]:
            gu = d["gu"][a:b].double()
            v = (gu[:, :K] * torch.sigmoid(gu[:, :K]) * gu[:, K:]).float()
        else:
            v = d["x"][src[a:b]].float()
        for j in range(0, K, 128):
            p = v[:, j: j + 128]
            top = p.abs().max(dim=1, keepdim=True).values
            # (scale and quotient are rounded to 32 bits by definition)
            s = top / 448
            s = torch.where(s > 0, s, torch.ones_like(s))
            q = _e4m3((p / s).double())
            w = value[d["w"][e, :, j: j + 128].long()]
            ws = d["ws"][e, :, j // 128].double()
            cols = torch.arange(N, device="cuda") // 128
            y[a:b] += torch.mm(q, w.t()) * s.double() * ws[cols]
    return y


def exact(case, seed):
    """The definitions in 64 bits.  (The 8-bit codes are those of the definition:
    quotient and scale rounded to 32 bits, then to the nearest code.)"""
    d = _inputs(case, seed)
    if case["op"] == "fp8":
        return _exact_fp8(d, case)
    T, k, E, N, K = (case[n] for n in ("T", "k", "E", "N", "K"))
    R, f64 = T * k, torch.float64
    start = d["offsets"].tolist()
    if case["op"] == "swiglu":
        src = torch.div(d["perm"].long(), k, rounding_mode="floor") if case["gather"] else (
            torch.arange(R, device="cuda"))
        p = torch.zeros((R, 2 * N), dtype=f64, device="cuda")
        for e in range(E):
            a, b = start[e], start[e + 1]
            p[a:b] = torch.mm(d["x"][src[a:b]].double(), d["w"][e].double().t())
        h = p[:, :N] * torch.sigmoid(p[:, :N]) * p[:, N:]
        return {"h": h, "gu": p} if case["keep"] else h
    dgu = torch.zeros((R, 2 * K), dtype=f64, device="cuda")
    h = torch.zeros((R, K), dtype=f64, device="cuda")
    for e in range(E):
        a, b = start[e], start[e + 1]
        dh = torch.mm(d["dy"][a:b].double(), d["w"][e].double())
        gate, up = d["gu"][a:b, :K].double(), d["gu"][a:b, K:].double()
        sig = torch.sigmoid(gate)
        dgu[a:b, :K] = dh * up * (sig + gate * sig * (1 - sig))
        dgu[a:b, K:] = dh * (gate * sig)
        h[a:b] = gate * sig * up
    return {"dgu": dgu, "h": h}
