"""Linear layers in 8-bit floating point with an fp32 scale for each block of 128, and the routing of tokens among experts, as cases
that can be timed and compared.

A layer's weights are quantized once, with a scale for each block of 128 x 128 (`mx_quantize_block128`, `block_rows=128`), its activations
at every step, with one for each 1 x 128 (`block_rows=1`); the product applies both (`mx_gemm_block128`).  An expert layer plans which expert
takes which token (`mx_moe_plan`), multiplies every expert's rows with that expert's weight, taking them from the tokens where they lie
(`mx_gemm_block128_grouped`), and adds the results up token by token (`mx_moe_combine`).  Sizes follow the FFN layers and the expert layer that
the benchmark runs (4096 -> 14336, 8192; 32 experts of 2880 x 2880, 4 a token, skewed load); others are generic.

kinds (each a range that `draw` samples):
  quant    rows of activations, or weights, quantized
  gemm     a product: one row to a batch of prompts
  grouped  an expert layer's product, rows through an index or in the experts' order already
  plan     the experts of every token, their weights, and places in the experts' order
  combine  the experts' rows added up

Everything that is not under `own` is the plain form: elementary torch operations on codes (uint8, the bits of torch.float8_e4m3fn or
torch.float8_e5m2) and scales [rows, K / 128] or [rows / 128, K / 128], cut off at the edges.
"""
from __future__ import annotations

import math

import torch

own = False

F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
TOP = {"e4m3": 448.0, "e5m2": 57344.0}
OUT = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # a decode step's activations: 17 requests
        dict(name="quant_rows_17", kind="quant", rows=17, K=4096, block_rows=1, elem="e4m3"),
        # activations of a batch of prompts
        dict(name="quant_rows_8192", kind="quant", rows=8192, K=8192, block_rows=1, elem="e4m3"),
        # a weight, quantized when it is loaded
        dict(name="quant_weight", kind="quant", rows=14336, K=4096, block_rows=128, elem="e4m3"),
        # one request decoding: latency, the weight read once
        dict(name="gemm_one_row", kind="gemm", M=1, N=4096, K=4096, a="e4m3", b="e4m3", out="bf16"),
        # a prompt of odd length against a weight of odd height, K ending inside a block
        dict(name="gemm_ragged", kind="gemm", M=1777, N=5001, K=2880, a="e5m2", b="e4m3", out="bf16"),
        # a batch of prompts through an FFN up-projection
        dict(name="gemm_prompts", kind="gemm", M=4096, N=14336, K=4096, a="e4m3", b="e4m3", out="bf16"),
        # 64 requests decoding through an expert layer: a few rows for every expert
        dict(name="grouped_decode", kind="grouped", tokens=64, experts=32, top_k=4, N=2880, K=2880, index=True, out="bf16"),
        # prompts through the same layer, skewed load
        dict(name="grouped_prompts", kind="grouped", tokens=8192, experts=32, top_k=4, N=2880, K=2880, index=True, out="bf16"),
        # the router of those 64 requests
        dict(name="plan_64", kind="plan", tokens=64, experts=32, top_k=4, logits="bf16", scoring="softmax", bias=False, renormalize=True),
        # many small experts, chosen under a bias that balances their load
        dict(name="plan_8192", kind="plan", tokens=8192, experts=128, top_k=8, logits="f32", scoring="sigmoid", bias=True, renormalize=True),
        dict(name="combine_64", kind="combine", tokens=64, top_k=4, N=2880, add=False, out="bf16"),
        # the experts' rows of prompts beside what every token went through
        dict(name="combine_8192", kind="combine", tokens=8192, top_k=4, N=2880, add=True, out="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["quant", "gemm", "gemm", "gemm", "grouped", "grouped", "plan", "plan", "combine"])
    elem = lambda: rng.choice(["e4m3", "e4m3", "e4m3", "e5m2"])  # noqa: E731
    if kind == "quant":
        return dict(kind=kind, rows=_log(rng, 1, 8192), K=16 * _log(rng, 8, 512), block_rows=rng.choice([1, 1, 128]), elem=elem())
    if kind == "gemm":
        c = dict(kind=kind, M=_log(rng, 1, 4096), N=_log(rng, 256, 14336), K=16 * _log(rng, 16, 512), a=elem(), b=elem(), out="bf16")
        while c["M"] * c["N"] * c["K"] > 4096 * 14336 * 4096:
            c["N"] = c["N"] * 3 // 4
        return c
    if kind == "grouped":
        c = dict(kind=kind, tokens=_log(rng, 1, 8192), experts=rng.choice([4, 8, 16, 32, 64, 128]), top_k=rng.choice([1, 2, 4]), N=_log(rng, 300, 4096),
                 K=16 * _log(rng, 16, 256), index=rng.random() < 0.5, out="bf16")
        while c["experts"] * c["N"] * c["K"] > 32 * 2880 * 2880:
            c["experts"] //= 2
        c["top_k"] = min(c["top_k"], c["experts"])
        while c["tokens"] * c["top_k"] * c["N"] * c["K"] > 32768 * 2880 * 2880:
            c["tokens"] = c["tokens"] * 3 // 4
        return c
    if kind == "plan":
        experts = rng.choice([4, 8, 16, 32, 60, 64, 128, 160, 256])
        scoring = rng.choice(["softmax", "sigmoid"])
        return dict(kind=kind, tokens=_log(rng, 1, 16384), experts=experts, top_k=rng.randint(1, min(8, experts)), logits=rng.choice(["bf16", "f32"]),
                    scoring=scoring, bias=scoring == "sigmoid" and rng.random() < 0.5, renormalize=rng.random() < 0.7)
    return dict(kind=kind, tokens=_log(rng, 1, 8192), top_k=rng.randint(1, 8), N=_log(rng, 256, 4096), add=rng.random() < 0.5, out="bf16")


def _blocks(n):
    return (n + 127) // 128


def work(case):
    kind = case["kind"]
    if kind == "quant":
        rows, K = case["rows"], case["K"]
        return dict(bytes=3 * rows * K + 4 * _blocks(K) * (rows if case["block_rows"] == 1 else _blocks(rows)), flops=0)
    if kind == "plan":
        T, E, k = case["tokens"], case["experts"], case["top_k"]
        return dict(bytes=T * E * (2 if case["logits"] == "bf16" else 4) + 16 * T * k + 8 * (E + 1) + (4 * E if case["bias"] else 0), flops=0)
    if kind == "combine":
        T, k, N = case["tokens"], case["top_k"], case["N"]
        return dict(bytes=2 * T * N * (k + 1 + int(case["add"])) + 8 * T * k, flops=0)
    N, K = case["N"], case["K"]
    if kind == "gemm":
        rows, weights, tokens = case["M"], 1, case["M"]
    else:
        rows = case["tokens"] * case["top_k"]
        # (with few tokens an expert may have no rows; then its weight need not be read)
        weights, tokens = min(case["experts"], rows), case["tokens"] if case["index"] else rows
    return dict(bytes=tokens * (K + 4 * _blocks(K)) + weights * (N * K + 4 * _blocks(N) * _blocks(K)) + 2 * rows * N, flops=2 * rows * N * K)


# ---- quantizing, plain --------------------------------------------------------------------------------------
def _tops(x, block_rows):
    """Largest magnitudes of the blocks of x [..., rows, K]: [..., rows / block_rows, K / 128]."""
    rows, K = x.shape[-2:]
    a = torch.nn.functional.pad(x.abs(), (0, -K % 128, 0, -rows % block_rows))
    return a.unflatten(-1, (-1, 128)).amax(-1).unflatten(-2, (-1, block_rows)).amax(-2)


def _spread(scales, block_rows, rows, K):
    """Scales of blocks, an element each."""
    s = scales.repeat_interleave(128, -1)[..., :K]
    return s if block_rows == 1 else s.repeat_interleave(block_rows, -2)[..., :rows, :]


def _quantize(x, block_rows, elem):
    """Codes (uint8) and scales of bf16 x [..., rows, K]: the codes nearest to x * largest code / largest magnitude.  Quotients are taken in
    64 bits, where one that lies midway between two codes is exact."""
    top = _tops(x, block_rows).double()
    top = torch.where(top > 0, torch.clamp(top, min=TOP[elem] * 2.0 ** -126), TOP[elem])
    q = x.double() * TOP[elem] / _spread(top, block_rows, *x.shape[-2:])
    return q.float().to(F8[elem]).view(torch.uint8), (top / TOP[elem]).float()


def _values(codes, scales, block_rows, elem):
    return codes.view(F8[elem]).float() * _spread(scales, block_rows, *codes.shape[-2:])


# ---- inputs -------------------------------------------------------------------------------------------------
def _activations(gen, rows, K):
    """What comes out of a norm: N(0, 1), a few channels larger, rows of different size."""
    x = torch.randn((rows, K), generator=gen, device="cuda")
    size = torch.ones(K, device="cuda")
    size[torch.randperm(K, generator=gen, device="cuda")[:max(1, K // 100)]] = 20.0
    x *= size
    x *= torch.exp(0.5 * torch.randn((rows, 1), generator=gen, device="cuda"))
    return x.to(torch.bfloat16)


def _weights(gen, rows, K):
    return (0.02 * torch.randn((rows, K), generator=gen, device="cuda")).to(torch.bfloat16)


def _routing(gen, tokens, experts, top_k):
    """Distinct experts of every token, P(e) ~ (e + 1)^-1.1, as the experts' rows: counts and the token of every row."""
    score = -1.1 * torch.log(torch.arange(1, experts + 1, device="cuda").float()) - torch.log(
        -torch.log(torch.rand((tokens, experts), generator=gen, device="cuda").clamp(1e-9, 1 - 1e-6)))
    chosen = score.topk(top_k, 1).indices.flatten()
    order = torch.sort(chosen, stable=True).indices
    return torch.bincount(chosen, minlength=experts), torch.div(order, top_k, rounding_mode="floor").int(), order


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind = case["kind"]
    s = dict(case)
    if kind == "quant":
        rows, K, br = case["rows"], case["K"], case["block_rows"]
        s.update(x=_activations(gen, rows, K) if br == 1 else _weights(gen, rows, K), codes=torch.zeros((rows, K), dtype=torch.uint8, device="cuda"),
                 scales=torch.zeros(((rows + br - 1) // br, _blocks(K)), device="cuda"))
    elif kind == "gemm":
        s.update(zip(("a_codes", "a_scales"), _quantize(_activations(gen, case["M"], case["K"]), 1, case["a"])))
        s.update(zip(("b_codes", "b_scales"), _quantize(_weights(gen, case["N"], case["K"]), 128, case["b"])))
        s.update(C=torch.zeros((case["M"], case["N"]), dtype=OUT[case["out"]], device="cuda"))
    elif kind == "grouped":
        E, N, K, T = case["experts"], case["N"], case["K"], case["tokens"]
        counts, token_of_row, _ = _routing(gen, T, E, case["top_k"])
        x = _activations(gen, T, K)
        codes, scales = _quantize(x if case["index"] else x[token_of_row.long()], 1, "e4m3")
        b = [_quantize(_weights(gen, N, K), 128, "e4m3") for _ in range(E)]
        rows = T * case["top_k"]
        s.update(a_codes=codes, a_scales=scales, b_codes=torch.cat([c for c, _ in b]), b_scales=torch.cat([c for _, c in b]),
                 a_rows=token_of_row if case["index"] else None, row_offsets=torch.nn.functional.pad(counts.cumsum(0), (1, 0)),
                 most=int(counts.max()), C=torch.zeros((rows, N), dtype=OUT[case["out"]], device="cuda"))
    elif kind == "plan":
        T, E, k = case["tokens"], case["experts"], case["top_k"]
        logits = 1.5 * torch.randn((T, E), generator=gen, device="cuda") + 0.7 * torch.randn(E, generator=gen, device="cuda")
        i32 = dict(dtype=torch.int32, device="cuda")
        s.update(logits=logits.to(OUT[case["logits"]]), bias=0.1 * torch.randn(E, generator=gen, device="cuda") if case["bias"] else None,
                 outputs=dict(experts=torch.zeros((T, k), **i32), weights=torch.zeros((T, k), device="cuda"),
                              row_offsets=torch.zeros(E + 1, dtype=torch.int64, device="cuda"), rows=torch.zeros((T, k), **i32),
                              tokens=torch.zeros(T * k, **i32)))
    else:
        T, k, N = case["tokens"], case["top_k"], case["N"]
        _, _, order = _routing(gen, T, max(32, k), k)
        rows = torch.empty_like(order)
        rows[order] = torch.arange(T * k, device="cuda")
        weights = torch.rand((T, k), generator=gen, device="cuda") + 0.1
        s.update(y=_activations(gen, T * k, N), rows=rows.view(T, k).int(), weights=weights / weights.sum(1, keepdim=True),
                 add=_activations(gen, T, N) if case["add"] else None, result=torch.zeros((T, N), dtype=OUT[case["out"]], device="cuda"))
    return s


# ---- one pass -----------------------------------------------------------------------------------------------
def run(s):
    if own:
        return _own(s)
    kind = s["kind"]
    if kind == "quant":
        codes, scales = _quantize(s["x"], s["block_rows"], s["elem"])
        return codes.view(F8[s["elem"]]), scales
    if kind == "gemm":
        a, b = _values(s["a_codes"], s["a_scales"], 1, s["a"]), _values(s["b_codes"], s["b_scales"], 128, s["b"])
        return torch.matmul(a, b.T.contiguous()).to(OUT[s["out"]])
    if kind == "grouped":
        return _grouped(s)
    if kind == "plan":
        return _plan(s)
    out = (s["weights"][..., None] * s["y"].float()[s["rows"].long()]).sum(1)
    return (out + s["add"].float() if s["add"] is not None else out).to(OUT[s["out"]])


def _own(s):
    import paper_2603_08713_amd as mx

    kind = s["kind"]
    if kind == "quant":
        mx.mx_quantize_block128(s["x"], s["elem"], s["block_rows"], codes=s["codes"], scales=s["scales"])
        return s["codes"].view(F8[s["elem"]]), s["scales"]
    if kind == "gemm":
        return mx.mx_gemm_block128(s["a"], s["a_codes"], s["a_scales"], s["b"], s["b_codes"], s["b_scales"], s["out"], out=s["C"])
    if kind == "grouped":
        return mx.mx_gemm_block128_grouped("e4m3", s["a_codes"], s["a_scales"], "e4m3", s["b_codes"], s["b_scales"], s["row_offsets"], s["N"], s["out"],
                                           a_rows=s["a_rows"], out=s["C"])
    if kind == "plan":
        mx.mx_moe_plan(s["logits"], s["top_k"], s["scoring"], s["bias"], s["renormalize"], **s["outputs"])
        return s["outputs"]
    return mx.mx_moe_combine(s["y"], s["rows"], s["weights"], s["add"], s["out"], out=s["result"])


def _grouped(s):
    """All experts padded to the one with the most rows."""
    E, N, K, offsets = s["experts"], s["N"], s["K"], s["row_offsets"]
    w = _values(s["b_codes"].view(E, N, K), s["b_scales"].view(E, _blocks(N), _blocks(K)), 128, "e4m3").transpose(1, 2).contiguous()
    x = _values(s["a_codes"], s["a_scales"], 1, "e4m3")
    i = torch.arange(s["most"], device=x.device)
    there = i[None, :] < (offsets[1:] - offsets[:-1])[:, None]
    row = (offsets[:-1, None] + i).clamp_max(s["C"].shape[0] - 1)
    a = x[row if s["a_rows"] is None else s["a_rows"].long()[row]]
    return torch.matmul(a, w)[there].to(OUT[s["out"]])


def _plan(s):
    """Choices under a bias are made in 64 bits: two experts may be next to each other."""
    T, E, k = s["tokens"], s["experts"], s["top_k"]
    logits = s["logits"].float()
    score = logits if s["bias"] is None else 1.0 / (1.0 + torch.exp(-logits.double())) + s["bias"].double()
    chosen = torch.sort(score, dim=1, descending=True, stable=True).indices[:, :k]
    if s["scoring"] == "softmax":
        weights = torch.exp(logits - logits.amax(1, keepdim=True))
        weights = weights / weights.sum(1, keepdim=True)
    else:
        weights = 1.0 / (1.0 + torch.exp(-logits))
    weights = weights.gather(1, chosen)
    if s["renormalize"]:
        weights = weights / weights.sum(1, keepdim=True)
    flat = chosen.flatten()
    order = torch.sort(flat, stable=True).indices
    rows = torch.empty_like(order)
    rows[order] = torch.arange(T * k, device=order.device)
    counts = (flat[:, None] == torch.arange(E, device=order.device)).sum(0)
    return dict(experts=chosen.int(), weights=weights, row_offsets=torch.nn.functional.pad(counts.cumsum(0), (1, 0)), rows=rows.view(T, k).int(),
                tokens=torch.div(order, k, rounding_mode="floor").int())


# ---- in 64 bits, from the definitions ---------------------------------------------------------------------------
def _code_table(elem):
    """What the 256 codes stand for, from their bits."""
    mantissa, bias = (3, 7) if elem == "e4m3" else (2, 15)
    c = torch.arange(256, device="cuda", dtype=torch.int64)
    e, m = (c & 127) >> mantissa, (c & ((1 << mantissa) - 1)).double()
    size = torch.where(e > 0, (1 + m / 2 ** mantissa) * torch.exp2((e - bias).double()), m / 2 ** mantissa * 2.0 ** (1 - bias))
    return torch.where(c > 127, -size, size)


def _exact_quantized(x, block_rows, elem):
    """The point of the format's grid that is nearest to x over the unrounded scale, block by block of columns."""
    mantissa, lowest = (3, -6) if elem == "e4m3" else (2, -14)
    rows, K = x.shape
    groups = torch.div(torch.arange(rows, device="cuda"), block_rows, rounding_mode="floor")
    values, scales = [], []
    for k in range(0, K, 128):
        part = x[:, k:k + 128].double()
        top = torch.zeros((rows + block_rows - 1) // block_rows, dtype=torch.float64, device="cuda").scatter_reduce(0, groups, part.abs().amax(1), "amax")
        top = torch.where(top > 0, top.clamp_min(TOP[elem] * 2.0 ** -126), torch.full_like(top, TOP[elem]))
        q = part * TOP[elem] / top[groups][:, None]
        _, e = torch.frexp(q)  # |q| = m 2^e, m in [0.5, 1)
        step = torch.exp2(((e - 1).clamp_min(lowest) - mantissa).double())
        values.append(torch.round(q / step) * step)  # (halves to even)
        scales.append(top / TOP[elem])
    return torch.cat(values, 1), torch.stack(scales, 1)


def _exact_product(a_codes, a_scales, a, b_codes, b_scales, b):
    """Block after block of K: the codes' product, then the scales."""
    M, K = a_codes.shape
    N = b_codes.shape[0]
    column = torch.div(torch.arange(N, device="cuda"), 128, rounding_mode="floor")
    ta, tb = _code_table(a), _code_table(b)
    out = torch.zeros((M, N), dtype=torch.float64, device="cuda")
    for g in range(_blocks(K)):
        k = slice(128 * g, min(K, 128 * g + 128))
        left = ta[a_codes[:, k].int()] * a_scales[:, g].double()[:, None]
        right = tb[b_codes[:, k].int()].T.contiguous() * b_scales[column, g].double()
        out.addmm_(left, right)
    return out


def exact(case, seed):
    kind = case["kind"]
    s = prepare(case, seed)
    if kind == "quant":
        return _exact_quantized(s["x"], case["block_rows"], case["elem"])
    if kind == "gemm":
        return _exact_product(s["a_codes"], s["a_scales"], case["a"], s["b_codes"], s["b_scales"], case["b"])
    if kind == "grouped":
        N, tiles = case["N"], _blocks(case["N"])
        at = s["row_offsets"].tolist()
        out = torch.zeros(s["C"].shape, dtype=torch.float64, device="cuda")
        for e in range(case["experts"]):
            if at[e] < at[e + 1]:
                rows = torch.arange(at[e], at[e + 1], device="cuda")
                rows = rows if s["a_rows"] is None else s["a_rows"][rows].long()
                out[at[e]:at[e + 1]] = _exact_product(s["a_codes"][rows], s["a_scales"][rows], "e4m3", s["b_codes"][e * N:(e + 1) * N],
                                                      s["b_scales"][e * tiles:(e + 1) * tiles], "e4m3")
        return out
    if kind == "combine":
        out = s["add"].double() if s["add"] is not None else torch.zeros(s["result"].shape, dtype=torch.float64, device="cuda")
        for j in range(case["top_k"]):
            out = out + s["weights"][:, j:j + 1].double() * s["y"][s["rows"][:, j].long()].double()
        return out
    x = s["logits"].double()
    by = x if s["bias"] is None else torch.sigmoid(x) + s["bias"].double()
    chosen = []
    for _ in range(case["top_k"]):  # the largest that is left, of equal ones the first
        e = (by == by.amax(1, keepdim=True)).int().argmax(1, keepdim=True)
        by = by.scatter(1, e, float("-inf"))
        chosen.append(e)
    chosen = torch.cat(chosen, 1)
    w = (torch.softmax(x, 1) if case["scoring"] == "softmax" else torch.sigmoid(x)).gather(1, chosen)
    if case["renormalize"]:
        w = w / w.sum(1, keepdim=True)
    return dict(experts=None, weights=w, row_offsets=None, rows=None, tokens=None)
