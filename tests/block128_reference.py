"""Plain 64-bit forms of the block-scaled FP8 operators and of the routing among experts (torch and numpy on whatever device the inputs are on)."""
import numpy as np
import torch

TOP = {"e4m3": 448.0, "e5m2": 57344.0}
F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


def blocks(n):
    return (n + 127) // 128


def code_values(elem):
    """fp64 values of the 256 codes."""
    m, bias = (3, 7) if elem == "e4m3" else (2, 15)
    out = []
    for c in range(256):
        e, f = (c & 127) >> m, c & ((1 << m) - 1)
        v = (1 + f / 2.0 ** m) * 2.0 ** (e - bias) if e else f / 2.0 ** m * 2.0 ** (1 - bias)
        if elem == "e4m3" and c & 127 == 127:
            v = float("nan")
        if elem == "e5m2" and e == 31:
            v = float("inf") if f == 0 else float("nan")
        out.append(-v if c & 128 else v)
    return torch.tensor(out, dtype=torch.float64)


def values(codes, scales, block_rows, elem):
    """What the codes [rows, K] and scales stand for, fp64."""
    rows, K = codes.shape
    v = code_values(elem).to(codes.device)[codes.long()]
    r = torch.arange(rows, device=codes.device) // block_rows
    k = torch.arange(K, device=codes.device) // 128
    return v * scales.double()[r[:, None], k[None, :]]


def quantize(x, block_rows, elem):
    """(codes, scales) of bf16 x [rows, K], from the definition: among all codes the nearest to x V / top, of two equally near the even one."""
    rows, K = x.shape
    V = TOP[elem]
    grid = code_values(elem)[:128].clone()
    grid[~torch.isfinite(grid)] = float("inf")
    grid = grid.numpy()
    limit = int(np.isfinite(grid).sum()) - 1
    codes = np.zeros((rows, K), np.uint8)
    scales = np.zeros((-(-rows // block_rows), blocks(K)), np.float32)
    xs = x.cpu().double().numpy()
    for i in range(scales.shape[0]):
        for g in range(scales.shape[1]):
            part = xs[i * block_rows:(i + 1) * block_rows, g * 128:(g + 1) * 128]
            if not np.isfinite(part).all():
                scales[i, g] = np.nan
                continue
            top = np.abs(part).max()
            if top == 0:
                scales[i, g] = 1.0
                q = np.zeros_like(part)
            elif top < V * 2.0 ** -126:
                scales[i, g] = 2.0 ** -126
                q = np.abs(part) * 2.0 ** 126
            else:
                scales[i, g] = np.float32(top / V)
                q = np.abs(part) * V / top  # (a quotient midway between two codes has few bits: it is exact)
            up = np.minimum(np.searchsorted(grid[:limit + 1], q), limit)
            down = np.maximum(up - 1, 0)
            a, b = q - grid[down], grid[up] - q
            c = np.where(a < b, down, np.where(b < a, up, np.where(down % 2 == 0, down, up)))
            c = np.where(grid[up] == q, up, c)
            codes[i * block_rows:(i + 1) * block_rows, g * 128:(g + 1) * 128] = c + 128 * np.signbit(part)
    return torch.from_numpy(codes), torch.from_numpy(scales)


def product(a, b):
    """C = A B^T of fp64 operands, and the sum of the products' magnitudes."""
    bt = b.T.contiguous()
    return a @ bt, a.abs() @ bt.abs()


def product_bound(exact, size, K, bf16):
    """How far the kernels' C may be off: a product loses less than 2^-14 of the largest of its group of 16 (15 of them: below 2^-10 of the sum of
    magnitudes, 2^-14 of it left over), the additions and the two scales' product 2^-23 each at most (ten, and two a block); bf16 rounds by 2^-8 at most."""
    off = size * (2.0 ** -10 + blocks(K) * 2.0 ** -21)
    return off + (exact.abs() + off) * 2.0 ** -8 if bf16 else off


def plan(logits, k, scoring, bias, renormalize, scale=1.0, num_tokens=None):
    """(experts, weights fp64, row_offsets, rows, tokens) as numpy arrays, token by token."""
    x = logits.detach().cpu().double().numpy()
    T, E = x.shape
    n = T if num_tokens is None else min(max(num_tokens, 0), T)
    experts, weights = np.full((T, k), -1, np.int32), np.zeros((T, k))
    with np.errstate(all="ignore"):
        for t in range(n):
            s = np.where(x[t] >= 0, 1 / (1 + np.exp(-np.abs(x[t]))), np.exp(-np.abs(x[t])) / (1 + np.exp(-np.abs(x[t]))))
            by = x[t].copy() if bias is None else s + bias.cpu().double().numpy()
            by[x[t] == -np.inf] = -np.inf
            if scoring == "softmax":
                p = np.exp(x[t] - (np.nan if np.isnan(x[t]).any() else x[t].max()))
                p[x[t] == -np.inf] = 0
            else:
                p = s
            order = sorted((e for e in range(E) if by[e] != -np.inf), key=lambda e: (not np.isnan(by[e]), 0 if np.isnan(by[e]) else -by[e], e))[:k]
            w = p[order]
            if renormalize:
                w = w / w.sum()
            elif scoring == "softmax":
                w = w / p.sum()
            experts[t, :len(order)], weights[t, :len(order)] = order, w * scale
    rows, tokens = np.full((T, k), -1, np.int32), np.full(T * k, -1, np.int32)
    offsets, at = np.zeros(E + 1, np.int64), 0
    for e in range(E):
        for t, j in np.argwhere(experts == e):
            rows[t, j], tokens[at] = at, t
            at += 1
        offsets[e + 1] = at
    return experts, weights, offsets, rows, tokens
