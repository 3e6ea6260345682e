"""Plain 64-bit implementations behind the tests of the paged MXFP4 cache: rows go through the C oracle, the rest is written out here on
the CPU from the definitions in include/mx4.h."""
import numpy as np
import torch

GRID = np.array([0, .5, 1, 1.5, 2, 3, 4, 6], np.float64)
STEP = 2.0 ** -8  # half a step of bf16, relative


def bits(x):
    return x.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def quantized_rows(oracle, x, rule, mbs):
    """codes [T, H, D/2], scales [T, H, D/32], words [T, H, W] or None of x [T, H, D] (bf16)."""
    T, H, D = x.shape
    c, s, w = oracle.quantize(bits(x).reshape(T * H, D), rule, mbs=mbs)
    return c.reshape(T, H, D // 2), s.reshape(T, H, D // 32), None if not mbs else w.reshape(T, H, -1)


def cached_rows(cache, is_key, slots):
    """The same three arrays of the rows at `slots`, taken out of a cache's arrays byte by byte."""
    codes, scales, words = (None if a is None else a.cpu().numpy() for a in cache)
    H, blocks, page = scales.shape[1:]
    P, at = np.asarray(slots) // page, np.asarray(slots) % page
    if is_key:
        c = codes[P, :, :, at, :].reshape(len(P), H, blocks * 16)
    else:
        c = codes[P, :, at // 4, :, at % 4, :].reshape(len(P), H, blocks * 16)
    return c, scales[P, :, :, at], None if words is None else words[P, :, :, at]


def values(codes, scales, words):
    """float64 [..., D]."""
    both = np.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[:-1] + (2 * codes.shape[-1],))
    x = GRID[both & 7] * np.where(both & 8, -1.0, 1.0)
    D = x.shape[-1]
    e = np.repeat(scales, 32, -1).astype(np.int64)
    x = np.where(e == 255, np.nan, np.ldexp(x, e - 127))
    if words is not None:
        x = x / (1.0 + np.repeat(words, 128, -1)[..., :D].astype(np.float64) / 256.0)
    return x


def norm_rope(x, positions, cos_sin, weight, eps, style):
    """float64 [T, H, D]."""
    y = x.cpu().double().numpy()
    if weight is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * weight.cpu().double().numpy()
    if cos_sin is None:
        return y
    R = cos_sin.shape[1]
    table = cos_sin.cpu().double().numpy()
    p = positions.cpu().numpy()
    angle = table[np.clip(p, 0, len(table) - 1)][:, None, :]
    angle = np.where((p < len(table))[:, None, None], angle, np.nan)
    c, s = angle[..., :R // 2], angle[..., R // 2:]
    out = y.copy()
    i, j = (np.arange(R // 2), np.arange(R // 2, R)) if style == "half" else (np.arange(0, R, 2), np.arange(1, R, 2))
    out[..., i] = y[..., i] * c - y[..., j] * s
    out[..., j] = y[..., j] * c + y[..., i] * s
    return out


def to_bf16(x):
    """float64 -> bf16 through fp32, as the definition says."""
    return torch.from_numpy(x).float().to(torch.bfloat16)


def plan(ctx, new, page, table, free, start, T):
    """numpy; returns row_offsets, kv_lens, slots, positions, free_next and the table."""
    table = table.copy()
    slots, positions = np.full(T, -1, np.int64), np.full(T, -1, np.int32)
    offsets, lens, at, t = [0], [], max(start, 0), 0
    for s, (c, n) in enumerate(zip(np.maximum(ctx, 0), np.maximum(new, 0))):
        held, need = -(-c // page), -(-(c + n) // page)
        for i in range(held, need):
            if i < table.shape[1]:
                table[s, i] = free[at] if at < len(free) else -1
            at += 1
        for p in range(c, c + n):
            if t < T:
                positions[t] = p
                if p // page < table.shape[1] and table[s, p // page] >= 0:
                    slots[t] = table[s, p // page] * page + p % page
            t += 1
        offsets.append(offsets[-1] + n)
        lens.append(c + n)
    return np.array(offsets, np.int64), np.array(lens, np.int32), slots, positions, at, table


def attention(q, offsets, lens, table, k_cache, v_cache, scale, causal, window):
    """(out, lse, bound on |out|'s error, bound on |lse|'s error, rows written), float64 [T, Hq, D] and [T, Hq].

    The bounds count what the kernel rounds.  d = largest error of a score: fp32 sums of D exact products and at most three factors more
    (scale, 1/F by a reciprocal within an ulp, log2 e), each relative to sum |q k|; a weight is off by d, by exp's ulps and by its
    rounding to bf16; the sum l by its n additions; the result is rounded once to bf16.  Relative bounds end where numbers do: the exp
    instruction, the products and their operands take less than 2^-126 (the smallest normal number) for 0, so that each of n weights, relative
    to a sum l >= 1, and then the result may lose that much: n 2^-126 max |v| from weights, as much again from products, and 2^-126."""
    q = q.cpu().double().numpy()
    T, Hq, D = q.shape
    H, page = k_cache[1].shape[1], k_cache[1].shape[3]
    pages = k_cache[1].shape[0]
    G = Hq // H
    offsets, lens, table = offsets.cpu().numpy(), lens.cpu().numpy(), table.cpu().numpy()
    out, lse = np.zeros((T, Hq, D)), np.full((T, Hq), -np.inf)
    tol, tol_lse, written = np.zeros((T, Hq, D)), np.zeros((T, Hq)), np.zeros(T, bool)
    u = 2.0 ** -24
    for s in range(len(lens)):
        b, e = offsets[s], offsets[s + 1]
        j = np.arange(max(0, min(lens[s], table.shape[1] * page)))
        P = table[s, j // page]
        there = (P >= 0) & (P < pages)
        slots = np.where(there, P, 0).astype(np.int64) * page + j % page
        k, v = values(*cached_rows(k_cache, True, slots)), values(*cached_rows(v_cache, False, slots))
        for t in range(b, min(e, T)):
            written[t] = True
            p = lens[s] - (e - b) + (t - b)
            sees = there.copy()
            if causal:
                sees &= j <= p
                if window:
                    sees &= j > p - window
            if not sees.any():
                continue
            n = int(sees.sum())
            for h in range(Hq):
                kk, vv = k[sees, h // G], v[sees, h // G]
                x = kk @ q[t, h] * scale
                d = (np.abs(kk) @ np.abs(q[t, h])).max() * abs(scale) * (D + 8) * u
                m = x.max()
                w = np.exp(x - m)
                total = w.sum()
                out[t, h] = w @ vv / total
                lse[t, h] = m + np.log(total)
                spread = (np.abs(w) @ np.abs(vv)) / total
                sums = (n + 64) * u
                tol[t, h] = STEP * np.abs(out[t, h]) + (STEP + 2 * d + 2 * sums) * 1.02 * spread + (2 * n * np.abs(vv).max(0) + 1) * 2.0 ** -126
                tol_lse[t, h] = 2 * d + 2 * sums + 8 * u * (abs(m) + abs(lse[t, h]))
    return out, lse, tol, tol_lse, written
