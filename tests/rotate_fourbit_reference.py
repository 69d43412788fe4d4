"""Plain 64-bit forms of the rotation of heads and of a cache in 4 bits, with bounds of what fp32 arithmetic may be off by.
NumPy only."""
import numpy as np

U = 2.0 ** -24                                    # rounding of one fp32 operation
HALF = {"bf16": 2.0 ** -8, "f32": U}              # rounding of one result to storage
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def rotate(x, weight, turns, style, eps, kind):
    """x [n, heads, D], turns [n, rot] -> y and a bound of its error."""
    D, rot = x.shape[2], turns.shape[1]
    half = rot // 2
    x = x.astype(np.float64)
    rel = 0.0
    if weight is not None:
        with np.errstate(invalid="ignore"):
            x = x / np.sqrt((x * x).mean(axis=2, keepdims=True) + eps) * weight.astype(np.float64)
        # D squares and sums, the division and eps: half of it under the root; the root's reciprocal to 1 unit (2 U), two products
        rel = ((D + 4) / 2 + 4) * U
    i = np.arange(half)
    a, b = (i, i + half) if style == "halves" else (2 * i, 2 * i + 1)
    c, s = turns[:, None, :half].astype(np.float64), turns[:, None, half:].astype(np.float64)
    y, size = x.copy(), np.abs(x)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    size[..., a], size[..., b] = (np.abs(x[..., a] * c) + np.abs(x[..., b] * s)), (np.abs(x[..., a] * s) + np.abs(x[..., b] * c))
    # each term carries rel and its product's rounding, the sum one more
    return y, size * (rel + 3 * U) + np.abs(y) * HALF[kind] + 1e-38


def to_fourbit(x):
    """[..., D] float32 values -> the numbers they become (float64), exponents' bytes [..., D / 32]."""
    g = x.astype(np.float64).reshape(*x.shape[:-1], -1, 32)
    nan = np.isnan(g).any(axis=-1)
    a = np.where(np.isnan(g), 0.0, np.abs(g))
    most = a.max(axis=-1)
    e = np.full(most.shape, -125)
    for i in range(-125, 125):
        e = np.where(most > 7 * 2.0 ** i, i + 1, e)
    y = np.minimum(a / 2.0 ** e[..., None], 6.0)
    d = np.abs(y[..., None] - GRID)
    d[..., 1::2] += 1e-9                          # ties to the even code (distances of different numbers are further apart than that or equal)
    got = GRID[d.argmin(axis=-1)] * 2.0 ** e[..., None] * np.where(np.signbit(g), -1.0, 1.0)
    got = np.where(nan[..., None], np.nan, got)
    return got.reshape(x.shape), np.where(nan, 255, e + 127).astype(np.uint8)


def values(codes, scales):
    """codes [..., D / 2], scales [..., D / 32] uint8 -> the numbers (float64)."""
    c = np.stack([codes & 15, codes >> 4], axis=-1).reshape(*codes.shape[:-1], -1)
    v = np.where(c & 8, -GRID[c & 7], GRID[c & 7])
    with np.errstate(over="ignore"):
        by = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(by, 32, axis=-1)


def attend(q, k, v, table, lengths, starts, scale, max_len, kind):
    """out, lse and bounds of their errors; k, v [n_pages, Hkv, page_size, width]: the numbers that stand in the cache."""
    B, Hq, D = q.shape
    n_pages, H, ps, Dv = v.shape
    G = Hq // H
    out, lse = np.zeros((B, Hq, Dv)), np.full((B, Hq), -np.inf)
    tol = [np.zeros_like(out), np.zeros_like(lse)]
    parts = 1 if kind == "bf16" else 3
    for b in range(B):
        pos = np.arange(max(0, 0 if starts is None else int(starts[b])), min(max(int(lengths[b]), 0), max_len))
        entry = table[b, pos // ps]
        there = (entry >= 0) & (entry < n_pages)
        pos, entry = pos[there], entry[there]
        if not pos.size:
            continue
        for h in range(Hq):
            kk, vv = k[entry, h // G, pos % ps], v[entry, h // G, pos % ps]
            qh = q[b, h].astype(np.float64)
            s, mag = scale * (kk @ qh), abs(scale) * (np.abs(kk) @ np.abs(qh))
            top = s.max()
            e = np.exp(s - top)
            p = e / e.sum()
            out[b, h], lse[b, h] = p @ vv, top + np.log(e.sum())
            # scores: a product and a sum for each of an element's parts, and the factor; exponentials: their reference point is at
            # most 8 below the maximum, its difference, the product with log2 e and that constant are rounded, and 2 units of its own
            ds = ((parts * 2 * D + 4) * U * mag).max() + 8 * U * (np.abs(s - top).clip(max=100).max() + 8)
            rel = 2 * ds + (pos.size + 16) * 2 * U       # ... in a term and in the sum; sums: one rounding per term
            tol[0][b, h] = rel * (p @ np.abs(vv)) + HALF[kind] * np.abs(out[b, h]) + 1e-38
            tol[1][b, h] = ds + (pos.size + 16) * 2 * U + 4 * U * abs(lse[b, h]) + 4 * U
    return (out, lse), tol
