"""Plain 64-bit forms of a decode step's operators (attention over a paged cache, eviction, the expert layer), with bounds of
what fp32 arithmetic may be off by.  NumPy only; sequence by sequence, head by head."""
import numpy as np
from scipy.special import erf

U = 2.0 ** -24                    # rounding of one fp32 operation
BF16 = 2.0 ** -8                  # rounding of one result to bf16, doubled


def gather(pages, table, b, positions):
    """Rows [Hkv, len(positions), width] of one sequence, and which of them stand on a page at all."""
    n_pages, H, ps, _ = pages.shape
    entry = table[b, positions // ps]
    there = (entry >= 0) & (entry < n_pages)
    rows = pages[np.where(there, entry, 0), :, positions % ps]
    return rows.transpose(1, 0, 2).astype(np.float64), there


def attend(q, k_pages, v_pages, table, lengths, starts, scale, max_len, bf16):
    """out, lse, weight [B, Hkv, max_len] summed over the heads of a group, and a bound for the error of each."""
    B, Hq, Dk = q.shape
    H, Dv = k_pages.shape[1], v_pages.shape[3]
    G = Hq // H
    out, lse = np.zeros((B, Hq, Dv)), np.full((B, Hq), -np.inf)
    weight = np.zeros((B, H, max_len))
    tol = [np.zeros_like(out), np.zeros_like(lse), np.zeros_like(weight)]
    for b in range(B):
        n = min(max(int(lengths[b]), 0), max_len)
        pos = np.arange(max(0, 0 if starts is None else int(starts[b])), n)
        k, there = gather(k_pages, table, b, pos)
        v, _ = gather(v_pages, table, b, pos)
        pos, k, v = pos[there], k[:, there], v[:, there]
        if not pos.size:
            continue
        for h in range(Hq):
            g = h // G
            qh = q[b, h].astype(np.float64)
            with np.errstate(invalid="ignore"):
                s = scale * (k[g] @ qh)
                mag = abs(scale) * (np.abs(k[g]) @ np.abs(qh))
            live = s > -np.inf
            if not live.any():
                continue
            top = s[live].max()
            e = np.where(live, np.exp(s - top), 0.0)
            p = e / e.sum()
            out[b, h] = p[live] @ v[g][live]
            lse[b, h] = top + np.log(e.sum())
            weight[b, g, pos] += p
            # scores: Dk products and sums, and the factor; exp: its argument s - top and a few units of its own; sums: one
            # rounding per term
            ds = ((Dk + 4) * U * mag[live] + 8 * U * np.abs(s[live])).max() + 8 * U * np.abs(s[live] - top).clip(max=100).max()
            rel = 2 * ds + (pos.size + 16) * 2 * U
            spread = p[live] @ np.abs(v[g][live])
            # bf16: the probabilities are multiplied in two bf16 parts, 16 bits, and the result is rounded
            tol[0][b, h] = (rel + (2.0 ** -15 if bf16 else 0)) * spread + (BF16 if bf16 else 2 * U) * np.abs(out[b, h]) + 1e-30
            tol[1][b, h] = ds + (pos.size + 16) * 2 * U + 4 * U * abs(lse[b, h])
            tol[2][b, g, pos] += rel * p + 2 * U * weight[b, g, pos] + 1e-30
    return (out, lse, weight), tol


def kept_positions(mass, n, budget, recent):
    """The ascending positions that one head keeps of n."""
    if n <= budget:
        return np.arange(n)
    old = n - recent
    rank = sorted(range(old), key=lambda p: (np.isnan(mass[p]), 0.0 if np.isnan(mass[p]) else -mass[p], p))
    return np.array(sorted(rank[:budget - recent]) + list(range(old, n)), dtype=np.int64)


def act(u, name):
    if name == "silu":
        return u / (1.0 + np.exp(-u))
    if name == "gelu":
        return 0.5 * u * (1.0 + erf(u * np.sqrt(0.5)))
    return u


def select(z, k, prob):
    idx = np.argsort(-z, axis=1, kind="stable")[:, :k]
    top = np.take_along_axis(z, idx, 1)
    if prob == "sigmoid":
        return idx, 1.0 / (1.0 + np.exp(-top))
    e = np.exp(top - top[:, :1])
    return idx, e / (e.sum(1, keepdims=True) if prob == "softmax_topk" else np.exp(z - top[:, :1]).sum(1, keepdims=True))


def experts(x, W13, W2, idx, probs, name, residual, bf16):
    """y [T, d] and a bound of its error, given the selection (ids outside [0, E) are skipped)."""
    T, d = x.shape
    E, _, f = W2.shape
    y = np.zeros((T, d)) if residual is None else residual.astype(np.float64).copy()
    size = np.abs(y)
    off = np.zeros((T, d))
    for e in sorted(set(int(i) for i in idx.ravel() if 0 <= i < E)):
        w13, w2 = W13[e].astype(np.float64), W2[e].astype(np.float64)
        for t in np.flatnonzero((idx == e).any(1)):
            p = probs[t][idx[t] == e].astype(np.float64).sum()
            xt = x[t].astype(np.float64)
            u, a = w13 @ xt, d * U * (np.abs(w13) @ np.abs(xt))        # both halves, and what their sums may be off by
            gate = act(u[:f], name)
            h = p * gate * u[f:]
            # the activations' slope is at most 1.13; their own error a few units; the row's weight; bf16: two bf16 parts
            dh = abs(p) * (1.13 * a[:f] * np.abs(u[f:]) + np.abs(gate) * a[f:] + 1.13 * a[:f] * a[f:]) \
                + np.abs(h) * (64 * U + (2.0 ** -16 if bf16 else 0)) + 1e-30
            y[t] += w2 @ h
            size[t] += np.abs(w2) @ np.abs(h)
            off[t] += np.abs(w2) @ dh
    k = idx.shape[1]
    return y, off + (k * f + 4) * U * size + (BF16 if bf16 else 2 * U) * np.abs(y) + 1e-30
