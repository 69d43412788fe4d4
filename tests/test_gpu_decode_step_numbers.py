"""The decode step's operators at the edges of their number types: how many bits what lies between their two products has,
infinite values and weights, sums and scores near the largest number.  Expected results are the formulas', in 64 bits."""
import numpy as np
import pytest
import torch

import decode_step_reference as R
from paper_2511_10676_amd import binding as B
from test_gpu_decode_step import _cache, _i32, _np, _pages, _storage, _to

pytestmark = pytest.mark.gpu


def _two_parts(x):
    """x as the sum of two bf16 numbers: the nearest, and the nearest to what is left."""
    high = _storage(x, "bf16").astype(np.float64)
    return high, _storage(x - high, "bf16").astype(np.float64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,where", [(3, (0, 1, 2)), (40, (5, 6, 7)), (40, (5, 38, 17)), (3000, (100, 1700, 2800)), (3000, (1700, 1701, 1702)), (20000, (19999, 0, 7777))])
def test_attend_multiplies_probabilities_of_32_bits(n, where, dtype):
    """Head h looks at three positions, with weights in the ratio 1 : e : e (e = exp(-s_h), s_h < 1); dimension h of their
    values is 1, -v1, -v2 with v1 + v2 close to 1 / e, so that the sum all but cancels and shows what the weights were off by.
    Of the sum, whose terms are 1 at most: e is off by its argument's rounding (2 U) and the exponential's (2 U), the products
    of bf16 numbers with parts of e are exact, and about 8 sums of terms up to 1 round (U each; their join over chunks 4 more):
    16 U.  A weight of 16 bits is off by up to 64 U."""
    H, G, D = 1, 16, 16
    kp, vp, table = _cache(np.random.default_rng(n), [n], H, D, D, 16, dtype)
    g = np.random.default_rng(40)
    s = _storage(g.uniform(0.2, 0.95, G), "bf16").astype(np.float64)       # exact in both types
    e = np.exp(-s)
    q = np.zeros((1, G, D))
    q[0, :, 0], q[0, :, 1] = s, 256.0
    pos = np.array(where)
    page, slot = table[0, np.arange(n) // 16], np.arange(n) % 16
    kp[page, 0, slot], vp[page, 0, slot] = 0.0, 0.0
    kp[page, 0, slot, 1] = -4.0                            # everyone else: a score of -1024, a weight of 0
    kp[page[pos], 0, slot[pos], 1] = 0.0
    kp[page[pos[1:]], 0, slot[pos[1:]], 0] = -1.0          # scores 0, -s, -s
    high, low = _two_parts(1.0 / e)
    vp[page[pos[0]], 0, slot[pos[0]]] = 1.0
    vp[page[pos[1]], 0, slot[pos[1]]], vp[page[pos[2]], 0, slot[pos[2]]] = -high, -low
    got = B.attend(_to(q, dtype), _pages(kp, dtype, "heads"), _pages(vp, dtype, "heads"), _i32(table), _i32([n]), scale=1.0)
    torch.cuda.synchronize()
    want = (1.0 - e[:, None] * (high + low)[None]) / (1.0 + 2.0 * e[:, None])          # [head, dimension]
    size = np.maximum(1.0, e[:, None] * np.abs(high + low)[None])
    tol = 16 * R.U * size / (1.0 + 2.0 * e[:, None]) + (R.BF16 if dtype == "bf16" else 4 * R.U) * np.abs(want)
    off = np.abs(_np(got.out)[0].astype(np.float64) - want)
    assert (off <= tol).all(), (off / tol).max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,f", [(1, 8), (5, 40), (16, 8), (40, 72), (64, 1000)])
def test_moe_experts_multiply_hidden_values_of_32_bits(T, f, dtype):
    """Token t has the weights p, r at experts 1 and 2, whose hidden values are p (unit 0) and r (units 0 and f - 1): gate and
    other rows are exactly 1 there.  Row t of the second matrices is 1 and -v1, -v2 with v1 + v2 close to p / r: the sum all but
    cancels.  Products are exact, about 8 sums of terms up to p round: 8 U p.  A hidden value of 16 bits is off by up to 64 U p."""
    E, d = 4, max(16, -(-T // 8) * 8)
    g = np.random.default_rng(T)
    p, r = (g.uniform(0.5, 1.0, T).astype(np.float32).astype(np.float64) for _ in range(2))
    x, W13, W2 = np.zeros((T, d)), np.zeros((E, 2 * f, d)), np.zeros((E, d, f))
    x[:, 3] = 1.0
    W13[1:3, [0, f - 1, f, 2 * f - 1], 3] = 1.0
    high, low = _two_parts(p / r)
    W2[1, :T, 0], W2[2, :T, 0], W2[2, :T, f - 1] = 1.0, -high, -low
    idx = _i32(np.tile([1, 2], (T, 1)))
    got = B.moe_experts(_to(x, dtype), _to(W13, dtype), _to(W2, dtype), idx, _to(np.stack([p, r], 1), "f32"), act="none")
    torch.cuda.synchronize()
    want = p[:, None] - r[:, None] * (high + low)[None]                                # [token, row]
    tol = 8 * R.U * np.maximum(p[:, None], r[:, None] * (high + low)[None]) + (R.BF16 if dtype == "bf16" else 2 * R.U) * np.abs(want)
    off = np.abs(_np(got)[:, :T].astype(np.float64) - want)
    assert (off <= tol).all(), (off / tol).max()
    assert not _np(got)[:, T:].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,f,residual", [(1, 8, False), (7, 200, True), (16, 1000, False), (40, 72, True), (64, 1000, True)])
def test_moe_experts_with_infinite_weights(T, f, residual, dtype):
    """Infinite entries of the second matrix, and hidden values that are infinite, or finite and above the largest bf16
    number: every row of y is what the formula gives, and where that is finite, as close as ever."""
    E, d, k = 6, 64, 2
    g = np.random.default_rng(T + f)
    x = _storage(g.standard_normal((T, d)), dtype)
    W13 = _storage(g.standard_normal((E, 2 * f, d)) / np.sqrt(d), dtype)
    W2 = _storage(g.standard_normal((E, d, f)) / np.sqrt(f), dtype)
    idx = np.stack([g.permutation(E - 1)[:k] for _ in range(T)])
    idx[0] = [0, 1]
    probs = g.uniform(0.2, 0.8, (T, k)).astype(np.float32)
    res = _storage(g.standard_normal((T, d)), dtype) if residual else None
    finite, tol = R.experts(x, W13, W2, idx, probs, "silu", res, dtype == "bf16")
    bad = W2.copy()
    bad[0, 5, 3], bad[1, 5, f - 1], bad[1, 9, 0] = np.inf, np.inf, -np.inf
    bad[2, 9, 2], bad[3, 63, f // 2], bad[4, 17, 1] = np.inf, np.nan, -np.inf
    want = np.zeros((T, d)) if res is None else res.astype(np.float64).copy()
    for t in range(T):
        for j in range(k):
            u = W13[idx[t, j]].astype(np.float64) @ x[t].astype(np.float64)
            with np.errstate(invalid="ignore"):
                want[t] += bad[idx[t, j]].astype(np.float64) @ (probs[t, j] * R.act(u[:f], "silu") * u[f:])
    got = B.moe_experts(_to(x, dtype), _to(W13, dtype), _to(bad, dtype), _i32(idx), _to(probs, "f32"),
                        residual=None if res is None else _to(res, dtype))
    torch.cuda.synchronize()
    y = _np(got).astype(np.float64)
    here = np.isfinite(want)
    assert not here.all() and here.any()
    assert np.array_equal(y[~here], want[~here], equal_nan=True)
    assert np.allclose(want[here], finite[here], rtol=1e-9, atol=1e-12) and (np.abs(y - finite)[here] <= tol[here]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [3, 40])
def test_moe_experts_with_infinite_hidden_values(T, dtype):
    """Hidden values p * 2^64 * u: infinite for u = 2^64 and p = 1, finite for p = 0.9985, where the nearest bf16 number is infinity."""
    E, d, f = 3, 64, 24
    x, W13, W2 = np.zeros((T, d)), np.zeros((E, 2 * f, d)), np.zeros((E, d, f))
    x[:, 0] = 1.0
    W13[:, 4, 0] = 2.0 ** 64                              # gate row 4; its other row:
    W13[0, f + 4, 0], W13[1, f + 4, 0] = 2.0 ** 64, -2.0 ** 64
    W2[:, :, 4] = 2.0 ** -10
    W2[:, 1, 4] = -2.0 ** -10
    W2[0, 2, 4] = np.inf
    p = np.full((T, 1), 1.0, dtype=np.float32)
    p[1:] = 0.9985
    idx = np.zeros((T, 1), dtype=np.int32)
    idx[2] = 1
    got = _np(B.moe_experts(_to(x, dtype), _to(W13, dtype), _to(W2, dtype), _i32(idx), _to(p, "f32"), act="none"))
    torch.cuda.synchronize()
    big = np.float32(0.9985).astype(np.float64) * 2.0 ** 118
    assert got[0, 0] == np.inf and got[0, 1] == -np.inf and got[0, 2] == np.inf
    tol = (R.BF16 if dtype == "bf16" else 8 * R.U) * big
    assert abs(got[1, 0] - big) <= tol and abs(got[1, 1] + big) <= tol and got[1, 2] == np.inf
    assert abs(got[2, 0] + big) <= tol and abs(got[2, 1] - big) <= tol and abs(got[2, 2] + big) <= tol


def _attend_given(g, lengths, H, G, D, page, dtype, values, scale=None):
    """attend and R.attend over random keys, the values being values(vp at the sequences' positions); masses too."""
    kp, vp, table = _cache(g, lengths, H, D, D, page, dtype)
    bad = vp.copy()
    for b, n in enumerate(lengths):
        p = np.arange(n)
        rows = bad[table[b, p // page], :, p % page]              # [n, H, D]
        bad[table[b, p // page], :, p % page] = values(b, rows)
    q = _storage(g.standard_normal((len(lengths), H * G, D)), dtype)
    mass = torch.zeros((len(lengths), H, table.shape[1] * page), device="cuda")
    got = B.attend(_to(q, dtype), _pages(kp, dtype, "heads"), _pages(bad, dtype, "heads"), _i32(table), _i32(lengths), mass=mass,
                   want_lse=True, scale=scale)
    alone = B.attend(_to(q, dtype), _pages(kp, dtype, "heads"), _pages(bad, dtype, "heads"), _i32(table), _i32(lengths), scale=scale)
    torch.cuda.synchronize()
    assert torch.equal(got.out.nan_to_num(7.0), alone.out.nan_to_num(7.0))
    return q, kp, vp, bad, table, got, _np(mass).astype(np.float64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lengths", [[1, 2, 50], [200, 33, 17], [5000, 1], [3000, 900, 2049]])
@pytest.mark.parametrize("H,G,D", [(1, 3, 64), (2, 17, 128), (1, 2, 256)])
def test_attend_with_infinite_values(H, G, D, lengths, dtype):
    """Infinite and NaN values at positions that are looked at: a dimension is what the formula gives; the others, and what
    does not depend on the values, are as close as ever."""
    def values(b, rows):
        n = len(rows)
        rows = rows.copy()
        rows[0, 0, 3], rows[n - 1, 0, 9] = np.inf, -np.inf
        rows[n // 2, 0, 20] = np.nan
        rows[0, -1, 30] = -np.inf
        if n > 1:
            rows[0, -1, 40], rows[n - 1, -1, 40] = np.inf, -np.inf
        rows[n // 3, -1, D - 1] = np.inf
        return rows
    q, kp, vp, bad, table, got, mass = _attend_given(np.random.default_rng(sum(lengths)), lengths, H, G, D, 16, dtype, values, scale=0.25 * D ** -0.5)
    cap = table.shape[1] * 16
    (out, lse, weight), tol = R.attend(q, kp, vp, table, lengths, None, 0.25 * D ** -0.5, cap, dtype == "bf16")
    o = _np(got.out).astype(np.float64)
    for b, n in enumerate(lengths):
        for h in range(H):
            p = np.arange(n)
            rows = bad[table[b, p // 16], h, p % 16].astype(np.float64)
            with np.errstate(invalid="ignore"):
                special = rows[~np.isfinite(rows).all(1)].sum(0)                       # infinite or NaN as the weighted sum is
            there = slice(h * G, (h + 1) * G)
            odd = ~np.isfinite(special)
            assert odd.any()
            assert np.array_equal(o[b, there][:, odd], np.broadcast_to(special[odd], (G, odd.sum())), equal_nan=True)
            assert (np.abs(o[b, there] - out[b, there]) <= tol[0][b, there])[:, ~odd].all()
    assert (np.abs(_np(got.lse) - lse) <= tol[1]).all() and (np.abs(mass - weight) <= tol[2] + 2 * R.U * weight).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_is_zero_where_every_score_is_minus_infinity_whatever_the_values(dtype):
    g = np.random.default_rng(44)
    lengths = [9, 700, 300]
    kp, vp, table = _cache(g, lengths, 1, 64, 64, 16, dtype)
    kp[..., 0] = -np.inf
    for b in range(2):
        p = np.arange(lengths[b])
        vp[table[b, p // 16], 0, p % 16] = [np.inf, -np.inf, np.nan, 1.0] * 16
    p = np.arange(256, 300)                               # the last sequence: its first positions only
    kp[table[2, p // 16], 0, p % 16, 0] = 0.0
    q = np.abs(_storage(g.standard_normal((3, 2, 64)), dtype)) + 0.5
    mass = torch.zeros((3, 1, 704), device="cuda")
    got = B.attend(_to(q, dtype), _pages(kp, dtype, "heads"), _pages(vp, dtype, "heads"), _i32(table), _i32(lengths), mass=mass, want_lse=True)
    torch.cuda.synchronize()
    assert not _np(got.out)[:2].any() and np.isfinite(_np(got.out)[2]).all() and _np(got.out)[2].any()
    assert (_np(got.lse)[:2] == -np.inf).all() and not _np(mass)[:2].any() and np.allclose(_np(mass)[2].sum(), 2.0, rtol=1e-5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lengths,size", [([40, 1, 700], 3.2e38), ([9000], 3.2e38), ([4000], 1.5e36), ([2000, 1800], 4e36), ([300, 5], 1e37)])
def test_attend_averages_values_near_the_largest_number(lengths, size, dtype):
    """The sum of the values would overflow; their average, the result, does not (keys equal: the weights are 1 / n)."""
    g = np.random.default_rng(50)
    kp, vp, table = _cache(g, lengths, 2, 64, 64, 16, dtype)
    kp[:], sign = 0.0, np.where(np.arange(64) % 3 == 0, -1.0, 1.0)
    vp[:] = _storage(sign * size * (1.0 - np.arange(64) / 200.0), dtype)
    q = _storage(g.standard_normal((len(lengths), 6, 64)), dtype)
    got = B.attend(_to(q, dtype), _pages(kp, dtype, "heads"), _pages(vp, dtype, "heads"), _i32(table), _i32(lengths), want_lse=True)
    torch.cuda.synchronize()
    want = vp[0, 0, 0].astype(np.float64)
    # a sum over n terms rounds n times at most, and so does the sum of the weights
    tol = (2 * (np.array(lengths) + 16) * 2 * R.U + (R.BF16 if dtype == "bf16" else 0))[:, None, None] * np.abs(want)
    assert (np.abs(_np(got.out).astype(np.float64) - want) <= tol).all()
    assert np.allclose(_np(got.lse), np.log(lengths)[:, None], rtol=1e-5, atol=1e-6)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [7, 600])
def test_attend_scores_near_the_largest_number(n, dtype):
    """Finite scores up to 3.3e38 in size: equal ones share the weight, lower ones get none."""
    kp, vp, table = _cache(np.random.default_rng(60), [n, n], 1, 64, 64, 16, dtype)
    kp[:] = 0.0
    vp[:] = _storage(np.random.default_rng(61).standard_normal(vp.shape), dtype)
    q = np.zeros((2, 4, 64))
    q[:, :, 0] = 1.0
    big, less = _storage([3.3e38, 2.6e38], dtype)
    kp[..., 0] = -big                                     # sequence 1: everywhere the lowest
    p = np.arange(n)
    kp[table[0, p // 16], 0, p % 16, 0] = less
    kp[table[0, 1 // 16], 0, 1, 0] = kp[table[0, (n - 1) // 16], 0, (n - 1) % 16, 0] = big
    mass = torch.zeros((2, 1, table.shape[1] * 16), device="cuda")
    got = B.attend(_to(q, dtype), _pages(kp, dtype, "heads"), _pages(vp, dtype, "heads"), _i32(table), _i32([n, n]), scale=1.0, mass=mass, want_lse=True)
    torch.cuda.synchronize()
    rows = vp[table[:, p // 16], 0, p % 16].astype(np.float64)
    want = np.stack([(rows[0, 1] + rows[0, n - 1]) / 2, rows[1].mean(0)])
    tol = (n + 16) * 4 * R.U * np.abs(rows).max() + (R.BF16 if dtype == "bf16" else 0) * np.abs(want)
    o = _np(got.out).astype(np.float64)
    assert (np.abs(o - want[:, None]) <= tol[:, None]).all()
    w = np.zeros((2, n))
    w[0, [1, n - 1]], w[1] = 2.0, 4.0 / n
    assert np.allclose(_np(mass)[:, 0, :n], w, rtol=1e-4, atol=0)
    assert np.allclose(_np(got.lse)[0], big, rtol=1e-6) and np.allclose(_np(got.lse)[1], -big, rtol=1e-6)
