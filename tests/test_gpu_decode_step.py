"""Attention over a paged cache, the cache's upkeep and the expert layer on the GPU against their plain 64-bit forms, at the
sizes, layouts and masks where they can go wrong.  Whatever no call may look at (slots behind a length or before a start, pages
that no sequence has, weights of experts that no token picked) holds NaN."""
import numpy as np
import pytest
import torch

import decode_step_reference as R
from paper_2511_10676_amd import binding as B

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _to(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DT[dtype] if isinstance(dtype, str) else dtype).cuda()


def _np(t):
    return t.detach().float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _pages(pages_np, dtype, order):
    """The pool with heads or slots as a page's outer dimension, as the view [n_pages, Hkv, page_size, width]."""
    if order == "heads":
        return _to(pages_np, dtype)
    return _to(pages_np.transpose(0, 2, 1, 3), dtype).permute(0, 2, 1, 3)


def _storage(a, dtype):
    """The values that the type can hold."""
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(DT[dtype]).float().numpy()


def _cache(g, lengths, H, Dk, Dv, page, dtype, starts=None, spare=2, width=None, kscale=1.0):
    """Pools with NaN everywhere but at the positions looked at, and a scattered page table, -1 behind the last page."""
    need = [-(-max(0, int(n)) // page) for n in lengths]
    width = max(1, max(need)) if width is None else width
    total = sum(need) + spare
    order = g.permutation(total)
    table = np.full((len(lengths), width), -1, dtype=np.int32)
    kp = np.full((total, H, page, Dk), np.nan, dtype=np.float32)
    vp = np.full((total, H, page, Dv), np.nan, dtype=np.float32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
        for p in range(0 if starts is None else max(0, int(starts[b])), max(0, int(lengths[b]))):
            kp[table[b, p // page], :, p % page] = g.standard_normal((H, Dk)) * kscale
            vp[table[b, p // page], :, p % page] = g.standard_normal((H, Dv))
    return _storage(kp, dtype), _storage(vp, dtype), table


def _i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def _check_attend(q, kp, vp, table, lengths, starts, dtype, order="heads", scale=None, max_len=None, mass=True, q_dev=None, **kw):
    B_, Hq, Dk = q.shape
    H, Dv = kp.shape[1], vp.shape[3]
    cap = table.shape[1] * kp.shape[2] if max_len is None else max_len
    scale = Dk ** -0.5 if scale is None else scale
    (out, lse, weight), tol = R.attend(q, kp, vp, table, lengths, starts, scale, cap, dtype == "bf16")
    m0 = np.random.default_rng(9).random((B_, H, cap + 5)).astype(np.float32)
    m = _to(m0, "f32") if mass else None
    got = B.attend(_to(q, dtype) if q_dev is None else q_dev, _pages(kp, dtype, order), _pages(vp, dtype, order),
                   _i32(table), _i32(lengths), starts=None if starts is None else _i32(starts), scale=scale, max_len=max_len,
                   mass=m, want_lse=True, **kw)
    torch.cuda.synchronize()
    o, l = _np(got.out).astype(np.float64), _np(got.lse).astype(np.float64)
    assert o.shape == out.shape and np.isfinite(o).all()
    assert (np.abs(o - out) <= tol[0]).all(), (np.abs(o - out) / tol[0]).max()
    assert np.array_equal(np.isinf(l), np.isinf(lse)) and not (l == np.inf).any()
    fin = np.isfinite(lse)
    assert (np.abs(l[fin] - lse[fin]) <= tol[1][fin]).all()
    if mass:
        got_m, want_m = _np(m).astype(np.float64), m0.astype(np.float64)
        assert np.array_equal(got_m[:, :, cap:], want_m[:, :, cap:])
        untouched = weight == 0
        assert np.array_equal(got_m[:, :, :cap][untouched], want_m[:, :, :cap][untouched])
        want = want_m[:, :, :cap] + weight
        assert (np.abs(got_m[:, :, :cap] - want) <= tol[2] + 2 * R.U * want).all()
    return got


EDGES = [0, 1, 2, 3, 7, 8, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 513]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page,order", [(1, "heads"), (2, "slots"), (4, "heads"), (16, "slots"), (64, "heads"), (1024, "slots")])
def test_attend_lengths_and_pages(page, order, dtype):
    g = np.random.default_rng(page)
    kp, vp, table = _cache(g, EDGES, 2, 64, 64, page, dtype)
    q = _storage(g.standard_normal((len(EDGES), 6, 64)) * 2, dtype)
    _check_attend(q, kp, vp, table, EDGES, None, dtype, order)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,Dk,Dv", [
    (1, 1, 8, 8), (3, 1, 16, 24), (2, 2, 40, 64), (1, 7, 72, 80), (2, 8, 80, 80), (1, 16, 96, 96), (1, 17, 128, 128), (2, 24, 128, 64),
    (1, 32, 64, 128), (1, 33, 136, 136), (2, 4, 192, 128), (1, 48, 256, 256), (4, 8, 128, 128), (1, 71, 104, 200), (16, 1, 128, 128),
    (2, 3, 256, 8), (2, 20, 8, 256), (1, 16, 160, 160), (5, 2, 224, 248)])
def test_attend_heads_and_widths(H, G, Dk, Dv, dtype):
    g = np.random.default_rng(H * 1000 + G * 10 + Dk)
    lengths = [300, 0, 77, 1]
    kp, vp, table = _cache(g, lengths, H, Dk, Dv, 16, dtype)
    q = _storage(g.standard_normal((4, H * G, Dk)) * 2, dtype)
    _check_attend(q, kp, vp, table, lengths, None, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_windows(dtype):
    g = np.random.default_rng(5)
    lengths = [200, 200, 200, 200, 200, 37, 0, 130, 129, 200]
    starts = [0, 1, 31, 128, 199, 37, 0, -4, 128, 500]
    kp, vp, table = _cache(g, lengths, 2, 128, 128, 8, dtype, starts)
    q = _storage(g.standard_normal((len(lengths), 10, 128)) * 2, dtype)
    _check_attend(q, kp, vp, table, lengths, starts, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,n,page,window", [(1, 8, 20011, 16, 0), (4, 1, 9001, 64, 0), (2, 16, 16384, 1, 5000), (1, 40, 6001, 128, 0)])
def test_attend_long(H, G, n, page, window, dtype):
    """Lengths whose work is split over workgroups and joined."""
    g = np.random.default_rng(n)
    lengths, starts = [n, 5, n // 3], [max(0, n - window), 0, 0] if window else None
    kp, vp, table = _cache(g, lengths, H, 64, 64, page, dtype, starts)
    q = _storage(g.standard_normal((3, H * G, 64)) * 2, dtype)
    _check_attend(q, kp, vp, table, lengths, starts, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_clamps_lengths_and_leaves_absent_pages_out(dtype):
    g = np.random.default_rng(11)
    page = 16
    kp, vp, table = _cache(g, [96] * 4, 2, 64, 64, page, dtype, width=6)
    table[1, 2], table[1, 5] = -1, kp.shape[0]            # no page, one past the pool
    table[2, :] = -7                                      # none at all
    lengths = [-3, 96, 96, 2000]                          # below zero; above max_len
    q = _storage(g.standard_normal((4, 4, 64)) * 2, dtype)
    got = _check_attend(q, kp, vp, table, lengths, None, dtype, max_len=90)
    assert not _np(got.out)[[0, 2]].any() and (_np(got.lse)[[0, 2]] == -np.inf).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_scores_of_minus_infinity_and_steep_scores(dtype):
    g = np.random.default_rng(12)
    lengths = [150, 150, 40, 600]
    kp, vp, table = _cache(g, lengths, 1, 64, 64, 16, dtype)
    q = np.abs(g.standard_normal((4, 4, 64))) + 0.5
    kp[table[0, 2], 0, 3, 5] = -np.inf                    # one position whose score is -infinity
    kp[table[1, :9], 0, 1::2, 0] = -np.inf                # every other one
    kp[table[2, :3], 0, :, 7] = -np.inf                   # all of them
    q[3] *= 60                                            # one position takes everything
    _check_attend(_storage(q, dtype), kp, vp, table, lengths, None, dtype)
    # the type's lowest value in the keys: finite scores, far below the others
    kp, vp, table = _cache(g, [50], 1, 64, 64, 16, dtype)
    kp[table[0, 1], 0, :8] = _storage(np.full(64, -3.0e38 / 64), dtype)
    _check_attend(_storage(q[:1], dtype), kp, vp, table, [50], None, dtype, mass=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_strided_queries_given_buffers_streams_and_repeats(dtype):
    g = np.random.default_rng(13)
    lengths = [400, 33, 1200]
    kp, vp, table = _cache(g, lengths, 2, 64, 64, 16, dtype)
    q = _storage(g.standard_normal((3, 4, 64)), dtype)
    fused = torch.full((3, 12, 72), float("nan"), dtype=DT[dtype], device="cuda")        # heads 72 apart, rows 12 heads apart
    fused[:, 4:8, :64] = _to(q, dtype)
    first = _check_attend(q, kp, vp, table, lengths, None, dtype, q_dev=fused[:, 4:8, :64])
    out = B.Attention(torch.full((3, 4, 64), 7.0, dtype=DT[dtype], device="cuda"), torch.full((3, 4), 7.0, device="cuda"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    args = (_to(q, dtype), _pages(kp, dtype, "heads"), _pages(vp, dtype, "heads"), _i32(table), _i32(lengths))
    torch.cuda.synchronize()
    got = B.attend(*args, out=out, stream=side)
    side.synchronize()
    assert got.out is out.out and torch.equal(out.out, first.out) and torch.equal(out.lse, first.lse)
    alone = B.attend(*args)
    torch.cuda.synchronize()
    assert alone.lse is None and torch.equal(alone.out, first.out)
    with pytest.raises(ValueError):
        B.attend(args[0].cpu(), *args[1:])
    with pytest.raises(ValueError):
        B.attend(args[0], args[1], args[2][:, :, :8], *args[3:])
    with pytest.raises(ValueError):
        B.attend(args[0], args[1], args[2], args[3].long(), args[4])
    with pytest.raises(ValueError):
        B.attend(*args, mass=torch.zeros((3, 2, 9), device="cuda"))
    with pytest.raises(B.PaepError, match="PAEP_ERR_SHAPE"):
        B.attend(args[0][:, :3], *args[1:])
    with pytest.raises(B.PaepError, match="PAEP_ERR_WORKSPACE"):
        B.attend(args[0], *args[1:], mass=torch.zeros((3, 2, 1200), device="cuda"), max_len=1200, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))


def test_attend_is_the_same_every_time_and_empty_batches_are_fine():
    g = np.random.default_rng(14)
    lengths = [3000, 100, 0, 2049]
    kp, vp, table = _cache(g, lengths, 2, 128, 128, 16, "bf16")
    args = (_to(g.standard_normal((4, 16, 128)), "bf16"), _pages(kp, "bf16", "heads"), _pages(vp, "bf16", "heads"), _i32(table), _i32(lengths))
    runs = []
    for _ in range(3):
        mass = torch.zeros((4, 2, table.shape[1] * 16), device="cuda")
        got = B.attend(*args, mass=mass, want_lse=True)
        runs.append((got.out, got.lse, mass))
    torch.cuda.synchronize()
    for r in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, runs[0]))
    none = B.attend(args[0][:0], args[1], args[2], args[3][:0], args[4][:0], want_lse=True)
    assert none.out.shape == (0, 16, 128) and none.lse.shape == (0, 16)
    zero = B.attend(*args, max_len=0, want_lse=True)
    torch.cuda.synchronize()
    assert not zero.out.any() and bool((zero.lse == -float("inf")).all())


# ---- the cache's upkeep ----

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Dk,Dv,page,order", [(1, 8, 8, 1, "heads"), (3, 72, 128, 16, "slots"), (8, 128, 128, 64, "heads"), (2, 256, 64, 2, "slots")])
def test_append_writes_rows_and_nothing_else(H, Dk, Dv, page, order, dtype):
    g = np.random.default_rng(H + Dk)
    S, cap = 5, 4 * page
    table = g.permutation(S * 4).reshape(S, 4).astype(np.int32)
    table[3, 1] = -1
    table[4, 0] = 77
    n = 2 * S * cap
    seq, pos = g.integers(-1, S + 1, n).astype(np.int32), g.integers(-2, cap + 2, n).astype(np.int32)
    seen, rows = set(), []
    for i in range(n):                                    # no place twice
        if (seq[i], pos[i]) not in seen:
            seen.add((seq[i], pos[i]))
            rows.append(i)
    seq, pos, n = seq[rows], pos[rows], len(rows)
    kp, vp = _storage(g.standard_normal((S * 4, H, page, Dk)), dtype), _storage(g.standard_normal((S * 4, H, page, Dv)), dtype)
    fused = _storage(g.standard_normal((n, H * (Dk + Dv) + 8)), dtype)
    mass0 = g.random((S, H, cap - 1)).astype(np.float32)
    kd, vd, md, f = _pages(kp, dtype, order), _pages(vp, dtype, order), _to(mass0, "f32"), _to(fused, dtype)
    k, v = f[:, :H * Dk].unflatten(1, (H, Dk)), f[:, H * Dk:H * (Dk + Dv)].unflatten(1, (H, Dv))
    B.cache_append(k, v, kd, vd, _i32(table), _i32(pos), sequences=_i32(seq), mass=md)
    torch.cuda.synchronize()
    for i in range(n):
        if 0 <= seq[i] < S and 0 <= pos[i] < cap and 0 <= table[seq[i], pos[i] // page] < S * 4:
            at = table[seq[i], pos[i] // page]
            kp[at, :, pos[i] % page] = fused[i, :H * Dk].reshape(H, Dk)
            vp[at, :, pos[i] % page] = fused[i, H * Dk:H * (Dk + Dv)].reshape(H, Dv)
            if pos[i] < cap - 1:
                mass0[seq[i], :, pos[i]] = 0
    assert np.array_equal(_np(kd), kp) and np.array_equal(_np(vd), vp) and np.array_equal(_np(md), mass0)
    # the new token of every sequence: sequences left out
    new = _to(g.standard_normal((S, H, Dk)), dtype), _to(g.standard_normal((S, H, Dv)), dtype)
    B.cache_append(*new, kd, vd, _i32(table), _i32([0, cap - 1, cap, 2 * page - 1, -1]))
    torch.cuda.synchronize()
    kp[table[0, 0], :, 0], kp[table[1, 3], :, page - 1] = _np(new[0])[0], _np(new[0])[1]
    vp[table[0, 0], :, 0], vp[table[1, 3], :, page - 1] = _np(new[1])[0], _np(new[1])[1]
    assert np.array_equal(_np(kd), kp) and np.array_equal(_np(vd), vp)
    B.cache_append(new[0][:0], new[1][:0], kd, vd, _i32(table), _i32([]))
    with pytest.raises(ValueError):
        B.cache_append(new[0], new[1][:, :, :Dv - 8] if Dv > 8 else new[1][:2], kd, vd, _i32(table), _i32([0] * S))
    with pytest.raises(B.PaepError, match="PAEP_ERR_SHAPE"):
        B.cache_append(torch.cat([new[0]] * 2), torch.cat([new[1]] * 2), kd, vd, _i32(table), _i32([0] * 2 * S))


def _check_evict(g, lengths, H, Dk, Dv, page, budget, recent, dtype="bf16", order="heads", masses=None, extra=3, max_len=None, out_width=None):
    cap = max(1, max(lengths)) if max_len is None else max_len
    width = max(1, -(-max(lengths) // page))
    wide = -(-budget // page) if out_width is None else out_width
    Bn = len(lengths)
    used = sum(-(-n // page) for n in lengths)
    total = used + Bn * wide + 2
    order_ = g.permutation(total)
    table, at = np.full((Bn, width), -1, dtype=np.int32), 0
    for b, n in enumerate(lengths):
        m = -(-n // page)
        table[b, :m] = order_[at:at + m]
        at += m
    out_table = order_[at:at + Bn * wide].reshape(Bn, wide).astype(np.int32)
    kp, vp = _storage(g.standard_normal((total, H, page, Dk)), dtype), _storage(g.standard_normal((total, H, page, Dv)), dtype)
    mass = g.random((Bn, H, cap + extra)).astype(np.float32) if masses is None else masses(Bn, H, cap + extra)
    kd, vd = _pages(kp, dtype, order), _pages(vp, dtype, order)
    got = B.cache_evict(kd, vd, _i32(table), _i32(lengths), _to(mass, "f32"), _i32(out_table), budget, recent, max_len=cap)
    torch.cuda.synchronize()
    kept, m_out = np.full((Bn, H, budget), -1), np.zeros_like(mass)
    for b, n in enumerate(lengths):
        n = min(n, cap)
        for h in range(H):
            ids = R.kept_positions(mass[b, h], n, budget, recent)
            kept[b, h, :len(ids)] = ids
            m_out[b, h, :len(ids)] = mass[b, h, ids]
            j = np.arange(len(ids))
            kp[out_table[b, j // page], h, j % page] = kp[table[b, ids // page], h, ids % page]
            vp[out_table[b, j // page], h, j % page] = vp[table[b, ids // page], h, ids % page]
    assert np.array_equal(_np(got.kept), kept)
    assert _np(got.lengths).tolist() == [min(n, cap, budget) for n in lengths]
    assert np.array_equal(_np(got.mass), m_out, equal_nan=True)
    assert np.array_equal(_np(kd), kp) and np.array_equal(_np(vd), vp)


@pytest.mark.parametrize("budget,recent", [(1, 0), (1, 1), (7, 3), (64, 0), (64, 64), (200, 16), (1000, 1)])
def test_evict_budgets(budget, recent):
    _check_evict(np.random.default_rng(budget), [0, 1, 7, 8, 63, 64, 65, 333, 1500], 2, 64, 64, 16, budget, recent)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Dk,Dv,page,order", [(1, 8, 8, 1, "heads"), (3, 72, 128, 4, "slots"), (8, 128, 64, 32, "heads"), (1, 256, 256, 128, "slots")])
def test_evict_layouts(H, Dk, Dv, page, order, dtype):
    _check_evict(np.random.default_rng(Dk), [400, 31, 129], H, Dk, Dv, page, 100, 9, dtype, order)


def test_evict_equal_and_special_masses():
    g = np.random.default_rng(3)

    def special(Bn, H, n):
        m = g.choice(np.array([0.0, -0.0, 1.0, 1.0, 2.5, np.inf, np.nan, -np.inf, -1.0, 1e-45, 2.0 ** -126], dtype=np.float32), (Bn, H, n))
        m[0, 0] = 0.0                                     # all equal: the lowest positions
        m[1, 0] = np.nan
        return m.astype(np.float32)
    for budget, recent in ((50, 5), (301, 0), (700, 100)):
        _check_evict(g, [1100, 900, 701], 2, 16, 16, 8, budget, recent, masses=special)


@pytest.mark.parametrize("n,budget,recent", [(40001, 4096, 256), (70007, 1000, 0), (33000, 32999, 100)])
def test_evict_long(n, budget, recent):
    """Lengths past what a workgroup holds at once."""
    _check_evict(np.random.default_rng(n), [n, 17], 1, 16, 16, 64, budget, recent)


def test_evict_cut_at_max_len_and_skipped_pages():
    _check_evict(np.random.default_rng(4), [500, 90], 2, 32, 32, 16, 64, 8, max_len=300)
    g = np.random.default_rng(5)
    kp = _to(g.standard_normal((12, 1, 4, 8)), "f32")
    vp, before = kp.clone(), kp.clone()
    mass = torch.arange(16, device="cuda", dtype=torch.float32).view(1, 1, 16)
    table, out_table = _i32([[0, -1, 99, 3]]), _i32([[8, -1, 10]])
    got = B.cache_evict(kp, vp, table, _i32([16]), mass, out_table, 12, 4)
    torch.cuda.synchronize()
    assert _np(got.kept)[0, 0].tolist() == list(range(4, 16))
    want = _np(before)
    want[10] = want[3]                                    # positions 12..15; 4..11 stand on no page, and so would 4..7 of the new ones
    assert np.array_equal(_np(kp), want) and np.array_equal(_np(vp), want)
    out = B.Eviction(got.lengths, got.kept, mass)
    with pytest.raises(ValueError):
        B.cache_evict(kp, vp, table, _i32([16]), mass, out_table, 12, 4, out=out)
    with pytest.raises(B.PaepError, match="PAEP_ERR_SHAPE"):
        B.cache_evict(kp, vp, table, _i32([16]), mass, out_table, 13, 4)


def test_attention_before_and_after_eviction_and_append():
    """Evicting what had no weight changes nothing; the token appended afterwards is attended."""
    g = np.random.default_rng(6)
    H, G, D, page, n, budget = 2, 4, 64, 16, 300, 128
    kp, vp, table = _cache(g, [n], H, D, D, page, "bf16", spare=budget // page + 3)
    kp, vp = np.nan_to_num(kp), np.nan_to_num(vp)
    live = g.permutation(n - 8)[:budget - 8]
    far = np.setdiff1d(np.arange(n - 8), live)
    q = np.abs(_storage(g.standard_normal((1, H * G, D)), "bf16")) + 0.5
    q = _storage(q, "bf16")
    kp[table[0, far // page], :, far % page] = -100.0     # scores so low that their weight is 0
    kd, vd, t, mass = _pages(kp, "bf16", "heads"), _pages(vp, "bf16", "heads"), _i32(table), torch.zeros((1, H, n), device="cuda")
    before = B.attend(_to(q, "bf16"), kd, vd, t, _i32([n]), mass=mass, max_len=n, want_lse=True)
    free = [p for p in range(kp.shape[0]) if p not in set(table.ravel().tolist())][:budget // page + 1]
    new_table = _i32([free])
    ev = B.cache_evict(kd, vd, t, _i32([n]), mass, new_table, budget, 8, max_len=n)
    torch.cuda.synchronize()
    assert sorted(_np(ev.kept)[0, 0].tolist()) == sorted(live.tolist() + list(range(n - 8, n)))
    after = B.attend(_to(q, "bf16"), kd, vd, new_table, ev.lengths, want_lse=True)
    torch.cuda.synchronize()
    assert np.allclose(_np(after.out), _np(before.out), rtol=2 ** -7, atol=1e-3) and np.allclose(_np(after.lse), _np(before.lse), atol=1e-4)
    # a token whose key matches the query best takes all the weight
    k = _to(np.full((1, H, D), 50.0), "bf16")
    v = _to(g.standard_normal((1, H, D)), "bf16")
    B.cache_append(k, v, kd, vd, new_table, ev.lengths)
    last = B.attend(_to(q, "bf16"), kd, vd, new_table, ev.lengths + 1)
    torch.cuda.synchronize()
    assert torch.equal(last.out.view(1, H, G, D), v.view(1, H, 1, D).expand(1, H, G, D))


# ---- the expert layer ----

def _moe_inputs(g, T, d, f, E, k, dtype):
    """Weights, and tokens whose first k + 1 scores stand apart (drawn again until they do)."""
    Wg = _storage(g.standard_normal((E, d)) / np.sqrt(d), dtype)
    W13 = _storage(g.standard_normal((E, 2 * f, d)) / np.sqrt(d), dtype)
    W2 = _storage(g.standard_normal((E, d, f)) / np.sqrt(f), dtype)
    x = np.zeros((T, d), dtype=np.float32)
    for t in range(T):
        for _ in range(100):
            x[t] = _storage(g.standard_normal(d) * 1.5, dtype)
            z = np.sort(Wg.astype(np.float64) @ x[t])[::-1][:k + 1]
            if len(z) < 2 or (z[:-1] - z[1:]).min() > 1e-4:
                break
    return x, Wg, W13, W2


def _check_moe(g, T, d, f, E, k, dtype, act="silu", prob="softmax", residual=False, bias=False, inplace=False):
    x, Wg, W13, W2 = _moe_inputs(g, T, d, f, E, k, dtype)
    bg = _storage(g.standard_normal(E) * 0.0 + np.arange(E) % 3, dtype) if bias else None      # whole numbers: the gaps stay
    z = x.astype(np.float64) @ Wg.astype(np.float64).T + (0 if bg is None else bg)
    if bg is not None:
        top = -np.sort(-z, axis=1)[:, :k + 1]
        assert top.shape[1] < 2 or (top[:, :-1] - top[:, 1:]).min() > 1e-6
    idx, probs = R.select(z, k, prob)
    res = _storage(g.standard_normal((T, d)), dtype) if residual else None
    for e in set(range(E)) - set(idx.ravel().tolist()):   # experts that nobody picked are not looked at
        W13[e], W2[e] = np.nan, np.nan
    y, tol = R.experts(x, W13, W2, idx, probs, act, res, dtype == "bf16")
    counts = torch.full((E,), 5, dtype=torch.int32, device="cuda")
    rd = None if res is None else _to(res, dtype)
    out = B.MoeOutput(rd, torch.empty((T, k), dtype=torch.int32, device="cuda"), torch.empty((T, k), device="cuda")) if inplace else None
    got = B.moe_layer(_to(x, dtype), _to(Wg, dtype), _to(W13, dtype), _to(W2, dtype), k, bg=None if bg is None else _to(bg, dtype),
                      act=act, prob=prob, residual=rd, counts=counts, out=out)
    torch.cuda.synchronize()
    assert np.array_equal(_np(got.idx), idx)
    assert np.allclose(_np(got.probs), probs, rtol=2e-5, atol=1e-7)
    assert np.array_equal(_np(counts), 5 + np.bincount(idx.ravel(), minlength=E))
    # the probabilities enter as the kernel has them: 2e-5 of every term at most
    off = np.abs(_np(got.y).astype(np.float64) - y)
    slack = 2e-5 * R.experts(x, W13, W2, idx, probs, act, None, False)[1] + 2e-5 * np.abs(y - (0 if res is None else res)).max()
    assert (off <= tol + slack).all(), (off / (tol + slack)).max()
    return got, (x, W13, W2, idx, probs)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,f,E,k", [(1, 8, 8, 1, 1), (1, 2048, 136, 16, 2), (2, 264, 40, 5, 5), (3, 72, 8, 100, 8), (15, 200, 104, 7, 2),
                                       (16, 1000, 64, 64, 6), (17, 512, 200, 3, 1), (31, 96, 72, 33, 4), (33, 256, 96, 128, 8), (48, 64, 24, 256, 3),
                                       (64, 136, 48, 16, 2), (64, 64, 64, 2, 1), (5, 32, 16, 40, 32), (64, 40, 24, 48, 32), (1, 1024, 704, 1024, 8)])
def test_moe_layer_shapes(T, d, f, E, k, dtype):
    _check_moe(np.random.default_rng(T * 31 + d), T, d, f, E, k, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act,prob,residual,bias,inplace", [("none", "softmax_topk", True, False, False), ("gelu", "sigmoid", False, True, False),
                                                            ("silu", "softmax_topk", True, True, True)])
@pytest.mark.parametrize("T", [1, 9, 40])
def test_moe_layer_options(T, act, prob, residual, bias, inplace, dtype):
    _check_moe(np.random.default_rng(T), T, 192, 88, 12, 3, dtype, act, prob, residual, bias, inplace)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_moe_experts_with_a_given_selection(dtype):
    g = np.random.default_rng(21)
    T, d, f, E, k = 37, 160, 56, 24, 4
    x, _, W13, W2 = _moe_inputs(g, T, d, f, E, 1, dtype)
    idx = g.integers(-2, E + 2, (T, k)).astype(np.int32)  # ids that are none, ids that stand twice
    idx[3], idx[4], idx[5] = -1, 7, [7, 7, -1, 8]
    idx[6:] = np.where(idx[6:] == 9, 10, idx[6:])         # expert 9: nobody
    idx[:3] = np.where(idx[:3] == 9, 10, idx[:3])
    W13[9], W2[9] = np.nan, np.nan
    probs = g.random((T, k)).astype(np.float32)
    probs[(idx < 0) | (idx >= E)] = np.nan                # not looked at
    res = _storage(g.standard_normal((T, d)), dtype)
    y, tol = R.experts(x, W13, W2, idx, np.where(np.isnan(probs), 0, probs), "silu", res, dtype == "bf16")
    dev = [_to(x, dtype), _to(W13, dtype), _to(W2, dtype), _i32(idx), _to(probs, "f32")]
    got = B.moe_experts(*dev, residual=_to(res, dtype))
    torch.cuda.synchronize()
    assert (np.abs(_np(got) - y) <= tol).all()
    assert np.array_equal(_np(got)[3], res[3])
    # one selection of all tokens, and none at all
    same = _i32(np.full((T, k), 2))
    y, tol = R.experts(x, W13, W2, np.full((T, k), 2), np.full((T, k), 0.25), "gelu", None, dtype == "bf16")
    got = B.moe_experts(*dev[:3], same, torch.full((T, k), 0.25, device="cuda"), act="gelu")
    none = B.moe_experts(*dev[:3], _i32(np.full((T, k), -1)), dev[4])
    torch.cuda.synchronize()
    assert (np.abs(_np(got) - y) <= tol).all() and not none.any()


def test_moe_layer_is_moe_experts_after_its_router_and_repeats_itself():
    g = np.random.default_rng(22)
    x, Wg, W13, W2 = (_to(a, "bf16") for a in _moe_inputs(g, 20, 256, 128, 32, 4, "bf16"))
    a = B.moe_layer(x, Wg, W13, W2, 4)
    b = B.moe_layer(x, Wg, W13, W2, 4)
    y = B.moe_experts(x, W13, W2, a.idx, a.probs)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c = B.moe_layer(x, Wg, W13, W2, 4, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(a.y, b.y) and torch.equal(a.y, y) and torch.equal(a.y, c.y) and torch.equal(a.idx, c.idx) and torch.equal(a.probs, c.probs)
    empty = B.moe_layer(x[:0], Wg, W13, W2, 4)
    assert empty.y.shape == (0, 256) and empty.idx.shape == (0, 4)
    with pytest.raises(ValueError):
        B.moe_layer(x, Wg[:, :8], W13, W2, 4)
    with pytest.raises(TypeError):
        B.moe_layer(x.float(), Wg, W13, W2, 4)
    with pytest.raises(ValueError):
        B.moe_layer(x, Wg, W13.transpose(1, 2), W2, 4)
    with pytest.raises(B.PaepError, match="PAEP_ERR_K"):
        B.moe_layer(x, Wg, W13, W2, 33)
    with pytest.raises(B.PaepError, match="PAEP_ERR_SHAPE"):
        B.moe_layer(x.repeat(4, 1), Wg, W13, W2, 4)
    with pytest.raises(ValueError):
        B.moe_experts(x, W13, W2, a.idx.long(), a.probs)


def test_moe_layer_ties_and_huge_values():
    """Equal scores go to the lower id; activations far out do not overflow."""
    d, f, E, k = 64, 32, 16, 4
    g = np.random.default_rng(23)
    for dtype in ("bf16", "f32"):
        Wg = np.zeros((E, d), dtype=np.float32)
        Wg[5], Wg[11], Wg[3] = 0.5, 0.5, 0.25
        x = np.ones((2, d), dtype=np.float32)
        x[1] = -60.0
        W13 = _storage(g.standard_normal((E, 2 * f, d)), dtype)
        W2 = _storage(g.standard_normal((E, d, f)), dtype)
        got = B.moe_layer(_to(x, dtype), _to(Wg, dtype), _to(W13, dtype), _to(W2, dtype), k, prob="softmax_topk")
        torch.cuda.synchronize()
        assert _np(got.idx).tolist() == [[5, 11, 3, 0], [0, 1, 2, 4]]
        idx, probs = R.select(x.astype(np.float64) @ Wg.T.astype(np.float64), k, "softmax_topk")
        y, tol = R.experts(x, W13, W2, idx, probs, "silu", None, dtype == "bf16")
        assert (np.abs(_np(got.y) - y) <= tol + 2e-5 * np.abs(y).max()).all()


def test_decode_step_in_a_graph():
    """append, attend with mass and the expert layer recorded once, replayed on new inputs."""
    g = np.random.default_rng(24)
    Bn, H, G, D, page, n = 3, 2, 4, 64, 16, 700
    d, E, k, f = 128, 16, 2, 64
    kp, vp, table = _cache(g, [n] * Bn, H, D, D, page, "bf16", width=64, spare=Bn * 64)
    kp, vp = np.nan_to_num(kp), np.nan_to_num(vp)
    free = iter(sorted(set(range(kp.shape[0])) - set(table.ravel().tolist())))
    table = np.array([[p if p >= 0 else next(free) for p in row] for row in table], dtype=np.int32)
    x, Wg, W13, W2 = (_to(a, "bf16") for a in _moe_inputs(g, Bn, d, f, E, k, "bf16"))
    tb = _i32(table)

    def fresh():
        return dict(k=_pages(kp, "bf16", "heads"), v=_pages(vp, "bf16", "heads"), mass=torch.zeros((Bn, H, 1024), device="cuda"),
                    q=torch.zeros((Bn, H * G, D), dtype=torch.bfloat16, device="cuda"), nk=torch.zeros((Bn, H, D), dtype=torch.bfloat16, device="cuda"),
                    pos=_i32([n, n - 50, 3]), x=x.clone(),
                    at=B.Attention(torch.empty((Bn, H * G, D), dtype=torch.bfloat16, device="cuda"), torch.empty((Bn, H * G), device="cuda")),
                    moe=B.MoeOutput(torch.empty_like(x), torch.empty((Bn, k), dtype=torch.int32, device="cuda"), torch.empty((Bn, k), device="cuda")))

    def step(s):
        B.cache_append(s["nk"], s["nk"], s["k"], s["v"], tb, s["pos"], mass=s["mass"])
        s["len"] = s["pos"] + 1
        B.attend(s["q"], s["k"], s["v"], tb, s["len"], mass=s["mass"], max_len=1024, out=s["at"])
        B.moe_layer(s["x"], Wg, W13, W2, k, out=s["moe"])
        s["pos"].add_(1)

    def feed(s, i):
        r = torch.Generator(device="cuda").manual_seed(i)
        for t in (s["q"], s["nk"], s["x"]):
            t.normal_(generator=r)

    eager, rec = fresh(), fresh()
    warm = fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(warm)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(rec)
    for i in range(4):
        feed(eager, i)
        step(eager)
        torch.cuda.synchronize()
        feed(rec, i)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in ((eager["at"].out, rec["at"].out), (eager["at"].lse, rec["at"].lse), (eager["mass"], rec["mass"]), (eager["k"], rec["k"]),
                     (eager["moe"].y, rec["moe"].y), (eager["moe"].idx, rec["moe"].idx), (eager["pos"], rec["pos"])):
            assert torch.equal(a, b), i


def test_example_runs_the_operators_together():
    import importlib.util
    import os
    import sys
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decode_step.py")
    spec = importlib.util.spec_from_file_location("decode_step_example", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    argv, sys.argv = sys.argv, ["decode_step.py", "--steps", "100"]      # past the first eviction
    try:
        assert example.main() > 0.5                          # by chance: 12 of 128
    finally:
        sys.argv = argv
