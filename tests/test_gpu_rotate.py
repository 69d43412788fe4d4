"""Rotation of queries and keys, alone and on the way into a paged cache, against 64-bit forms."""
import numpy as np
import pytest
import torch

import rotate_fourbit_reference as R
from paper_2511_10676_amd import binding as B

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _np(t):
    return t.double().cpu().numpy()


def _i32(*a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def _rows(g, n, heads, D, dtype, pad=0, std=1.5):
    """[n, heads, D], rows `pad` elements further apart than they have to be, heads as well."""
    t = torch.randn((n, heads * (D + pad) + pad), generator=g, device="cuda") * std
    return t.to(dtype)[:, :heads * (D + pad)].unflatten(1, (heads, D + pad))[..., :D]


def _check(got, want, tol, where):
    off = np.abs(_np(got) - want)
    worst = (off - tol).max() if off.size else 0.0
    assert worst <= 0, f"{where}: {worst:.3g} past the bound, error {off.max():.3g}"


SHAPES = [  # n, Hq, Hk, D, rot, pad
    (1, 16, 16, 128, 128, 0), (7, 5, 1, 128, 64, 8), (301, 32, 4, 128, 128, 0), (3, 3, 3, 8, 2, 0), (5, 2, 1, 8, 8, 8), (9, 7, 1, 256, 256, 0),
    (33, 21, 3, 80, 32, 0), (4, 6, 2, 96, 24, 0), (2, 1, 1, 40, 40, 8), (1, 1, 0, 64, 64, 0), (6, 0, 3, 64, 48, 0), (8, 4, 2, 248, 246, 0),
    (64, 9, 9, 72, 16, 0), (11, 2, 2, 16, 16, 0), (2, 1024, 8, 32, 32, 0)]


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("style", ["halves", "pairs"])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_rotate(kind, style, norm, shape):
    n, Hq, Hk, D, rot, pad = shape
    dtype = TYPES[kind]
    g = torch.Generator(device="cuda").manual_seed(hash((shape, norm)) % 1000)
    q, k = (_rows(g, n, h, D, dtype, pad) if h else None for h in (Hq, Hk))
    weights = [1 + 0.3 * torch.randn(D, generator=g, device="cuda").to(dtype) if norm and t is not None else None for t in (q, k)]
    table = B.rotation_table(500, rot)
    pos = torch.randint(0, 500, (n,), generator=g, device="cuda").to(torch.int32)
    if n > 4:
        pos[2], pos[4] = -1, 500                 # at no row of the table: left out
    here = (pos >= 0) & (pos < 500)
    out = B.Rotated(*(None if t is None else torch.full((n, t.shape[1], D + 8), 7.0, dtype=dtype, device="cuda")[..., :D] for t in (q, k)))
    got = B.rotate(q, k, pos, table, style=style, q_weight=weights[0], k_weight=weights[1], out=out)
    assert got is out
    turns = table[pos.clamp(0, 499).long()].cpu().numpy()
    for x, w, y, name in zip((q, k), weights, got, "qk"):
        if x is None:
            assert y is None
            continue
        want, tol = R.rotate(_np(x), None if w is None else _np(w), turns, style, float(np.float32(1e-6)), kind)
        keep = here.cpu().numpy()
        _check(y[here], want[keep], tol[keep], name)
        assert bool((y[~here] == 7.0).all())
        assert bool((y.as_strided((n, x.shape[1], 8), y.stride(), D) == 7.0).all())           # what lies between rows
    fresh = B.rotate(q, k, pos.clamp(0, 499), table, style=style, q_weight=weights[0], k_weight=weights[1])
    same = B.Rotated(q, k)
    B.rotate(q, k, pos.clamp(0, 499), table, style=style, q_weight=weights[0], k_weight=weights[1], out=same)
    for a, b in zip(fresh, same):
        assert a is None or torch.equal(a, b)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("D,rot", [(64, 64), (96, 24)])
def test_rotate_rows_at_the_ends_of_the_numbers(kind, D, rot):
    """Squares that leave the range of fp32, heads of zeros, infinities and NaN, each in its own row alone."""
    dtype, g = TYPES[kind], torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn((1, 9, D), generator=g, device="cuda")
    x[0, 1] *= 1e37 / x[0, 1].abs().max()
    x[0, 2] *= 1e-30
    x[0, 3] = 0.0
    x[0, 4, 5] = float("inf")
    x[0, 5, 5] = float("nan")
    x[0, 6] *= 1e-36
    x[0, 7, ::2] *= 1e20
    x = x.to(dtype)
    weight = torch.ones(D, dtype=dtype, device="cuda")
    table = B.rotation_table(100, rot)
    for eps in (1e-6, 1e-37):
        got = B.rotate(x, None, _i32(63), table, q_weight=weight, eps=eps).q
        want, tol = R.rotate(_np(x), _np(weight), table[63:64].cpu().numpy(), "halves", float(np.float32(eps)), kind)
        fine = [0, 1, 2, 3, 6, 7, 8]
        _check(got[:, fine], want[:, fine], tol[:, fine], "finite rows")
        assert bool((got[0, 3] == 0).all()) and bool(got[0, 5].isnan().all())
        rest = torch.ones(D, dtype=torch.bool, device="cuda")
        rest[[5, rot // 2 + 5]] = False
        assert bool((got[0, 4, rest] == 0).all()) and not bool(got[0, 4, 5].isfinite())
    plain = B.rotate(x, None, _i32(63), table).q                    # no norm: only its own pair
    want, tol = R.rotate(_np(x), None, table[63:64].cpu().numpy(), "halves", 0.0, kind)
    fine = np.isfinite(want)
    assert np.array_equal(fine, np.isfinite(_np(plain)))
    _check(torch.where(plain.isfinite(), plain, 0), np.where(fine, want, 0), np.where(fine, tol, 0), "no norm")


def _cache(g, pages, H, ps, width, dtype, order):
    t = torch.randn((pages, H, ps, width) if order == "heads" else (pages, ps, H, width), generator=g, device="cuda").to(dtype)
    return t if order == "heads" else t.transpose(1, 2)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("style,norm,D,Dv,rot", [("halves", True, 128, 128, 128), ("pairs", False, 80, 256, 32), ("halves", True, 96, 64, 24),
                                                 ("halves", False, 8, 128, 8), ("pairs", True, 256, 8, 250)])
@pytest.mark.parametrize("ps,order", [(16, "heads"), (1, "slots"), (64, "slots")])
def test_rotate_append_is_rotate_and_append(kind, style, norm, D, Dv, rot, ps, order):
    dtype, g = TYPES[kind], torch.Generator(device="cuda").manual_seed(11)
    n, Hq, H, S, pages = 23, 6, 2, 5, 40
    q, k, v = _rows(g, n, Hq, D, dtype), _rows(g, n, H, D, dtype, 8), _rows(g, n, H, Dv, dtype, 16)
    weights = [torch.randn(D, generator=g, device="cuda").to(dtype) if norm else None for _ in range(2)]
    kp, vp = _cache(g, pages, H, ps, D, dtype, order), _cache(g, pages, H, ps, Dv, dtype, order)
    width = 8
    table = torch.randperm(pages, generator=g, device="cuda")[:S * width].view(S, width).to(torch.int32).contiguous()
    table[1, 3], table[2, 0] = -1, pages                            # pages that are none
    seq = torch.arange(n, device="cuda").remainder(S).to(torch.int32)
    pos = (torch.arange(n, device="cuda") // S * 3 % (width * ps)).to(torch.int32)
    seq[3], seq[4], pos[5], pos[6] = -1, S, -1, width * ps          # no sequence, no position
    angles = torch.randint(0, 300, (n,), generator=g, device="cuda").to(torch.int32)
    angles[7], angles[8] = -5, 300                                  # at no row of the table
    turns = B.rotation_table(300, rot)
    kw = dict(style=style, q_weight=weights[0], k_weight=weights[1], eps=1e-5)
    mass = torch.rand((S, H, 16), generator=g, device="cuda")
    kp2, vp2, mass2 = (t.clone(memory_format=torch.preserve_format) for t in (kp, vp, mass))
    out = torch.full((n, Hq, D), 3.0, dtype=dtype, device="cuda")
    got = B.rotate_append(q, k, v, kp, vp, table, pos, turns, sequences=seq, angles=angles, mass=mass, out=out, **kw)
    want = B.Rotated(torch.full_like(out, 3.0), k.clone().contiguous())
    B.rotate(q, k, angles, turns, out=want, **kw)
    left_out = (angles < 0) | (angles >= 300)
    seq2 = torch.where(left_out, -1, seq)
    B.cache_append(want.k, v.contiguous(), kp2, vp2, table, pos, sequences=seq2, mass=mass2)
    assert torch.equal(got, want.q) and torch.equal(kp, kp2) and torch.equal(vp, vp2) and torch.equal(mass, mass2)
    assert bool((got[left_out] == 3.0).all())
    # a token per sequence, positions that are the angles
    pos = torch.randint(0, width * ps, (S,), generator=g, device="cuda").to(torch.int32)
    turns = B.rotation_table(width * ps, rot)
    got = B.rotate_append(q[:S], k[:S], v[:S], kp, vp, table, pos, turns, **kw)
    want = B.rotate(q[:S], k[:S], pos, turns, **kw)
    B.cache_append(want.k, v[:S].contiguous(), kp2, vp2, table, pos)
    assert torch.equal(got, want.q) and torch.equal(kp, kp2) and torch.equal(vp, vp2)


def test_rotate_append_of_nothing_and_into_no_sequence():
    g = torch.Generator(device="cuda").manual_seed(1)
    kp, vp, turns = torch.zeros((4, 2, 16, 32), device="cuda"), torch.zeros((4, 2, 16, 32), device="cuda"), B.rotation_table(64, 32)
    x = _rows(g, 0, 2, 32, torch.float32)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    table = torch.empty((0, 4), dtype=torch.int32, device="cuda")
    assert B.rotate_append(x, x, x, kp, vp, table, none, turns).shape == (0, 2, 32)
    assert B.rotate(x, x, none, turns).k.shape == (0, 2, 32)
    x = _rows(g, 3, 2, 32, torch.float32)
    got = B.rotate_append(x, x, x, kp, vp, table, _i32(1, 2, 3), turns, sequences=_i32(0, 0, 0))
    assert torch.equal(got, B.rotate(x, x, _i32(1, 2, 3), turns).q) and not bool(kp.any())


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_offsets_past_32_bits(kind):
    dtype, g = TYPES[kind], torch.Generator(device="cuda").manual_seed(2)
    far = (9 << 29) // (2 if kind == "bf16" else 4)                 # elements of 4.5 GiB
    big = torch.empty(far + 4096, dtype=dtype, device="cuda")
    x = big.as_strided((2, 2, 128), (far, 128, 1))
    x.copy_(torch.randn((2, 2, 128), generator=g, device="cuda"))
    turns, pos = B.rotation_table(10, 128), _i32(3, 9)
    want = B.rotate(x.contiguous(), None, pos, turns).q
    assert torch.equal(B.rotate(x, None, pos, turns).q, want)
    pools = big.as_strided((2, 1, 16, 128), (far, 128, 128, 1))
    k = x[:, :1].contiguous()
    B.rotate_append(k, k, k, pools, pools.clone(), _i32([1], [0]), _i32(3, 9), turns)
    assert torch.equal(pools[1, 0, 3], want[0, 0]) and torch.equal(pools[0, 0, 9], want[1, 0])
    del big, x, pools
    torch.cuda.empty_cache()


def test_many_tokens_and_positions_far_out():
    g = torch.Generator(device="cuda").manual_seed(6)
    n = 70001
    q, k = _rows(g, n, 3, 64, torch.bfloat16), _rows(g, n, 1, 64, torch.bfloat16)
    turns = B.rotation_table(1 << 20, 64, base=1e6)
    pos = torch.randint(0, 1 << 20, (n,), generator=g, device="cuda").to(torch.int32)
    got = B.rotate(q, k, pos, turns)
    for x, y in ((q, got.q), (k, got.k)):
        want, tol = R.rotate(_np(x), None, turns[pos.long()].cpu().numpy(), "halves", 1e-6, "bf16")
        _check(y, want, tol, "rows")


@pytest.mark.parametrize("kind,n", [("bf16", 8200), ("f32", 4111)])
def test_results_written_past_the_caches_are_the_same(kind, n):
    """Calls large enough for that, in place too, and their rows in a smaller call."""
    g = torch.Generator(device="cuda").manual_seed(8)
    q, k = _rows(g, n, 32, 128, TYPES[kind]), _rows(g, n, 2, 128, TYPES[kind])
    w, turns = torch.randn(128, generator=g, device="cuda").to(TYPES[kind]), B.rotation_table(n, 128)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    pos[7] = -1
    out = B.Rotated(torch.zeros_like(q), torch.zeros_like(k))
    B.rotate(q, k, pos, turns, q_weight=w, k_weight=w, out=out)
    part = slice(n - 600, n)
    few = B.rotate(q[part], k[part], pos[part].contiguous(), turns, q_weight=w, k_weight=w)
    assert torch.equal(out.q[part], few.q) and torch.equal(out.k[part], few.k) and not bool(out.q[7].any())
    want, tol = R.rotate(_np(q[:300]), _np(w), turns[pos[:300].clamp(min=0).long()].cpu().numpy(), "halves", float(np.float32(1e-6)), kind)
    want[7] = 0
    _check(out.q[:300], want, tol, "rows")
    seventh = q[7].clone()
    B.rotate(q, k, pos, turns, q_weight=w, k_weight=w, out=B.Rotated(q, k))
    out.q[7] = seventh
    assert torch.equal(q, out.q)


def test_python_calls_refuse():
    q, k, turns = torch.zeros((3, 4, 32), device="cuda"), torch.zeros((3, 2, 32), device="cuda"), B.rotation_table(8, 32)
    pos, w = _i32(0, 1, 2), torch.ones(32, device="cuda")
    kp = torch.zeros((4, 2, 16, 32), device="cuda")
    table = _i32([0], [1], [2])
    bad = [
        lambda: B.rotate(q, k.bfloat16(), pos, turns), lambda: B.rotate(q, k[:2], pos, turns), lambda: B.rotate(q, k[..., :24], pos, turns),
        lambda: B.rotate(q.transpose(1, 2), None, pos, turns), lambda: B.rotate(q, k, pos.long(), turns), lambda: B.rotate(q, k, pos[:2], turns),
        lambda: B.rotate(q, k, pos, turns.double()), lambda: B.rotate(q, k, pos, turns[0]), lambda: B.rotate(q, k, pos, turns.cpu()),
        lambda: B.rotate(q, k, pos, turns[:, ::2]), lambda: B.rotate(q, None, pos, turns, k_weight=w), lambda: B.rotate(q, k, pos, turns, q_weight=w[:16]),
        lambda: B.rotate(q, k, pos, turns, q_weight=w.bfloat16()), lambda: B.rotate(q, k, pos, turns, out=B.Rotated(q, None)),
        lambda: B.rotate(q, k, pos, turns, out=B.Rotated(q, q)), lambda: B.rotate_append(q, k, k, kp, kp, table, pos, turns, angles=pos[:2]),
        lambda: B.rotate_append(q, k[:, :1], k, kp, kp, table, pos, turns), lambda: B.rotate_append(q, k, k[:, :1], kp, kp, table, pos, turns),
        lambda: B.rotate_append(q.bfloat16(), k.bfloat16(), k.bfloat16(), kp, kp, table, pos, turns),
        lambda: B.rotate_append(q, k, k, kp, kp, table, pos, turns, sequences=pos.long())]
    for call in bad:
        with pytest.raises((ValueError, TypeError)):
            call()
    with pytest.raises(KeyError):
        B.rotate(q, k, pos, turns, style="both")
    for call in (lambda: B.rotate(q, k, pos, turns, eps=0.0), lambda: B.rotate_append(q, k, k, kp, kp.clone(), table[:2].contiguous(), pos, turns),
                 lambda: B.rotate(torch.zeros((3, 4, 30), device="cuda"), None, pos, turns)):
        with pytest.raises(B.PaepError):
            call()
    assert not bool(kp.any())
