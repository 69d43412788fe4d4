"""A key-value cache in 4 bits: written, read and attended to, against 64-bit forms."""
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


class Cache:
    """Pools of random codes and bytes (seldom NaN: never), and a table of scattered pages."""

    def __init__(self, g, B_, H, Dk, Dv, ps, width, order="heads", spare=3, scale_at=127, spread=3):
        pages = B_ * width + spare

        def codes(w):
            shape = (pages, H, ps, w // 2) if order == "heads" else (pages, ps, H, w // 2)
            t = torch.randint(0, 256, shape, generator=g, device="cuda").to(torch.uint8)
            return t if order == "heads" else t.transpose(1, 2)

        def scales(w):
            return torch.randint(scale_at - spread, scale_at + spread + 1, (pages, H, w // 32, ps), generator=g, device="cuda").to(torch.uint8)
        self.kp, self.vp, self.ks, self.vs = codes(Dk), codes(Dv), scales(Dk), scales(Dv)
        self.table = torch.randperm(pages, generator=g, device="cuda")[:B_ * width].view(B_, width).to(torch.int32).contiguous()

    @property
    def tensors(self):
        return self.kp, self.vp, self.ks, self.vs, self.table

    def values(self):
        return [R.values(p.cpu().numpy(), s.transpose(2, 3).cpu().numpy()) for p, s in ((self.kp, self.ks), (self.vp, self.vs))]


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("Dk,Dv,ps,order", [(128, 128, 16, "heads"), (32, 96, 1, "slots"), (256, 32, 8, "heads"), (64, 160, 64, "slots")])
def test_append_rounds_as_defined_and_read_gives_it_back(kind, Dk, Dv, ps, order):
    dtype, g = TYPES[kind], torch.Generator(device="cuda").manual_seed(5)
    n, H, S, width = 41, 3, 6, 9
    c = Cache(g, S, H, Dk, Dv, ps, width, order)
    c.table[1, 2], c.table[4, 0] = -1, c.kp.shape[0]
    x = [torch.randn((n, H * (D + 8)), generator=g, device="cuda") * torch.exp2(torch.randint(-20, 20, (n, 1), generator=g, device="cuda").float())
         for D in (Dk, Dv)]
    k, v = (t.to(dtype).unflatten(1, (H, -1))[..., :-8] for t in x)
    k[0, 0, :32] = torch.arange(32, device="cuda") / 4              # ties, up to 7.75
    k[0, 1, :32] = torch.arange(32, device="cuda") / -8
    k[1, 0], k[1, 1, :32] = 0.0, -0.0
    k[2, 0, 3], k[2, 1, 4], k[2, 2, 5] = float("inf"), -float("inf"), float("nan")
    k[3, 0], k[3, 1] = 3e38, torch.linspace(-3.3e38, 3.3e38, Dk, device="cuda").to(dtype)
    k[4, 0], k[4, 1, ::2] = 1e-39, 3e-38
    v[5, 0, :32] = 7.0
    v[5, 1, 0:32:2], v[5, 1, 1] = 7.0, 7.03125
    seq = torch.arange(n, device="cuda").remainder(S).to(torch.int32)
    pos = (torch.arange(n, device="cuda") // S * 5 % (width * ps)).to(torch.int32)
    seq[7], seq[8], pos[9], pos[10] = -1, S, -1, width * ps
    before = [t.clone() for t in c.tensors]
    B.cache_append_fourbit(k, v, *c.tensors, pos, sequences=seq)
    entry = torch.where((seq >= 0) & (seq < S) & (pos >= 0) & (pos < width * ps), 0, -1)
    table = c.table.cpu().numpy()
    pages = np.array([table[s, p // ps] if e == 0 and 0 <= table[s, p // ps] < c.kp.shape[0] else -1
                      for s, p, e in zip(seq.tolist(), pos.tolist(), entry.tolist())])
    there, slot = pages >= 0, pos.cpu().numpy() % ps
    assert there.sum() < n - 4
    for x, pool, scales, was, was_scales in ((k, c.kp, c.ks, before[0], before[2]), (v, c.vp, c.vs, before[1], before[3])):
        want, byte = R.to_fourbit(x.float().cpu().numpy())
        pool, scales = pool.cpu().numpy(), scales.cpu().numpy()
        got = R.values(pool[pages, :, slot], scales[pages, :, :, slot])
        assert np.array_equal(scales[pages, :, :, slot][there], byte[there])
        assert np.array_equal(got[there], want[there], equal_nan=True)
        touched = np.zeros(pool.shape[:3], bool)
        touched[pages[there], :, slot[there]] = True
        assert np.array_equal(pool[~touched], was.cpu().numpy()[~touched])
        assert np.array_equal(scales.swapaxes(2, 3)[~touched], was_scales.cpu().numpy().swapaxes(2, 3)[~touched])
    for out_kind, out_type in TYPES.items():
        rows = B.cache_read_fourbit(*c.tensors, pos, sequences=seq, dtype=out_type)
        for x, got in ((k, rows.k), (v, rows.v)):
            want, _ = R.to_fourbit(x.float().cpu().numpy())
            assert got.dtype == out_type and np.array_equal(_np(got), np.where(there[:, None, None], want, 0.0), equal_nan=True)
    twice = B.cache_read_fourbit(*c.tensors, _i32(3, 3, 0), sequences=_i32(2, 2, 0), dtype=dtype)
    assert torch.equal(twice.k[0], twice.k[1])
    again = B.cache_read_fourbit(*c.tensors, _i32(3, 3, 0), sequences=_i32(2, 2, 0), out=twice)
    assert again is twice


def test_every_code_and_byte_reads_as_it_is_defined():
    codes = torch.arange(256, device="cuda").to(torch.uint8).view(1, 1, 16, 16).repeat(16, 1, 1, 1)
    scales = torch.arange(256, device="cuda").to(torch.uint8).view(16, 1, 1, 16).clone()
    scales[0, 0, 0, :2], scales[15, 0, 0, 13:15] = 2, 252          # (bytes that no cache holds)
    table = torch.arange(16, dtype=torch.int32, device="cuda").view(1, 16)
    pos, seq = torch.arange(256, dtype=torch.int32, device="cuda"), torch.zeros(256, dtype=torch.int32, device="cuda")
    for dtype in TYPES.values():
        got = B.cache_read_fourbit(codes, codes, scales, scales, table, pos, sequences=seq, dtype=dtype)
        want = R.values(codes.cpu().numpy()[0, 0][pos.cpu().numpy() % 16], scales.cpu().numpy().reshape(256, 1))
        assert np.array_equal(_np(got.k)[:, 0], want, equal_nan=True) and np.array_equal(_np(got.v)[:, 0], want, equal_nan=True)


ATTEND = [  # Dk, Dv, Hq, Hkv, page, order, lengths, starts
    (128, 128, 8, 8, 16, "heads", [151], None),
    (128, 128, 8, 2, 16, "slots", [0, 1, 2, 15, 16, 17, 31, 32, 33, 127, 128, 129, 300], None),
    (64, 64, 7, 1, 64, "heads", [1, 63, 64, 65, 500], [0, 60, 64, 3, 499]),
    (32, 32, 2, 2, 32, "heads", [5, 40, 400], [-3, 39, 17]),
    (96, 160, 21, 3, 32, "slots", [900, 37, 0], [0, 36, 0]),
    (256, 256, 24, 1, 16, "heads", [200, 513], None),
    (192, 128, 40, 1, 128, "heads", [130, 1000], [129, 501]),
    (64, 256, 3, 3, 16, "slots", [77], None),
    (128, 64, 17, 1, 16, "heads", [300], [299]),
    (256, 32, 4, 4, 1, "heads", [1, 70, 33], [0, 3, 40]),
    (32, 128, 6, 2, 2, "slots", [100, 9], None),
    (128, 128, 4, 4, 8, "heads", [1000, 8, 7], [500, 0, 7]),
    (160, 96, 5, 5, 4, "slots", [65], [2]),
    (128, 256, 2, 1, 16, "slots", [2100], [1033]),
    (64, 128, 1, 1, 65536, "heads", [4000], None),
]


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("case", ATTEND, ids=str)
def test_attend(kind, case):
    Dk, Dv, Hq, H, ps, order, lengths, starts = case
    dtype, g = TYPES[kind], torch.Generator(device="cuda").manual_seed(Dk + Dv + Hq)
    width = max(1, -(-max(lengths) // ps)) + 1
    c = Cache(g, len(lengths), H, Dk, Dv, ps, width, order, spare=1)
    if width > 3:
        c.table[0, 1] = -1                                          # a page that is none, and one that is past the pools
        c.table[-1, 2] = c.kp.shape[0]
    q = torch.randn((len(lengths), Hq, Dk + 8), generator=g, device="cuda").to(dtype)[..., :Dk]
    k, v = c.values()
    # what stands in slots that nobody looks at may be anything
    seen = np.zeros((c.kp.shape[0], ps), bool)
    table = c.table.cpu().numpy()
    for b, n in enumerate(lengths):
        p = np.arange(max(0, starts[b] if starts else 0), n)
        e = table[b, p // ps]
        ok = (e >= 0) & (e < c.kp.shape[0])
        seen[e[ok], p[ok] % ps] = True
    dead = torch.from_numpy(~seen).cuda()[:, None, None, :]
    for s in (c.ks, c.vs):
        s.copy_(torch.where(dead, 255, s))
    lens, st = _i32(*lengths), None if starts is None else _i32(*starts)
    got = B.attend_fourbit(q, *c.tensors, lens, starts=st, want_lse=True)
    want, tol = R.attend(_np(q), k, v, table, lengths, starts, float(np.float32(Dk ** -0.5)), width * ps, kind)
    for x, w, t, name in zip(got, want, tol, ("out", "lse")):
        x = _np(x)
        none = ~np.isfinite(w)
        assert np.array_equal(x[none], w[none]), name
        off = np.where(none, 0, np.abs(np.where(none, 0, x) - np.where(none, 0, w)) - t)
        assert off.max() <= 0, f"{name}: {off.max():.3g} past the bound"
    # a bound on the lengths, buffers given, another scale of 0
    need = max(max(lengths), 1)
    again = B.attend_fourbit(q, *c.tensors, lens, starts=st, max_len=need, want_lse=True, out=B.Attention(torch.empty_like(got.out), torch.empty_like(got.lse)))
    assert np.all(np.abs(_np(again.out) - want[0]) <= tol[0])
    flat = B.attend_fourbit(q, *c.tensors, lens, starts=st, scale=0.0)
    want, tol = R.attend(_np(q), k, v, table, lengths, starts, 0.0, width * ps, kind)
    assert np.all(np.abs(_np(flat.out) - want[0]) <= tol[0])


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_attend_over_long_ranges(kind):
    """Hundreds of chunks joined, and page tables that do not fit in LDS at once."""
    g = torch.Generator(device="cuda").manual_seed(9)
    c = Cache(g, 1, 2, 64, 64, 1, 9000, spare=0)
    q = torch.randn((1, 4, 64), generator=g, device="cuda").to(TYPES[kind])
    for c, n, cap in ((c, 8999, 9000), (Cache(g, 1, 2, 64, 64, 32, 4400, spare=0), 140001, 140800)):
        k, v = c.values()
        got = B.attend_fourbit(q, *c.tensors, _i32(n), max_len=cap, want_lse=True)
        want, tol = R.attend(_np(q), k, v, c.table.cpu().numpy(), [n], None, 0.125, cap, kind)
        assert np.all(np.abs(_np(got.out) - want[0]) <= tol[0]) and np.all(np.abs(_np(got.lse) - want[1]) <= tol[1])
        # a bound far above the length: one long chunk walks a table in stretches
        wide = torch.full((1, 4 * c.table.shape[1]), -1, dtype=torch.int32, device="cuda")
        wide[:, :c.table.shape[1]] = c.table
        got = B.attend_fourbit(q, *c.tensors[:4], wide, _i32(n))
        assert np.all(np.abs(_np(got.out) - want[0]) <= tol[0])


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_attend_large_scores_and_values_near_the_largest_number(kind):
    g = torch.Generator(device="cuda").manual_seed(10)
    c = Cache(g, 2, 1, 32, 64, 16, 20, spare=0)
    c.vp.fill_(0x77)                                                # all 6
    c.vs.fill_(252)                                                 # ... times 2^125
    q = torch.zeros((2, 3, 32), device="cuda")
    q[0, 0], q[1, 1] = 1.0, 100.0
    q[0, 2, 0] = 3e38 / 192.0                                       # scores up to the largest number
    q = q.to(TYPES[kind])
    k, v = c.values()
    got = B.attend_fourbit(q, *c.tensors, _i32(300, 17), scale=1.0, want_lse=True)
    want, tol = R.attend(_np(q), k, v, c.table.cpu().numpy(), [300, 17], None, 1.0, 320, kind)
    assert bool(got.out.isfinite().all())
    assert np.all(np.abs(_np(got.out) - want[0]) <= tol[0]) and np.all(np.abs(_np(got.lse) - want[1]) <= tol[1])


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_attend_nan_groups_reach_what_they_belong_to(kind):
    g = torch.Generator(device="cuda").manual_seed(12)
    c = Cache(g, 3, 2, 128, 128, 16, 40, spare=0)
    q = torch.randn((3, 4, 128), generator=g, device="cuda").to(TYPES[kind])
    lens = _i32(600, 600, 600)
    whole = B.attend_fourbit(q, *c.tensors, lens, want_lse=True)
    want, tol = R.attend(_np(q), *c.values(), c.table.cpu().numpy(), [600, 600, 600], None, float(np.float32(128 ** -0.5)), 640, kind)
    c.ks[c.table[0, 20].long(), 1, 3, 5] = 255                      # a key's last 32 dimensions: all of its head
    c.vs[c.table[1, 30].long(), 0, 2, 7] = 255                      # a value's third 32 dimensions: those of its head
    got = B.attend_fourbit(q, *c.tensors, lens, want_lse=True)
    nan = torch.zeros_like(got.out, dtype=torch.bool)
    nan[0, 2:] = True
    nan[1, :2, 64:96] = True
    assert torch.equal(got.out.isnan(), nan) and bool(got.lse[0, 2:].isnan().all())
    assert np.all(np.abs(_np(got.lse[1]) - want[1][1]) <= tol[1][1])        # (no value is in it)
    assert torch.allclose(got.out[~nan].float(), whole.out[~nan].float(), rtol=2 ** -7, atol=1e-6)


def test_attend_bits_of_fp32_queries_and_of_probabilities():
    """Scores of queries whose last bits decide, and an output whose terms cancel."""
    ps, n = 16, 64
    kp = torch.zeros((4, 1, ps, 16), dtype=torch.uint8, device="cuda")
    kp[..., 0] = 0xA2                                               # 1 and -1 in the first two dimensions
    vp = torch.zeros((4, 1, ps, 16), dtype=torch.uint8, device="cuda")
    vp[0, 0, 0, 0], vp[0, 0, 1, 0] = 0x02, 0x0A                     # 1 and -1
    one = torch.full((4, 1, 1, ps), 127, dtype=torch.uint8, device="cuda")
    ks = one.clone()
    ks[0, 0, 0, 1] = 128                                            # position 1 has twice the score
    q = torch.zeros((1, 1, 32), device="cuda")
    q[0, 0, 0], q[0, 0, 1] = 1.0 + 2.0 ** -23 * 4097, 1.0
    table = torch.arange(4, dtype=torch.int32, device="cuda").view(1, 4)
    got = B.attend_fourbit(q, kp, vp, ks, one, table, _i32(2), scale=1.0).out[0, 0, 0].item()
    d = 2.0 ** -23 * 4097                                           # the scores are d and 2 d
    want = -np.tanh(d / 2)
    # exponentials of numbers below 2^-9: 2 units each and in the sum; P in three parts of 8 bits; the difference is exact but for those
    assert abs(got - want) <= 8 * 2.0 ** -24


def test_offsets_past_32_bits():
    g = torch.Generator(device="cuda").manual_seed(3)
    far = 9 << 29
    big = torch.zeros(far + 65536, dtype=torch.uint8, device="cuda")
    pool = big.as_strided((2, 1, 16, 64), (far, 64, 64, 1))
    scales = torch.full((2, 1, 4, 16), 127, dtype=torch.uint8, device="cuda")
    k = torch.randn((2, 1, 128), generator=g, device="cuda").bfloat16()
    table, pos = _i32([1], [0]), _i32(0, 0)
    small = [torch.zeros((2, 1, 16, 64), dtype=torch.uint8, device="cuda") for _ in range(2)]
    B.cache_append_fourbit(k, k, pool, pool.clone(), scales, scales.clone(), table, pos)
    sc = torch.full_like(scales, 127)
    B.cache_append_fourbit(k, k, *small, sc, sc.clone(), table, pos)
    assert torch.equal(pool, small[0]) and torch.equal(sc, scales)
    assert torch.equal(B.cache_read_fourbit(pool, small[1], scales, sc, table, pos).k, B.cache_read_fourbit(*small, scales, sc, table, pos).k)
    q = torch.randn((2, 2, 128), generator=g, device="cuda").bfloat16()
    a = B.attend_fourbit(q, pool, pool, scales, scales, table, _i32(1, 1)).out
    assert torch.equal(a, B.attend_fourbit(q, small[0], small[0], scales, scales, table, _i32(1, 1)).out)
    # slots so far apart that a lane's offset from the first of 16 has more than 31 bits
    pool = big.as_strided((1, 1, 16, 64), (far, far, 1 << 28, 1))
    pool.copy_(torch.randint(0, 256, pool.shape, generator=g, device="cuda").to(torch.uint8))
    one = scales[:1].contiguous()
    a = B.attend_fourbit(q[:1], pool, pool, one, one, _i32([0]), _i32(16)).out
    assert torch.equal(a, B.attend_fourbit(q[:1], pool.contiguous(), pool.contiguous(), one, one, _i32([0]), _i32(16)).out)
    del big, pool
    torch.cuda.empty_cache()


def test_python_calls_refuse():
    kp, ks, table = torch.zeros((4, 2, 16, 32), dtype=torch.uint8, device="cuda"), torch.full((4, 2, 2, 16), 127, dtype=torch.uint8, device="cuda"), _i32([0, 1], [2, 3])
    x, q, pos = torch.ones((2, 2, 64), device="cuda"), torch.zeros((2, 4, 64), device="cuda"), _i32(0, 1)
    c = (kp, kp, ks, ks, table)
    bad = [
        lambda: B.cache_append_fourbit(x.half(), x.half(), *c, pos), lambda: B.cache_append_fourbit(x, x.bfloat16(), *c, pos),
        lambda: B.cache_append_fourbit(x[..., :32], x, *c, pos), lambda: B.cache_append_fourbit(x, x[:, :1], *c, pos),
        lambda: B.cache_append_fourbit(x, x, kp.float(), kp, ks, ks, table, pos), lambda: B.cache_append_fourbit(x, x, kp, kp, ks[..., :8], ks, table, pos),
        lambda: B.cache_append_fourbit(x, x, kp, kp, ks, ks.transpose(2, 3), table, pos), lambda: B.cache_append_fourbit(x, x, kp, kp[:2], ks, ks, table, pos),
        lambda: B.cache_append_fourbit(x, x, *c, pos.long()), lambda: B.cache_append_fourbit(x, x, *c, pos, sequences=pos[:1]),
        lambda: B.cache_append_fourbit(x, x, kp[..., ::2], kp, ks, ks, table, pos),
        lambda: B.cache_read_fourbit(*c, pos, dtype=torch.float16), lambda: B.cache_read_fourbit(*c, pos[:, None]),
        lambda: B.cache_read_fourbit(*c, pos, out=B.CacheRows(x[:1], x)), lambda: B.cache_read_fourbit(*c, pos, out=B.CacheRows(x, x.bfloat16())),
        lambda: B.attend_fourbit(q[:1], *c, pos), lambda: B.attend_fourbit(q[..., :32], *c, pos), lambda: B.attend_fourbit(q, *c, pos.long()),
        lambda: B.attend_fourbit(q, *c, pos, starts=pos[:1]), lambda: B.attend_fourbit(q, *c, pos, max_len=1 << 31),
        lambda: B.attend_fourbit(q, *c, pos, out=B.Attention(x, None)), lambda: B.attend_fourbit(q, *c, pos, workspace=torch.empty(9)),
        lambda: B.attend_fourbit(q.half(), *c, pos)]
    for call in bad:
        with pytest.raises((ValueError, TypeError)):
            call()
    for call in (lambda: B.attend_fourbit(q, *c, pos, max_len=33), lambda: B.attend_fourbit(q[:, :3], *c, pos), lambda: B.attend_fourbit(q, *c, pos, scale=float("inf")),
                 lambda: B.cache_append_fourbit(x.repeat(2, 1, 1), x.repeat(2, 1, 1), *c, _i32(0, 1, 2, 3)), lambda: B.cache_read_fourbit(*c, _i32(0, 1, 2))):
        with pytest.raises(B.PaepError):
            call()
    assert not bool(kp.any())
    none = torch.empty((0, 2), dtype=torch.int32, device="cuda")
    assert B.attend_fourbit(q[:0], kp, kp, ks, ks, none, pos[:0]).out.shape == (0, 4, 64)
    assert not bool(B.cache_read_fourbit(kp, kp, ks, ks, none, pos, sequences=pos).k.any())
    B.cache_append_fourbit(x, x, kp, kp, ks, ks, none, pos, sequences=pos)
    assert not bool(kp.any())


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("n", [4095, 8198])
def test_many_tokens_at_once(kind, n):
    """Threads that work on several tokens each: as one token after the other, the last ones and skipped ones among them."""
    g = torch.Generator(device="cuda").manual_seed(n)
    c = Cache(g, 3, 8, 128, 160, 16, 200, "slots")
    k, v = (torch.randn((n, 8, D), generator=g, device="cuda").to(TYPES[kind]) for D in (128, 160))
    seq, pos = (torch.arange(n, device="cuda") % 3).to(torch.int32), (torch.arange(n, device="cuda") // 3).to(torch.int32)
    pos[5::7] = -1
    B.cache_append_fourbit(k, v, *c.tensors, pos, sequences=seq)
    got = B.cache_read_fourbit(*c.tensors, pos, sequences=seq, dtype=TYPES[kind])
    here = (pos >= 0).cpu().numpy()
    for x, y in ((k, got.k), (v, got.v)):
        want, _ = R.to_fourbit(x.float().cpu().numpy()[here])
        assert np.array_equal(_np(y)[here], want) and not _np(y)[~here].any()


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_attend_more_sequences_than_one_launch_takes(kind):
    g = torch.Generator(device="cuda").manual_seed(21)
    n, ps = 1500, 16
    c = Cache(g, n, 1, 32, 32, ps, 20, spare=0)
    lengths = torch.randint(0, 320, (n,), generator=g, device="cuda").to(torch.int32)
    lengths[1023:1026], lengths[0], lengths[-1] = 320, 0, 0
    starts = torch.where(torch.arange(n, device="cuda") % 3 == 0, lengths // 2, 0).to(torch.int32)
    q = torch.randn((n, 2, 32), generator=g, device="cuda").to(TYPES[kind])
    got = B.attend_fourbit(q, *c.tensors, lengths, starts=starts, want_lse=True)
    want, tol = R.attend(_np(q), *c.values(), c.table.cpu().numpy(), lengths.tolist(), starts.tolist(), float(np.float32(32 ** -0.5)), 320, kind)
    none = ~np.isfinite(want[1])
    lse = _np(got.lse)
    assert np.all(np.abs(_np(got.out) - want[0]) <= tol[0]) and np.array_equal(none, lse == -np.inf)
    assert np.all(np.abs(lse[~none] - want[1][~none]) <= tol[1][~none])


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_attend_joins_more_pieces_than_fit_at_once(kind):
    g = torch.Generator(device="cuda").manual_seed(22)
    c = Cache(g, 2, 1, 64, 96, 64, 2200, spare=0)
    q = torch.randn((2, 3, 64), generator=g, device="cuda").to(TYPES[kind])
    lengths, k_v = [140001, 700], c.values()
    got = B.attend_fourbit(q, *c.tensors, _i32(*lengths), want_lse=True)
    want, tol = R.attend(_np(q), *k_v, c.table.cpu().numpy(), lengths, None, 0.125, 140800, kind)
    assert np.all(np.abs(_np(got.out) - want[0]) <= tol[0]) and np.all(np.abs(_np(got.lse) - want[1]) <= tol[1])
