"""The way into a key-value cache, and a cache held in 4 bits, as timed cases.

A case is one pass through one of these:

* ``rotate``   the position rotation of the queries and keys of some tokens, behind a norm of each head;
* ``place``    the same with the keys and values going into the pages of a cache (``rotate_append``);
* ``append4``  keys and values rounded to 4 bits into the pages of a cache, and what then stands there read back
               (``cache_append_fourbit``, ``cache_read_fourbit``);
* ``read4``    a stretch of such a cache read back (``cache_read_fourbit``);
* ``attend4``  attention of one new token per sequence over such a cache (``attend_fourbit``).

Four bits: 32 neighbours of a row share a power of two, 2^(byte - 127), and each is a sign and one of the magnitudes
0, 0.5, 1, 1.5, 2, 3, 4, 6; the even neighbour stands in a byte's lower half.  The power is the smallest with which none
is more than 7 times it, from 2^-125 to 2^125; each element goes to the nearest number, of two the even code.

With ``own`` false ``run`` computes them in elementary torch operations in 32
bits, with ``own`` true it calls this package.  ``exact`` computes them in 64
bits, head by head and sequence by sequence.
"""
import itertools
import math

import torch

own = False

DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
MAGNITUDE = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
EPS = 1e-6


# ----------------------------------------------------------------------------
# cases
# ----------------------------------------------------------------------------
def _rotate(name, n, Hq, Hk, D, rot=None, style="halves", norm=True, dtype="bf16", far=4096):
    """n tokens at positions up to far; the first rot dimensions are rotated."""
    c = dict(kind="rotate", n=n, Hq=Hq, Hk=Hk, D=D, rot=rot or D, style=style, norm=norm, dtype=dtype, far=far)
    return dict(c, name=name) if name else c


def _place(name, n, per_seq, Hq, Hk, D, page, hi, rot=None, style="halves", norm=True, Dv=None, dtype="bf16", order="heads",
           moved=0):
    """per_seq consecutive tokens of each sequence, behind a history of up to hi positions of which `moved` were evicted."""
    c = dict(kind="place", n=n, per_seq=per_seq, Hq=Hq, Hk=Hk, D=D, Dv=Dv or D, rot=rot or D, style=style, norm=norm, dtype=dtype,
             page=page, hi=hi, order=order, moved=moved)
    return dict(c, name=name) if name else c


def _append4(name, n, per_seq, Hk, D, page, hi, Dv=None, dtype="bf16", order="heads"):
    c = dict(kind="append4", n=n, per_seq=per_seq, Hk=Hk, D=D, Dv=Dv or D, dtype=dtype, page=page, hi=hi, order=order)
    return dict(c, name=name) if name else c


def _read4(name, B, lo, hi, Hk, D, page, Dv=None, dtype="bf16", order="heads"):
    """All positions of B sequences of lo to hi."""
    c = dict(kind="read4", B=B, lo=lo, hi=hi, Hk=Hk, D=D, Dv=Dv or D, dtype=dtype, page=page, order=order)
    return dict(c, name=name) if name else c


def _attend4(name, B, Hq, Hk, D, lo, hi, page, Dv=None, dtype="bf16", order="heads", window=0, lse=False, empty=0):
    """lo, hi: the lengths, spread evenly on a logarithmic scale; empty: every empty-th sequence has length zero;
    window: only so many of the last positions are attended (0: all)."""
    c = dict(kind="attend4", B=B, Hq=Hq, Hk=Hk, D=D, Dv=Dv or D, lo=lo, hi=hi, page=page, dtype=dtype, order=order, window=window,
             lse=lse, empty=empty)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the new token of one conversation, no norms, a key-value head to every query head: latency is all that counts
        _rotate("rotate_token", n=1, Hq=16, Hk=16, D=128, norm=False),
        # a long prompt through norms and rotation
        _rotate("rotate_prompt", n=8191, Hq=32, Hk=4, D=128, far=131072),
        # the new token of every sequence of a batch, straight into the cache
        _place("place_decode", n=61, per_seq=1, Hq=32, Hk=8, D=128, page=16, hi=8192),
        # chunks of two prompts, fp32 storage, neighbours as pairs, a part of each head rotated, positions behind an eviction
        _place("place_chunk", n=4096, per_seq=2048, Hq=21, Hk=3, D=80, rot=32, style="pairs", norm=False, page=16, hi=4096,
               dtype="f32", order="slots", moved=1000),
        # the new token of every sequence of a batch, into 4 bits
        _append4("append4_decode", n=61, per_seq=1, Hk=8, D=128, page=16, hi=8192),
        # chunks of four prompts
        _append4("append4_chunk", n=8192, per_seq=2048, Hk=8, D=128, page=16, hi=4096, order="slots"),
        # a shared beginning of a conversation, back into bf16
        _read4("read4_prefix", B=1, lo=511, hi=511, Hk=8, D=128, page=16),
        # several sessions of another width of key and value, back into fp32
        _read4("read4_sessions", B=5, lo=1000, hi=9001, Hk=4, D=192, Dv=128, page=64, dtype="f32", order="slots"),
        # the first tokens of one short conversation
        _attend4("attend4_short", B=1, Hq=16, Hk=16, D=128, lo=151, hi=151, page=16),
        # one user, a long document, eight query heads to a key-value head
        _attend4("attend4_long", B=1, Hq=32, Hk=4, D=128, lo=131071, hi=131071, page=64, lse=True),
        # a serving batch of long sessions, some slots empty, pages that hold their slots outside their heads
        _attend4("attend4_batch", B=31, Hq=64, Hk=8, D=128, lo=2000, hi=32768, page=16, order="slots", lse=True, empty=15),
        # fp32 queries and results, odd group, narrow heads, a sliding window
        _attend4("attend4_f32_window", B=5, Hq=21, Hk=3, D=96, lo=900, hi=6000, page=32, dtype="f32", window=4096),
    ]


_MOST = 3.0e8               # bytes of attend4_batch


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    Hk = rng.choice([1, 2, 3, 4, 8, 16])
    G = rng.choice([1, 2, 4, 7, 8, 16, 24])
    while Hk * G > 64:
        G = max(1, G // 2)
    return Hk * G, Hk


def draw(rng):
    kind = rng.choice(["rotate", "place", "append4", "read4", "attend4", "attend4"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    order = rng.choice(["heads", "slots"])
    page = rng.choice([1, 8, 16, 16, 32, 64, 128])
    Hq, Hk = _heads(rng)
    per_seq = rng.choice([1, 1, _log_int(rng, 2, 2048)])
    seqs = max(1, _log_int(rng, 1, 4096) // per_seq)
    hi = _log_int(rng, 16, 8192)
    if kind in ("rotate", "place"):
        D = rng.choice([64, 128, 128, 256, 8 * rng.randint(4, 32)])
        rot = rng.choice([D, D, D // 2, 2 * rng.randint(1, D // 2)])
        style, norm = rng.choice(["halves", "halves", "pairs"]), rng.random() < 0.6
        while 2 * seqs * per_seq * (Hq + 2 * Hk) * D * SIZE[dtype] > 0.9 * _MOST:
            seqs, per_seq = (seqs + 1) // 2, per_seq if seqs > 1 else (per_seq + 1) // 2
        if kind == "rotate":
            return _rotate(None, seqs * per_seq, Hq, Hk, D, rot, style, norm, dtype, hi + per_seq)
        while 2 * seqs * (hi + per_seq) * Hk * D * SIZE[dtype] > 4 * _MOST:
            hi = hi // 2 + 1
        return _place(None, seqs * per_seq, per_seq, Hq, Hk, D, page, hi, rot, style, norm, rng.choice([D, D, 64, 128]), dtype, order,
                      rng.choice([0, 0, 500]))
    D = rng.choice([64, 128, 128, 128, 256, 32 * rng.randint(1, 8)])
    Dv = rng.choice([D, D, D, 64, 128])
    if kind == "append4":
        while seqs * per_seq * Hk * (D + Dv) * (2 * SIZE[dtype] + 2) > 0.9 * _MOST:
            seqs, per_seq = (seqs + 1) // 2, per_seq if seqs > 1 else (per_seq + 1) // 2
        while seqs * (hi + per_seq) * Hk * (D + Dv) > 4 * _MOST:
            hi = hi // 2 + 1
        return _append4(None, seqs * per_seq, per_seq, Hk, D, page, hi, Dv, dtype, order)
    B = rng.choice([1, _log_int(rng, 1, 96)])
    hi = _log_int(rng, 1, 131072 if B < 4 else 16384)
    row = Hk * (D + Dv) * (17 / 32 + (SIZE[dtype] if kind == "read4" else 0))
    while B * hi * row > 0.9 * _MOST:
        hi = hi // 2 + 1
    lo = rng.choice([hi, _log_int(rng, 1, hi)])
    if kind == "read4":
        return _read4(None, B, lo, hi, Hk, D, page, Dv, dtype, order)
    return _attend4(None, B, Hq, Hk, D, lo, hi, page, Dv, dtype, order, rng.choice([0, 0, 1 + hi // 3]), rng.random() < 0.5,
                    rng.choice([0, 0, 5]))


def _lengths(case):
    """A case's lengths: fixed by the case, spread evenly over the logarithm of lo..hi in a scattered order."""
    lo, hi, n = case["lo"], case["hi"], case["B"]
    got = [int(round(lo * (hi / lo) ** ((0.61803398875 * (i + 1)) % 1.0))) for i in range(n)]
    got[0] = hi
    if case.get("empty"):
        got = [0 if i % case["empty"] == case["empty"] - 1 else x for i, x in enumerate(got)]
    return got


def _past(case):
    """What each sequence holds before the new tokens."""
    return [(i * 7919) % case["hi"] for i in range(case["n"] // case["per_seq"])]


# ----------------------------------------------------------------------------
# 4 bits, plain
# ----------------------------------------------------------------------------
def _power(e):
    """2^e in fp32, from its bits; e from -126 to 127."""
    return ((e + 127).to(torch.int32) << 23).view(torch.float32)


def _to_fp4(x):
    """[..., D] -> two codes to a byte [..., D / 2], powers [..., D / 32], both uint8."""
    x = x.float().unflatten(-1, (-1, 32))
    m, e = torch.frexp(x.abs().amax(dim=-1))                            # the largest is m 2^e, m in [0.5, 1); 7 2^e = 0.875 2^(e + 3)
    e = torch.where(m > 0.875, e - 2, e - 3)
    e = torch.where(m == 0, -125, e).clamp(-125, 125)
    y = x * _power(-e)[..., None]
    a = y.abs()
    code = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    code = (code + 8 * torch.signbit(y)).to(torch.uint8).flatten(-2).unflatten(-1, (-1, 2))
    return code[..., 0] | code[..., 1] << 4, (e + 127).to(torch.uint8)


def _from_fp4(codes, scales):
    """[..., D / 2], [..., D / 32] -> [..., D] fp32."""
    one = torch.tensor(MAGNITUDE + tuple(-m for m in MAGNITUDE), device=codes.device)
    both = torch.stack([one.repeat(16), one.repeat_interleave(16)], dim=1)
    x = both[codes.to(torch.int32)].flatten(-2).unflatten(-1, (-1, 32))
    return (x * _power(scales.to(torch.int32) - 127)[..., None]).flatten(-2)


# ----------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------
def _tables(g, lengths, page):
    """Page tables over a pool in scattered order, -1 behind a sequence's last page; and the number of pages used."""
    need = [-(-n // page) for n in lengths]
    used = sum(need)
    order = torch.randperm(used, generator=g, device="cuda").to(torch.int32)
    before = torch.tensor([0, *itertools.accumulate(need)][:-1], device="cuda")
    at = torch.arange(max(1, max(need)), device="cuda")
    live = at < torch.tensor(need, device="cuda")[:, None]
    at = before[:, None] + at
    table = torch.where(live, order[at.clamp(max=max(0, used - 1))] if used else -1, -1).to(torch.int32)
    return table.contiguous(), max(1, used)


def _ordered(t, order):
    """Pages [n, Hk, page, width] that lie in memory as the case says."""
    return t if order == "heads" else t.transpose(1, 2).contiguous().transpose(1, 2)


def _pool4(g, pages, case, width):
    """Pages of rounded rows, as earlier calls left them: channels of unequal size."""
    H, ps = case["Hk"], case["page"]
    x = torch.randn((pages, H, ps, width), generator=g, device="cuda")
    x *= torch.exp(0.5 * torch.randn((H, 1, width), generator=g, device="cuda"))
    codes, scales = _to_fp4(x)
    return _ordered(codes, case["order"]), scales.transpose(2, 3).contiguous()


def _turns(case, rows):
    """[rows, rot]: the cosines of the rot / 2 angles of each position, then the sines."""
    rot = case["rot"]
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    a = torch.arange(rows, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.cat([a.cos(), a.sin()], dim=1).float()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dtype = DTYPE[case["dtype"]]
    kind, Hk, D = case["kind"], case["Hk"], case["D"]

    def randn(*shape, std=1.0):
        return torch.randn(shape, generator=g, device="cuda").mul_(std).to(dtype)

    s = dict(case=case)
    if kind in ("rotate", "place"):
        n, Hq = case["n"], case["Hq"]
        Dv = case.get("Dv", D)
        # a fused projection's rows: queries, keys, values side by side
        qkv = randn(n, (Hq + Hk) * D + Hk * Dv, std=1.5)
        s.update(q=qkv[:, :Hq * D].unflatten(1, (Hq, D)), k=qkv[:, Hq * D:(Hq + Hk) * D].unflatten(1, (Hk, D)),
                 v=qkv[:, (Hq + Hk) * D:].unflatten(1, (Hk, Dv)))
        s["q_weight"], s["k_weight"] = ((1 + randn(D, std=0.2), 1 + randn(D, std=0.2)) if case["norm"] else (None, None))
    if kind == "rotate":
        first = torch.randint(0, max(1, case["far"] - n + 1), (1,), generator=g, device="cuda")
        s["pos"] = (first + torch.arange(n, device="cuda") % case["far"]).to(torch.int32)
        s["turns"] = _turns(case, max(case["far"], n))
        return s
    if kind in ("place", "append4"):
        past, per, Dv = _past(case), case["per_seq"], case["Dv"]
        s["table"], pages = _tables(g, [p + per for p in past], case["page"])
        s["pos"] = (torch.tensor(past, device="cuda")[:, None] + torch.arange(per, device="cuda")).reshape(-1).to(torch.int32)
        s["seq"] = None if per == 1 else torch.arange(len(past), device="cuda").repeat_interleave(per).to(torch.int32)
        if kind == "place":
            for name, width in (("k_pages", D), ("v_pages", Dv)):
                pool = torch.empty((pages, Hk, case["page"], width), dtype=dtype, device="cuda").normal_(generator=g)
                s[name] = _ordered(pool, case["order"])
            s["angles"] = s["pos"] + case["moved"] if case["moved"] else None
            s["turns"] = _turns(case, max(past) + per + case["moved"])
            return s
        kv = randn(case["n"], Hk * (D + Dv), std=1.5)
        s.update(k=kv[:, :Hk * D].unflatten(1, (Hk, D)), v=kv[:, Hk * D:].unflatten(1, (Hk, Dv)))
    else:
        lengths = _lengths(case)
        s["table"], pages = _tables(g, lengths, case["page"])
        s["lengths"], s["cap"] = torch.tensor(lengths, dtype=torch.int32, device="cuda"), max(1, max(lengths))
    s["k_pages"], s["k_scales"] = _pool4(g, pages, case, D)
    s["v_pages"], s["v_scales"] = _pool4(g, pages, case, case["Dv"])
    if kind == "read4":
        s["pos"] = torch.cat([torch.arange(n, device="cuda") for n in lengths]).to(torch.int32)
        s["seq"] = torch.repeat_interleave(torch.arange(len(lengths), device="cuda"), s["lengths"].long()).to(torch.int32)
    if kind == "attend4":
        s["q"] = randn(case["B"], case["Hq"], D, std=2.0)
        s["starts"] = (s["lengths"] - case["window"]).clamp(min=0) if case["window"] else None
    return s


# ----------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------
def _run_own(s):
    from paper_2511_10676_amd import binding as B
    case = s["case"]
    cache = [s[n] for n in ("k_pages", "v_pages", "k_scales", "v_scales", "table") if n in s]
    if case["kind"] == "rotate":
        got = B.rotate(s["q"], s["k"], s["pos"], s["turns"], style=case["style"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS)
        return [got.q, got.k]
    if case["kind"] == "place":
        q = B.rotate_append(s["q"], s["k"], s["v"], *cache, s["pos"], s["turns"], sequences=s["seq"], angles=s["angles"],
                            style=case["style"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS)
        return [q, s["k_pages"], s["v_pages"]]
    if case["kind"] == "attend4":
        got = B.attend_fourbit(s["q"], *cache, s["lengths"], starts=s["starts"], max_len=s["cap"], want_lse=case["lse"])
        return [x for x in (got.out, got.lse) if x is not None]
    if case["kind"] == "append4":
        B.cache_append_fourbit(s["k"], s["v"], *cache, s["pos"], sequences=s["seq"])
    got = B.cache_read_fourbit(*cache, s["pos"], sequences=s["seq"], dtype=DTYPE[case["dtype"]])
    return [got.k, got.v]


def _turned(x, weight, at, case):
    """Norm and rotation of [n, heads, D]; `at`: [n, rot] rows of the table."""
    x, half, rot = x.float(), case["rot"] // 2, case["rot"]
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + EPS) * weight.float()
    c, n = at[:, None, :half], at[:, None, half:]
    if case["style"] == "halves":
        a, b = x[..., :half], x[..., half:rot]
        return torch.cat([a * c - b * n, a * n + b * c, x[..., rot:]], dim=-1)
    a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    return torch.cat([torch.stack([a * c - b * n, a * n + b * c], dim=-1).flatten(-2), x[..., rot:]], dim=-1)


def _plain_rotate(s):
    case, at = s["case"], s["turns"][s["pos"].long()]
    dtype = s["q"].dtype
    return [_turned(s["q"], s["q_weight"], at, case).to(dtype), _turned(s["k"], s["k_weight"], at, case).to(dtype)]


def _where(s):
    """Sequence, page and slot of every token."""
    seq = s["seq"].long() if s["seq"] is not None else torch.arange(s["pos"].shape[0], device="cuda")
    pos = s["pos"].long()
    return s["table"][seq, pos // s["case"]["page"]].long(), pos % s["case"]["page"]


def _plain_place(s):
    case, dtype = s["case"], s["q"].dtype
    at = s["turns"][(s["pos"] if s["angles"] is None else s["angles"]).long()]
    page, slot = _where(s)
    s["k_pages"][page, :, slot] = _turned(s["k"], s["k_weight"], at, case).to(dtype)
    s["v_pages"][page, :, slot] = s["v"]
    return [_turned(s["q"], s["q_weight"], at, case).to(dtype), s["k_pages"], s["v_pages"]]


def _plain_read(s):
    page, slot = _where(s)
    dtype = DTYPE[s["case"]["dtype"]]
    return [_from_fp4(s["k_pages"][page, :, slot], s["k_scales"][page, :, :, slot]).to(dtype),
            _from_fp4(s["v_pages"][page, :, slot], s["v_scales"][page, :, :, slot]).to(dtype)]


def _plain_append(s):
    page, slot = _where(s)
    s["k_pages"][page, :, slot], s["k_scales"][page, :, :, slot] = _to_fp4(s["k"])
    s["v_pages"][page, :, slot], s["v_scales"][page, :, :, slot] = _to_fp4(s["v"])
    return _plain_read(s)


def _dense(pages, scales, table):
    """The positions of every sequence in order: [B, Hk, positions, width]."""
    at = table.long().clamp(min=0)
    return _from_fp4(pages[at], scales.transpose(2, 3)[at]).transpose(1, 2).flatten(2, 3)


def _plain_attend(s):
    case, q = s["case"], s["q"].float()
    B, Hq, D = q.shape
    H = case["Hk"]
    k, v = _dense(s["k_pages"], s["k_scales"], s["table"]), _dense(s["v_pages"], s["v_scales"], s["table"])
    pos = torch.arange(k.shape[2], device="cuda")
    live = pos < s["lengths"][:, None]
    if s["starts"] is not None:
        live = live & (pos >= s["starts"][:, None])
    sc = torch.matmul(q.view(B, H, Hq // H, D), k.transpose(2, 3).contiguous()) * D ** -0.5
    sc = torch.where(live[:, None, None, :], sc, -math.inf)
    top = sc.amax(dim=3, keepdim=True)
    e = torch.exp(sc - torch.where(top == -math.inf, 0.0, top))
    z = e.sum(dim=3, keepdim=True)
    out = torch.matmul(e / torch.where(z > 0, z, 1.0), v).reshape(B, Hq, case["Dv"]).to(s["q"].dtype)
    return [out, (top + torch.log(z)).view(B, Hq)] if case["lse"] else [out]


def run(state):
    if own:
        return _run_own(state)
    return {"rotate": _plain_rotate, "place": _plain_place, "append4": _plain_append, "read4": _plain_read,
            "attend4": _plain_attend}[state["case"]["kind"]](state)


# ----------------------------------------------------------------------------
# the same from the definitions, in 64 bits
# ----------------------------------------------------------------------------
def _exact_turn(x, weight, turns, style):
    """[n, heads, D]: every pair of dimensions as a complex number, multiplied by the position's."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt((x * x).sum(dim=-1, keepdim=True) / x.shape[-1] + EPS) * weight.double()
    half = turns.shape[1] // 2
    by = torch.complex(turns[:, :half].double(), turns[:, half:].double())[:, None]
    out = x.clone()
    i = torch.arange(half, device="cuda")
    one, two = (i, i + half) if style == "halves" else (2 * i, 2 * i + 1)
    z = torch.complex(x[..., one], x[..., two]) * by
    out[..., one], out[..., two] = z.real, z.imag
    return out


def _exact_values(codes, scales):
    """[..., D / 2], [..., D / 32] -> [..., D] in 64 bits, from the code's fields."""
    code = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).long()
    field, last = code >> 1 & 3, (code & 1).double()
    size = torch.where(field == 0, last * 0.5, (1 + last / 2) * 2.0 ** (field.double() - 1))
    return torch.where(code > 7, -size, size) * (2.0 ** (scales.double() - 127)).repeat_interleave(32, dim=-1)


def _exact_rounded(x):
    """[..., D] -> the nearest of the numbers that its group of 32 can hold, ties to the even code."""
    x = x.double().unflatten(-1, (-1, 32))
    most = x.abs().amax(dim=-1, keepdim=True)
    e = torch.full_like(most, -125.0)
    for i in range(-125, 125):
        e = torch.where(most > 7 * 2.0 ** i, i + 1.0, e)
    y = x.abs() / 2.0 ** e
    grid = torch.tensor(MAGNITUDE, dtype=torch.float64, device="cuda")
    near = torch.full_like(y, math.inf)
    got = torch.zeros_like(y)
    for c in (0, 2, 4, 6, 1, 3, 5, 7):                                 # even codes first: an odd one has to be nearer
        d = (y - grid[c]).abs()
        got, near = torch.where(d < near, grid[c], got), torch.minimum(d, near)
    return (torch.copysign(got, x) * 2.0 ** e).flatten(-2)


def _rows4(pages, scales, table, b, n, page):
    """[Hk, n, width] in 64 bits: the first n positions of sequence b."""
    at = table[b, :-(-n // page)].long()
    values = _exact_values(pages[at], scales[at].transpose(2, 3))
    return values.transpose(0, 1).flatten(1, 2)[:, :n]


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "rotate":
        at = s["turns"][s["pos"].long()]
        return [_exact_turn(s["q"], s["q_weight"], at, case["style"]), _exact_turn(s["k"], s["k_weight"], at, case["style"])]
    if kind == "place":
        at = s["turns"][s["pos"].long() + case["moved"]]
        k, v = _exact_turn(s["k"], s["k_weight"], at, case["style"]), s["v"].double()
        k_pages, v_pages = s["k_pages"].double(), s["v_pages"].double()
        seqs = s["seq"].tolist() if s["seq"] is not None else range(case["n"])
        table = s["table"].tolist()
        for i, (q, p) in enumerate(zip(seqs, s["pos"].tolist())):
            page = table[q][p // case["page"]]
            k_pages[page, :, p % case["page"]] = k[i]
            v_pages[page, :, p % case["page"]] = v[i]
        return [_exact_turn(s["q"], s["q_weight"], at, case["style"]), k_pages, v_pages]
    if kind == "append4":
        return [_exact_rounded(s["k"]), _exact_rounded(s["v"])]
    lengths = _lengths(case)
    if kind == "read4":
        return [torch.cat([_rows4(s[p], s[c], s["table"], b, n, case["page"]) for b, n in enumerate(lengths)], dim=1).transpose(0, 1)
                for p, c in (("k_pages", "k_scales"), ("v_pages", "v_scales"))]
    B, Hq, D = s["q"].shape
    H, G = case["Hk"], Hq // case["Hk"]
    out = torch.zeros((B, Hq, case["Dv"]), dtype=torch.float64, device="cuda")
    lse = torch.full((B, Hq), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lengths):
        first = max(0, n - case["window"]) if case["window"] else 0
        if n == first:
            continue
        k = _rows4(s["k_pages"], s["k_scales"], s["table"], b, n, case["page"])[:, first:]
        v = _rows4(s["v_pages"], s["v_scales"], s["table"], b, n, case["page"])[:, first:]
        for h in range(H):
            sc = s["q"][b, h * G:(h + 1) * G].double() @ k[h].t() / math.sqrt(D)
            out[b, h * G:(h + 1) * G] = torch.softmax(sc, dim=1) @ v[h]
            lse[b, h * G:(h + 1) * G] = torch.logsumexp(sc, dim=1)
    return [out, lse] if case["lse"] else [out]


def work(case):
    s, kind, Hk, D = SIZE[case["dtype"]], case["kind"], case["Hk"], case["D"]
    if kind in ("rotate", "place"):
        n, rows = case["n"], case["Hq"] + Hk
        seen = min(n, case["far"]) if kind == "rotate" else len({p + j for p in _past(case) for j in range(case["per_seq"])})
        values = 2 * n * Hk * case["Dv"] * s + 4 * n if kind == "place" else 0
        return {"bytes": 2 * n * rows * D * s + seen * case["rot"] * 4 + 4 * n + values,
                "flops": n * rows * (3.0 * case["rot"] + (4.0 * D if case["norm"] else 0))}
    wide = Hk * (D + case["Dv"])
    if kind == "append4":
        return {"bytes": case["n"] * (wide * (2 * s + 2 * 17 / 32) + 8), "flops": 2.0 * case["n"] * wide}
    lengths = _lengths(case)
    if kind == "read4":
        return {"bytes": sum(lengths) * (wide * (s + 17 / 32) + 8), "flops": 1.0 * sum(lengths) * wide}
    seen = sum(min(n, case["window"]) if case["window"] else n for n in lengths)
    rows = case["B"] * case["Hq"]
    return {"bytes": seen * wide * 17 / 32 + rows * (D + case["Dv"]) * s + (4 * rows if case["lse"] else 0)
            + 4 * sum(-(-n // case["page"]) for n in lengths),
            "flops": 2.0 * seen * case["Hq"] * (D + case["Dv"])}
