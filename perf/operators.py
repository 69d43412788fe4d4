"""The operators of a decode step beside the predictor, as timed cases.

While a layer's experts are fetched, its attention runs, and then the experts
themselves.  A case is one pass through one of the operators for that:

* ``attend``  attention of one new token per sequence over a paged key-value
  cache, with ragged lengths and, where asked for, the log-sum-exp per head and
  the attention weight accumulated per cached position;
* ``append``  new keys and values written into the pages;
* ``evict``   the positions of least accumulated weight dropped and the rest
  moved together into other pages;
* ``moe``     a whole mixture-of-experts layer for a few tokens: router, top-k,
  gated experts, weighted sum.

With ``own`` false ``run`` computes them in elementary torch operations in 32
bits, with ``own`` true it calls this package.  ``exact`` computes them in 64
bits, sequence by sequence and expert by expert.
"""
import itertools
import math

import torch

own = False

DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}


# ----------------------------------------------------------------------------
# cases
# ----------------------------------------------------------------------------
def _attend(name, B, Hq, Hkv, Dk, lo, hi, page, Dv=None, dtype="bf16", order="heads", window=0, mass=False, lse=False,
            empty=0):
    """lo, hi: the lengths, spread evenly on a logarithmic scale; empty: every empty-th sequence has length zero;
    window: only so many of the last positions are attended (0: all); order: whether a page holds its heads or its
    slots as the outer dimension."""
    c = dict(kind="attend", B=B, Hq=Hq, Hkv=Hkv, Dk=Dk, Dv=Dv or Dk, lo=lo, hi=hi, page=page, dtype=dtype, order=order,
             window=window, mass=mass, lse=lse, empty=empty)
    return dict(c, name=name) if name else c


def _append(name, n, per_seq, Hkv, Dk, page, hi, Dv=None, dtype="bf16", order="heads"):
    """n tokens, per_seq consecutive ones of each sequence, behind a history of up to hi positions."""
    c = dict(kind="append", n=n, per_seq=per_seq, Hkv=Hkv, Dk=Dk, Dv=Dv or Dk, page=page, hi=hi, dtype=dtype, order=order)
    return dict(c, name=name) if name else c


def _evict(name, B, Hkv, Dk, lo, hi, page, budget, recent, Dv=None, dtype="bf16", order="heads"):
    c = dict(kind="evict", B=B, Hkv=Hkv, Dk=Dk, Dv=Dv or Dk, lo=lo, hi=hi, page=page, budget=budget, recent=recent,
             dtype=dtype, order=order)
    return dict(c, name=name) if name else c


def _moe(name, T, d, f, E, k, dtype="bf16", act="silu", prob="softmax", residual=False):
    c = dict(kind="moe", T=T, d=d, f=f, E=E, k=k, dtype=dtype, act=act, prob=prob, residual=residual)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the first tokens of one short conversation, a key-value head to every query head: latency is all that counts
        _attend("attend_short", B=1, Hq=16, Hkv=16, Dk=128, lo=151, hi=151, page=16),
        # one user, a long document, eight query heads to a key-value head: few rows, the work lies along the cache
        _attend("attend_long", B=1, Hq=32, Hkv=4, Dk=128, lo=131071, hi=131071, page=64, lse=True),
        # a serving batch of everything from a greeting to a long session, some slots empty, weights accumulated for
        # a later eviction, pages that hold their slots outside their heads
        _attend("attend_ragged_mass", B=61, Hq=32, Hkv=8, Dk=128, lo=17, hi=8192, page=16, order="slots", mass=True,
                lse=True, empty=15),
        # fp32 storage, odd group and width, a sliding window
        _attend("attend_f32_window", B=5, Hq=21, Hkv=3, Dk=80, lo=900, hi=6000, page=32, dtype="f32", window=4096),
        # the new token of every sequence of a batch
        _append("append_decode", n=61, per_seq=1, Hkv=8, Dk=128, page=16, hi=8192),
        # chunks of two prompts, fp32 storage, slots outside heads
        _append("append_chunk", n=4096, per_seq=2048, Hkv=8, Dk=128, page=16, hi=4096, dtype="f32", order="slots"),
        # one long session cut down to what a small card can hold
        _evict("evict_long", B=1, Hkv=4, Dk=128, lo=32749, hi=32749, page=64, budget=4096, recent=256),
        # a batch trimmed to a budget that some of it does not reach
        _evict("evict_batch", B=32, Hkv=8, Dk=128, lo=300, hi=6011, page=16, budget=2048, recent=128, order="slots"),
        # one token through a layer of 128 narrow experts
        _moe("moe_t1", T=1, d=2048, f=768, E=128, k=8, prob="softmax_topk"),
        # a small batch through a layer of few, short experts behind a wide hidden state
        _moe("moe_t16", T=16, d=4096, f=960, E=16, k=2, residual=True),
        # a large, odd batch that wakes every expert
        _moe("moe_t61", T=61, d=2048, f=1408, E=64, k=6),
        # fp32 storage, a few tokens, exact GELU
        _moe("moe_f32", T=7, d=1024, f=704, E=32, k=4, dtype="f32", act="gelu", prob="sigmoid"),
    ]


_MOST = 1.1e9               # bytes of moe_t61


def _log_int(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n + 1 if n == 3072 else n


def _heads(rng):
    Hkv = rng.choice([1, 2, 3, 4, 8, 16])
    G = rng.choice([1, 2, 4, 7, 8, 16, 24])
    while Hkv * G > 64:
        G = max(1, G // 2)
    return Hkv * G, Hkv


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "append", "evict", "moe", "moe", "moe"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind == "moe":
        T = _log_int(rng, 1, 64)
        d = rng.choice([2048, 4096, 8 * rng.randint(32, 380)])
        f = rng.choice([768, 1408, 8 * rng.randint(16, 250)])
        E = rng.choice([16, 64, 128, _log_int(rng, 4, 256)])
        while 3 * E * f * d * SIZE[dtype] > _MOST:
            E = max(4, E // 2)
            f = f if E > 4 else 768
            d = d if E > 4 else 2048
        return _moe(None, T, d, f, E, rng.randint(1, min(E, 8)), dtype, rng.choice(["silu", "silu", "gelu", "none"]),
                    rng.choice(["softmax", "softmax_topk", "sigmoid"]), rng.random() < 0.4)
    Hq, Hkv = _heads(rng)
    Dk = rng.choice([64, 128, 128, 128, 256, 8 * rng.randint(4, 32)])
    Dv = rng.choice([Dk, Dk, Dk, 64, 128])
    page = rng.choice([1, 8, 16, 16, 32, 64, 128])
    order = rng.choice(["heads", "slots"])
    row = Hkv * (Dk + Dv) * SIZE[dtype]
    if kind == "append":
        per_seq = rng.choice([1, 1, _log_int(rng, 2, 2048)])
        seqs = max(1, _log_int(rng, 1, 4096) // per_seq)
        seqs = seqs + 1 if seqs * per_seq == 3072 else seqs
        hi = _log_int(rng, 16, 8192)
        while seqs * (hi + per_seq) * row > 4 * _MOST and hi > 1:
            hi = hi // 2
        return _append(None, seqs * per_seq, per_seq, Hkv, Dk, page, hi, Dv, dtype, order)
    B = rng.choice([1, _log_int(rng, 1, 96)])
    hi = _log_int(rng, 1, 131072 if B < 4 else 16384)
    while B * hi * row > (0.4 * _MOST if kind == "evict" else _MOST):
        hi = hi // 2 + 1
    lo = rng.choice([hi, _log_int(rng, 1, hi)])
    if kind == "attend":
        return _attend(None, B, Hq, Hkv, Dk, lo, hi, page, Dv, dtype, order, rng.choice([0, 0, 1 + hi // 3]), rng.random() < 0.3,
                       rng.random() < 0.5, rng.choice([0, 0, 5]))
    budget = _log_int(rng, 1, max(1, hi))
    return _evict(None, B, Hkv, Dk, lo, hi, page, budget, rng.randint(0, budget), Dv, dtype, order)


def _lengths(case):
    """A case's lengths: fixed by the case, spread evenly over the logarithm of lo..hi in a scattered order."""
    lo, hi, n = case["lo"], case["hi"], case["B"]
    got = [int(round(lo * (hi / lo) ** ((0.61803398875 * (i + 1)) % 1.0))) for i in range(n)]
    got[0] = hi
    if case.get("empty"):
        got = [0 if i % case["empty"] == case["empty"] - 1 else x for i, x in enumerate(got)]
    return got


# ----------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------
def _pool(g, pages, case, width):
    """Pages of unit-variance entries (past keys and values; what an unused page holds is as good as anything)."""
    H, ps = case["Hkv"], case["page"]
    shape = (pages, H, ps, width) if case["order"] == "heads" else (pages, ps, H, width)
    t = torch.empty(shape, dtype=DTYPE[case["dtype"]], device="cuda").normal_(generator=g)
    return t if case["order"] == "heads" else t.permute(0, 2, 1, 3)


def _tables(g, lengths, page, spare=0):
    """Page tables over a pool in scattered order, -1 behind a sequence's last page; and the number of pages used."""
    need = [-(-n // page) for n in lengths]
    used = sum(need)
    order = torch.randperm(used + spare, generator=g, device="cuda").to(torch.int32)
    width = max(1, max(need))
    before = torch.tensor([0, *itertools.accumulate(need)][:-1], device="cuda")
    at = before[:, None] + torch.arange(width, device="cuda")
    live = torch.arange(width, device="cuda") < torch.tensor(need, device="cuda")[:, None]
    table = torch.where(live, order[at.clamp(max=max(0, used - 1))] if used else -1, -1).to(torch.int32)
    return table.contiguous(), order[used:].contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dtype = DTYPE[case["dtype"]]

    def randn(*shape, std=1.0):
        return torch.randn(shape, generator=g, device="cuda").mul_(std).to(dtype)

    if case["kind"] == "moe":
        T, d, f, E, k = (case[n] for n in ("T", "d", "f", "E", "k"))
        Wg = randn(E, d, std=d ** -0.5)
        W13 = torch.empty((E, 2 * f, d), dtype=dtype, device="cuda").normal_(std=d ** -0.5, generator=g)
        W2 = torch.empty((E, d, f), dtype=dtype, device="cuda").normal_(std=f ** -0.5, generator=g)
        # post-norm states with a few outlier channels.  A token two of whose first k + 1 scores are as good as equal has
        # two right selections: it is drawn again
        x = torch.empty((T, d), dtype=dtype, device="cuda")
        redo = torch.ones(T, dtype=torch.bool, device="cuda")
        for _ in range(16):
            h = torch.randn((T, d), generator=g, device="cuda")
            h[:, torch.randperm(d, generator=g, device="cuda")[:max(4, d // 512)]] *= 8.0
            h = (h * h.square().mean(dim=1, keepdim=True).rsqrt()).to(dtype)
            x = torch.where(redo[:, None], h, x)
            top = torch.sort(x.double() @ Wg.double().t(), dim=1, descending=True).values[:, :k + 1]
            redo = (top[:, :-1] - top[:, 1:]).amin(dim=1) < 1e-4 if top.shape[1] > 1 else torch.zeros_like(redo)
        return dict(case=case, x=x, Wg=Wg, W13=W13, W2=W2, residual=randn(T, d) if case["residual"] else None)

    H, Dk, Dv, page = case["Hkv"], case["Dk"], case["Dv"], case["page"]
    if case["kind"] == "append":
        seqs, per = case["n"] // case["per_seq"], case["per_seq"]
        past = [(i * 7919) % case["hi"] for i in range(seqs)]
        table, _ = _tables(g, [p + per for p in past], page)
        pages = int(table.max()) + 1
        pos = (torch.tensor(past, device="cuda")[:, None] + torch.arange(per, device="cuda")).reshape(-1).to(torch.int32)
        seq = torch.arange(seqs, device="cuda").repeat_interleave(per).to(torch.int32)
        # the keys and values as a fused projection leaves them: columns of one row per token
        qkv = randn(case["n"], H * (Dk + Dv))
        return dict(case=case, k=qkv[:, :H * Dk].unflatten(1, (H, Dk)), v=qkv[:, H * Dk:].unflatten(1, (H, Dv)),
                    k_pages=_pool(g, pages, case, Dk), v_pages=_pool(g, pages, case, Dv), table=table, pos=pos,
                    seq=None if per == 1 else seq)

    lengths = _lengths(case)
    B, cap = case["B"], max(1, max(lengths))
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    if case["kind"] == "evict":
        wide = -(-case["budget"] // page)
        table, spare = _tables(g, lengths, page, B * wide)
        # accumulated weight: a few positions hold most of it, many were hardly ever looked at and hold the same
        mass = torch.rand((B, H, cap), generator=g, device="cuda").pow_(8) * 50.0
        mass = torch.where(mass < 1e-3, torch.zeros_like(mass), mass)
        pages = sum(-(-n // page) for n in lengths) + B * wide
        return dict(case=case, k_pages=_pool(g, pages, case, Dk), v_pages=_pool(g, pages, case, Dv), table=table, lengths=lens,
                    mass=mass, out_table=spare.view(B, wide), cap=cap)
    table, _ = _tables(g, lengths, page)
    pages = max(1, sum(-(-n // page) for n in lengths))
    return dict(case=case, q=randn(B, case["Hq"], Dk, std=2.0), k_pages=_pool(g, pages, case, Dk), v_pages=_pool(g, pages, case, Dv),
                table=table, lengths=lens, starts=(lens - case["window"]).clamp(min=0) if case["window"] else None, cap=cap,
                mass=torch.rand((B, H, cap), generator=g, device="cuda") if case["mass"] else None)


# ----------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------
def _run_own(s):
    from paper_2511_10676_amd import binding as B
    case = s["case"]
    if case["kind"] == "attend":
        got = B.attend(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lengths"], starts=s["starts"], max_len=s["cap"],
                       mass=s["mass"], want_lse=case["lse"])
        return [x for x in (got.out, got.lse, s["mass"]) if x is not None]
    if case["kind"] == "append":
        B.cache_append(s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["pos"], sequences=s["seq"])
        return [s["k_pages"], s["v_pages"]]
    if case["kind"] == "evict":
        got = B.cache_evict(s["k_pages"], s["v_pages"], s["table"], s["lengths"], s["mass"], s["out_table"], case["budget"],
                            case["recent"], max_len=s["cap"])
        return [s["k_pages"], s["v_pages"], got.lengths, got.kept, got.mass]
    got = B.moe_layer(s["x"], s["Wg"], s["W13"], s["W2"], case["k"], act=case["act"], prob=case["prob"], residual=s["residual"])
    return [got.y, got.idx, got.probs]


def _dense(pages, table):
    """The positions of every sequence in order: [B, Hkv, positions, width]."""
    t = pages[table.long().clamp(min=0)].transpose(1, 2)
    return t.reshape(t.shape[0], t.shape[1], -1, t.shape[-1])


def _plain_attend(s):
    case, q = s["case"], s["q"].float()
    B, Hq, Dk = q.shape
    H, Dv = case["Hkv"], case["Dv"]
    k, v = _dense(s["k_pages"], s["table"]).float(), _dense(s["v_pages"], s["table"]).float()
    pos = torch.arange(k.shape[2], device="cuda")
    live = pos < s["lengths"][:, None]
    if s["starts"] is not None:
        live = live & (pos >= s["starts"][:, None])
    live = live[:, None, None, :]
    sc = torch.matmul(q.view(B, H, Hq // H, Dk), k.transpose(2, 3).contiguous()) * Dk ** -0.5
    sc = torch.where(live, sc, -math.inf)
    top = sc.amax(dim=3, keepdim=True)
    e = torch.exp(sc - torch.where(top == -math.inf, 0.0, top))
    z = e.sum(dim=3, keepdim=True)
    p = e / torch.where(z > 0, z, 1.0)
    out = [torch.matmul(p, torch.where(live.transpose(2, 3), v, 0.0)).view(B, Hq, Dv).to(s["q"].dtype)]
    if case["lse"]:
        out.append((top + torch.log(z)).view(B, Hq))
    if case["mass"]:
        s["mass"] += p.sum(dim=2)[:, :, :s["cap"]]
        out.append(s["mass"])
    return out


def _plain_append(s):
    page = s["case"]["page"]
    seq = s["seq"].long() if s["seq"] is not None else torch.arange(s["pos"].shape[0], device="cuda")
    pos = s["pos"].long()
    at, slot = s["table"][seq, pos // page].long(), pos % page
    s["k_pages"][at, :, slot] = s["k"]
    s["v_pages"][at, :, slot] = s["v"]
    return [s["k_pages"], s["v_pages"]]


def _plain_evict(s):
    case, mass = s["case"], s["mass"]
    page, budget = case["page"], case["budget"]
    B, H, cap = mass.shape
    lens, pos = s["lengths"].long()[:, None, None], torch.arange(cap, device="cuda")
    # ranks by falling weight, the recent ones before all others, what is not there behind them
    key = torch.where(pos >= lens - case["recent"], math.inf, mass)
    key = torch.where(pos < lens, key, -math.inf)
    rank = torch.sort(torch.sort(key, dim=2, descending=True, stable=True).indices, dim=2).indices
    keep = (rank < budget) & (pos < lens)
    # the kept ones in ascending order, behind them what is dropped
    src = torch.sort((~keep).to(torch.int32), dim=2, stable=True).indices[:, :, :budget]
    src = torch.nn.functional.pad(src, (0, budget - src.shape[2]))
    there = torch.arange(budget, device="cuda") < lens
    j = torch.arange(budget, device="cuda")
    to, slot = s["out_table"].long()[:, None, j // page].expand(B, H, budget), (j % page).expand(B, H, budget)
    head = torch.arange(H, device="cuda")[None, :, None].expand(B, H, budget)
    frm = torch.gather(s["table"].long()[:, None, :].expand(B, H, -1), 2, src // page)
    for_k, for_v = s["k_pages"][frm.clamp(min=0), head, src % page], s["v_pages"][frm.clamp(min=0), head, src % page]
    s["k_pages"][to, head, slot] = torch.where(there[..., None], for_k, s["k_pages"][to, head, slot])
    s["v_pages"][to, head, slot] = torch.where(there[..., None], for_v, s["v_pages"][to, head, slot])
    kept = torch.where(there, src, -1).to(torch.int32)
    got = torch.where(there, torch.gather(mass, 2, src), 0.0)
    got = torch.nn.functional.pad(got, (0, max(0, cap - budget)))[:, :, :cap]
    return [s["k_pages"], s["v_pages"], s["lengths"].clamp(max=budget), kept, got]


def _activation(v, act):
    if act == "silu":
        return v / (1.0 + torch.exp(-v))
    if act == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * 0.5 ** 0.5))
    return v


def _plain_moe(s):
    case, x = s["case"], s["x"].float()
    T, f, E, k = case["T"], case["f"], case["E"], case["k"]
    z = x @ s["Wg"].float().t()
    idx = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :k]
    top = torch.gather(z, 1, idx)
    if case["prob"] == "sigmoid":
        probs = 1.0 / (1.0 + torch.exp(-top))
    else:
        e = torch.exp(top - top[:, :1])
        probs = e / (e.sum(dim=1, keepdim=True) if case["prob"] == "softmax_topk"
                     else torch.exp(z - top[:, :1]).sum(dim=1, keepdim=True))
    if T * k <= E:                                                     # fewer rows than experts: the weights of each row's own
        W13, W2 = s["W13"][idx.reshape(-1)].float(), s["W2"][idx.reshape(-1)].float()
        xs, p = x.repeat_interleave(k, dim=0)[:, :, None], probs.reshape(-1, 1, 1)
    else:                                                              # every expert on every token
        W13, W2 = s["W13"].float(), s["W2"].float()
        xs = x.t().expand(E, -1, T)
        p = torch.zeros_like(z).scatter_(1, idx, probs).t()[:, None, :]
    h = torch.matmul(W13, xs)
    h = _activation(h[:, :f], case["act"]) * h[:, f:] * p
    y = torch.matmul(W2, h)
    y = y[:, :, 0].view(T, k, -1).sum(dim=1) if T * k <= E else y.sum(dim=0).t()
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return [y.to(s["x"].dtype), idx.to(torch.int32), probs]


def run(state):
    if own:
        return _run_own(state)
    return {"attend": _plain_attend, "append": _plain_append, "evict": _plain_evict, "moe": _plain_moe}[state["case"]["kind"]](state)


# ----------------------------------------------------------------------------
# the same from the definitions, in 64 bits
# ----------------------------------------------------------------------------
def _rows(pages, table, b, n, page):
    """[Hkv, n, width]: the first n positions of sequence b."""
    at = table[b, :-(-n // page)].long()
    return torch.cat(list(pages[at]), dim=1)[:, :n] if n else pages[0][:, :0]


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "attend":
        B, Hq, Dk = s["q"].shape
        H, G = case["Hkv"], case["Hq"] // case["Hkv"]
        out = torch.zeros((B, Hq, case["Dv"]), dtype=torch.float64, device="cuda")
        lse = torch.full((B, Hq), -math.inf, dtype=torch.float64, device="cuda")
        mass = s["mass"].double() if case["mass"] else None
        for b, n in enumerate(_lengths(case)):
            first = max(0, n - case["window"]) if case["window"] else 0
            if n == first:
                continue
            k = _rows(s["k_pages"], s["table"], b, n, case["page"])[:, first:].double()
            v = _rows(s["v_pages"], s["table"], b, n, case["page"])[:, first:].double()
            for h in range(H):
                sc = s["q"][b, h * G:(h + 1) * G].double() @ k[h].t() / math.sqrt(Dk)
                p = torch.softmax(sc, dim=1)
                out[b, h * G:(h + 1) * G] = p @ v[h]
                lse[b, h * G:(h + 1) * G] = torch.logsumexp(sc, dim=1)
                if mass is not None:
                    mass[b, h, first:n] += p.sum(dim=0)
        return [x for x in (out, lse if case["lse"] else None, mass) if x is not None]
    if case["kind"] == "append":
        seqs = range(case["n"]) if s["seq"] is None else s["seq"].tolist()
        table = s["table"].tolist()
        for i, (q, p) in enumerate(zip(seqs, s["pos"].tolist())):
            at = table[q][p // case["page"]]
            s["k_pages"][at, :, p % case["page"]] = s["k"][i]
            s["v_pages"][at, :, p % case["page"]] = s["v"][i]
        return [s["k_pages"].double(), s["v_pages"].double()]
    if case["kind"] == "evict":
        B, H, budget, page = case["B"], case["Hkv"], case["budget"], case["page"]
        kept = torch.full((B, H, budget), -1, dtype=torch.int32)
        got = torch.zeros(s["mass"].shape, dtype=torch.float64)
        mass, out_table = s["mass"].cpu().numpy(), s["out_table"]
        for b, n in enumerate(_lengths(case)):
            m = min(n, budget)
            k, v = _rows(s["k_pages"], s["table"], b, n, page), _rows(s["v_pages"], s["table"], b, n, page)
            j = torch.arange(m, device="cuda")
            for h in range(H):
                old = max(0, n - case["recent"]) if n > budget else 0
                best = (-mass[b, h, :old]).argsort(kind="stable")[:max(0, budget - (n - old))]
                at = sorted(best.tolist()) + list(range(old, n))
                kept[b, h, :m] = torch.tensor(at, dtype=torch.int32)
                got[b, h, :m] = torch.from_numpy(mass[b, h, at]).double()
                at = torch.tensor(at, dtype=torch.long, device="cuda")
                s["k_pages"][out_table[b].long()[j // page], h, j % page] = k[h, at]
                s["v_pages"][out_table[b].long()[j // page], h, j % page] = v[h, at]
        lens = torch.tensor([min(n, budget) for n in _lengths(case)], dtype=torch.int32)
        return [s["k_pages"].double(), s["v_pages"].double(), lens, kept, got]
    T, f, k = case["T"], case["f"], case["k"]
    x = s["x"].double()
    z = torch.stack([(s["Wg"].double() * x[t]).sum(dim=1) for t in range(T)])
    idx = z.cpu().numpy().argsort(axis=1, kind="stable")[:, ::-1][:, :k].copy()
    idx = torch.from_numpy(idx).to("cuda")
    top = torch.gather(z, 1, idx)
    probs = {"softmax": lambda: torch.gather(torch.softmax(z, dim=1), 1, idx), "softmax_topk": lambda: torch.softmax(top, dim=1),
             "sigmoid": lambda: torch.sigmoid(top)}[case["prob"]]()
    act = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "none": lambda t: t}[case["act"]]
    y = s["residual"].double() if s["residual"] is not None else torch.zeros_like(x)
    for e in sorted(set(idx.reshape(-1).tolist())):
        t, j = (idx == e).nonzero(as_tuple=True)
        u = x[t] @ s["W13"][e].double().t()
        y.index_add_(0, t, (act(u[:, :f]) * u[:, f:]) @ s["W2"][e].double().t() * probs[t, j][:, None])
    return [y, idx.to(torch.int32), probs]


def work(case):
    s = SIZE[case["dtype"]]
    if case["kind"] == "moe":
        T, d, f, E, k = (case[n] for n in ("T", "d", "f", "E", "k"))
        active = E * (1.0 - (1.0 - k / E) ** T)                       # distinct experts that T tokens pick evenly
        return {"bytes": s * (E * d + active * 3 * f * d + T * d * (3 if case["residual"] else 2)) + 8 * T * k,
                "flops": 2.0 * T * (E * d + 3 * k * f * d)}
    row = case["Hkv"] * (case["Dk"] + case["Dv"]) * s
    if case["kind"] == "append":
        return {"bytes": 2 * case["n"] * row + 8 * case["n"], "flops": 0}
    lengths = _lengths(case)
    if case["kind"] == "evict":
        kept = sum(min(n, case["budget"]) for n in lengths)
        return {"bytes": 2 * kept * row + 4 * case["Hkv"] * (sum(lengths) + case["B"] * (max(lengths) + case["budget"])), "flops": 0}
    seen = sum(min(n, case["window"]) if case["window"] else n for n in lengths)
    rows = case["B"] * case["Hq"]
    return {"bytes": seen * (row + (8 * case["Hkv"] if case["mass"] else 0)) + rows * (case["Dk"] + case["Dv"]) * s
            + (4 * rows if case["lse"] else 0) + 4 * sum(-(-n // case["page"]) for n in lengths),
            "flops": 2.0 * seen * case["Hq"] * (case["Dk"] + case["Dv"])}
