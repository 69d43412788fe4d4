"""Host-side checks of the decode step's operators that need no GPU: every bad argument is refused before any HIP call (the
pointers used here are never dereferenced), and the plain forms that the GPU tests compare with agree with other ways of
computing the same."""
import ctypes

import numpy as np
import pytest
import torch

import decode_step_reference as R
from paper_2511_10676_amd import binding as B

OK, E_NULL, E_SHAPE, E_K, E_DTYPE, E_ALIGN, E_WS, E_HIP, E_UNSUP = range(9)
FAKE = ctypes.c_void_p(0x10000)
ODD = ctypes.c_void_p(0x10008)
HUGE = 1 << 40


def _cache(**kw):
    c = dict(B=2, Hkv=2, Dk=64, Dv=64, page_size=16, n_pages=8, max_pages=4, dtype=B.BF16)
    c.update({n: v for n, v in kw.items() if n in c})
    k = dict(k_page_stride=c["Hkv"] * c["page_size"] * c["Dk"], k_head_stride=c["page_size"] * c["Dk"], k_slot_stride=c["Dk"],
             v_page_stride=c["Hkv"] * c["page_size"] * c["Dv"], v_head_stride=c["page_size"] * c["Dv"], v_slot_stride=c["Dv"])
    c.update(k)
    c.update(kw)
    return B.CacheDesc(**c)


BAD_CACHES = [(dict(dtype=7), E_DTYPE), (dict(B=-1), E_SHAPE), (dict(Hkv=0), E_SHAPE), (dict(Hkv=1025), E_SHAPE),
              (dict(Dk=60), E_SHAPE), (dict(Dk=0), E_SHAPE), (dict(Dk=264), E_SHAPE), (dict(Dv=12), E_SHAPE), (dict(Dv=264), E_SHAPE),
              (dict(page_size=0), E_SHAPE), (dict(page_size=24), E_SHAPE), (dict(page_size=1 << 17), E_SHAPE), (dict(n_pages=0), E_SHAPE),
              (dict(max_pages=0), E_SHAPE), (dict(k_page_stride=-8), E_SHAPE), (dict(v_slot_stride=56), E_SHAPE),
              (dict(k_head_stride=0), E_SHAPE), (dict(k_slot_stride=HUGE + 8), E_SHAPE), (dict(k_slot_stride=65), E_ALIGN),
              (dict(v_head_stride=1028), E_ALIGN), (dict(dtype=B.F32, k_page_stride=2050), E_ALIGN)]


def _attend(cache=None, Hq=4, max_len=64, scale=0.125, reserved=0, qs=256, qh=64, ms=64, q=FAKE, kp=FAKE, vp=FAKE, table=FAKE,
            lengths=FAKE, out=FAKE, mass=None, ws=FAKE, ws_bytes=1 << 40):
    c = _cache() if cache is None else cache
    a = B.AttendDesc(Hq, max_len, scale, reserved, qs, qh, ms)
    return B.lib().paep_attend(ctypes.byref(c), ctypes.byref(a), q, kp, vp, table, lengths, None, out, None, mass, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_every_call_refuses_a_bad_cache(kw, status):
    c = _cache(**kw)
    assert _attend(c, Hq=max(1, c.Hkv)) == status
    assert _append(c) == status
    assert _evict(c) == status


def test_attend_refuses_bad_arguments():
    a = B.AttendDesc(4, 64, 0.125, 0, 256, 64, 64)
    c = _cache()
    assert B.lib().paep_attend(None, ctypes.byref(a), *[FAKE] * 10, 0, None) == E_NULL
    assert B.lib().paep_attend(ctypes.byref(c), None, *[FAKE] * 10, 0, None) == E_NULL
    for kw in (dict(Hq=3), dict(Hq=0), dict(Hq=1026), dict(max_len=-1), dict(max_len=65), dict(scale=float("nan")),
               dict(scale=float("inf")), dict(reserved=1), dict(qs=-8), dict(qh=HUGE + 8), dict(mass=FAKE, ms=63)):
        assert _attend(**kw) == E_SHAPE, kw
    assert _attend(_cache(page_size=65536, max_pages=1 << 20), max_len=0x7FFF8000) == E_SHAPE
    for kw in (dict(qs=252), dict(qh=68), dict(q=ODD), dict(kp=ODD), dict(vp=ODD), dict(out=ODD)):
        assert _attend(**kw) == E_ALIGN, kw
    for name in ("q", "kp", "vp", "table", "lengths", "out"):
        assert _attend(**{name: None}) == E_NULL, name
    # an empty batch needs nothing but the pools; a grid that no launch can hold is refused
    assert _attend(_cache(B=0), q=None, table=None, lengths=None, out=None) == OK
    assert _attend(_cache(B=1 << 20, Hkv=1024), Hq=1024) == E_SHAPE
    mass = B.lib().paep_attend_workspace_bytes(ctypes.byref(c), ctypes.byref(a), 1)
    if mass:
        assert _attend(mass=FAKE, ws=None) == E_WS and _attend(mass=FAKE, ws_bytes=mass - 1) == E_WS and _attend(mass=FAKE, ws=ODD) == E_WS
    assert B.lib().paep_attend_workspace_bytes(ctypes.byref(_cache(Dk=60)), ctypes.byref(a), 0) == 0


def _append(cache=None, n=2, k=FAKE, kr=128, v=FAKE, vr=128, kp=FAKE, vp=FAKE, table=FAKE, seq=None, pos=FAKE, mass=None, ms=0):
    c = _cache() if cache is None else cache
    if cache is not None and c.B < 2:
        n = min(n, 1)
    return B.lib().paep_cache_append(ctypes.byref(c), n, k, kr, v, vr, kp, vp, table, seq, pos, mass, ms, None)


def test_append_refuses_bad_arguments():
    for kw in (dict(n=-1), dict(n=3), dict(n=1 << 25, seq=FAKE), dict(kr=120), dict(vr=-128), dict(kr=HUGE + 8), dict(mass=FAKE, ms=-1)):
        assert _append(**kw) == E_SHAPE, kw
    for kw in (dict(kr=132), dict(vr=132), dict(k=ODD), dict(v=ODD), dict(kp=ODD), dict(vp=ODD)):
        assert _append(**kw) == E_ALIGN, kw
    for name in ("k", "v", "kp", "vp", "table", "pos"):
        assert _append(**{name: None}) == E_NULL, name
    assert _append(n=0, k=None, v=None, table=None, pos=None) == OK


def _evict(cache=None, max_len=64, budget=16, recent=4, kp=FAKE, vp=FAKE, table=FAKE, lengths=FAKE, mass=FAKE, ms=64, ot=FAKE, op=2,
           kept=FAKE, mo=FAKE, mos=64, lo=FAKE):
    c = _cache() if cache is None else cache
    return B.lib().paep_cache_evict(ctypes.byref(c), max_len, budget, recent, kp, vp, table, lengths, mass, ms, ot, op, kept, mo, mos, lo, None)


def test_evict_refuses_bad_arguments():
    for kw in (dict(max_len=-1), dict(max_len=65), dict(budget=0), dict(budget=33), dict(recent=-1), dict(recent=17), dict(op=0),
               dict(ms=63), dict(mos=15), dict(mos=1 << 31), dict(ms=HUGE + 1)):
        assert _evict(**kw) == E_SHAPE, kw
    for kw in (dict(kp=ODD), dict(vp=ODD)):
        assert _evict(**kw) == E_ALIGN, kw
    for name in ("kp", "vp", "table", "lengths", "mass", "ot", "kept", "mo", "lo"):
        assert _evict(**{name: None}) == E_NULL, name
    assert _evict(_cache(B=0), table=None, lengths=None, mass=None, ot=None, kept=None, mo=None, lo=None) == OK
    assert _evict(_cache(B=1 << 20, Hkv=1024)) == E_SHAPE


def _moe(layer=True, x=FAKE, Wg=FAKE, W13=FAKE, W2=FAKE, res=None, y=FAKE, idx=FAKE, probs=FAKE, ws=FAKE, ws_bytes=1 << 40, **kw):
    d = dict(T=4, d=64, f=32, E=8, k=2, dtype=B.BF16, act=1, prob=0)
    d.update(kw)
    d = B.MoeDesc(**d)
    if layer:
        return B.lib().paep_moe_layer(ctypes.byref(d), x, Wg, None, W13, W2, res, y, idx, probs, None, ws, ws_bytes, None)
    return B.lib().paep_moe_experts(ctypes.byref(d), x, W13, W2, idx, probs, res, y, ws, ws_bytes, None)


@pytest.mark.parametrize("layer", [True, False])
def test_expert_layer_refuses_bad_arguments(layer):
    call = lambda **kw: _moe(layer, **kw)
    for kw in (dict(dtype=3), dict(act=3), dict(act=-1), dict(prob=3)):
        assert call(**kw) == E_DTYPE, kw
    for kw in (dict(T=-1), dict(T=65), dict(d=60), dict(d=0), dict(f=12), dict(f=0), dict(E=0), dict(E=1025), dict(d=(1 << 20) + 8)):
        assert call(**kw) == E_SHAPE, kw
    for kw in (dict(k=0), dict(k=9), dict(E=64, k=33)):
        assert call(**kw) == E_K, kw
    for name in ("x", "W13", "W2", "y", "idx", "probs") + (("Wg",) if layer else ()):
        assert call(**{name: None}) == E_NULL, name
    for name in ("x", "W13", "W2", "y", "res") + (("Wg",) if layer else ()):
        assert call(**{name: ODD}) == E_ALIGN, name
    need = B.lib().paep_moe_workspace_bytes(ctypes.byref(B.MoeDesc(4, 64, 32, 8, 2, B.BF16, 1, 0)))
    assert need > 0 and call(ws=None) == E_WS and call(ws=ODD) == E_WS and call(ws_bytes=need - 1) == E_WS
    assert call(T=0, x=None, y=None, idx=None, probs=None) == OK
    assert B.lib().paep_moe_workspace_bytes(ctypes.byref(B.MoeDesc(65, 64, 32, 8, 2, B.BF16, 1, 0))) == 0
    assert B.lib().paep_moe_layer(None, *[FAKE] * 11, 0, None) == E_NULL


def test_workspaces_do_not_shrink_with_more_tokens_or_longer_caches():
    def moe(**kw):
        d = dict(T=4, d=2048, f=768, E=64, k=6, dtype=B.BF16, act=1, prob=0)
        d.update(kw)
        return B.lib().paep_moe_workspace_bytes(ctypes.byref(B.MoeDesc(**d)))
    sizes = [moe(T=t) for t in range(0, 65)]
    assert sizes == sorted(sizes)
    assert moe(k=5) <= moe(k=6) and moe(f=760) <= moe(f=768) and moe(E=60) <= moe(E=64)


# ---- the plain forms themselves ----

def test_reference_attention_is_softmax_attention():
    g = np.random.default_rng(1)
    H, G, Dk, Dv, ps, n = 2, 3, 16, 24, 4, 11
    kp, vp = g.standard_normal((5, H, ps, Dk)), g.standard_normal((5, H, ps, Dv))
    table = np.array([[3, 0, 4]])
    q = g.standard_normal((1, H * G, Dk))
    (out, lse, weight), tol = R.attend(q, kp, vp, table, [n], [2], 0.25, 12, False)
    k = torch.from_numpy(np.concatenate([kp[i] for i in table[0]], axis=1)[:, 2:n])
    v = torch.from_numpy(np.concatenate([vp[i] for i in table[0]], axis=1)[:, 2:n])
    qt = torch.from_numpy(q).view(H, G, Dk)
    want = torch.nn.functional.scaled_dot_product_attention(qt, k, v, scale=0.25)
    assert np.allclose(out, want.reshape(1, H * G, Dv).numpy(), atol=1e-13)
    s = torch.matmul(qt, k.transpose(1, 2)) * 0.25
    assert np.allclose(lse[0], torch.logsumexp(s, 2).reshape(-1).numpy(), atol=1e-13)
    assert np.allclose(weight[0, :, 2:n], torch.softmax(s, 2).sum(1).numpy(), atol=1e-13) and not weight[0, :, :2].any()
    assert all((t >= 0).all() for t in tol) and tol[0].max() < 1e-4


def test_reference_attention_leaves_absent_pages_and_empty_ranges_out():
    g = np.random.default_rng(2)
    kp, vp = g.standard_normal((4, 1, 2, 8)), g.standard_normal((4, 1, 2, 8))
    q = g.standard_normal((3, 1, 8))
    table = np.array([[1, -1, 2], [0, 9, 3], [0, 1, 2]])
    (out, lse, weight), _ = R.attend(q, kp, vp, table, [6, 3, 4], [0, 2, 4], 1.0, 6, False)
    s = np.concatenate([kp[1, 0], kp[2, 0]]) @ q[0, 0]
    assert np.isclose(lse[0, 0], np.log(np.exp(s).sum())) and weight[0, 0, 2:4].sum() == 0
    assert not out[1:].any() and (lse[1:] == -np.inf).all() and not weight[1:].any()


def test_reference_eviction_by_hand():
    mass = np.array([0.5, 2.0, np.nan, 0.0, 2.0, -0.0, 1.0, 9.0])
    assert R.kept_positions(mass, 8, 4, 2).tolist() == [1, 4, 6, 7]
    assert R.kept_positions(mass, 8, 3, 2).tolist() == [1, 6, 7]             # equal: the lower position
    assert R.kept_positions(mass, 8, 6, 2).tolist() == [0, 1, 3, 4, 6, 7]    # 0 before -0 and NaN
    assert R.kept_positions(mass, 8, 7, 0).tolist() == [0, 1, 3, 4, 5, 6, 7]
    assert R.kept_positions(mass, 3, 3, 1).tolist() == [0, 1, 2]
    assert R.kept_positions(mass, 8, 2, 2).tolist() == [6, 7]


def test_reference_experts_are_gated_mlps():
    g = np.random.default_rng(3)
    T, d, f, E, k = 5, 16, 24, 6, 3
    x, W13, W2 = g.standard_normal((T, d)), g.standard_normal((E, 2 * f, d)), g.standard_normal((E, d, f))
    z = g.standard_normal((T, E))
    for name, fn in (("silu", torch.nn.functional.silu), ("gelu", torch.nn.functional.gelu), ("none", lambda t: t)):
        idx, probs = R.select(z, k, "softmax")
        y, tol = R.experts(x, W13, W2, idx, probs, name, None, False)
        xt, p = torch.from_numpy(x), torch.softmax(torch.from_numpy(z), 1)
        all_h = torch.stack([fn(xt @ torch.from_numpy(W13[e, :f]).t()) * (xt @ torch.from_numpy(W13[e, f:]).t()) for e in range(E)])
        all_y = torch.stack([all_h[e] @ torch.from_numpy(W2[e]).t() for e in range(E)])
        keep = torch.zeros(T, E, dtype=torch.float64).scatter_(1, torch.topk(torch.from_numpy(z), k).indices, 1.0)
        want = torch.einsum("te,etd->td", keep * p, all_y)
        assert np.allclose(y, want.numpy(), rtol=1e-12, atol=1e-12) and tol.max() < 1e-2
    # a repeated id weighs the sum, an absent one nothing
    y1, _ = R.experts(x[:1], W13, W2, np.array([[2, 2, -1]]), np.array([[0.25, 0.5, 7.0]]), "silu", x[:1], False)
    y2, _ = R.experts(x[:1], W13, W2, np.array([[2]]), np.array([[0.75]]), "silu", x[:1], False)
    assert np.allclose(y1, y2, rtol=1e-14)
