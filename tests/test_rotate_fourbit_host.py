"""Host-side checks of the rotation's and the 4-bit cache's calls that need no GPU: every bad argument is refused before any HIP
call (the pointers used here are never dereferenced), workspaces asked for do not shrink, and the plain forms that the GPU tests
compare with agree with other ways of computing the same."""
import ctypes

import numpy as np
import pytest
import torch

import rotate_fourbit_reference as R
from paper_2511_10676_amd import binding as B

OK, E_NULL, E_SHAPE, E_K, E_DTYPE, E_ALIGN, E_WS, E_HIP, E_UNSUP = range(9)
FAKE, ODD = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10008)
HUGE = 1 << 40


def _cache(fourbit=True, **kw):
    c = dict(B=2, Hkv=2, Dk=64, Dv=64, page_size=16, n_pages=8, max_pages=4, dtype=B.BF16)
    c.update({n: v for n, v in kw.items() if n in c})
    c.update(k_page_stride=c["Hkv"] * c["page_size"] * c["Dk"], k_head_stride=c["page_size"] * c["Dk"], k_slot_stride=c["Dk"],
             v_page_stride=c["Hkv"] * c["page_size"] * c["Dv"], v_head_stride=c["page_size"] * c["Dv"], v_slot_stride=c["Dv"])
    c.update(kw)
    return B.CacheDesc(**c)


def _rotate(append=False, cache=None, q=FAKE, k=FAKE, v=FAKE, vr=128, vh=64, qw=None, kw_=None, pos=FAKE, table=FAKE, qo=FAKE, ko=FAKE,
            kp=FAKE, vp=FAKE, pt=FAKE, seq=None, mass=None, ms=0, angles=None, **kw):
    d = dict(n=2, Hq=4, Hk=2, D=64, rot=64, table_rows=100, dtype=B.BF16, style=0, eps=1e-6, reserved=0, q_row_stride=256, q_head_stride=64,
             k_row_stride=128, k_head_stride=64, q_out_row_stride=256, q_out_head_stride=64, k_out_row_stride=128, k_out_head_stride=64)
    d.update(kw)
    d = ctypes.byref(B.RotateDesc(**d))
    if not append:
        return B.lib().paep_rotate(d, q, k, qw, kw_, pos, table, qo, ko, None)
    c = _cache() if cache is None else cache
    return B.lib().paep_rotate_append(d, ctypes.byref(c), q, k, v, vr, vh, qw, kw_, table, angles, qo, kp, vp, pt, seq, pos, mass, ms, None)


@pytest.mark.parametrize("append", [False, True])
def test_rotate_refuses_bad_arguments(append):
    for kw in (dict(n=-1), dict(n=(1 << 24) + 1), dict(Hq=-1), dict(Hq=1025), dict(Hk=-1), dict(Hk=1025), dict(Hq=0, Hk=0), dict(D=60),
               dict(D=0), dict(D=264), dict(rot=0), dict(rot=63), dict(rot=66), dict(table_rows=0), dict(reserved=1), dict(eps=0.0),
               dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(q_row_stride=-8), dict(q_head_stride=56),
               dict(k_head_stride=HUGE + 8), dict(q_out_row_stride=0), dict(q_out_head_stride=32)):
        assert _rotate(append, **kw) == E_SHAPE, kw
    for kw in (dict(dtype=2), dict(style=2), dict(style=-1)):
        assert _rotate(append, **kw) == E_DTYPE, kw
    for kw in (dict(q_row_stride=260), dict(k_head_stride=68), dict(q=ODD), dict(k=ODD), dict(qw=ODD), dict(kw_=ODD), dict(table=ODD), dict(qo=ODD)):
        assert _rotate(append, **kw) == E_ALIGN, kw
    for name in ("q", "k", "pos", "table", "qo"):
        assert _rotate(append, **{name: None}) == E_NULL, name
    lib = B.lib()
    assert lib.paep_rotate(None, *[FAKE] * 8, None) == E_NULL
    assert _rotate(append, n=0, q=None, k=None, v=None, qo=None, ko=None, pos=None, pt=None) == OK


def test_rotate_refuses_outputs_that_overlap():
    assert _rotate(q_out_row_stride=64, q_out_head_stride=64) == E_SHAPE              # a row's second head on the next row's first
    assert _rotate(k_out_row_stride=64, k_out_head_stride=64) == E_SHAPE
    assert _rotate(n=1 << 24, q_out_row_stride=HUGE, q_out_head_stride=HUGE) == E_SHAPE
    assert _rotate(q_out_row_stride=64, q_out_head_stride=128, k_out_row_stride=64, k_out_head_stride=128, n=0) == OK
    for rows, heads in ((256, 64), (64, 128)):                                         # heads within rows, rows within heads: not refused for that
        assert _rotate(q_out_row_stride=rows, q_out_head_stride=heads, table=None) == E_NULL


def test_rotate_alone_refuses_bad_outputs_of_keys():
    assert _rotate(ko=None) == E_NULL and _rotate(ko=ODD) == E_ALIGN
    assert _rotate(k_out_row_stride=0) == E_SHAPE and _rotate(k_out_head_stride=68) == E_ALIGN


def test_rotate_append_refuses_bad_arguments():
    call = lambda **kw: _rotate(True, **kw)
    for kw in (dict(cache=_cache(Hkv=1)), dict(cache=_cache(Dk=128)), dict(cache=_cache(Dv=12)), dict(cache=_cache(page_size=24)), dict(n=3),
               dict(vr=-8), dict(vh=56), dict(mass=FAKE, ms=-1)):
        assert call(**kw) == E_SHAPE, kw
    assert call(cache=_cache(dtype=B.F32)) == E_DTYPE
    for kw in (dict(v=ODD), dict(kp=ODD), dict(vp=ODD), dict(vr=132)):
        assert call(**kw) == E_ALIGN, kw
    for name in ("v", "kp", "vp", "pt"):
        assert call(**{name: None}) == E_NULL, name
    assert B.lib().paep_rotate_append(ctypes.byref(B.RotateDesc()), None, *[FAKE] * 3, 0, 0, *[FAKE] * 11, 0, None) != OK


def _append(cache=None, n=2, k=FAKE, kr=128, kh=64, v=FAKE, vr=128, vh=64, kp=FAKE, vp=FAKE, ks=FAKE, vs=FAKE, pt=FAKE, seq=None, pos=FAKE):
    c = _cache() if cache is None else cache
    return B.lib().paep_cache_append_fourbit(ctypes.byref(c), min(n, max(c.B, 0)) if cache is not None else n, k, kr, kh, v, vr, vh, kp, vp, ks, vs,
                                             pt, seq, pos, None)


def _read(cache=None, n=2, kp=FAKE, vp=FAKE, ks=FAKE, vs=FAKE, pt=FAKE, seq=None, pos=FAKE, ko=FAKE, vo=FAKE):
    c = _cache() if cache is None else cache
    return B.lib().paep_cache_read_fourbit(ctypes.byref(c), n, kp, vp, ks, vs, pt, seq, pos, ko, vo, None)


def _attend(cache=None, Hq=4, max_len=64, scale=0.125, reserved=0, qs=256, qh=64, q=FAKE, kp=FAKE, vp=FAKE, ks=FAKE, vs=FAKE, pt=FAKE,
            lengths=FAKE, out=FAKE, ws=FAKE, ws_bytes=1 << 40):
    c = _cache() if cache is None else cache
    a = B.AttendDesc(Hq, max_len, scale, reserved, qs, qh, 0)
    return B.lib().paep_attend_fourbit(ctypes.byref(c), ctypes.byref(a), q, kp, vp, ks, vs, pt, lengths, None, out, None, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=7), E_DTYPE), (dict(B=-1), E_SHAPE), (dict(Hkv=0), E_SHAPE), (dict(Hkv=1025), E_SHAPE), (dict(Dk=48), E_SHAPE),
    (dict(Dk=8), E_SHAPE), (dict(Dk=288), E_SHAPE), (dict(Dv=40), E_SHAPE), (dict(Dv=0), E_SHAPE), (dict(page_size=0), E_SHAPE),
    (dict(page_size=24), E_SHAPE), (dict(page_size=1 << 17), E_SHAPE), (dict(n_pages=0), E_SHAPE), (dict(max_pages=0), E_SHAPE),
    (dict(k_page_stride=-32), E_SHAPE), (dict(v_slot_stride=32), E_SHAPE), (dict(k_head_stride=0), E_SHAPE),
    (dict(k_slot_stride=HUGE + 32), E_SHAPE), (dict(k_slot_stride=80), E_ALIGN), (dict(v_head_stride=1040), E_ALIGN)])
def test_every_call_refuses_a_bad_fourbit_cache(kw, status):
    c = _cache(**kw)
    assert _attend(c, Hq=max(1, c.Hkv)) == status
    assert _append(c) == status
    assert _read(c) == status


def test_append_and_read_refuse_bad_arguments():
    for kw in (dict(n=-1), dict(n=3), dict(n=(1 << 24) + 1, seq=FAKE), dict(kh=56), dict(vr=-128), dict(kr=HUGE + 8)):
        assert _append(**kw) == E_SHAPE, kw
    for kw in (dict(kr=132), dict(vh=68), dict(k=ODD), dict(v=ODD), dict(kp=ODD), dict(vp=ODD), dict(ks=ODD), dict(vs=ODD)):
        assert _append(**kw) == E_ALIGN, kw
    for name in ("k", "v", "kp", "vp", "ks", "vs", "pt", "pos"):
        assert _append(**{name: None}) == E_NULL, name
    assert _append(n=0, k=None, v=None, pt=None, pos=None) == OK
    for kw in (dict(n=-1), dict(n=3), dict(n=(1 << 24) + 1, seq=FAKE)):
        assert _read(**kw) == E_SHAPE, kw
    for kw in (dict(kp=ODD), dict(vp=ODD), dict(ks=ODD), dict(vs=ODD), dict(ko=ODD), dict(vo=ODD)):
        assert _read(**kw) == E_ALIGN, kw
    for name in ("kp", "vp", "ks", "vs", "pt", "pos", "ko", "vo"):
        assert _read(**{name: None}) == E_NULL, name
    assert _read(n=0, pt=None, pos=None, ko=None, vo=None) == OK


def test_attend_fourbit_refuses_bad_arguments():
    a, c, lib = B.AttendDesc(4, 64, 0.125, 0, 256, 64, 0), _cache(), B.lib()
    assert lib.paep_attend_fourbit(None, ctypes.byref(a), *[FAKE] * 11, 0, None) == E_NULL
    assert lib.paep_attend_fourbit(ctypes.byref(c), None, *[FAKE] * 11, 0, None) == E_NULL
    for kw in (dict(Hq=3), dict(Hq=0), dict(Hq=1026), dict(max_len=-1), dict(max_len=65), dict(scale=float("nan")),
               dict(scale=float("inf")), dict(reserved=1), dict(qs=-8), dict(qh=HUGE + 8)):
        assert _attend(**kw) == E_SHAPE, kw
    assert _attend(_cache(page_size=65536, max_pages=1 << 20), max_len=0x7FFF8000) == E_SHAPE
    for kw in (dict(qs=252), dict(qh=68), dict(q=ODD), dict(kp=ODD), dict(vp=ODD), dict(ks=ODD), dict(vs=ODD), dict(out=ODD)):
        assert _attend(**kw) == E_ALIGN, kw
    for name in ("q", "kp", "vp", "ks", "vs", "pt", "lengths", "out"):
        assert _attend(**{name: None}) == E_NULL, name
    assert _attend(_cache(B=0), q=None, pt=None, lengths=None, out=None) == OK
    assert _attend(_cache(B=1 << 20, Hkv=1024), Hq=1024) == E_SHAPE
    big, d = _cache(max_pages=1000), B.AttendDesc(4, 16000, 0.125, 0, 256, 64, 0)
    need = lib.paep_attend_fourbit_workspace_bytes(ctypes.byref(big), ctypes.byref(d))
    assert need > 0
    for kw in (dict(ws=None), dict(ws_bytes=need - 1), dict(ws=ODD)):
        assert _attend(big, max_len=16000, **kw) == E_WS
    assert lib.paep_attend_fourbit_workspace_bytes(ctypes.byref(_cache(Dk=48)), ctypes.byref(a)) == 0


@pytest.mark.parametrize("Hq,Hkv,Dv", [(1, 1, 32), (8, 2, 128), (40, 1, 256), (64, 64, 96)])
def test_attend_fourbit_workspace_does_not_shrink(Hq, Hkv, Dv):
    lib, before = B.lib(), {}
    for batch in (1, 2, 3, 7, 40, 200):
        last = 0
        for n in [*range(0, 700, 13), *range(700, 9000, 331), *range(9000, 140000, 4099), 600000, 1 << 22]:
            c = _cache(B=batch, Hkv=Hkv, Dv=Dv, max_pages=1 << 18)
            need = lib.paep_attend_fourbit_workspace_bytes(ctypes.byref(c), ctypes.byref(B.AttendDesc(Hq, n, 0.1, 0, 8 * 64, 64, 0)))
            assert need >= last and need >= before.get(n, 0), (batch, n)
            last = before[n] = need


def test_reference_rounding_is_to_the_nearest_and_never_half_a_step_off():
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((200, 64)) * 2.0 ** rng.integers(-140, 125, (200, 1))).astype(np.float32)
    x[0] = 0.0
    x[1, :32] = np.arange(32) * 0.25                     # 7.75 is the largest: a power of 2, and ties
    x[2, 3] = np.nan
    x[3, 40] = -np.inf
    got, byte = R.to_fourbit(x)
    assert byte[0, 0] == 2 and byte[1, 0] == 128 and byte[2, 0] == 255 and byte[3, 1] == 252 and got[3, 40] == -6 * 2.0 ** 125
    assert np.isnan(got[2, :32]).all() and np.isfinite(got[2, 32:]).all()
    assert (got[1, :8] == [0, 0, 0, 1, 1, 1, 2, 2]).all()            # 0.25 to 1.75 in steps of 1: 0.5 and 1.5 are ties
    fine = np.isfinite(x) & np.repeat(byte != 255, 32, axis=1) & (np.abs(x) < 2e38)
    power = np.repeat(2.0 ** (byte.astype(float) - 127), 32, axis=1)
    a, step = np.abs(x.astype(float)) / power, np.full(x.shape, 0.5)
    step[a > 2] = 1.0
    step[a > 4] = 2.0
    assert (np.abs(got - x.astype(float)) / power <= step / 2)[fine].all()
    # no smaller power would do
    smaller = power / 2
    most = np.where(np.isnan(x), 0, np.abs(x.astype(float))).reshape(200, 2, 32).max(axis=2).repeat(32, axis=1)
    assert ((most > 7 * smaller) | (np.repeat(byte, 32, axis=1) == 2))[fine].all()


def test_reference_attention_and_rotation_against_torch():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((1, 4, 32)), rng.standard_normal((3, 2, 8, 32)), rng.standard_normal((3, 2, 8, 32))
    table = np.array([[2, 0, 1]])
    (out, lse), _ = R.attend(q, k, v, table, np.array([21]), None, 0.2, 24, "f32")
    kk = torch.from_numpy(k[[2, 0, 1]]).transpose(0, 1).reshape(2, 24, 32)[:, :21].repeat_interleave(2, 0)
    vv = torch.from_numpy(v[[2, 0, 1]]).transpose(0, 1).reshape(2, 24, 32)[:, :21].repeat_interleave(2, 0)
    s = 0.2 * (kk @ torch.from_numpy(q)[0, :, :, None])[..., 0]
    want = (torch.softmax(s, 1)[:, None] @ vv)[:, 0]
    assert np.allclose(out[0], want.numpy(), atol=1e-12) and np.allclose(lse[0], torch.logsumexp(s, 1).numpy(), atol=1e-12)
    x, turns = rng.standard_normal((5, 2, 16)), B.rotation_table(50, 8, device="cpu")[[0, 3, 49, 7, 7]].numpy()
    y, _ = R.rotate(x, None, turns, "pairs", 1e-6, "f32")
    z = torch.view_as_complex(torch.from_numpy(x[..., :8].reshape(5, 2, 4, 2).copy())) * torch.complex(*map(torch.from_numpy, (turns[:, None, :4].astype(float), turns[:, None, 4:].astype(float))))
    assert np.allclose(y[..., :8], torch.view_as_real(z).flatten(-2).numpy(), atol=1e-12) and (y[..., 8:] == x[..., 8:]).all()


def test_rotation_table_at_far_positions():
    t = B.rotation_table(1 << 20, 4, base=500000.0, device="cpu")
    p = (1 << 20) - 1
    a = p * 500000.0 ** np.array([0.0, -0.5])
    assert t.shape == (1 << 20, 4) and t.dtype == torch.float32
    assert np.abs(t[p].numpy() - np.concatenate([np.cos(a), np.sin(a)])).max() <= 2.0 ** -25 + 1e-9
    for bad in ((0, 4), (8, 3), (8, 0)):
        with pytest.raises(ValueError):
            B.rotation_table(*bad, device="cpu")


def test_python_calls_refuse_host_tensors():
    x, pos, table = torch.zeros((2, 1, 32)), torch.zeros(2, dtype=torch.int32), torch.zeros((4, 32))
    pages, scales, pt = torch.zeros((2, 1, 16, 16), dtype=torch.uint8), torch.zeros((2, 1, 1, 16), dtype=torch.uint8), torch.zeros((2, 1), dtype=torch.int32)
    for call in (lambda: B.rotate(x, x, pos, table), lambda: B.rotate(None, None, pos, table),
                 lambda: B.rotate_append(x, x, x, torch.zeros((2, 1, 16, 32)), torch.zeros((2, 1, 16, 32)), pt, pos, table),
                 lambda: B.cache_append_fourbit(x, x, pages, pages, scales, scales, pt, pos),
                 lambda: B.cache_read_fourbit(pages, pages, scales, scales, pt, pos),
                 lambda: B.attend_fourbit(x, pages, pages, scales, scales, pt, pos)):
        with pytest.raises(ValueError):
            call()
