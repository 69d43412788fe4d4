"""Paths of the decode step's operators that only some sizes take, against the 64-bit forms: workgroups of the expert layer that
go on to further items, parts of rows added afterwards, every width of the selection, joins of several hundred chunks."""
import ctypes

import numpy as np
import pytest
import torch

import decode_step_reference as R
from paper_2511_10676_amd import binding as B
from test_gpu_decode_step import _cache, _check_attend, _check_moe, _i32, _np, _pages, _storage, _to

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,f,E,k", [
    (9, 64, 768, 128, 8), (16, 72, 520, 64, 8), (1, 16, 2000, 32, 8),        # up to 16 tokens, more items than workgroups
    (64, 64, 768, 16, 8), (64, 40, 1000, 24, 12), (33, 48, 2400, 8, 6),      # more tokens: experts of more than 16 among others, several items each
    (20, 96, 264, 300, 5), (5, 96, 40, 300, 6), (20, 64, 24, 1024, 7), (5, 64, 40, 700, 32)])      # selections of more than 256 experts
def test_moe_layer_paths(T, d, f, E, k, dtype):
    _check_moe(np.random.default_rng(T + d + f), T, d, f, E, k, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,f,E,k", [(16, 256, 704, 64, 6), (40, 136, 512, 24, 4), (64, 1000, 264, 16, 2)])
@pytest.mark.parametrize("inplace", [False, True])
def test_moe_layer_parts_with_residual(T, d, f, E, k, inplace, dtype):
    _check_moe(np.random.default_rng(T + d), T, d, f, E, k, dtype, "silu", "softmax_topk", residual=True, inplace=inplace)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_moe_experts_every_token_to_the_same_few(dtype):
    """64 tokens at each of two experts among others: every block of columns, more than one item of a workgroup."""
    g = np.random.default_rng(70)
    T, d, f, E, k = 64, 96, 712, 40, 4
    x = _storage(g.standard_normal((T, d)), dtype)
    W13 = _storage(g.standard_normal((E, 2 * f, d)) / np.sqrt(d), dtype)
    W2 = _storage(g.standard_normal((E, d, f)) / np.sqrt(f), dtype)
    idx = np.stack([np.concatenate([[7, 30], g.choice(np.setdiff1d(np.arange(E), [7, 30]), 2, replace=False)]) for _ in range(T)])
    probs = g.random((T, k)).astype(np.float32)
    y, tol = R.experts(x, W13, W2, idx, probs, "gelu", None, dtype == "bf16")
    got = B.moe_experts(_to(x, dtype), _to(W13, dtype), _to(W2, dtype), _i32(idx), _to(probs, "f32"), act="gelu")
    torch.cuda.synchronize()
    assert (np.abs(_np(got) - y) <= tol).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,n,window", [(1, 1, 131072, 0), (1, 3, 70001, 0), (2, 2, 100003, 99000), (1, 20, 66000, 0)])
def test_attend_joins_hundreds_of_chunks(H, G, n, window, dtype):
    g = np.random.default_rng(n)
    starts = [n - window] if window else None
    kp, vp, table = _cache(g, [n], H, 8, 8, 64, dtype, starts)
    q = _storage(g.standard_normal((1, H * G, 8)) * 2, dtype)
    _check_attend(q, kp, vp, table, [n], starts, dtype)


def test_attend_walks_more_pages_than_a_workgroup_holds():
    """One position per page and chunks of more than 2048 positions: the page table is read in stretches."""
    g = np.random.default_rng(71)
    n, D = 600011, 8
    order = g.permutation(n + 1)
    kp, vp = (_storage(g.standard_normal((n + 1, 1, 1, D)), "bf16") for _ in range(2))
    kp[order[n]], vp[order[n]] = np.nan, np.nan
    table = order[:n].reshape(1, n).astype(np.int32)
    table[0, 4444] = -1
    q = _storage(g.standard_normal((1, 2, D)), "bf16")
    _check_attend(q, kp, vp, table, [n], [3], "bf16")


@pytest.mark.parametrize("mass", [False, True])
@pytest.mark.parametrize("batch,H,G", [(1, 2, 4), (5, 1, 3), (61, 8, 1)])
def test_attend_in_one_workspace_for_every_length(batch, H, G, mass):
    """A workspace asked for once, for the table's capacity and the whole batch, is enough for tight bounds and parts of the batch."""
    g = np.random.default_rng(batch)
    page, width, D = 16, 130, 64
    kp, vp, table = _cache(g, [width * page] * batch, H, D, D, page, "bf16")
    q, kd, vd, td = _to(g.standard_normal((batch, H * G, D)), "bf16"), _pages(kp, "bf16", "heads"), _pages(vp, "bf16", "heads"), _i32(table)
    c = B.CacheDesc(batch, H, D, D, page, kp.shape[0], width, B.BF16, H * page * D, page * D, D, H * page * D, page * D, D)
    d = B.AttendDesc(H * G, width * page, 0.125, 0, H * G * D, D, width * page)
    workspace = torch.empty(B.lib().paep_attend_workspace_bytes(ctypes.byref(c), ctypes.byref(d), mass), dtype=torch.uint8, device="cuda")
    for n, few in ((1, batch), (241, batch), (242, 1), (260, batch), (272, batch), (400, (batch + 1) // 2), (1025, batch), (2080, batch)):
        lengths = _i32([max(0, n - i) for i in range(few)])
        sums = [torch.zeros((few, H, n), device="cuda") if mass else None for _ in range(2)]
        got = B.attend(q[:few], kd, vd, td[:few], lengths, max_len=n, mass=sums[0], workspace=workspace)
        want = B.attend(q[:few], kd, vd, td[:few], lengths, max_len=n, mass=sums[1])
        torch.cuda.synchronize()
        assert torch.equal(got.out, want.out) and (not mass or torch.equal(*sums))
