"""Attention over a cache in 4 bits at the ends of the range of scores, where the answers are known without a bound that grows with
them: one position far above all others, or all of them equal."""
import numpy as np
import pytest
import torch

import rotate_fourbit_reference as R
from paper_2511_10676_amd import binding as B

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
PARTS = {"bf16": 1, "f32": 3}
U = R.U


def _np(t):
    return t.double().cpu().numpy()


class Rows:
    """Sequences of 1, 20, 300 and 5000 positions (the last one is cut into pieces), each three times.  A key is `key` in its first 32
    dimensions, of 128, times its power, and 0 in the others; values are random."""

    def __init__(self, g, ps, n=(1, 20, 300, 5000) * 3, pattern="equal"):
        self.lengths, width = list(n), -(-max(n) // ps)
        pages = len(n) * width
        self.table = torch.randperm(pages, generator=g, device="cuda").view(len(n), width).to(torch.int32).contiguous()
        kp, ks = torch.zeros((pages, 1, ps, 64), dtype=torch.uint8), torch.full((pages, 1, 4, ps), 127, dtype=torch.uint8)
        self.best = [x * 3 // 8 for x in n]
        table = self.table.cpu().long()
        # 6 in the best place; elsewhere the same, -6, 0; or -6 there and -12 elsewhere
        kp[..., :16] = {"equal": 0x77, "above": 0xFF, "zeros": 0x00, "below": 0xFF}[pattern]
        ks[:, :, 0] = 128 if pattern == "below" else 127
        for b, p in enumerate(self.best):
            kp[table[b, p // ps], 0, p % ps, :16] = 0xFF if pattern == "below" else 0x77
            ks[table[b, p // ps], 0, 0, p % ps] = 127
        self.kp, self.ks = kp.cuda(), ks.cuda()
        self.vp = torch.randint(0, 256, (pages, 1, ps, 64), generator=g, device="cuda").to(torch.uint8)
        self.vs = torch.randint(124, 130, (pages, 1, 4, ps), generator=g, device="cuda").to(torch.uint8)
        self.v = R.values(self.vp.cpu().numpy(), self.vs.transpose(2, 3).cpu().numpy())
        self.factor = -6.0 if pattern == "below" else 6.0
        self.ps = ps

    def attend(self, q, scale):
        lens = torch.tensor(self.lengths, dtype=torch.int32, device="cuda")
        got = B.attend_fourbit(q, self.kp, self.vp, self.ks, self.vs, self.table, lens, scale=scale, want_lse=True)
        return _np(got.out), _np(got.lse)

    def values(self, b):
        """[length, 128]: the sequence's values."""
        p = np.arange(self.lengths[b])
        return self.v[self.table.cpu().numpy()[b, p // self.ps], 0, p % self.ps]


def _queries(g, size, scale, kind, n):
    """[n, 3, 128]: three heads whose scores with a key of sixes are near size, size / 2 and size / 10, none of them round."""
    q = torch.zeros((n, 3, 128), device="cuda")
    q[..., :32] = (0.5 + torch.rand((n, 3, 32), generator=g, device="cuda")) * (size / (192 * abs(scale)))
    q *= torch.tensor([1.0, 0.5, 0.1], device="cuda")[:, None] * (1.0 if scale > 0 else -1.0)
    return q.to(TYPES[kind])


SIZES = [(None, s) for s in (1e6, 3e7, 1e9, 3e9, 1e10, 1e15, 1e20, 1e30, 3e36)] + [(1.0, 1e38), (-0.7, 4e9), (-0.7, 8e37), (1e-20, 1e10), (1e20, 1e12)]


@pytest.mark.parametrize("heads", [1, 3])
@pytest.mark.parametrize("ps", [16, 4])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("pattern", ["above", "zeros", "below"])
def test_one_position_far_above_the_others(pattern, kind, ps, heads):
    """Every weight but one is 0 in any arithmetic (the others' scores are at least 5e4 lower), so out is that position's value, and
    lse its score."""
    g = torch.Generator(device="cuda").manual_seed(31)
    r = Rows(g, ps, pattern=pattern)
    best = np.stack([r.values(b)[p] for b, p in enumerate(r.best)])[:, None]
    for scale, size in SIZES:
        by = float(np.float32(128 ** -0.5 if scale is None else scale))
        q = _queries(g, size, by, kind, len(r.lengths))[:, :heads]
        out, lse = r.attend(q, scale)
        score = by * r.factor * _np(q).sum(axis=2)
        # Three parts of the weight, which leave 1 U, their products' sums up to 2 each, three factors and 1 / sum to 2, and the join's
        # weight, its exponential's 2, and its sum: below 16.  A value is a bf16 number, which less than 2^-9 does not move.
        assert np.all(np.abs(out - best) <= (0 if kind == "bf16" else 16 * U * np.abs(best))), (scale, size)
        # a score: a product and a sum for each of 32 elements' parts, the factor; then its way through units of log2 and back, 6
        assert np.all(np.abs(lse - score) <= (PARTS[kind] * 64 + 1 + 6) * U * np.abs(score)), (scale, size)


@pytest.mark.parametrize("ps", [16, 4])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_equal_scores_of_any_size(kind, ps):
    g = torch.Generator(device="cuda").manual_seed(32)
    r = Rows(g, ps)
    values = [r.values(b) for b in range(len(r.lengths))]
    for sign in (1.0, -1.0):
        for scale, size in SIZES:
            by = float(np.float32(128 ** -0.5 if scale is None else scale))
            q = _queries(g, size, by, kind, len(r.lengths)) * sign
            out, lse = r.attend(q, scale)
            score = by * 6.0 * _np(q).sum(axis=2)
            for b, v in enumerate(values):
                n = len(v)
                # one rounding for each position in the weighted sum and in the sum of weights, as many again for the parts of a weight, 16 more
                tol = (n + 16) * 4 * U * np.abs(v).mean(axis=0) + R.HALF[kind] * np.abs(v.mean(axis=0))
                assert np.all(np.abs(out[b] - v.mean(axis=0)) <= tol), (scale, size, n)
                off = (PARTS[kind] * 64 + 1 + 6) * U * np.abs(score[b]) + ((n + 16) * 2 + 4 * np.log(n)) * U
                assert np.all(np.abs(lse[b] - score[b] - np.log(n)) <= off), (scale, size, n)


@pytest.mark.parametrize("ps", [16, 4])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_scales_of_zero_and_next_to_it(kind, ps):
    """Products up to 1e38: by 0 they are equal; by numbers too small to be normal ones they are scores of size 1e-2 to 1e-7."""
    g = torch.Generator(device="cuda").manual_seed(33)
    for pattern in ("above", "zeros", "below"):
        r = Rows(g, ps, pattern=pattern)
        q = _queries(g, 1e38, 1.0, kind, len(r.lengths))
        k = R.values(r.kp.cpu().numpy(), r.ks.transpose(2, 3).cpu().numpy())
        for scale in (0.0, -0.0, 1e-40, -1e-40, 1e-45):
            out, lse = r.attend(q, scale)
            want, tol = R.attend(_np(q), k, r.v, r.table.cpu().numpy(), r.lengths, None, float(np.float32(scale)), r.table.shape[1] * ps, kind)
            assert np.all(np.abs(out - want[0]) <= tol[0]) and np.all(np.abs(lse - want[1]) <= tol[1]), (pattern, scale)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_scales_of_zero_and_next_to_it_over_rows_that_are_left_out(kind):
    """Rows before the start, behind the end and on pages that are none take no part, whatever the scale."""
    g = torch.Generator(device="cuda").manual_seed(34)
    for ps in (16, 4):
        r = Rows(g, ps, n=(300, 37, 5))
        r.table[0, 2] = -1
        r.vs.fill_(127)
        lens, starts = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ((300, 37, 5), (21, 36, 5)))
        v = R.values(r.vp.cpu().numpy(), r.vs.transpose(2, 3).cpu().numpy())
        k = R.values(r.kp.cpu().numpy(), r.ks.transpose(2, 3).cpu().numpy())
        q = _queries(g, 1e38, 1.0, kind, 3)
        for scale in (0.0, 1e-40):
            got = B.attend_fourbit(q, r.kp, r.vp, r.ks, r.vs, r.table, lens, starts=starts, scale=scale, want_lse=True)
            want, tol = R.attend(_np(q), k, v, r.table.cpu().numpy(), [300, 37, 5], [21, 36, 5], float(np.float32(scale)), r.table.shape[1] * ps, kind)
            assert np.all(np.abs(_np(got.out) - want[0]) <= tol[0])
            lse = _np(got.lse)
            assert np.all(lse[2] == -np.inf) and np.all(np.abs(lse[:2] - want[1][:2]) <= tol[1][:2])
