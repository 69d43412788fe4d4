"""The calls on the way into and out of a cache one after the other, as a decode step makes them: eager, on another stream, and
captured into graphs that are replayed with eager work between."""
import numpy as np
import pytest
import torch

import rotate_fourbit_reference as R
from paper_2511_10676_amd import binding as B

pytestmark = pytest.mark.gpu


def _step(fourbit, seqs=3, Hq=8, H=2, D=64, ps=16, width=8, seed=1):
    """A decode step's buffers and the step itself, which works in place."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    pages = seqs * width
    s = dict(table=torch.randperm(pages, generator=g, device="cuda").view(seqs, width).to(torch.int32).contiguous(),
             lengths=torch.tensor([0, 17, 100][:seqs], dtype=torch.int32, device="cuda"), turns=B.rotation_table(ps * width, D),
             x=torch.randn((seqs, Hq + 2 * H, D), generator=g, device="cuda").bfloat16(), w=torch.randn(D, generator=g, device="cuda").bfloat16())
    if fourbit:
        s["cache"] = [torch.randint(0, 256, (pages, H, ps, D // 2), generator=g, device="cuda").to(torch.uint8) for _ in range(2)] + \
                     [torch.full((pages, H, D // 32, ps), 126, dtype=torch.uint8, device="cuda") for _ in range(2)]
    else:
        s["cache"] = [torch.randn((pages, H, ps, D), generator=g, device="cuda").bfloat16() for _ in range(2)]
    q, k, v = s["x"][:, :Hq], s["x"][:, Hq:Hq + H], s["x"][:, Hq + H:]
    out = B.Attention(torch.empty((seqs, Hq, D), dtype=torch.bfloat16, device="cuda"), torch.empty((seqs, Hq), device="cuda"))
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")

    def step(stream=None):
        kw = dict(q_weight=s["w"], k_weight=s["w"], stream=stream)
        if fourbit:
            B.rotate(q, k, s["lengths"], s["turns"], out=B.Rotated(qo, ko), **kw)
            B.cache_append_fourbit(ko, v, *s["cache"], s["table"], s["lengths"], stream=stream)
        else:
            B.rotate_append(q, k, v, *s["cache"], s["table"], s["lengths"], s["turns"], out=qo, **kw)
        with (torch.cuda.stream(stream) if stream is not None else torch.cuda.stream(torch.cuda.current_stream())):
            s["lengths"] += 1
        attend = B.attend_fourbit if fourbit else B.attend
        attend(qo, *s["cache"], s["table"], s["lengths"], out=out, workspace=ws, stream=stream)
    return s, step, out


@pytest.mark.parametrize("fourbit", [False, True])
def test_a_run_of_steps_against_the_formulas(fourbit):
    s, step, out = _step(fourbit)
    Hq, H, D = 8, 2, 64
    for turn in range(4):
        n = s["lengths"].cpu().numpy()
        before = [t.clone() for t in s["cache"]]
        step()
        torch.cuda.synchronize()
        x, w = s["x"].double().cpu().numpy(), s["w"].double().cpu().numpy()
        turns = s["turns"].cpu().numpy()[n]
        table = s["table"].cpu().numpy()
        qr, qtol = R.rotate(x[:, :Hq], w, turns, "halves", float(np.float32(1e-6)), "bf16")
        # the step's own rounded queries and keys, which the tests of rotate alone hold to the formula; here: that they are the ones used
        got = B.rotate(s["x"][:, :Hq], s["x"][:, Hq:Hq + H], torch.from_numpy(n).cuda(), s["turns"], q_weight=s["w"], k_weight=s["w"])
        assert np.all(np.abs(got.q.double().cpu().numpy() - qr) <= qtol)
        if fourbit:
            k, v = (R.values(p.cpu().numpy(), c.transpose(2, 3).cpu().numpy()) for p, c in ((before[0], before[2]), (before[1], before[3])))
            new = [R.to_fourbit(t.float().cpu().numpy())[0] for t in (got.k, s["x"][:, Hq + H:])]
        else:
            k, v = (t.double().cpu().numpy() for t in before)
            new = [t.double().cpu().numpy() for t in (got.k, s["x"][:, Hq + H:])]
        for b in range(3):
            k[table[b, n[b] // 16], :, n[b] % 16], v[table[b, n[b] // 16], :, n[b] % 16] = new[0][b], new[1][b]
        want, tol = R.attend(got.q.double().cpu().numpy(), k, v, table, n + 1, None, 0.125, 128, "bf16")
        # (attend over bf16 rows has its own tests: two parts of P and twice the rounding are what those allow)
        extra = 0 if fourbit else 2.0 ** -15 * np.abs(v).max()
        assert np.all(np.abs(out.out.double().cpu().numpy() - want[0]) <= tol[0] + extra), turn
        assert np.all(np.abs(out.lse.cpu().numpy() - want[1]) <= tol[1] + (0 if fourbit else 1e-5))


@pytest.mark.parametrize("fourbit", [False, True])
def test_a_captured_step_replayed_with_eager_work_between(fourbit):
    s, step, out = _step(fourbit)
    r, eager, want = _step(fourbit)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)                                                      # warm up on another stream
    side.synchronize()
    eager()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    other, other_step, other_out = _step(fourbit, seed=2)
    for turn in range(5):
        s["x"].copy_(r["x"].roll(1, 0))
        r["x"].copy_(s["x"])
        graph.replay()
        other_step()                                                # eager work between
        torch.cuda.synchronize()
        eager()
        torch.cuda.synchronize()
        assert torch.equal(out.out, want.out) and torch.equal(out.lse, want.lse) and torch.equal(s["lengths"], r["lengths"]), turn
        assert all(torch.equal(a, b) for a, b in zip(s["cache"], r["cache"])), turn


def test_two_captured_attentions_share_a_workspace():
    a = []
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(8)
    for n in (3000, 5000):
        pages = -(-n // 16)
        kp, vp = (torch.randint(0, 256, (pages, 2, 16, 64), generator=g, device="cuda").to(torch.uint8) for _ in range(2))
        ks, vs = (torch.randint(124, 130, (pages, 2, 4, 16), generator=g, device="cuda").to(torch.uint8) for _ in range(2))
        args = (torch.randn((1, 8, 128), generator=g, device="cuda").bfloat16(), kp, vp, ks, vs,
                torch.arange(pages, dtype=torch.int32, device="cuda").view(1, -1), torch.tensor([n], dtype=torch.int32, device="cuda"))
        want = B.attend_fourbit(*args)
        out = B.Attention(torch.empty_like(want.out))
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            B.attend_fourbit(*args, out=out, workspace=ws)
        a.append((graph, out, want, args))                          # (a graph does not keep its tensors)
    for turn in range(4):
        for graph, out, _, _ in (a if turn % 2 else a[::-1]):
            out.out.zero_()
            graph.replay()
        torch.cuda.synchronize()
        for _, out, want, _ in a:
            assert torch.equal(out.out, want.out)
        ws.random_()


def test_results_are_the_same_every_time():
    g = torch.Generator(device="cuda").manual_seed(8)
    kp, vp = (torch.randint(0, 256, (600, 4, 16, 64), generator=g, device="cuda").to(torch.uint8) for _ in range(2))
    ks, vs = (torch.randint(124, 130, (600, 4, 4, 16), generator=g, device="cuda").to(torch.uint8) for _ in range(2))
    table = torch.randperm(600, generator=g, device="cuda").view(3, 200).to(torch.int32).contiguous()
    q, lengths = torch.randn((3, 16, 128), generator=g, device="cuda"), torch.tensor([3200, 100, 2000], dtype=torch.int32, device="cuda")
    first = B.attend_fourbit(q, kp, vp, ks, vs, table, lengths, want_lse=True)
    for _ in range(5):
        again = B.attend_fourbit(q, kp, vp, ks, vs, table, lengths, want_lse=True)
        assert torch.equal(first.out, again.out) and torch.equal(first.lse, again.lse)
