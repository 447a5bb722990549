"""Global gradient norm, clipping and the clipped AdamW step against plain fp64.

Tolerances.  A thread adds at most 64 squares in two fp32 chains of 32, each within
2^-24 of a partial sum, and the rest in fp64: the sum of squares is within 34 2^-24
relative, the norm within 17 2^-24 plus its own rounding, the coefficient within one
rounding more.  A clipped element adds the rounding of the product: 2^-24 for fp32,
2^-8 for bf16.  Where a result has to be the same bits, it is compared for equality."""

import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32
E_NORM = 18 * 2.0 ** -24
E_COEF = E_NORM + 2.0 ** -24


def tensors(spec, seed, std=1e-2):
    """(numel, dtype, elements before it in its storage) -> views and their storages."""
    gen = torch.Generator().manual_seed(seed)
    views, stores = [], []
    for n, dtype, offset in spec:
        store = torch.full((offset + n + 9,), 3.0, dtype=dtype)
        store[offset:offset + n] = (torch.randn(n, generator=gen) * std).to(dtype)
        store = store.cuda()
        views.append(store[offset:offset + n])
        stores.append(store)
    return views, stores


def norm64(ts):
    return math.sqrt(math.fsum(float((t.double() ** 2).sum()) for t in ts))


SETS = {
    "one": [(1, FP, 0)],
    "one_bf16_odd": [(7, BF, 3)],
    "mixed": [(5, BF, 1), (4096, FP, 0), (16385, BF, 5), (8193, FP, 3), (100003, BF, 8), (1, BF, 7), (33333, FP, 1)],
    "empty_inside": [(0, FP, 0), (777, BF, 0), (0, BF, 0), (9, FP, 2)],
    "large": [(3_000_001, BF, 0), (2_500_000, FP, 0)],
    "many": [(1 + 13 * i % 500, BF if i % 3 else FP, i % 5) for i in range(2500)],
}


@pytest.mark.parametrize("name", list(SETS))
def test_norm_matches_fp64(name):
    from paper_2502_16982_b200 import binding as b

    ts, _ = tensors(SETS[name], 11)
    want = norm64(ts)
    r = b.muon_grad_norm(ts, max_norm=0.25 * want)
    assert abs(float(r.sum_sq) - want * want) <= 34 * 2.0 ** -24 * want * want
    assert abs(float(r.norm) - want) <= E_NORM * want
    coef = min(1.0, 0.25 * want / (want + 1e-6))
    assert abs(float(r.coef) - coef) <= E_COEF * coef
    again = b.muon_grad_norm(ts, max_norm=0.25 * want)
    assert all(torch.equal(x, y) for x, y in zip(r, again))


@pytest.mark.parametrize("name", list(SETS))
@pytest.mark.parametrize("out", [None, BF, FP])
def test_clipping_matches_fp64_and_stays_inside(name, out):
    from paper_2502_16982_b200 import binding as b

    ts, stores = tensors(SETS[name], 12)
    before = [t.clone() for t in ts]
    want = norm64(ts)
    outs = out_stores = None
    if out is not None:  # other alignments than the gradients'
        outs, out_stores = tensors([(n, out, (o + 2) % 6) for n, _, o in SETS[name]], 13)
    r = b.muon_clip_grads(ts, 0.3 * want, out=outs)
    coef = 0.3 * want / (want + 1e-6)
    assert abs(float(r.norm) - want) <= E_NORM * want and abs(float(r.coef) - coef) <= E_COEF * coef
    for i, g in enumerate(before):
        got = ts[i] if outs is None else outs[i]
        step = 2.0 ** -8 if got.dtype == BF else 2.0 ** -24
        exact = g.double() * coef
        assert bool(((got.double() - exact).abs() <= (step + 1.01 * E_COEF) * exact.abs()).all()), i
        assert torch.equal(got, (g.float() * r.coef).to(got.dtype))
        if outs is not None:
            assert torch.equal(ts[i], g)
    for (n, _, o), s in zip(SETS[name], stores):
        assert bool((s[:o] == 3).all()) and bool((s[o + n:] == 3).all())
    for (n, _, o), s in zip(SETS[name], out_stores or []):
        o = (o + 2) % 6
        assert bool((s[:o] == 3).all()) and bool((s[o + n:] == 3).all())


def test_below_the_limit_nothing_changes():
    from paper_2502_16982_b200 import binding as b

    ts, _ = tensors(SETS["mixed"], 14)
    before = [t.clone() for t in ts]
    for limit in (2.0 * norm64(ts), float("inf")):
        r = b.muon_clip_grads(ts, limit)
        assert float(r.coef) == 1.0 and all(torch.equal(x, y) for x, y in zip(ts, before))
    outs = [torch.empty_like(t, dtype=FP) for t in ts]
    b.muon_clip_grads(ts, 2.0 * norm64(ts), out=outs)
    assert all(torch.equal(o, t.float()) for o, t in zip(outs, ts))
    # a norm of 0: nothing to clip, whatever the limit; a limit of 0 makes everything 0
    zeros = [torch.zeros(5000, device="cuda"), torch.zeros(3, dtype=BF, device="cuda")]
    r = b.muon_clip_grads(zeros, 1.0)
    assert float(r.norm) == 0.0 and float(r.coef) == 1.0
    r = b.muon_clip_grads(zeros, 0.0, eps=0.0)
    assert float(r.norm) == 0.0 and float(r.coef) == 1.0
    r = b.muon_clip_grads(ts, 0.0)
    assert float(r.coef) == 0.0 and all(bool((t == 0).all()) for t in ts)


@pytest.mark.parametrize("magnitude", [1e-38, 1e-30, 1e-20, 1e20, 3e37])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_norm_of_any_magnitude(magnitude, dtype):
    """Squares that fp32 cannot hold."""
    from paper_2502_16982_b200 import binding as b

    gen = torch.Generator().manual_seed(15)
    t = ((torch.rand(50001, generator=gen) + 0.5) * magnitude).to(dtype).cuda()
    small = (torch.randn(777, generator=gen) * 1e-3).cuda()
    for ts in ([t], [t, small]):
        want = norm64(ts)
        r = b.muon_grad_norm(ts)
        assert abs(float(r.sum_sq) - want * want) <= 34 * 2.0 ** -24 * want * want
        if want < 3e38:
            assert abs(float(r.norm) - want) <= E_NORM * want
        else:
            assert float(r.norm) == float("inf")


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_a_norm_that_is_not_finite_clips_nothing(bad):
    from paper_2502_16982_b200 import binding as b

    ts, _ = tensors(SETS["mixed"], 16)
    ts[4][99_990] = bad
    before = [t.clone() for t in ts]
    r = b.muon_clip_grads(ts, 1e-3)
    assert not math.isfinite(float(r.norm)) and math.isnan(float(r.coef))
    same = lambda x, y: torch.equal(torch.nan_to_num(x, 7.0), torch.nan_to_num(y, 7.0))
    assert all(same(x, y) for x, y in zip(ts, before))
    # and the AdamW step that is given the coefficient changes nothing
    p, m, v = (torch.randn(5000, device="cuda") for _ in range(3))
    kept = p.clone(), m.clone(), v.clone()
    b.muon_adamw_step([p], [torch.ones(5000, device="cuda")], [m], [v], 3, lr=0.1, wd=0.1, coef=r.coef)
    assert all(torch.equal(x, y) for x, y in zip((p, m, v), kept))


@pytest.mark.parametrize("pdt,gdt", [(FP, FP), (FP, BF), (BF, BF), (BF, FP)])
def test_clipped_adamw_is_adamw_on_scaled_gradients(pdt, gdt):
    from paper_2502_16982_b200 import binding as b

    sizes = [(2048, 0), (64_000, 0), (7, 1), (42_957, 1), (1, 0)] + [(64, 0)] * 50

    def state(seed):
        gen = torch.Generator().manual_seed(seed)
        out = []
        for n, o in sizes:
            row = []
            for dt, std in ((pdt, 0.02), (gdt, 1e-2), (FP, 1e-3), (FP, 1e-3)):
                t = (torch.randn(n + o, generator=gen) * std).to(dt).cuda()
                row.append(t[o:])
            row[3].abs_()
            out.append(row)
        return [list(c) for c in zip(*out)]

    for limit, expect in ((0.5, None), (1e9, 1.0)):
        p, g, m, v = state(17)
        r = b.muon_grad_norm(g, max_norm=limit * norm64(g) if expect is None else limit)
        if expect is not None:
            assert float(r.coef) == expect
        b.muon_adamw_step(p, g, m, v, 4, lr=1e-3, wd=0.1, coef=r.coef)
        p2, g2, m2, v2 = state(17)
        b.muon_adamw_step(p2, [x.float() * r.coef for x in g2], m2, v2, 4, lr=1e-3, wd=0.1)
        for x, y in zip(p + m + v, p2 + m2 + v2):
            assert torch.equal(x, y)


def test_sums_of_ranks_are_added_before_the_coefficient():
    """Two ranks that own different tensors: each scales its own by the coefficient of all."""
    from paper_2502_16982_b200 import binding as b

    ts, _ = tensors(SETS["mixed"], 18)
    before = [t.clone() for t in ts]
    want = norm64(ts)
    mine, theirs = b.MuonGrads(ts[:3]), b.MuonGrads(ts[3:])
    total = mine.muon_grad_norm().sum_sq + theirs.muon_grad_norm().sum_sq
    for h in (mine, theirs):
        r = h.muon_clip_grads(0.5 * want, sum_sq=total)
        assert abs(float(r.norm) - want) <= E_NORM * want
    for t, g in zip(ts, before):
        assert torch.equal(t, (g.float() * r.coef).to(t.dtype))


def test_other_stream_and_captured_graph():
    from paper_2502_16982_b200 import binding as b

    ts, _ = tensors(SETS["mixed"], 19)
    outs = [torch.zeros_like(t) for t in ts]
    h = b.MuonGrads(ts, out=outs)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    r = h.muon_clip_grads(0.1, stream=side)
    side.synchronize()
    for o, g in zip(outs, ts):
        assert torch.equal(o, (g.float() * r.coef).to(o.dtype))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = h.muon_clip_grads(0.1)
    for k in (1.0, 4.0):
        for t in ts:
            t.mul_(k)
        graph.replay()
        torch.cuda.synchronize()
        want = norm64(ts)
        assert abs(float(r.norm) - want) <= E_NORM * want
        for o, g in zip(outs, ts):
            assert torch.equal(o, (g.float() * r.coef).to(o.dtype))


def test_a_tensor_past_32_bit_offsets():
    from paper_2502_16982_b200 import binding as b

    n = (1 << 31) + 12345
    t = torch.zeros(n, dtype=BF, device="cuda")
    t[-5:] = 2.0
    t[(1 << 31) - 1] = 1.0
    r = b.muon_clip_grads([t], math.sqrt(21.0) / 4, eps=0.0)
    assert float(r.sum_sq) == 21.0
    assert torch.equal(t[-5:], torch.full((5,), 0.5, dtype=BF, device="cuda")) and float(t[(1 << 31) - 1]) == 0.25
    assert int((t != 0).sum()) == 6


def test_norm_before_muon_and_adamw_steps():
    """A step's gradients clipped together: matrices for Muon in place, the rest inside AdamW."""
    from oracle import adamw_oracle as aw, muon_oracle as orc
    from paper_2502_16982_b200 import binding as b

    gen = torch.Generator().manual_seed(20)
    rand = lambda *s: torch.randn(*s, generator=gen).cuda()
    W, G, M = rand(128, 256) * 0.02, rand(128, 256), rand(128, 256) * 0.1
    p, g = rand(3000) * 0.02, rand(3000).to(BF)
    m, v = torch.zeros(3000, device="cuda"), torch.zeros(3000, device="cuda")
    before = [t.double().cpu().numpy() for t in (W, G, M, p, g)]
    want = norm64([G, g])
    ctx = b.MuonContext([([W], [G], [M])])
    total = b.muon_grad_norm([G, g], max_norm=0.1 * want)
    b.muon_clip_grads([G], 0.1 * want, sum_sq=total.sum_sq)
    ctx.muon_step(b.Hyper(lr=1e-2))
    b.muon_adamw_step([p], [g], [m], [v], 1, lr=1e-2, wd=0.1, coef=total.coef)
    assert ctx.muon_status() == (0, -1)
    coef = 0.1 * want / (want + 1e-6)
    W0, G0, M0, p0, g0 = before
    ref = orc.muon_step(W0, G0 * coef, M0, orc.Hyper(lr=1e-2, wd=0.1, mu=0.95, nesterov=True, ns_steps=5, eps=1e-7))
    err = np.linalg.norm(M.double().cpu().numpy() - ref["M"]) / np.linalg.norm(ref["M"])
    assert err <= 1e-5
    dW, dref = W.double().cpu().numpy() - W0, ref["W"] - W0
    assert np.linalg.norm(dW - dref) <= 2e-2 * np.linalg.norm(dref)
    pr, mr, vr = aw.adamw_step(p0, g0 * coef, np.zeros(3000), np.zeros(3000), 1, lr=1e-2, wd=0.1)
    for got, ref1 in ((p, pr), (m, mr), (v, vr)):
        assert np.linalg.norm(got.double().cpu().numpy() - ref1) <= 1e-5 * np.linalg.norm(ref1)


def test_refusals_of_the_handle():
    from paper_2502_16982_b200 import binding as b

    t = torch.ones(100, device="cuda")
    for bad in (dict(grads=[]), dict(grads=[torch.ones(4, 4, device="cuda").t()]), dict(grads=[t, torch.ones(3)]),
                dict(grads=[t.half()]), dict(grads=[t], out=[torch.ones(99, device="cuda")]), dict(grads=[t], out=[]),
                dict(grads=[t], workspace=torch.zeros(4, device="cuda"))):
        with pytest.raises(b.MuonError):
            b.MuonGrads(**bad)
    twice = b.MuonGrads([t, t])
    assert float(twice.muon_grad_norm().sum_sq) == 200.0
    with pytest.raises(b.MuonError):
        twice.muon_clip_grads(1.0)
    for limit, eps in ((-1.0, 0.0), (float("nan"), 0.0), (1.0, -1.0), (1.0, float("inf"))):
        with pytest.raises(b.MuonError):
            b.MuonGrads([t]).muon_grad_norm(limit, eps)
    with pytest.raises(b.MuonError):
        b.MuonGrads([t], workspace=torch.zeros(100, dtype=torch.uint8, device="cuda")).muon_grad_norm()
    with pytest.raises(b.MuonError):
        b.MuonGrads([t]).muon_grad_norm(norm=torch.zeros(2, device="cuda"))
    with pytest.raises(b.MuonError):
        b.muon_adamw_step([t], [t.clone()], [t.clone()], [t.clone()], 1, lr=0.1, wd=0.0, coef=torch.ones(1))
    assert float(t.sum()) == 100.0


def test_owner_computes_step_clips_its_gradients():
    from paper_2502_16982_b200 import binding as b
    from paper_2502_16982_b200.distributed import DistributedMuon

    m = DistributedMuon([(128, 192, 3, FP, FP), (64, 64, 2, BF, BF)], "cuda")
    gen = torch.Generator().manual_seed(21)
    for group in m.grads:
        for g in group:
            g.copy_(torch.randn(g.shape, generator=gen))
    before = [g.clone() for group in m.grads for g in group]
    other = torch.randn(1000, generator=gen).cuda()
    want = norm64(before + [other])
    r = m.clip_grads(0.5 * want, others=b.muon_grad_norm([other]).sum_sq)
    assert abs(float(r.norm) - want) <= E_NORM * want
    clipped = [g for group in m.grads for g in group]
    for g, x in zip(clipped, before):
        assert torch.equal(g, (x.float() * r.coef).to(x.dtype))
    before = [g.clone() for g in clipped]
    r = m.clip_grads(float("inf"))  # the handle is kept
    assert float(r.coef) == 1.0 and abs(float(r.norm) - norm64(before)) <= E_NORM * norm64(before)
    assert all(torch.equal(g, x) for g, x in zip(clipped, before))
    m.step(b.Hyper(lr=1e-2))
    assert m.status() == (0, -1)
    m.close()
