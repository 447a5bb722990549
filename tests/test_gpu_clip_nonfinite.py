"""A gradient norm that is not finite stops the whole step, wherever the bad element is: the
Muon matrices keep weight and momentum as AdamW's tensors do, and the status says so."""

import math

import numpy as np
import pytest
import torch

from oracle import muon_oracle as orc

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32


def same(xs, ys):
    return all(torch.equal(x, y) for x, y in zip(xs, ys))


def problem(cols, wdt, gdt, seed=91):
    gen = torch.Generator().manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=gen).cuda()
    W = [(rand(136, cols) * 0.02).to(wdt) for _ in range(3)] + [(rand(cols, 136) * 0.02).to(wdt)]
    G = [torch.randn(w.shape, generator=gen).cuda().to(gdt) for w in W]
    M = [torch.randn(w.shape, generator=gen).cuda() * 0.1 for w in W]
    return W, G, M, gen


def context(b, W, G, M):
    return b.MuonContext([(W[:3], G[:3], M[:3]), (W[3:], G[3:], M[3:])])


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("cols", [264, 203])  # both momentum kernels
@pytest.mark.parametrize("wdt,gdt", [(FP, FP), (FP, BF), (BF, BF)])
@pytest.mark.parametrize("protect", [False, True])
def test_a_bad_element_of_adamw_stops_muon(bad, cols, wdt, gdt, protect):
    from paper_2502_16982_b200 import binding as b

    W, G, M, gen = problem(cols, wdt, gdt)
    p, g = torch.randn(3000, generator=gen).cuda(), torch.randn(3000, generator=gen).cuda()
    m, v = torch.zeros(3000, device="cuda"), torch.zeros(3000, device="cuda")
    ctx = context(b, W, G, M)
    hp = b.Hyper(lr=1e-2, protect_momentum=protect)
    good = float(g[1234])
    g[1234] = bad
    before = [t.clone() for t in W + M + [p, m, v]]

    def step():
        total = b.muon_grad_norm(G + [g], max_norm=1.0)
        b.muon_clip_grads(G, 1.0, sum_sq=total.sum_sq)
        ctx.muon_step(hp, coef=total.coef)
        b.muon_adamw_step([p], [g], [m], [v], 1, lr=1e-2, wd=0.1, coef=total.coef)
        return total

    total = step()
    assert math.isnan(float(total.coef))
    assert ctx.muon_status()[0] == b.MUON_ERR_NONFINITE  # of all matrices one
    assert same(W + M + [p, m, v], before)
    # the next batch is finite: the step is muon_step's, to the bit
    g[1234] = good
    W2, G2, M2, _ = problem(cols, wdt, gdt)
    plain = context(b, W2, G2, M2)
    total = step()
    assert 0.0 < float(total.coef) < 1.0 and ctx.muon_status() == (0, -1)
    b.muon_clip_grads(G2, 1.0, sum_sq=total.sum_sq)
    plain.muon_step(hp)
    assert same(W + M, W2 + M2) and not same(W, before) and not torch.equal(p, before[-3])
    ctx.muon_destroy()
    plain.muon_destroy()


def test_a_replayed_step_reads_the_coefficient_of_the_moment():
    from paper_2502_16982_b200 import binding as b

    W, G, M, _ = problem(264, FP, BF)
    ctx = context(b, W, G, M)
    coef = torch.ones(1, device="cuda")
    ctx.muon_step(b.Hyper(lr=1e-2), coef=coef)
    W2, G2, M2, _ = problem(264, FP, BF)
    plain = context(b, W2, G2, M2)
    plain.muon_step(b.Hyper(lr=1e-2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.muon_step(b.Hyper(lr=1e-2), coef=coef)
    assert same(W + M, W2 + M2)
    for value in (float("nan"), 0.25, float("nan"), 1.0):
        coef.fill_(value)
        graph.replay()
        if not math.isnan(value):
            plain.muon_step(b.Hyper(lr=1e-2))
        assert same(W + M, W2 + M2)
        assert (ctx.muon_status()[0] == b.MUON_ERR_NONFINITE) == math.isnan(value)
    del graph
    ctx.muon_destroy()
    plain.muon_destroy()


def test_other_ranks_parameters_stop_the_owner_computes_step():
    from paper_2502_16982_b200 import binding as b
    from paper_2502_16982_b200.distributed import DistributedMuon

    m = DistributedMuon([(128, 192, 3, FP, FP), (64, 64, 2, BF, BF)], "cuda")
    gen = torch.Generator().manual_seed(92)
    for group in m.grads:
        for g in group:
            g.copy_(torch.randn(g.shape, generator=gen))
    weights = [w for group in m.weights for w in group]
    momenta = [t[2] for mats in m.unit_mats for t in mats]
    before = [t.clone() for t in weights + momenta]
    r = m.clip_grads(1.0, others=torch.tensor([float("nan")], dtype=torch.float64, device="cuda"))
    m.step(b.Hyper(lr=1e-2), coef=r.coef)
    assert m.status()[0] == b.MUON_ERR_NONFINITE and same(weights + momenta, before)
    r = m.clip_grads(1.0, others=torch.tensor([2.0], dtype=torch.float64, device="cuda"))
    m.step(b.Hyper(lr=1e-2), coef=r.coef)
    assert m.status() == (0, -1) and not same(weights + momenta, before)
    m.close()


def test_the_examples_step():
    import os
    import sys

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    sys.path.insert(0, os.path.join(root, "examples"))
    import train_and_distill as ex

    model = ex.Model(512, 64, 5, max_norm=1.0)
    tokens = ex.Chain(512, 1).batch(8, 10)
    state = lambda: [t.clone() for t in [model.embed, model.head, model.embed16, model.head16] + list(model.moments) + [model.mats, model.mats16, model.momentum]]
    x, kept = model.hidden(tokens)
    d = torch.randn(x.shape, device="cuda").to(x.dtype)
    model.backward(d, kept)
    model.head_grad.normal_()
    model.head_grad[3, 5] = float("nan")
    before = state()
    model.step(1e-2)
    assert same(state(), before) and model.muon.muon_status()[0] != 0
    model.head_grad[3, 5] = 0.0
    model.step(1e-2)
    assert not same(state(), before) and model.muon.muon_status() == (0, -1)


def test_refusals():
    from paper_2502_16982_b200 import binding as b

    W, G, M, _ = problem(264, FP, FP)
    ctx = context(b, W, G, M)
    before = [w.clone() for w in W]
    for bad in (torch.ones(1), torch.ones(2, device="cuda"), torch.ones(1, device="cuda", dtype=torch.float64)):
        for call in (lambda: ctx.muon_step(b.Hyper(), coef=bad), lambda: ctx.muon_step_bucket(b.Hyper(), 0, coef=bad)):
            with pytest.raises(b.MuonError):
                call()
    assert same(W, before)
    ctx.muon_destroy()
