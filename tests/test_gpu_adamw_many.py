"""AdamW over more tensors than one launch holds (600), and over the sizes at which a launch
deals its blocks out in another way, against the oracle.

Tolerances.  1 - 0.9f and 1 - 0.95f are 2^-22 off 0.1 and 0.05, and so are the corrections'
1 - beta^3; an operation rounds by 2^-24.  With a = |beta1 m| + |(1 - beta1) g|, m is within
2^-22 + 3 2^-24 < 2^-21 of a, v within 2^-22 + 5 2^-24 < 2^-20 of itself, the update within half
of v's, m's, 1.5 2^-22 of the corrections and 6 2^-24, < 2^-19, of lr a / (corrections, root); the
weight rounds by 2^-24 three times at most, and a bf16 weight by 2^-8 once more."""

import numpy as np
import pytest
import torch

from oracle import adamw_oracle as aw

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32
LR, WD, STEP = 1e-2, 0.1, 3


def f64(t):
    return t.double().cpu().numpy()


def state(sizes, seed):
    """Tensors of mixed types at mixed alignments, each with a guard behind it."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    out, guards = [], []
    for i, n in enumerate(sizes):
        off = i % 5 if i % 3 == 0 else 0
        row = []
        for dt, std in ((BF if i % 4 == 1 else FP, 0.02), (FP if i % 2 else BF, 1e-2), (FP, 1e-3), (FP, 1e-2)):
            store = torch.full((off + n + 3,), 5.0, dtype=dt, device="cuda")
            store[off:off + n] = (torch.randn(n, generator=gen, device="cuda") * std).to(dt)
            row.append(store[off:off + n])
            guards.append((store, off, n))
        row[3].square_()
        out.append(row)
    return [list(c) for c in zip(*out)], guards


SIZES = {
    "600": [1 + 37 * i % 300 for i in range(600)],
    "601": [1 + 37 * i % 300 for i in range(600)] + [5001],
    "1301": [1 + 41 * i % 200 for i in range(1300)] + [100003],
    "48": [1 + 37 * i % 300 for i in range(48)],
    "49": [20011] + [1 + 37 * i % 300 for i in range(48)],
    "few_elements": [65536, 1408, 7, 42957],
    "lone": [3_000_001, 1_000_000, 4097],
    "both_ways": [9_000_000, 70_001, 128],   # bf16 gradients a vector a thread, fp32 two
    "large": [17_000_003, 2048, 2049, 30],
}


@pytest.mark.parametrize("name", list(SIZES))
@pytest.mark.parametrize("coef", [None, 0.3])
def test_every_tensor_is_stepped_once(name, coef):
    from paper_2502_16982_b200 import binding as b

    (p, g, m, v), guards = state(SIZES[name], 81)
    before = [[t.clone() for t in c] for c in (p, g, m, v)]
    c = None if coef is None else torch.tensor([coef], device="cuda")
    b.muon_adamw_step(p, g, m, v, STEP, lr=LR, wd=WD, coef=c)
    factor = 1.0 if coef is None else float(c)
    for i in range(len(p)):
        p0, g0, m0, v0 = (f64(x[i]) for x in before)
        pr, mr, vr = aw.adamw_step(p0, g0 * factor, m0, v0, STEP, lr=LR, wd=WD)
        terms = 0.9 * np.abs(m0) + 0.1 * np.abs(g0) * factor
        assert np.all(np.abs(f64(m[i]) - mr) <= 2.0 ** -21 * terms + 1e-37), i
        assert np.all(np.abs(f64(v[i]) - vr) <= 2.0 ** -20 * vr + 1e-37), i
        root = np.sqrt(vr / (1 - 0.95 ** STEP)) + 1e-8
        tol = LR * 2.0 ** -19 * terms / (1 - 0.9 ** STEP) / root + 2.0 ** -22 * np.abs(p0)
        if p[i].dtype == BF:
            tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(pr)
        assert np.all(np.abs(f64(p[i]) - pr) <= tol), i
        assert torch.equal(g[i], before[1][i])
    for store, off, n in guards:
        assert bool((store[:off] == 5).all()) and bool((store[off + n:] == 5).all())
    # again, from the same state: the same bits
    (p2, g2, m2, v2), _ = state(SIZES[name], 81)
    b.muon_adamw_step(p2, g2, m2, v2, STEP, lr=LR, wd=WD, coef=c)
    assert all(torch.equal(x, y) for x, y in zip(p + m + v, p2 + m2 + v2))


def test_a_coefficient_that_is_nan_stops_every_launch():
    from paper_2502_16982_b200 import binding as b

    (p, g, m, v), _ = state(SIZES["1301"], 82)
    before = [t.clone() for t in p + m + v]
    b.muon_adamw_step(p, g, m, v, STEP, lr=LR, wd=WD, coef=torch.full((1,), float("nan"), device="cuda"))
    assert all(torch.equal(x, y) for x, y in zip(p + m + v, before))
