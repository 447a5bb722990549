"""Masks of finite numbers far below every logit, at any logit scale: -1e30, -1e10 and the
lowest number of the type are out like minus infinity; -1e9 and -1e4 are numbers.

Tolerances: those of test_gpu_logits_logprob.py, whose exponents are measured from the
reference m, the rounded exponent of the largest logit.  That rounding, at most |m| 2^-24,
is in every exponent of a row: it adds to the distances from the reference, and to log2 of
the sum, whose own rounding is 2^-23 of it."""

import numpy as np
import pytest
import torch

from oracle import logprob_oracle as lo
from test_gpu_logits_logprob import check_rows, expect, f64, strided

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32
V = 20003


def rows(T, mask, dtype, seed):
    """Masked in nine of ten columns, in all but 2 %, and, the first row, throughout."""
    gen = torch.Generator().manual_seed(seed)
    z = torch.randn(T, V, generator=gen) * 2
    share = torch.where(torch.arange(T) % 2 == 0, 0.9, 0.98)[:, None]
    masked = torch.rand(T, V, generator=gen) < share
    masked[:, 77] = False
    masked[0] = True
    value = torch.finfo(dtype).min if mask == "lowest" else mask
    return torch.where(masked, torch.tensor(value), z), masked, gen


@pytest.mark.parametrize("scale", [0.5, 0.7, 1.0, 1.6])
@pytest.mark.parametrize("mask", [-1e4, -1e9, -1e10, -1e30, -3e38, "lowest"])
@pytest.mark.parametrize("T", [6, 600])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_finite_masks(T, mask, scale, dtype):
    from paper_2502_16982_b200 import binding as b

    z, masked, gen = rows(T, mask, dtype, 71)
    d = strided(z, dtype, 3, 2)
    y = torch.full((T,), 77)
    r = b.muon_logits_logprob(d, y.cuda(), top=20, logit_scale=scale)
    again = b.muon_logits_logprob(d, y.cuda(), top=20, logit_scale=scale)
    assert all(torch.equal(p, q) for p, q in zip(r, again))
    zz, some = f64(d), slice(1, min(T, 40))
    want, tol, log_q, counts = check_rows(b.LogitsLogprob(*[t[some] for t in r]), zz[some], y[some].numpy(), scale, 20)
    rr, hh = torch.randn(T, generator=gen), torch.randn(T, generator=gen) * 0.1
    g = b.muon_logits_logprob_grad(d, y.cuda(), r, g_logprob=rr.cuda(), g_entropy=hh.cuda(), logit_scale=scale)
    assert bool(torch.isfinite(g).all()) and not g[1:][masked[1:].cuda()].any()
    exact = lo.logprob_grad(log_q, want["entropy"], counts, y[some].numpy(), rr[some].double().numpy(), hh[some].double().numpy(), scale)
    u = 2.0 ** -22
    t, q = np.where(log_q > -1e4, np.abs(log_q), 0.0), np.exp(log_q)
    ra, ha = np.abs(rr[some].double().numpy()), np.abs(hh[some].double().numpy())
    size = ra[:, None] + ha[:, None] * (t + want["entropy"][:, None])
    err = scale * (q * size * (tol["lse"][:, None] + u * (3 + t)) + q * ha[:, None] * (tol["lse"] + tol["entropy"])[:, None]
                   + u * ra[:, None] * (q > 0))
    bound = err + (2.0 ** -8 if dtype == BF else 2.0 ** -24) * (np.abs(exact) + err) + 1e-36 * (1 + size)
    assert np.all(np.abs(f64(g[some]) - exact) <= bound)

    # the row of masks alone
    exponent = zz[0, 0] * scale * np.log2(np.e)
    if exponent <= -2.0 ** 31:
        assert float(r.lse[0]) == float(r.logprob[0]) == -float("inf") and float(r.entropy[0]) == 0.0
        assert not g[0].any()
        assert bool((r.top_logprob[0] == -float("inf")).all())
    else:
        far = abs(exponent) * 2.0 ** -24 + 16
        one, tol = expect(zz[:1], y[:1].numpy(), scale)[:2]
        n_c = (V / 4096 + 64) * 2.0 ** -24
        assert abs(float(r.logprob[0]) - one["logprob"][0]) <= tol["logprob"][0] + far * 2.0 ** -22
        assert abs(float(r.entropy[0]) - one["entropy"][0]) <= tol["entropy"][0] + far * (2.0 ** -22 + 2 * n_c)
        assert abs(float(r.lse[0]) - one["lse"][0]) <= tol["lse"][0]
        if abs(one["lse"][0]) >= 2.0 ** 24:
            assert not g[0].any()
    assert np.array_equal(r.top_ids[0].cpu().numpy(), np.arange(20))
    assert np.array_equal(f64(r.top_logits[0]), zz[0, :20])


@pytest.mark.parametrize("dtype", [BF, FP])
def test_a_target_that_is_masked(dtype):
    """Its log probability is the number that l - lse is."""
    from paper_2502_16982_b200 import binding as b

    z, masked, _ = rows(40, -1e30, dtype, 72)
    masked[1:, 5] = True
    z[1:, 5] = -1e30
    d = z.to(dtype).cuda()
    r = b.muon_logits_logprob(d, torch.full((40,), 5, device="cuda"), logit_scale=0.5)
    want = 0.5 * f64(d)[1:, 5]
    assert np.all(np.abs(f64(r.logprob)[1:] - want) <= 2.0 ** -22 * np.abs(want))


@pytest.mark.parametrize("dtype", [BF, FP])
def test_a_logit_far_above_counts_as_infinity(dtype):
    from paper_2502_16982_b200 import binding as b

    z = torch.randn(8, 3001, generator=torch.Generator().manual_seed(73))
    for i, value in enumerate((1e10, 1e30, torch.finfo(dtype).max)):
        z[i, 100] = z[i + 3, 3000] = value
    for times in (1, 120):
        d = strided(z.repeat(times, 1), dtype, 1, 1)
        r = b.muon_logits_logprob(d, torch.full((len(d),), 7, device="cuda"), top=2, logit_scale=0.9)
        for name in ("logprob", "entropy", "lse"):
            got = getattr(r, name).view(times, 8)
            assert bool(torch.isnan(got[:, :6]).all()) and not bool(torch.isnan(got[:, 6:]).any()), name
        assert np.array_equal(r.top_ids.cpu().numpy(), lo.best(f64(d), 2))
