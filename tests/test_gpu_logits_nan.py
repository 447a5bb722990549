"""A NaN anywhere in a row makes the row's statistics and gradient NaN: in the elements outside
whole 16-byte vectors as well, whatever else the row holds."""

import numpy as np
import pytest
import torch

from oracle import logprob_oracle as lo
from test_gpu_logits_logprob import check_rows, f64, strided

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32
INF = float("inf")


@pytest.mark.parametrize("V", [1, 3, 5, 17, 2003, 30001])
@pytest.mark.parametrize("offset", [0, 1, 3, 7])
@pytest.mark.parametrize("rest", ["normal", "minus_infinity", "minus_infinity_but_one"])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_a_nan_at_a_rows_ends(V, offset, rest, dtype):
    from paper_2502_16982_b200 import binding as b

    gen = torch.Generator().manual_seed(10 * V + offset)
    base = torch.randn(V, generator=gen) * 2
    if rest != "normal":
        base[:] = -INF
        if rest == "minus_infinity_but_one":
            base[V // 2] = 1.5
    places = sorted({0, 1, 6, V // 2, V - 7, V - 2, V - 1} & set(range(V)))
    z = base.repeat(len(places) + 1, 1)
    for i, p in enumerate(places):
        z[i, p] = float("nan")  # the last row has none
    rows = len(places)
    for times in (1, 120):  # a cluster a row, a block a row
        d = strided(z.repeat(times, 1), dtype, 0, offset)
        y = torch.full((len(d),), V // 3, dtype=torch.int64, device="cuda")
        top = min(V, 4)
        r = b.muon_logits_logprob(d, y, top=top, logit_scale=0.5)
        for name in ("logprob", "entropy", "lse"):
            got = getattr(r, name).view(times, rows + 1)
            assert bool(torch.isnan(got[:, :rows]).all()), name
            assert not bool(torch.isnan(got[:, rows]).any()), name
        ids = lo.best(f64(d), top)
        assert np.array_equal(r.top_ids.cpu().numpy(), ids)
        g = b.muon_logits_logprob_grad(d, y, r, g_logprob=torch.ones(len(d), device="cuda"), g_entropy=torch.ones(len(d), device="cuda"),
                                       logit_scale=0.5)
        g = g.reshape(times, rows + 1, V)
        assert bool(torch.isnan(g[:, :rows]).all()) and bool(torch.isfinite(g[:, rows]).all())
        one = b.LogitsLogprob(*[t[rows:rows + 1] for t in r])
        check_rows(one, f64(d[rows:rows + 1]), y[:1].cpu().numpy(), 0.5, top)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_infinities_at_a_rows_ends(dtype):
    """Plus infinity makes a row NaN, minus infinity is probability 0, there too."""
    from paper_2502_16982_b200 import binding as b

    gen = torch.Generator().manual_seed(9)
    for V in (1, 3, 17, 2003):
        z = torch.randn(6, V, generator=gen)
        z[0, 0] = z[1, -1] = INF
        z[2, 0] = z[3, -1] = -INF
        z[4, 1:] = -INF
        z[5, :-1] = -INF
        d = strided(z, dtype, 3, 1)
        y = torch.tensor([0, 0, V // 2, 0, 0, V - 1], device="cuda")
        r = b.muon_logits_logprob(d, y, top=1)
        assert all(bool(torch.isnan(t[:2]).all()) for t in (r.logprob, r.entropy, r.lse))
        part = b.LogitsLogprob(*[t[2:] for t in r])
        check_rows(part, f64(d[2:]), y[2:].cpu().numpy(), 1.0, 1)
