"""The LM-head losses where numbers, sizes or layouts are extreme.

Tolerances are those of test_gpu_head_loss.py, derived there."""

import numpy as np
import pytest
import torch

from oracle import head_oracle as ho
from test_gpu_head_loss import BF, FP, check, coefficients, f64, knobs, make  # noqa: F401

pytestmark = pytest.mark.gpu


def shifted(T, D, V, seed, shift, spread):
    """Logits of about `shift`, spread around it: one column of x and w carries the shift."""
    x, w, gen = make(T, D, V, seed, gain=spread)
    x[:, 0] = abs(shift) ** 0.5
    w[:, 0] = abs(shift) ** 0.5 * (1 if shift > 0 else -1)
    return x, w, gen


@pytest.mark.parametrize("codes", [1, 2])
@pytest.mark.parametrize("T", [70, 300])
@pytest.mark.parametrize("shift,spread", [(3000, 3.0), (-3000, 3.0), (10000, 3.0), (-10000, 3.0), (0, 1000.0), (0, 4000.0)])
def test_logits_of_thousands(knobs, codes, T, shift, spread):  # noqa: F811
    """The rounding of a row's largest logit must not cost it its gradient; the largest is
    hardly ever the target here.  Few tokens and gathered ones, codes and second product."""
    b = knobs
    b.muon_debug_set_head_codes(codes)
    V = 1500
    x, w, gen = shifted(T, 64, V, 41 + T, shift, spread) if shift else make(T, 64, V, 43 + T, gain=spread)
    t = torch.randint(0, V, (T,), generator=gen)
    r = b.muon_head_xent(x, w, t.cuda(), dx=True, dw=True)
    rows = ho.target_rows(t.numpy(), V)
    ref = ho.head_loss(f64(x), f64(w), rows)
    check(r, ref, f64(x), f64(w), rows, 1.0, BF, BF, coefficients(ref["counts"], None, True, 1.0, 0.0))


@pytest.mark.parametrize("codes", [1, 2])
def test_low_temperature(knobs, codes):  # noqa: F811
    """Logits of 30 - 40 at a temperature of 0.01."""
    b = knobs
    b.muon_debug_set_head_codes(codes)
    T, V, K = 300, 1500, 8
    x, w, gen = shifted(T, 64, V, 51, 36, 1.0)
    ids = torch.stack([torch.randperm(V, generator=gen)[:K] for _ in range(T)])
    z = torch.randn(T, K, generator=gen) * 0.02
    r = b.muon_head_distill(x, w, ids.cuda(), z.cuda(), temperature=0.01, scale=1e-4, dx=True, dw=True)
    rows = ho.teacher_rows(ids.numpy(), f64(z), V, 0.01)
    ref = ho.head_loss(f64(x), f64(w), rows, temperature=0.01, scale=1e-4)
    check(r, ref, f64(x), f64(w), rows, 100.0, BF, BF, coefficients(ref["counts"], None, True, 1e-4, 0.0))


@pytest.mark.parametrize("bad", ["inf", "nan"])
@pytest.mark.parametrize("T,pad", [(40, 0), (40, 1), (256, 0), (257, 0)])
@pytest.mark.parametrize("top", [0, 3])
def test_masked_rows_are_zero_whatever_the_head_holds(bad, T, pad, top):
    from paper_2502_16982_b200 import binding as b

    V = 600
    x, w, gen = make(T, 64, V, 61, pad_x=pad)
    w[5, 3] = float(bad)
    if top:
        ids = torch.randint(0, V, (T, top), generator=gen)
        ids[::3] = -1
        r = b.muon_head_distill(x, w, ids.cuda(), torch.randn(T, top, generator=gen).cuda(), dx=True, dw=True)
    else:
        t = torch.randint(0, V, (T,), generator=gen)
        t[::3] = -100
        r = b.muon_head_xent(x, w, t.cuda(), dx=True, dw=True)
    assert not r.loss[::3].any() and not r.lse[::3].any() and not r.dx[::3].any()
    assert not torch.isfinite(r.loss).all() and torch.isnan(r.dx[1::3]).any()  # the others show it


@pytest.mark.parametrize("D", [64, 2048])
@pytest.mark.parametrize("T", [60, 300])
def test_logits_without_fraction_bits_give_finite_results(D, T):
    """Logits of about 2^24, where an fp32 value has no bits below 1: the target is the
    largest, so that its two values stand against each other in the softmax sum."""
    from paper_2502_16982_b200 import binding as b

    scale = 1e6
    x, w, _ = make(T, D, 3000, 71)
    l = scale * (x.double() @ w.double().t())
    r = b.muon_head_xent(x, w, l.argmax(1), dx=True, dw=True, logit_scale=scale)
    for k in ("loss", "lse", "total", "dx", "dw"):
        assert torch.isfinite(getattr(r, k)).all(), k
    e_l = scale * (D / 16 + 8) * 2.0 ** -23 * float((x.double().abs() @ w.double().abs().t()).max())
    assert float((r.lse.double() - torch.logsumexp(l, 1)).abs().max()) <= 2 * e_l


@pytest.mark.parametrize("T,D,V", [(100, 512, 40000), (2000, 64, 20000), (700, 1024, 20000)])
def test_many_tiles_a_pair_give_the_same_bits(T, D, V):
    """Both accumulators of every CTA pair are handed over many times, short products and
    long ones, with the stores of codes, of dX and of dW in between."""
    from paper_2502_16982_b200 import binding as b

    x, w, gen = make(T, D, V, 81)
    t = torch.randint(0, V, (T,), generator=gen).cuda()
    first = b.muon_head_xent(x, w, t, dx=True, dw=True)
    for _ in range(20):
        again = b.muon_head_xent(x, w, t, dx=True, dw=True)
        for k in ("loss", "lse", "total", "dx", "dw"):
            assert torch.equal(getattr(first, k), getattr(again, k)), k


@pytest.mark.parametrize("top", [0, 20])
def test_least_workspace(knobs, top):  # noqa: F811
    """The argument takes the smallest workspace and changes nothing but its size and,
    to rounding, how the gradient of the logits is formed."""
    b = knobs
    T, D, V = 600, 512, 4000
    x, w, gen = make(T, D, V, 91)
    b.muon_debug_set_head_piece_bytes(T * 256 * 2 * 2)  # eight pieces
    if top:
        ids = torch.stack([torch.randperm(V, generator=gen)[:top] for _ in range(T)])
        z = torch.randn(T, top, generator=gen)
        rows = ho.teacher_rows(ids.numpy(), f64(z), V, 1.0)
        ids, z = ids.cuda(), z.cuda()
    else:
        t = torch.randint(0, V, (T,), generator=gen)
        rows = ho.target_rows(t.numpy(), V)
        t = t.cuda()
    ref = ho.head_loss(f64(x), f64(w), rows)
    for least in (False, True):
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_stats()["requested_bytes.all.current"]
        r = (b.muon_head_distill(x, w, ids, z, dx=True, dw=True, least_workspace=least) if top else
             b.muon_head_xent(x, w, t, dx=True, dw=True, least_workspace=least))
        # what was asked for: the allocator's blocks may be larger, as its history has it
        peak = torch.cuda.memory_stats()["requested_bytes.all.peak"] - before
        outputs = 2 * (T + V) * D + 8 * T + 4
        need = b.muon_head_workspace_bytes(T, D, V, top=top, least=least)
        assert need <= peak <= need + outputs + 4096
        check(r, ref, f64(x), f64(w), rows, 1.0, BF, BF, coefficients(ref["counts"], None, True, 1.0, 0.0))


@pytest.mark.parametrize("aligned", [True, False])
@pytest.mark.parametrize("T,D,V,K,opts", [
    (100, 64, 700, 33, dict(tail=True, weights=True)),
    (200, 128, 1500, 16, dict(temperature=2.0, masked=0.3)),
    (60, 64, 900, 20, dict(twice=True, dw=FP)),
    (40, 256, 3000, 100, dict(z_bf16=True, strided=True, temperature=0.7, scale=0.49, mean=False)),
    (30, 72, 5000, 128, dict(masked=0.4, weights=True)),
    (256, 64, 1000, 16, dict(tail=True, temperature=3.0, masked=0.2, twice=True, dx=FP)),
    (150, 128, 2600, 5, dict(dx=None, dw=None, tail=True)),
    (90, 64, 1300, 40, dict(dx=None, neg_inf=True)),
    (20, 512, 4096, 16, dict(dw=None, logit_scale=0.5, weights=True, z_bf16=True)),
    (256, 2048, 600, 1, dict(masked=0.1)),
])
def test_distillation_of_few_tokens(T, D, V, K, opts, aligned):
    """Every option where nothing is gathered (aligned rows of x) and where it is."""
    from paper_2502_16982_b200 import binding as b

    o = dict(opts)
    x, w, gen = make(T, D, V, 91 * T + K, pad_x=0 if aligned else 1)
    tau = o.get("temperature", 1.0)
    ids = torch.stack([torch.randperm(V, generator=gen)[:K] for _ in range(T)])
    z = torch.randn(T, K, generator=gen) * 2
    if o.pop("z_bf16", False):
        z = z.to(BF)
    if o.pop("twice", False):
        ids[:, 1] = ids[:, 0]
        ids[:, 5] = ids[:, 2]
        ids[:, 9] = ids[:, 2]
    hide = torch.rand(T, generator=gen) < o.pop("masked", 0.0)
    ids[hide] = torch.tensor([-1, V])[torch.randint(0, 2, (int(hide.sum()), K), generator=gen)]
    some = torch.rand(T, K, generator=gen) < 0.1
    some[:, 0] = False
    ids[some] = -5
    if o.pop("neg_inf", False):
        z[torch.rand(T, K, generator=gen) < 0.3] = -float("inf")
        z[3] = -float("inf")
    weight = (torch.rand(T, generator=gen) + 0.5).cuda() if o.pop("weights", False) else None
    tlse = (torch.logsumexp(z.double() / tau, 1) + 0.3).float().cuda() if o.pop("tail", False) else None
    hidden = torch.tensor(~ho.teacher_rows(ids.numpy(), f64(z), V, tau)[2].any(1))
    x[hidden.cuda()] = float("nan")
    dxt, dwt = o.pop("dx", BF), o.pop("dw", BF)
    ids_d, z_d = ids.cuda(), z.cuda()
    if o.pop("strided", False):
        ids_d = torch.cat([ids_d, ids_d[:, :3] * 0 - 9], 1)[:, :K]
        z_d = torch.cat([z_d, z_d[:, :1] * 0 + 99], 1)[:, :K]
    dx = None if dxt is None else torch.full((T, D), 7.0, dtype=dxt, device="cuda")
    dw = None if dwt is None else torch.full((V, D), 7.0, dtype=dwt, device="cuda")
    ws = torch.full((b.muon_head_workspace_bytes(T, D, V, top=K, dx=dx is not None, dw=dw is not None),), 255,
                    dtype=torch.uint8, device="cuda")
    r = b.muon_head_distill(x, w, ids_d, z_d, teacher_lse=tlse, weight=weight, dx=dx, dw=dw, workspace=ws, **o)
    assert b.muon_head_status(ws) == 0
    rows = ho.teacher_rows(ids.numpy(), f64(z), V, tau, None if tlse is None else f64(tlse))
    xr, wr = np.where(rows[2].any(1)[:, None], f64(x), 0.0), f64(w)
    ref = ho.head_loss(xr, wr, rows, weight=None if weight is None else f64(weight), **o)
    coef = coefficients(ref["counts"], weight, o.get("mean", True), o.get("scale", 1.0), 0.0)
    check(r, ref, xr, wr, rows, o.get("logit_scale", 1.0) / tau, dxt, dwt, coef)


@pytest.mark.parametrize("T", [96, 320])
def test_distillation_adds_to_dw_inside_margins(T):
    """accumulate_dw of a distillation, into rows inside a larger array, fp32 and bf16."""
    from paper_2502_16982_b200 import binding as b

    D, V, K = 72, 900, 12
    x, w, gen = make(T, D, V, 101)
    ids = torch.stack([torch.randperm(V, generator=gen)[:K] for _ in range(T)])
    z = torch.randn(T, K, generator=gen)
    rows = ho.teacher_rows(ids.numpy(), f64(z), V, 2.0)
    ref = ho.head_loss(f64(x), f64(w), rows, temperature=2.0)
    for dt in (FP, BF):
        dx = torch.full((T + 2, D + 12), 5.0, dtype=dt, device="cuda")
        dw = torch.full((V + 2, D + 12), 0.5, dtype=dt, device="cuda")
        first = b.muon_head_distill(x, w, ids.cuda(), z.cuda(), temperature=2.0, dx=dx[1:-1, 4:-8],
                                    dw=torch.empty(V, D, dtype=FP, device="cuda"))
        r = b.muon_head_distill(x, w, ids.cuda(), z.cuda(), temperature=2.0, dx=dx[1:-1, 4:-8], dw=dw[1:-1, 4:-8],
                                accumulate_dw=True)
        check(first, ref, f64(x), f64(w), rows, 0.5, dt, FP, coefficients(ref["counts"], None, True, 1.0, 0.0))
        # the same gradients of logits on both sides; what differs is one addition to 0.5, rounded once
        err = (r.dw.double() - 0.5 - first.dw.double()).abs()
        assert bool((err <= (2.0 ** -23 if dt == FP else 2.0 ** -8) * (0.5 + first.dw.double().abs())).all())
        for m, v in ((dx, 5.0), (dw, 0.5)):
            m[1:-1, 4:-8] = v
            assert bool((m == v).all())


def head_loss64(x, w, ids, p, g, a, z_loss):
    """The oracle's formulas in fp64 on the GPU, for sizes that the host takes too long for."""
    x, w = x.double(), w.double()
    l = a * (x @ w.t())
    lse = torch.logsumexp(l, 1)
    log_q = l - lse[:, None]
    loss = (torch.xlogy(p, p) - p * log_q.gather(1, ids)).sum(1) + z_loss * lse ** 2
    d = torch.exp(log_q) * (p.sum(1) + 2 * z_loss * lse)[:, None]
    d.scatter_add_(1, ids, -p)
    d *= (g * a)[:, None]
    counts = (p > 0).any(1)
    e_l = abs(a) * (x.shape[1] / 16 + 8) * 2.0 ** -23 * float((x.abs() @ w.abs().t())[counts].max())
    absg = d.abs()
    absg_at = torch.zeros_like(d).scatter_add_(1, ids, (p > 0).double() * ((g * a).abs() * (4 * e_l + 2.0 ** -20))[:, None])
    absg_at += (g * a).abs()[:, None] * 2.0 ** -31
    return dict(loss=loss * counts, lse=lse * counts, total=(g * loss * counts).sum(), dx=d @ w, dw=d.t() @ x, e_l=e_l, counts=counts,
                bound=dict(dx=(absg @ w.abs(), absg_at @ w.abs()), dw=(absg.t() @ x.abs(), absg_at.t() @ x.abs())))


def check64(r, ref, V, T, g, z_loss):
    """test_gpu_head_loss.check on the GPU."""
    e_l, rel = ref["e_l"], (V / 256 + 64) * 2.0 ** -24
    zl = 1 + 2 * abs(z_loss) * ref["lse"].abs()
    tol = (2 * e_l + rel * (1 + ref["lse"].abs()) * zl) * zl + 1e-30
    for name in ("loss", "lse"):
        assert bool(((getattr(r, name).double() - ref[name]).abs() <= tol).all()), name
    assert abs(float(r.total) - float(ref["total"])) <= float((g.abs() * (tol + 2.0 ** -20 * ref["loss"].abs())).sum())
    for name, steps in (("dx", V / 16 + 64), ("dw", T / 16 + 16)):
        main, slack = ref["bound"][name]
        bound = (2.0 ** -8 + 4 * e_l + 2.0 ** -12 + steps * 2.0 ** -23) * main + 1.01 * slack
        bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * ref[name].abs() + 1e-30
        err = (getattr(r, name).double() - ref[name]).abs()
        assert bool((err <= bound).all()), (name, float((err / bound).max()))


@pytest.mark.parametrize("T,D,V,top,masked,z_loss", [
    (1000, 2048, 163840, 0, 0.3, 1e-4),   # two pieces kept as codes, the second converted beside the products
    (4100, 512, 100000, 0, 0.2, 0.0),     # four pieces
    (1200, 64, 163840, 0, 0.1, 0.0),      # a narrow head: two pieces, each by a second product
    (700, 96, 20000, 8, 0.2, 0.0),        # the same in one piece
    (900, 1536, 163840, 20, 0.1, 0.0),    # distillation, two pieces of codes
    (1500, 320, 110000, 5, 0.0, 0.0),     # and by a second product
    (100, 2048, 163840, 0, 0.1, 0.0),     # few tokens on the full vocabulary
])
def test_sizes_that_take_several_pieces(T, D, V, top, masked, z_loss):
    from paper_2502_16982_b200 import binding as b

    x, w, gen = make(T, D, V, 111)
    hide = torch.rand(T, generator=gen) < masked
    if top:
        ids = (torch.randint(0, V, (T, 1), generator=gen) + torch.arange(top) * (V // top)) % V
        z = torch.randn(T, top, generator=gen) * 2
        p = torch.softmax(z.double(), 1)
        ids[hide] = -1
        x[hide.cuda()] = float("nan")
        r = b.muon_head_distill(x, w, ids.cuda(), z.cuda(), dx=True, dw=True)
    else:
        ids = torch.randint(0, V, (T, 1), generator=gen)
        p = torch.ones(T, 1, dtype=torch.float64)
        ids[hide] = -100
        x[hide.cuda()] = float("nan")
        r = b.muon_head_xent(x, w, ids[:, 0].cuda(), z_loss=z_loss, dx=True, dw=True)
    x[hide.cuda()] = 0
    p[hide] = 0
    g = ((~hide).double() / int((~hide).sum())).cuda()
    ref = head_loss64(x, w, ids.clamp(min=0).cuda(), p.cuda(), g, 1.0, z_loss)
    assert not r.dx[hide.cuda()].any()
    check64(r, ref, V, T, g, z_loss)


@pytest.mark.parametrize("T,masked,opts", [
    (40, 0, {}), (230, 1, {}), (367, 0, {}), (367, 2, dict(scale=0.37, mean=False)), (367, 0, dict(logit_scale=0.6, scale=-1.0)),
    (1500, 30, {}), (367, 0, dict(distill=True)), (40, 0, dict(distill=True)),
])
@pytest.mark.parametrize("codes", [1, 2])
def test_the_tokens_common_coefficient_is_not_rounded(knobs, codes, T, masked, opts):  # noqa: F811
    """1 / tokens, scale and logit_scale are the same for every token.  Rounded to bf16 with
    each gradient of a logit they would make all of dX and dW too large or too small,
    by up to 2^-8.

    The factor by which an output is too large is its projection on the oracle's, less 1.
    The logits here are small and the vocabulary is large, q = 2^-14 on average: the
    entries of a target distribution make up the gradient, and for cross entropy (p = 1)
    what they lose is the rounding of 1 - q to 1, 2^-14 on average.  Distillation: of
    p over four equal entries 1/4 - q, that is 2^-12.  The q's, rounded
    independently, add less than 2^-8 / sqrt(T V) of a norm that is itself a small part;
    outputs are fp32.  2^-11 in all."""
    b = knobs
    b.muon_debug_set_head_codes(codes)
    o = dict(opts)
    V, D = 20000, 64
    x, w, gen = make(T, D, V, 121 + T, gain=0.5)
    hide = torch.arange(T) < masked
    dx, dw = torch.empty(T, D, device="cuda"), torch.empty(V, D, device="cuda")
    if o.pop("distill", False):
        ids = (torch.randint(0, V, (T, 1), generator=gen) + torch.arange(4) * (V // 4)) % V
        ids[hide] = -1
        z = torch.zeros(T, 4)
        r = b.muon_head_distill(x, w, ids.cuda(), z.cuda(), dx=dx, dw=dw, **o)
        rows = ho.teacher_rows(ids.numpy(), f64(z), V, 1.0)
    else:
        t = torch.randint(0, V, (T,), generator=gen)
        t[hide] = -100
        r = b.muon_head_xent(x, w, t.cuda(), dx=dx, dw=dw, **o)
        rows = ho.target_rows(t.numpy(), V)
    ref = ho.head_loss(f64(x), f64(w), rows, **o)
    for name in ("dx", "dw"):
        factor = float((f64(getattr(r, name)) * ref[name]).sum() / (ref[name] ** 2).sum())
        assert abs(factor - 1) <= 2.0 ** -11, (name, factor - 1)
