"""The LM-head losses where numbers, sizes or layouts are extreme.

Tolerances are those of test_gpu_head_loss.py, derived there."""

import pytest
import torch

from oracle import head_oracle as ho
from test_gpu_head_loss import BF, check, coefficients, f64, knobs, make  # noqa: F401

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
        before = torch.cuda.memory_allocated()
        r = (b.muon_head_distill(x, w, ids, z, dx=True, dw=True, least_workspace=least) if top else
             b.muon_head_xent(x, w, t, dx=True, dw=True, least_workspace=least))
        peak = torch.cuda.max_memory_allocated() - before
        outputs = 2 * (T + V) * D + 8 * T + 4
        need = b.muon_head_workspace_bytes(T, D, V, top=top, least=least)
        assert need <= peak <= need + outputs + 4096
        check(r, ref, f64(x), f64(w), rows, 1.0, BF, BF, coefficients(ref["counts"], None, True, 1.0, 0.0))
