"""Results of muon_head_logprob written into an earlier result, and then its gradients: nothing
of the earlier pass reaches them.  Tolerances: those of test_gpu_head_logprob.py."""

import contextlib

import numpy as np
import pytest
import torch

from test_gpu_head_logprob import Reference, f64, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("second", ["keep", "keep_false", "no_grad", "workspace"])
@pytest.mark.parametrize("use", ["returned", "given"])
@pytest.mark.parametrize("T,D,V", [(300, 136, 3000), (24, 512, 4096)])
def test_an_earlier_result_written_again(second, use, T, D, V):
    from paper_2502_16982_b200 import binding as b

    x1, w1, _ = make(T, D, V, 51)
    x2, w2, gen = make(T, D, V, 52)
    y1, y2 = (torch.randint(0, V, (T,), generator=gen) for _ in range(2))
    y1[::5] = -100
    y2[::7] = -100
    r = b.muon_head_logprob(x1, w1, y1.cuda())
    assert r.kept is not None
    more = {}
    if second == "keep_false":
        more["keep"] = False
    elif second == "workspace":
        n = b.muon_head_logprob_workspace_bytes(T, D, V, grads=False)
        more["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    with torch.no_grad() if second == "no_grad" else contextlib.nullcontext():
        again = b.muon_head_logprob(x2, w2, y2.cuda(), logit_scale=0.8, out=r, **more)
    assert again.logprob is r.logprob and again.entropy is r.entropy and again.lse is r.lse
    assert (again.kept is not None) == (second == "keep") and r.kept is again.kept
    saved = again if use == "returned" else r
    ref = Reference(f64(x2), f64(w2), y2.numpy(), 0.8)
    ref.check(saved)
    rr, hh = torch.randn(T, generator=gen) / T, torch.randn(T, generator=gen) * 0.1 / T
    d = b.muon_head_logprob_grad(x2, w2, y2.cuda(), saved, g_logprob=rr.cuda(), g_entropy=hh.cuda(), logit_scale=0.8, dx=True, dw=True)
    counted = lambda v: np.where(y2.numpy() < 0, 0.0, v.double().numpy())
    ref.check_grads(d, counted(rr), counted(hh), kept=second == "keep")


def test_a_call_that_is_refused_leaves_what_an_earlier_one_kept():
    from paper_2502_16982_b200 import binding as b

    x, w, gen = make(300, 136, 3000, 53)
    y = torch.randint(0, 3000, (300,), generator=gen).cuda()
    r = b.muon_head_logprob(x, w, y)
    kept = r.kept
    with pytest.raises(b.MuonError):
        b.muon_head_logprob(x, w, y, out=r, workspace=torch.zeros(1024, dtype=torch.uint8, device="cuda"))
    assert r.kept is kept
    plain = b.muon_head_logprob(x, w, y, out=tuple(r), keep=False)
    assert type(plain) is b.HeadLogprob and plain.kept is None and r.kept is kept


def test_the_gradients_workspace_beside_what_was_kept():
    """Both carved from one buffer, one behind the other in either order; overlapping is refused."""
    from paper_2502_16982_b200 import binding as b

    T, D, V = 300, 136, 3000
    x, w, gen = make(T, D, V, 54)
    y = torch.randint(0, V, (T,), generator=gen)
    n = b.muon_head_logprob_workspace_bytes(T, D, V, grads=False, keep=True) - 1024
    m = b.muon_head_logprob_workspace_bytes(T, D, V, grads=True, keep=True) - 1024
    buffer = torch.zeros(n + m + 1024, dtype=torch.uint8, device="cuda")
    buffer = buffer[-buffer.data_ptr() % 1024:]
    rr = torch.randn(T, generator=gen) / T
    ref = Reference(f64(x), f64(w), y.numpy(), 1.0)
    for own in (buffer[n:n + m], buffer[:m]):
        kept = buffer[:n] if own.data_ptr() != buffer.data_ptr() else buffer[m:m + n]
        r = b.muon_head_logprob(x, w, y.cuda(), workspace=kept, keep=True)
        ref.check(r)
        for bad in (kept, buffer[1024:]):  # (the entropy's sums, behind what is kept, may be overwritten)
            with pytest.raises(b.MuonError) as e:
                b.muon_head_logprob_grad(x, w, y.cuda(), r, g_logprob=rr.cuda(), dx=True, dw=True, workspace=bad)
            assert e.value.code == b.MUON_ERR_WORKSPACE
        d = b.muon_head_logprob_grad(x, w, y.cuda(), r, g_logprob=rr.cuda(), dx=True, dw=True, workspace=own)
        ref.check_grads(d, rr.double().numpy(), None, kept=True)


@pytest.mark.parametrize("other", ["tokens", "more_tokens", "dim", "vocab", "scale", "alignment", "codes", "kept_nothing", "in_place", "loss"])
def test_what_another_call_kept_gives_no_gradient(other):
    """The binding refuses what it can see; the kernel compares what lies in the workspace."""
    from paper_2502_16982_b200 import binding as b

    T, D, V, S = 200, 128, 3000, 0.8
    sizes = {"tokens": (70, D, V, S), "more_tokens": (260, D, V, S), "dim": (T, 64, V, S), "vocab": (T, D, 2900, S), "scale": (T, D, V, 0.9)}
    t, d, v, s = sizes.get(other, (T, D, V, S))
    ws = torch.zeros(32 << 20, dtype=torch.uint8, device="cuda")
    x, w, gen = make(t, d, v, 55, offset_w=1 if other == "alignment" else 0)
    y = torch.randint(0, v, (t,), generator=gen).cuda()
    made = None
    if other == "loss":
        b.muon_head_xent(x, w, y, dx=True, workspace=ws)
    else:
        mode = b.muon_debug_set_head_codes(1 if other == "codes" else 0)
        made = b.muon_head_logprob(x, w, y, logit_scale=s, workspace=ws, keep=other not in ("kept_nothing", "in_place"))
        b.muon_debug_set_head_codes(mode)
    if other == "in_place":  # over what was kept before
        b.muon_head_logprob(x, w, y, logit_scale=s, workspace=ws, keep=True)
        b.muon_head_logprob(x, w, y, logit_scale=s, workspace=ws)
    x, w, gen = make(T, D, V, 56)
    y = torch.randint(0, V, (T,), generator=gen).cuda()
    r = b.muon_head_logprob(x, w, y, logit_scale=S, keep=False)
    r.kept = ws
    g = torch.full((T,), 0.5, device="cuda")
    own = torch.zeros(b.muon_head_logprob_workspace_bytes(T, D, V, grads=True, keep=True), dtype=torch.uint8, device="cuda")
    dw = torch.full((V, D), 7.0, device="cuda")
    dx = torch.full((T, D), 7.0, device="cuda")
    grad = lambda **k: b.muon_head_logprob_grad(x, w, y, r, g_logprob=g, g_entropy=g, logit_scale=S, workspace=own, **k)
    grad(dx=dx, dw=dw, accumulate_dw=True)
    assert b.muon_head_status(own) == b.MUON_ERR_INVALID_ARG
    assert not dx.any() and bool((dw == 7.0).all())
    grad(dw=dw)
    assert b.muon_head_status(own) == b.MUON_ERR_INVALID_ARG and not dw.any()
    if other in sizes:
        r.kept_for = made.kept_for
        with pytest.raises(b.MuonError) as e:
            grad(dx=True)
        assert e.value.code == b.MUON_ERR_INVALID_ARG


def test_what_the_same_call_kept_after_others_used_the_workspace():
    from paper_2502_16982_b200 import binding as b

    T, D, V = 200, 128, 3000
    ws = torch.zeros(32 << 20, dtype=torch.uint8, device="cuda")
    own = torch.zeros(32 << 20, dtype=torch.uint8, device="cuda")
    for seed, (t, d, v) in enumerate(((T, D, V), (20, 64, 500), (T, D, V), (0, D, V), (T, D, V))):
        x, w, gen = make(t, d, v, 57 + seed)
        y = torch.randint(0, v, (t,), generator=gen)
        r = b.muon_head_logprob(x, w, y.cuda(), logit_scale=0.8, workspace=ws, keep=True)
        rr, hh = torch.randn(t, generator=gen), torch.randn(t, generator=gen) * 0.1
        g = b.muon_head_logprob_grad(x, w, y.cuda(), r, g_logprob=rr.cuda(), g_entropy=hh.cuda(), logit_scale=0.8, dx=True, dw=True, workspace=own)
        assert b.muon_head_status(own) == 0
        if t:
            Reference(f64(x), f64(w), y.numpy(), 0.8).check_grads(g, rr.double().numpy(), hh.double().numpy(), kept=True)
        else:
            assert not g.dw.any()


def test_no_tokens_after_a_call_that_kept_nothing():
    """The first call's 200 tokens are still counted in the workspace; none of them is looked at."""
    from paper_2502_16982_b200 import binding as b

    T, D, V = 200, 128, 3000
    ws, own = (torch.zeros(32 << 20, dtype=torch.uint8, device="cuda") for _ in range(2))
    x, w, gen = make(T, D, V, 63)
    y = torch.randint(0, V, (T,), generator=gen).cuda()
    b.muon_head_logprob(x, w, y, workspace=ws, keep=True)
    b.muon_head_logprob(x, w, y, workspace=ws)
    r = b.muon_head_logprob(x[:0], w, y[:0], keep=False)
    r.kept = ws
    dw = torch.full((V, D), 7.0, device="cuda")
    b.muon_head_logprob_grad(x[:0], w, y[:0], r, g_logprob=r.lse, dw=dw, workspace=own)
    assert b.muon_head_status(own) == b.MUON_ERR_INVALID_ARG and not dw.any()
