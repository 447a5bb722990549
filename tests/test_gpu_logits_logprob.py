"""Log probabilities over stored logits (muon_logits_logprob and its gradient) against
the fp64 oracle.

Tolerances, from the arithmetic.  With l the scaled logits, lmax a row's largest,
D1 = sum q |l - lmax| and D2 = sum q (l - lmax)^2: an exponent is one fused
multiply-add of an fp32 factor, within 2^-23 of its distance from lmax (the factor's own
rounding shows in lmax too, where it stands alone); exponentials are within 2^-22; a sum
is a chain of 16 terms, one per tile of 4096 columns or more, and a tree, n_c = (V / 4096
+ 64) 2^-24 in all.
    e_s      = 2^-22 (1 + D1) + n_c                              relative error of S
    logprob  : e_s + 2^-22 (1 + |l_y - lmax| + |logprob|)
    lse      : e_s + 2^-22 (1 + |lmax| + |lse|)
    entropy  : e_s + D1 (2^-22 + 2 n_c) + 2^-22 (D1 + D2 + H)
A gradient's q has the relative error e_q = err(lse) + 2^-22 (1 + |log q|); the factor in
brackets adds the errors of log q and H, and the result is rounded once to its type.
The alternatives are exact: ids equal, logits the same numbers."""

import numpy as np
import pytest
import torch

from oracle import logprob_oracle as lo

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def strided(z, dtype, pad, offset):
    """z on the device with row stride V + pad, its first row `offset` elements from an
    aligned address; what lies between the rows is NaN."""
    T, V = z.shape
    store = torch.full((offset + T * (V + pad),), float("nan"), dtype=dtype)
    store[offset:].view(T, V + pad)[:, :V] = z.to(dtype)
    return store.cuda()[offset:].view(T, V + pad)[:, :V]


def rows_of(kind, T, V, gen):
    z = torch.randn(T, V, generator=gen) * 3
    if kind == "ties":  # a few values only, many at the top
        z = (z * 0.7).round() * 0.5
    elif kind == "constant":
        z = torch.full((T, V), -1.25)
    elif kind == "ascending":
        z = torch.arange(V).float().expand(T, V) * (20.0 / V) - 5
    elif kind == "descending":
        z = -torch.arange(V).float().expand(T, V) * (20.0 / V)
    elif kind == "few":  # most of the vocabulary is forbidden
        z = torch.where(torch.rand(T, V, generator=gen) < 3.0 / V, z, -float("inf"))
        z[:, V // 2] = 1.0
    elif kind == "spread":
        z = z * 40
    return z.contiguous()


def expect(z, targets, scale):
    logprob, entropy, lse, log_q, counts = lo.logprob_rows(z, targets, scale)
    V = z.shape[1]
    with np.errstate(invalid="ignore"):
        top = (z * scale).max(1)
        far = np.where(log_q > -np.inf, (top - lse)[:, None] - log_q, 0.0)
    q = np.where(log_q > -np.inf, np.exp(log_q), 0.0)
    d1, d2 = (q * far).sum(1), (q * far * far).sum(1)
    n_c = (V / 4096 + 64) * 2.0 ** -24
    u = 2.0 ** -22
    e_s = u * (1 + d1) + n_c
    with np.errstate(invalid="ignore"):
        tol = {"logprob": e_s + u * (1 + 2 * np.abs(logprob) + np.abs(top - lse)), "lse": e_s + u * (1 + np.abs(top) + np.abs(lse)),
               "entropy": e_s + d1 * (u + 2 * n_c) + u * (d1 + d2 + entropy)}
    return {"logprob": logprob, "entropy": entropy, "lse": lse}, tol, log_q, counts


def check_rows(r, z, targets, scale, top):
    want, tol, log_q, counts = expect(z, targets, scale)
    for name in ("logprob", "entropy", "lse"):
        got = getattr(r, name)
        if got is None:
            assert targets is None and name == "logprob"
            continue
        got = f64(got)
        finite = np.isfinite(want[name])
        assert np.array_equal(got[~finite], want[name][~finite]), name
        err = np.abs(got - want[name])[finite]
        assert np.all(err <= tol[name][finite]), (name, float((err / tol[name][finite]).max()))
        assert np.all(got[~counts] == 0)
    if top:
        ids = r.top_ids.cpu().numpy()
        order = lo.best(z, top)
        assert np.array_equal(ids[counts], order[counts])
        assert np.all(ids[~counts] == -1)
        vals = np.where(np.isnan(z), -np.inf, z)
        picked = np.take_along_axis(vals, order, 1)
        assert np.array_equal(f64(r.top_logits)[counts], picked[counts])
        assert np.all(f64(r.top_logits)[~counts] == 0) and np.all(f64(r.top_logprob)[~counts] == 0)
        with np.errstate(invalid="ignore"):
            want_lp = picked * scale - want["lse"][:, None]
        want_lp = np.where((want["lse"] == -np.inf)[:, None], -np.inf, want_lp)[counts]
        got_lp = f64(r.top_logprob)[counts]
        ok = np.isfinite(want_lp)
        assert np.array_equal(got_lp[~ok], want_lp[~ok])
        d1tol = np.broadcast_to((tol["logprob"])[counts][:, None], want_lp.shape) + 2.0 ** -21 * np.where(ok, np.abs(want_lp), 0)
        assert np.all(np.abs(got_lp - want_lp)[ok] <= d1tol[ok])
    return want, tol, log_q, counts


@pytest.mark.parametrize("T,V,top,kind,opts", [
    (1, 1, 1, "normal", {}),
    (1, 7, 7, "normal", dict(offset=3)),
    (3, 128, 128, "normal", dict(pad=1)),
    (5, 129, 128, "ties", dict(offset=1, pad=3)),
    (1, 8192, 5, "normal", {}),
    (2, 5003, 64, "ties", dict(offset=7)),
    (17, 9001, 20, "normal", dict(pad=8, scale=0.7, masked=0.3)),
    (2, 163840, 64, "normal", {}),                        # a cluster's blocks share a row
    (2, 163839, 128, "ties", dict(offset=5)),
    (300, 2100, 100, "normal", dict(masked=0.4)),
    (700, 4999, 50, "normal", dict(pad=3, scale=1.25)),   # a block a row
    (700, 40000, 128, "normal", {}),
    (700, 25001, 64, "ascending", {}),                    # every tile raises the threshold
    (2, 100000, 128, "ascending", {}),
    (610, 20000, 33, "descending", {}),
    (610, 20000, 128, "constant", {}),                    # more equal logits than the list holds
    (3, 50000, 64, "constant", {}),
    (610, 20000, 40, "few", dict(masked=0.1)),
    (3, 30000, 128, "few", {}),
    (40, 30000, 0, "normal", dict(masked=0.2)),
    (1000, 12345, 0, "spread", dict(pad=1)),
    (70001, 9, 3, "normal", {}),                          # more rows than a grid's dimension
    (2000, 2003, 64, "ties", dict(pad=2, masked=0.1)),    # short rows: blocks of half the threads
    (700, 3001, 64, "constant", dict(offset=3)),
    (300, 1000, 64, "ascending", {}),
    (620, 32768, 0, "normal", {}),                        # at the limits of short rows, and behind them
    (620, 32776, 0, "normal", {}),
    (310, 65536, 64, "ascending", {}),
    (310, 65544, 64, "ties", {}),
    (1, 1 << 24, 128, "normal", {}),
])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_rows_match_the_oracle(T, V, top, kind, opts, dtype):
    from paper_2502_16982_b200 import binding as b

    gen = torch.Generator().manual_seed(100 * T + V)
    z = strided(rows_of(kind, T, V, gen), dtype, opts.get("pad", 0), opts.get("offset", 0))
    targets = torch.randint(0, V, (T,), generator=gen)
    hide = torch.rand(T, generator=gen) < opts.get("masked", 0.0)
    targets[hide] = torch.tensor([-100, -1, V, 1 << 40])[torch.randint(0, 4, (int(hide.sum()),), generator=gen)]
    z[hide.cuda()] = float("nan")  # nothing of a masked row is read
    scale = opts.get("scale", 1.0)
    r = b.muon_logits_logprob(z, targets.cuda(), top=top, logit_scale=scale)
    again = b.muon_logits_logprob(z, targets.cuda(), top=top, logit_scale=scale)
    for x, y in zip(r, again):
        assert x is None and y is None or torch.equal(x, y)
    some = np.arange(T) if T < 5000 else np.r_[0:300, 65400:65700, T - 300:T]
    pick = torch.as_tensor(some, device="cuda")
    part = b.LogitsLogprob(*[None if t is None else t[pick] for t in r])
    zz = f64(z[pick])
    hidden = hide.numpy()[some]
    zz[hidden] = 0.0
    check_rows(part, zz, targets.numpy()[some], scale, top)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_infinities_and_nan(dtype):
    from paper_2502_16982_b200 import binding as b

    V = 30001
    gen = torch.Generator().manual_seed(5)
    z = torch.randn(6, V, generator=gen)
    z[0] = -float("inf")                      # nothing left
    z[1] = -float("inf")
    z[1, 7] = 2.0                             # one entry left
    z[2, ::2] = -float("inf")
    z[3, 5:25000] = float("nan")              # statistics NaN; alternatives from the others
    z[4, 100] = float("inf")
    z[5] = float("nan")
    d = z.to(dtype).cuda()
    targets = torch.tensor([3, 7, 1, 2, 3, 0], device="cuda")
    for rows in (d, d.repeat(200, 1)):        # a cluster a row, a block a row
        t = targets.repeat(rows.shape[0] // 6)
        r = b.muon_logits_logprob(rows, t, top=16)
        zz = f64(rows[:3])
        part = b.LogitsLogprob(*[x[:3] for x in r])
        check_rows(part, zz, targets[:3].cpu().numpy(), 1.0, 16)
        for k in (3, 4, 5):
            assert all(torch.isnan(x[k]) for x in (r.logprob, r.entropy, r.lse)), k
        ids = r.top_ids[3:6].cpu().numpy()
        zc = z.to(dtype).double().numpy()
        assert np.array_equal(ids, lo.best(zc[3:6], 16))
        g = b.muon_logits_logprob_grad(rows, t, r, g_logprob=torch.ones(len(t), device="cuda"), g_entropy=torch.ones(len(t), device="cuda"))
        assert torch.equal(g[0], torch.zeros_like(g[0])) and torch.equal(g[1], torch.zeros_like(g[1]))
        assert bool((g[2, ::2] == 0).all()) and bool(torch.isfinite(g[2]).all())
        assert bool(torch.isnan(g[5]).all())


@pytest.mark.parametrize("T,V,opts", [
    (1, 1, {}), (1, 5, dict(offset=1)), (3, 8192, {}), (9, 8193, dict(pad=1, scale=0.7)), (33, 20011, dict(pad=2, masked=0.4, offset=3)),
    (400, 3001, dict(masked=0.2)), (6, 40000, dict(kind="few")), (7, 1000, dict(kind="spread", scale=1.5)),
])
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("which", ["both", "logprob", "entropy", "entropy_without_targets"])
def test_gradient_matches_the_formula(T, V, opts, dtype, which):
    from paper_2502_16982_b200 import binding as b

    gen = torch.Generator().manual_seed(7 * T + V)
    z = strided(rows_of(opts.get("kind", "normal"), T, V, gen), dtype, opts.get("pad", 0), opts.get("offset", 0))
    targets = torch.randint(0, V, (T,), generator=gen)
    hide = torch.rand(T, generator=gen) < opts.get("masked", 0.0)
    if which == "entropy_without_targets":
        hide[:] = False
    targets[hide] = -100
    z[hide.cuda()] = float("nan")
    scale = opts.get("scale", 1.0)
    tg = None if which == "entropy_without_targets" else targets.cuda()
    rr = torch.randn(T, generator=gen) if which in ("both", "logprob") else None
    hh = torch.randn(T, generator=gen) if which != "logprob" else None
    r = b.muon_logits_logprob(z, tg, logit_scale=scale)
    up = dict(g_logprob=None if rr is None else rr.cuda(), g_entropy=None if hh is None else hh.cuda(), logit_scale=scale)
    got = b.muon_logits_logprob_grad(z, tg, r, **up)
    # other strides and alignment, and in place
    other = strided(torch.zeros(T, V), dtype, 5, 1)
    b.muon_logits_logprob_grad(z, tg, r, dlogits=other, **up)
    assert torch.equal(other, got)
    copy = strided(torch.zeros(T, V), dtype, opts.get("pad", 0), opts.get("offset", 0))
    copy.copy_(z)
    zz = f64(z)
    assert b.muon_logits_logprob_grad(copy, tg, r, dlogits=copy, **up) is copy and torch.equal(copy, got)
    zz[hide.numpy()] = 0.0
    tn = None if tg is None else targets.numpy()
    want, tol, log_q, counts = expect(zz, tn, scale)
    r64, h64 = (None if x is None else x.double().numpy() for x in (rr, hh))
    exact = lo.logprob_grad(log_q, want["entropy"], counts, targets.numpy(), r64, h64, scale)
    ra, ha = (np.zeros(T) if x is None else np.abs(x) for x in (r64, h64))
    t = np.where(log_q > -np.inf, np.abs(log_q), 0.0)
    q = np.where(log_q > -np.inf, np.exp(log_q), 0.0)
    u = 2.0 ** -22
    e_q = tol["lse"][:, None] + u * (1 + t)
    size = ra[:, None] + ha[:, None] * (t + want["entropy"][:, None])
    err = scale * (q * size * (e_q + 2 * u) + q * ha[:, None] * (tol["lse"] + tol["entropy"])[:, None] + u * ra[:, None] * (q > 0))
    bound = err + (2.0 ** -8 if dtype == BF else 2.0 ** -24) * (np.abs(exact) + err) + 1e-36 * (1 + size)
    assert np.all(np.abs(f64(got) - exact) <= bound), float((np.abs(f64(got) - exact) / bound).max())
    assert np.all(f64(got)[~counts] == 0)


def test_gradient_against_differences():
    """dJ along a direction, from the operator's own forward pass."""
    from paper_2502_16982_b200 import binding as b

    gen = torch.Generator().manual_seed(8)
    z = torch.randn(12, 301, generator=gen).cuda()
    y = torch.randint(0, 301, (12,), generator=gen).cuda()
    rr, hh, way = torch.randn(12, generator=gen).cuda(), torch.randn(12, generator=gen).cuda(), torch.randn(12, 301, generator=gen).cuda()
    r = b.muon_logits_logprob(z, y, logit_scale=0.9)
    d = b.muon_logits_logprob_grad(z, y, r, g_logprob=rr, g_entropy=hh, logit_scale=0.9)

    def value(zz):
        v = b.muon_logits_logprob(zz, y, logit_scale=0.9)
        return ((rr.double() * v.logprob.double()) + hh.double() * v.entropy.double())

    step = 2.0 ** -6
    slope = (value(z + step * way) - value(z - step * way)) / (2 * step)
    along = (d.double() * way.double()).sum(1)
    # fp32 values of up to 10 (2^-20 each) over the step; third derivatives of order 10 |way|^3
    scale_of = rr.abs().double() + 10 * hh.abs().double()
    assert bool(((slope - along).abs() <= scale_of * (2.0 ** -20 / step + 30 * step ** 2)).all())


def test_outputs_may_be_left_out_and_stay_inside():
    from paper_2502_16982_b200 import binding as b

    gen = torch.Generator().manual_seed(9)
    z = (torch.randn(20, 6000, generator=gen) * 2).cuda()
    y = torch.randint(0, 6000, (20,), generator=gen).cuda()
    full = b.muon_logits_logprob(z, y, top=9)
    store = torch.full((20 * 9 + 16,), -7, dtype=torch.int64, device="cuda")
    only = b.LogitsLogprob(None, None, None, store[8:-8].view(20, 9), None, None)
    b.muon_logits_logprob(z, y, top=9, out=only)
    assert torch.equal(only.top_ids, full.top_ids) and bool((store[:8] == -7).all()) and bool((store[-8:] == -7).all())
    part = b.muon_logits_logprob(z, y, out=b.LogitsLogprob(None, torch.empty(20, device="cuda"), None))
    assert torch.allclose(part.entropy, full.entropy, rtol=1e-5)
    free = b.muon_logits_logprob(z, top=9)
    assert free.logprob is None and torch.equal(free.top_ids, full.top_ids) and torch.equal(free.lse, full.lse)
    none = b.muon_logits_logprob(z[:0], y[:0], top=3)
    assert none.top_ids.shape == (0, 3) and none.logprob.shape == (0,)
    assert b.muon_logits_logprob_grad(z[:0], y[:0], none, g_logprob=none.lse).shape == (0, 6000)


def test_other_stream_and_captured_graph():
    from paper_2502_16982_b200 import binding as b

    gen = torch.Generator().manual_seed(10)
    z = torch.randn(30, 7001, generator=gen).to(BF).cuda()
    y = torch.randint(0, 7001, (30,), generator=gen).cuda()
    g = torch.randn(30, generator=gen).cuda()
    want = b.muon_logits_logprob(z, y, top=20)
    dwant = b.muon_logits_logprob_grad(z, y, want, g_logprob=g, g_entropy=g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    r = b.muon_logits_logprob(z, y, top=20, stream=side)
    side.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(r, want))
    held = torch.zeros_like(z)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = b.muon_logits_logprob(held, y, top=20)
        d = b.muon_logits_logprob_grad(held, y, r, g_logprob=g, g_entropy=g)
    held.copy_(z)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(r, want)) and torch.equal(d, dwant)


def test_rows_past_32_bit_offsets():
    from paper_2502_16982_b200 import binding as b

    T, V = 13200, 163840
    z = torch.zeros(T, V, dtype=BF, device="cuda")
    gen = torch.Generator().manual_seed(11)
    rows = [0, 13106, 13107, T - 1]  # on both sides of 2^31 elements
    z[rows] = torch.randn(4, V, generator=gen).to(BF).cuda()
    y = torch.full((T,), V - 1, dtype=torch.int64, device="cuda")
    r = b.muon_logits_logprob(z, y, top=4)
    part = b.LogitsLogprob(*[t[rows] for t in r])
    check_rows(part, f64(z[rows]), np.full(4, V - 1), 1.0, 4)
    g = torch.ones(T, device="cuda")
    b.muon_logits_logprob_grad(z, y, r, g_logprob=g, dlogits=z)
    _, _, log_q, counts = expect(f64(z[[1]]) * 0, np.array([V - 1]), 1.0)
    assert abs(float(z[1, -1]) - 1) < 2.0 ** -7 and abs(float(z[T - 2, -1]) - 1) < 2.0 ** -7
    assert abs(float(z[T - 2, 0]) * V + 1) < 2.0 ** -7


def test_a_teachers_entries_feed_distillation():
    """logits -> alternatives and log-sum-exp -> the distillation loss at the student's head."""
    from oracle import head_oracle as ho
    from paper_2502_16982_b200 import binding as b

    gen = torch.Generator().manual_seed(12)
    T, V, D, top, tau = 70, 3000, 64, 16, 2.0
    z = (torch.randn(T, V, generator=gen) * 2).to(BF).cuda()
    mask = torch.zeros(T, dtype=torch.int64)
    mask[::5] = -100
    t = b.muon_logits_logprob(z, mask.cuda(), top=top, logit_scale=1 / tau)
    x = torch.randn(T, D, generator=gen).to(BF).cuda()
    w = (torch.randn(V, D, generator=gen) * 0.2).to(BF).cuda()
    r = b.muon_head_distill(x, w, t.top_ids, t.top_logits, temperature=tau, teacher_lse=t.lse, dx=True, dw=True)
    zz = f64(z)
    ids = lo.best(zz, top)
    picked = np.take_along_axis(zz, ids, 1)
    lse = np.log(np.exp(zz / tau).sum(1))
    ids[mask.numpy() < 0] = -1
    rows = ho.teacher_rows(ids, picked, V, tau, lse)
    ref = ho.head_loss(f64(x), f64(w), rows, temperature=tau)
    assert np.abs(f64(r.loss) - ref["loss"]).max() <= 1e-4 and np.all(f64(r.loss)[::5] == 0)
    for got, want in ((r.dx, ref["dx"]), (r.dw, ref["dw"])):
        assert np.linalg.norm(f64(got) - want) <= 1e-2 * np.linalg.norm(want)  # two roundings to bf16


def test_refusals_of_the_binding():
    from paper_2502_16982_b200 import binding as b

    z, y = torch.zeros(4, 100, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    r = b.muon_logits_logprob(z, y)
    f = lambda **k: dict(dict(logits=z, targets=y), **k)
    for bad in (f(logits=z.half()), f(logits=z[0]), f(logits=z.t()), f(logits=z.cpu()), f(targets=y.int()), f(targets=y[:3]),
                f(targets=y.cpu()), f(top=129), f(top=-1), f(top=101), f(logit_scale=0.0), f(logit_scale=float("nan")),
                f(logits=z[:1].expand(4, 100)), f(top=2, out=b.LogitsLogprob(None, None, None, y)),
                f(out=b.LogitsLogprob(None, None, None)), f(targets=None, out=r)):
        with pytest.raises(b.MuonError):
            b.muon_logits_logprob(**bad)
    g = torch.zeros(4, device="cuda")
    f = lambda **k: dict(dict(logits=z, targets=y, saved=r, g_logprob=g), **k)
    for bad in (f(saved=r._replace(lse=None)), f(saved=r._replace(entropy=None), g_entropy=g), f(targets=None), f(g_logprob=g[:3]),
                f(g_logprob=g.double()), f(dlogits=torch.zeros(4, 100)), f(dlogits=torch.zeros(4, 100, device="cuda", dtype=BF)),
                f(dlogits=torch.zeros(4, 99, device="cuda"))):
        with pytest.raises(b.MuonError):
            b.muon_logits_logprob_grad(**bad)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("T", [6, 600])
def test_masks_of_the_lowest_number(dtype, T):
    """Entries masked with the dtype's lowest number are out, like those of minus infinity; a row
    of them alone has nothing left."""
    from paper_2502_16982_b200 import binding as b

    V = 20003
    gen = torch.Generator().manual_seed(31)
    z = torch.randn(T, V, generator=gen).to(dtype)
    masked = torch.rand(T, V, generator=gen) < 0.9
    masked[:, 77] = False
    masked[0] = True
    low = torch.where(masked, torch.tensor(torch.finfo(dtype).min, dtype=dtype), z).cuda()
    inf = torch.where(masked, torch.tensor(-float("inf"), dtype=dtype), z).cuda()
    y = torch.full((T,), 77).cuda()
    r, s = b.muon_logits_logprob(low, y, top=20), b.muon_logits_logprob(inf, y, top=20)
    assert all(torch.equal(getattr(r, k), getattr(s, k)) for k in ("logprob", "entropy", "lse", "top_ids"))
    assert float(r.lse[0]) == -float("inf") and float(r.entropy[0]) == 0.0
    g = torch.ones(T, device="cuda")
    d, e = (b.muon_logits_logprob_grad(q, y, v, g_logprob=g, g_entropy=g) for q, v in ((low, r), (inf, s)))
    assert torch.equal(d, e) and not d[0].any() and not d[masked.cuda()].any()


def test_calls_of_two_streams_at_once():
    from paper_2502_16982_b200 import binding as b

    gen = torch.Generator().manual_seed(32)
    z = [(torch.randn(64, 50000, generator=gen) * 2).to(BF).cuda() for _ in range(2)]
    y = torch.randint(0, 50000, (64,), generator=gen).cuda()
    want = [b.muon_logits_logprob(v, y, top=32) for v in z]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[b.muon_logits_logprob(z[k], y, top=32, stream=streams[k]) for k in range(2)] for _ in range(20)]
    torch.cuda.synchronize()
    for pair in got:
        for r, w in zip(pair, want):
            assert all(torch.equal(p, q) for p, q in zip(r, w))


def test_a_scale_that_its_field_does_not_hold_is_refused():
    from paper_2502_16982_b200 import binding as b

    z, y = torch.zeros(4, 100, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    with pytest.raises(b.MuonError):
        b.muon_logits_logprob(z, y, logit_scale=1e300)
