"""Log probabilities at the LM head (muon_head_logprob and its gradient) against the fp64
oracle.

Tolerances, from the arithmetic the header states.  A logit is an fp32 sum of exact
products in steps of 16 (D/16 additions, each within 2^-23 of a partial sum that
sum |x_i w_i| bounds), so it is within
    e_l = scale (D/16 + 8) 2^-23 A,   A = max over tokens and entries of sum |x_i w_i|.
To first order d logprob = d l_y - sum q d l, within 2 e_l, d lse within e_l and
d H = - sum q (log q + H) d l within 2 e_l H.  The sums over the vocabulary add, with D1 =
sum q |l - lmax|, D2 = sum q (l - lmax)^2 and n_c = (V/256 + 64) 2^-24,
    e_s = 2^-22 (1 + D1) + n_c;  to H: e_s + D1 (2^-22 + 2 n_c) + 2^-22 (D1 + D2 + H).
The gradient of a logit is q (..): q is within e_q = 3 e_l + err(lse) + 2^-21 (1 + |log q|)
relative, the bracket r + h (log q + H) within |h| (2 e_l + err(lse) + err(H) + 2^-22 |log q|);
it is rounded to bf16 once, 2^-8.  At the target r (1 - q) of fp32 values adds |r| (2 e_l +
2^-20).  dx and dw are fp32 sums of those products (V/16 + 64 or T/16 + 16 steps of 2^-23)
and rounded once where they are bf16.  Logits kept as codes: q is within e_k = 2^-12 more and what
lies 2^-32 below the largest of its columns is 0, log q within e_k absolutely."""

import numpy as np
import pytest
import torch

from oracle import logprob_oracle as lo

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def make(T, D, V, seed, offset_x=0, offset_w=0, pad_x=0, pad_w=0, gain=3.0):
    gen = torch.Generator().manual_seed(seed)

    def matrix(rows, cols, std, offset, pad):
        flat = torch.zeros(offset + rows * (cols + pad), dtype=BF)
        flat[offset:].view(rows, cols + pad)[:, :cols] = (torch.randn(rows, cols, generator=gen) * std).to(BF)
        return flat.cuda()[offset:].view(rows, cols + pad)[:, :cols]

    return matrix(T, D, 1.0, offset_x, pad_x), matrix(V, D, gain / D ** 0.5, offset_w, pad_w), gen


class Reference:
    def __init__(self, x, w, targets, scale):
        self.x, self.w, self.targets, self.scale = x, w, targets, scale
        T, V, D = x.shape[0], w.shape[0], x.shape[1]
        z = x @ w.T
        self.logprob, self.entropy, self.lse, self.log_q, self.counts = lo.logprob_rows(z, targets, scale)
        self.e_l = scale * (D / 16 + 8) * 2.0 ** -23 * (float((np.abs(x) @ np.abs(w).T).max()) if T else 0.0)
        top = (z * scale).max(1) if T else np.zeros(0)
        far = np.where(self.counts[:, None], (top - self.lse)[:, None] - self.log_q, 0.0)
        q = np.where(self.counts[:, None], np.exp(self.log_q), 0.0)
        d1, d2 = (q * far).sum(1), (q * far * far).sum(1)
        u, n_c = 2.0 ** -22, (V / 256 + 64) * 2.0 ** -24
        e_s = u * (1 + d1) + n_c
        self.tol = {"logprob": 2 * self.e_l + e_s + u * (1 + 2 * np.abs(self.logprob) + np.abs(top - self.lse)),
                    "lse": self.e_l + e_s + u * (1 + np.abs(top) + np.abs(self.lse)),
                    "entropy": 2.01 * self.e_l * self.entropy + e_s + d1 * (u + 2 * n_c) + u * (d1 + d2 + self.entropy)}
        self.q = q

    def check(self, r):
        for name, tol in self.tol.items():
            got = getattr(r, name)
            if got is None:
                continue
            err = np.abs(f64(got) - getattr(self, name))
            assert np.all(err <= tol), (name, float((err / tol).max()))
            assert np.all(f64(got)[~self.counts] == 0)

    def check_grads(self, d, r, h, before=None, kept=False):
        T, V = self.log_q.shape
        G = lo.logprob_grad(self.log_q, self.entropy, self.counts, self.targets, r, h, self.scale)
        ra, ha = (np.zeros(T) if v is None else np.where(self.counts, np.abs(v), 0.0) for v in (r, h))
        t, u = np.abs(self.log_q), 2.0 ** -22
        e_k = 2.0 ** -12 if kept else 0.0
        e_q = 3 * self.e_l + self.tol["lse"][:, None] + 2 * u * (1 + t) + e_k
        size = ra[:, None] + ha[:, None] * (t + self.entropy[:, None])
        err = self.q * (size * e_q + ha[:, None] * (2 * self.e_l + e_k + (self.tol["lse"] + self.tol["entropy"])[:, None] + u * t))
        if kept:
            err = err + 2.0 ** -31 * size
        for i in np.flatnonzero(self.counts):
            err[i, self.targets[i]] += ra[i] * (2 * self.e_l + 2.0 ** -20)
        err = self.scale * err
        G_abs = np.abs(G) + err
        xs = np.where(self.counts[:, None], self.x, 0.0)
        for name, exact, pick, like, steps in (("dx", G @ self.w, lambda m, o: m @ o, np.abs(self.w), V / 16 + 64),
                                               ("dw", G.T @ xs, lambda m, o: m.T @ o, np.abs(xs), T / 16 + 16)):
            got = getattr(d, name)
            if got is None:
                continue
            bound = pick(2.0 ** -8 * G_abs + err, like) + (steps * 2.0 ** -23 + 2.0 ** -22) * pick(G_abs, like) + 1e-37
            if name == "dw" and before is not None:
                exact = exact + before
                bound = bound + 2.0 ** -24 * np.abs(exact)
            if got.dtype == BF:
                bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(exact)
            e = np.abs(f64(got) - exact)
            assert np.all(e <= bound), (name, float((e / bound).max()))
        if d.dx is not None:
            assert np.all(f64(d.dx)[~self.counts] == 0)


CASES = [
    (1, 64, 300, 0.0, {}),
    (1, 2048, 5000, 0.0, {}),
    (2, 8, 1, 0.0, {}),                                  # one vocabulary entry: probability 1
    (7, 1, 3, 0.0, {}),                                  # one dimension: rows TMA cannot address
    (24, 512, 4096, 0.3, {}),                            # tokens as rows
    (130, 72, 257, 0.3, {}),                             # an entry past a tile
    (256, 128, 512, 0.0, dict(dx=FP, dw=FP)),
    (257, 129, 1000, 0.5, dict(scale=1.3)),
    (513, 200, 1031, 0.1, dict(scale=0.5)),
    (300, 320, 2049, 1.0, {}),                           # every token masked
    (20, 320, 2049, 1.0, {}),
    (64, 1000, 777, 0.2, dict(dx=None)),
    (640, 96, 1500, 0.2, dict(dw=None)),
    (200, 264, 4096, 0.0, dict(pad_x=3, pad_w=8, offset_x=1, offset_w=8)),
    (200, 264, 900, 0.2, dict(offset_w=1, pad_w=1, dw=FP)),
    (1100, 520, 3001, 0.4, {}),
    (20011, 24, 300, 0.6, {}),                           # tokens counted in runs first
    (1200, 776, 9100, 0.3, dict(dx=FP)),
    (700, 256, 5000, 0.1, dict(gain=12.0)),              # confident rows, small entropies
]


@pytest.mark.parametrize("T,D,V,masked,opts", CASES)
def test_values_and_gradients_match_the_oracle(T, D, V, masked, opts):
    from paper_2502_16982_b200 import binding as b

    o = dict(opts)
    scale = o.pop("scale", 1.0)
    dxt, dwt = o.pop("dx", BF), o.pop("dw", BF)
    x, w, gen = make(T, D, V, 1000 * T + D, **o)
    targets = torch.randint(0, V, (T,), generator=gen)
    hide = torch.rand(T, generator=gen) < masked
    targets[hide] = torch.tensor([-100, -1, V, 1 << 40])[torch.randint(0, 4, (int(hide.sum()),), generator=gen)]
    x[hide.cuda()] = float("nan")  # what a masked token holds reaches nothing
    if hide.any():
        x[int(hide.nonzero()[0])] = float("inf")
    y = targets.cuda()
    ws = torch.full((b.muon_head_logprob_workspace_bytes(T, D, V, grads=False, packed_head=False),), 255, dtype=torch.uint8, device="cuda")
    r = b.muon_head_logprob(x, w, y, logit_scale=scale, workspace=ws)
    assert b.muon_head_status(ws) == 0
    plain = b.muon_head_logprob(x, w, y, logit_scale=scale, entropy=False)
    assert plain.entropy is None and torch.equal(plain.logprob, r.logprob) and torch.equal(plain.lse, r.lse)
    ref = Reference(np.where(hide.numpy()[:, None], 0.0, f64(x)), f64(w), targets.numpy(), scale)
    ref.check(r)
    rr, hh = torch.randn(T, generator=gen) / T, torch.randn(T, generator=gen) * 0.1 / T
    rr[hide], hh[hide] = float("nan"), float("inf")
    for g, e in ((rr, hh), (rr, None), (None, hh), (torch.full((T,), -0.7 / T), None)):
        dx = None if dxt is None else torch.full((T, D), 7.0, dtype=dxt, device="cuda")
        dw = None if dwt is None else torch.full((V, D), 7.0, dtype=dwt, device="cuda")
        n = b.muon_head_logprob_workspace_bytes(T, D, V, grads=True, dx=dxt is not None, dw=dwt is not None, packed_head=False)
        ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
        up = dict(g_logprob=None if g is None else g.cuda(), g_entropy=None if e is None else e.cuda(), logit_scale=scale)
        d = b.muon_head_logprob_grad(x, w, y, r, dx=dx, dw=dw, workspace=ws, **up)
        assert b.muon_head_status(ws) == 0
        zero = lambda v: None if v is None else np.where(hide.numpy(), 0.0, v.double().numpy())
        ref.check_grads(d, zero(g), zero(e))


@pytest.mark.parametrize("T,D,V,masked,opts", CASES + [(900, 512, 20000, 0.3, {}), (3000, 512, 9000, 0.1, dict(scale=0.8))])
@pytest.mark.parametrize("tiles", [None, 2, 3])
def test_gradients_from_kept_logits(T, D, V, masked, opts, tiles):
    """Codes of all logits kept by the forward pass, in one piece or in several of them."""
    from paper_2502_16982_b200 import binding as b

    o = dict(opts)
    scale = o.pop("scale", 1.0)
    dxt, dwt = o.pop("dx", BF), o.pop("dw", BF)
    x, w, gen = make(T, D, V, 2000 * T + D, **o)
    targets = torch.randint(0, V, (T,), generator=gen)
    hide = torch.rand(T, generator=gen) < masked
    targets[hide] = -100
    x[hide.cuda()] = float("nan")
    y = targets.cuda()
    ref = Reference(np.where(hide.numpy()[:, None], 0.0, f64(x)), f64(w), targets.numpy(), scale)
    rr, hh = torch.randn(T, generator=gen) / T, torch.randn(T, generator=gen) * 0.1 / T
    before, mode = b.muon_debug_set_head_piece_bytes(0 if tiles is None else tiles * T * 512), b.muon_debug_set_head_codes(2)
    try:
        n = b.muon_head_logprob_workspace_bytes(T, D, V, grads=False, packed_head=False, keep=True)
        ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
        r = b.muon_head_logprob(x, w, y, logit_scale=scale, workspace=ws, keep=True)
        assert r.kept is ws
        ref.check(r)
        held = ws.clone()
        for g, e in ((rr, hh), (None, hh)):
            dx = None if dxt is None else torch.full((T, D), 7.0, dtype=dxt, device="cuda")
            dw = None if dwt is None else torch.full((V, D), 7.0, dtype=dwt, device="cuda")
            n = b.muon_head_logprob_workspace_bytes(T, D, V, grads=True, dx=dxt is not None, dw=dwt is not None, packed_head=False, keep=True)
            gs = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
            up = dict(g_logprob=None if g is None else g.cuda(), g_entropy=e.cuda(), logit_scale=scale)
            d = b.muon_head_logprob_grad(x, w, y, r, dx=dx, dw=dw, workspace=gs, **up)
            assert b.muon_head_status(gs) == 0
            zero = lambda v: None if v is None else np.where(hide.numpy(), 0.0, v.double().numpy())
            ref.check_grads(d, zero(g), zero(e), kept=True)
        assert torch.equal(ws, held)  # only read: it may be asked for again
        again = b.muon_head_logprob_grad(x, w, y, r, dx=dx is not None, dw=dw is not None, **up)
        for p, q in zip(again, d):
            assert p is None and q is None or p.dtype != q.dtype or torch.equal(p, q)
    finally:
        b.muon_debug_set_head_piece_bytes(before)
        b.muon_debug_set_head_codes(mode)


def test_what_other_pieces_kept_gives_no_gradient_but_a_status():
    from paper_2502_16982_b200 import binding as b

    x, w, gen = make(300, 512, 3000, 3)
    y = torch.randint(0, 3000, (300,), generator=gen).cuda()
    r = b.muon_head_logprob(x, w, y, keep=True)
    before = b.muon_debug_set_head_piece_bytes(2 * 300 * 512)
    try:
        n = b.muon_head_logprob_workspace_bytes(300, 512, 3000, grads=True, keep=True)
        ws = torch.zeros(n, dtype=torch.uint8, device="cuda")
        d = b.muon_head_logprob_grad(x, w, y, r, g_logprob=torch.ones(300, device="cuda"), dx=True, dw=True, workspace=ws)
        assert b.muon_head_status(ws) == b.MUON_ERR_INVALID_ARG
        assert not d.dx.any() and not d.dw.any()
    finally:
        b.muon_debug_set_head_piece_bytes(before)
    with pytest.raises(b.MuonError):
        short = b.HeadLogprob(*r)
        short.kept = r.kept[:4096]
        b.muon_head_logprob_grad(x, w, y, short, g_logprob=torch.ones(300, device="cuda"), dx=True)


def test_scoring_keeps_nothing():
    from paper_2502_16982_b200 import binding as b

    x, w, gen = make(300, 512, 3000, 4)
    y = torch.randint(0, 3000, (300,), generator=gen).cuda()
    with torch.no_grad():
        assert b.muon_head_logprob(x, w, y).kept is None
    r = b.muon_head_logprob(x, w, y)
    assert r.kept is not None and r._replace(lse=r.lse).kept is None
    assert b.muon_head_logprob(x, w, y, keep=False).kept is None


@pytest.mark.parametrize("T,D,V", [(300, 136, 3000), (1100, 256, 2100), (70, 96, 5000)])
def test_several_pieces_and_adding_to_dw(T, D, V):
    from paper_2502_16982_b200 import binding as b

    x, w, gen = make(T, D, V, 77)
    targets = torch.randint(0, V, (T,), generator=gen)
    targets[::9] = -100
    y = targets.cuda()
    r = b.muon_head_logprob(x, w, y, keep=False)
    assert r.kept is None
    ref = Reference(np.where(targets.numpy()[:, None] < 0, 0.0, f64(x)), f64(w), targets.numpy(), 1.0)
    ref.check(r)
    rr, hh = torch.randn(T, generator=gen), torch.randn(T, generator=gen) * 0.1
    z = np.where(targets.numpy() < 0, 0.0, 1.0)
    up = dict(g_logprob=rr.cuda(), g_entropy=hh.cuda())
    before = b.muon_debug_set_head_piece_bytes(2 * T * 512)  # two tiles a piece
    try:
        base = torch.randn(V, D, generator=gen)
        dw = base.cuda()
        d = b.muon_head_logprob_grad(x, w, y, r, dx=True, dw=dw, accumulate_dw=True, **up)
        again = b.muon_head_logprob_grad(x, w, y, r, dx=True, dw=base.cuda(), accumulate_dw=True, **up)
    finally:
        b.muon_debug_set_head_piece_bytes(before)
    assert torch.equal(d.dx, again.dx) and torch.equal(d.dw, again.dw)
    ref.check_grads(d, rr.double().numpy() * z, hh.double().numpy() * z, before=base.double().numpy())


def test_gradient_against_differences():
    from paper_2502_16982_b200 import binding as b

    T, D, V = 40, 64, 500
    x, w, gen = make(T, D, V, 5)
    y = torch.randint(0, V, (T,), generator=gen).cuda()
    rr, hh = torch.randn(T, generator=gen).cuda(), (torch.randn(T, generator=gen) * 0.3).cuda()
    r = b.muon_head_logprob(x, w, y)
    d = b.muon_head_logprob_grad(x, w, y, r, g_logprob=rr, g_entropy=hh, dx=torch.empty(T, D, device="cuda"))
    # steps that bf16 holds: to the next values on both sides, as far apart as they came out
    way = torch.sign(torch.randn(T, D, generator=gen)).cuda() * 2.0 ** -5
    up, down = (x.float() + way).to(BF), (x.float() - way).to(BF)
    moved = (up.double() - down.double())

    def value(xx):
        v = b.muon_head_logprob(xx, w, y)
        return rr.double() * v.logprob.double() + hh.double() * v.entropy.double()

    along = (d.dx.double() * moved).sum(1)
    # a change of the logits of at most c = 0.05 |w|_1: third-order terms c^3 and, as the two steps
    # are not quite equal, second-order ones of their difference; bf16 of the gradient of logits
    c = float((w.double().abs() * 2.0 ** -5).sum(1).max())
    skew = float(((up.double() + down.double() - 2 * x.double()).abs().sum(1)).max()) * float(w.abs().max())
    size = rr.abs().double() + 10 * hh.abs().double()
    bound = size * (c ** 3 + 2 * c * skew + 2.0 ** -18) + 2.0 ** -8 * 4 * size * c
    assert bool(((value(up) - value(down) - along).abs() <= bound).all())


def test_other_stream_and_captured_graph():
    from paper_2502_16982_b200 import binding as b

    T, D, V = 300, 128, 2000
    x, w, gen = make(T, D, V, 6)
    y = torch.randint(0, V, (T,), generator=gen).cuda()
    g, e = torch.randn(T, generator=gen).cuda(), torch.randn(T, generator=gen).cuda()

    def step(xx, **k):
        r = b.muon_head_logprob(xx, w, y, **k)
        return tuple(r) + tuple(b.muon_head_logprob_grad(xx, w, y, r, g_logprob=g, g_entropy=e, dx=True, dw=True, **k))

    want = step(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(x, stream=side)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    held = torch.zeros_like(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(held)
    held.copy_(x)
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_agrees_with_the_cross_entropy():
    """REINFORCE with one advantage for all tokens is the cross entropy: the same losses and gradients."""
    from paper_2502_16982_b200 import binding as b

    T, D, V = 400, 256, 3000
    x, w, gen = make(T, D, V, 7)
    y = torch.randint(0, V, (T,), generator=gen).cuda()
    y[::7] = -100
    n = int((y >= 0).sum())
    r = b.muon_head_logprob(x, w, y)
    d = b.muon_head_logprob_grad(x, w, y, r, g_logprob=torch.full((T,), -1.0 / n, device="cuda"), dx=torch.empty(T, D, device="cuda"),
                                 dw=torch.empty(V, D, device="cuda"))
    ref = b.muon_head_xent(x, w, y, dx=torch.empty(T, D, device="cuda"), dw=torch.empty(V, D, device="cuda"))
    assert torch.allclose(-r.logprob, ref.loss, rtol=1e-6, atol=1e-5) and torch.allclose(r.lse, ref.lse, rtol=1e-6)
    for p, q in ((d.dx, ref.dx), (d.dw, ref.dw)):
        assert float((p - q).norm()) <= 4e-3 * float(q.norm())  # both within 2^-8 of the sums, at most


def test_a_policy_step():
    """Log probabilities -> a clipped ratio objective with an entropy bonus -> gradients at the
    head -> their norm -> clipped AdamW on the head; everything again in fp64."""
    from oracle import adamw_oracle as aw
    from paper_2502_16982_b200 import binding as b

    T, D, V = 320, 128, 1500
    x, _, gen = make(T, D, V, 8)
    master = torch.randn(V, D, generator=gen).cuda() * 0.2
    w = master.to(BF)
    y = torch.randint(0, V, (T,), generator=gen).cuda()
    y[:40] = -100
    counts = (y >= 0)
    adv = torch.randn(T, generator=gen).cuda()
    old = b.muon_head_logprob(x, (master + 0.01).to(BF), y, entropy=False).logprob
    m, v = torch.zeros_like(master), torch.zeros_like(master)

    r = b.muon_head_logprob(x, w, y)
    n = counts.sum()

    def upstream(logprob):
        ratio = torch.exp(logprob - old.to(logprob.dtype))
        kept = ((adv >= 0) & (ratio < 1.2)) | ((adv < 0) & (ratio > 0.8))
        return torch.where(counts & kept, -adv.to(logprob.dtype) * ratio / n, 0.0)

    g, e = upstream(r.logprob), torch.where(counts, -0.01 / n, 0.0)
    d = b.muon_head_logprob_grad(x, w, y, r, g_logprob=g, g_entropy=e, dx=True, dw=torch.empty(V, D, device="cuda"))
    grads = b.MuonGrads([d.dx, d.dw])
    limit = 0.5 * float(torch.sqrt((d.dx.double() ** 2).sum() + (d.dw.double() ** 2).sum()))
    c = grads.muon_grad_norm(limit)
    before = f64(master)
    b.muon_adamw_step([master], [d.dw], [m], [v], 1, lr=1e-2, wd=0.1, coef=c.coef)

    ref = Reference(np.where(counts.cpu().numpy()[:, None], f64(x), 0.0), f64(w), y.cpu().numpy(), 1.0)
    ref.check(r)
    ref.check_grads(d, f64(g), f64(e), kept=True)
    G = lo.logprob_grad(ref.log_q, ref.entropy, ref.counts, ref.targets, f64(upstream(torch.as_tensor(ref.logprob, device="cuda"))), f64(e))
    dx, dw = G @ ref.w, G.T @ ref.x
    coef = limit / (np.sqrt((dx ** 2).sum() + (dw ** 2).sum()) + 1e-6)
    assert abs(float(c.coef) - coef) <= 2.0 ** -7 * coef
    pr, mr, vr = aw.adamw_step(before, f64(d.dw) * float(c.coef), np.zeros((V, D)), np.zeros((V, D)), 1, lr=1e-2, wd=0.1)
    for got, want in ((master, pr), (m, mr), (v, vr)):
        assert np.linalg.norm(f64(got) - want) <= 1e-5 * np.linalg.norm(want)


def test_no_tokens():
    from paper_2502_16982_b200 import binding as b

    w = torch.ones(300, 64, dtype=BF, device="cuda")
    x, y = torch.zeros(0, 64, dtype=BF, device="cuda"), torch.zeros(0, dtype=torch.int64, device="cuda")
    r = b.muon_head_logprob(x, w, y)
    assert r.logprob.shape == r.entropy.shape == r.lse.shape == (0,)
    dw = torch.full((300, 64), 7.0, device="cuda")
    d = b.muon_head_logprob_grad(x, w, y, r, g_logprob=r.lse, dx=True, dw=dw)
    assert d.dx.shape == (0, 64) and bool((dw == 0).all())


def test_refusals_of_the_binding():
    from paper_2502_16982_b200 import binding as b

    x, w, gen = make(4, 64, 100, 9)
    y = torch.zeros(4, dtype=torch.int64, device="cuda")
    r = b.muon_head_logprob(x, w, y)
    f = lambda **k: dict(dict(x=x, w=w, targets=y), **k)
    for bad in (f(x=x[0]), f(x=x.float()), f(w=w[:, :32]), f(w=w.t()), f(x=x.cpu()), f(w=w.cpu()), f(targets=y.int()), f(targets=y[:3]),
                f(logit_scale=0.0), f(logit_scale=float("inf")), f(workspace=torch.zeros(1024, dtype=torch.uint8, device="cuda")),
                f(workspace=torch.zeros(1 << 20, device="cuda")), f(out=r._replace(logprob=None)), f(out=r._replace(lse=r.lse[:3]))):
        with pytest.raises(b.MuonError):
            b.muon_head_logprob(**bad)
    g = torch.zeros(4, device="cuda")
    f = lambda **k: dict(dict(x=x, w=w, targets=y, saved=r, g_logprob=g, dx=True), **k)
    for bad in (f(dx=None), f(dx=False, dw=False), f(saved=r._replace(lse=None)), f(saved=r._replace(logprob=None)),
                f(saved=r._replace(entropy=None), g_entropy=g), f(g_logprob=g[:2]), f(g_logprob=g.double()), f(dx=torch.zeros(4, 64)),
                f(dx=torch.zeros(4, 64, device="cuda", dtype=torch.float16)), f(dw=True, accumulate_dw=True),
                f(dx=torch.zeros(4, 63, device="cuda")), f(workspace=torch.zeros(1024, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(b.MuonError):
            b.muon_head_logprob_grad(**bad)


@pytest.mark.parametrize("T,D,V", [(1100, 256, 2100), (300, 129, 3000)])
def test_kept_without_codes_or_entropy(T, D, V):
    """Where codes are not faster the forward pass keeps only what it gathered."""
    from paper_2502_16982_b200 import binding as b

    x, w, gen = make(T, D, V, 41)
    targets = torch.randint(0, V, (T,), generator=gen)
    targets[::5] = -100
    y, z = targets.cuda(), np.where(targets.numpy() < 0, 0.0, 1.0)
    ref = Reference(f64(x) * z[:, None], f64(w), targets.numpy(), 1.0)
    rr = torch.randn(T, generator=gen)
    for mode in (1, 2):
        before, piece = b.muon_debug_set_head_codes(mode), b.muon_debug_set_head_piece_bytes(2 * T * 512)
        try:
            r = b.muon_head_logprob(x, w, y, keep=True, entropy=False)
            assert r.kept is not None and r.entropy is None
            d = b.muon_head_logprob_grad(x, w, y, r, g_logprob=rr.cuda(), dx=True, dw=True)
        finally:
            b.muon_debug_set_head_codes(before)
            b.muon_debug_set_head_piece_bytes(piece)
        ref.check(r)
        ref.check_grads(d, rr.double().numpy() * z, None, kept=True)


def test_more_logits_than_are_kept():
    """3 GiB of codes, the rest of the logits formed again: REINFORCE with one advantage against
    the cross entropy (both within 2^-8 of the sums, at most)."""
    from paper_2502_16982_b200 import binding as b

    T, D, V = 17000, 64, 110000
    gen = torch.Generator(device="cuda").manual_seed(42)
    x = torch.randn(T, D, generator=gen, device="cuda").to(BF)
    w = (torch.randn(V, D, generator=gen, device="cuda") * 0.3).to(BF)
    y = torch.randint(0, V, (T,), generator=gen, device="cuda")
    y[::11] = -1
    before = b.muon_debug_set_head_codes(2)
    try:
        r = b.muon_head_logprob(x, w, y)
        assert 3 << 30 > r.kept.numel() - T * V // 8 > (3 << 30) - (2 << 28)  # whole pieces beside the statistics
        n = int((y >= 0).sum())
        f32 = dict(device="cuda")
        d = b.muon_head_logprob_grad(x, w, y, r, g_logprob=torch.full((T,), -1.0 / n, device="cuda"), dx=torch.empty(T, D, **f32),
                                     dw=torch.empty(V, D, **f32))
        del r
        ref = b.muon_head_xent(x, w, y, dx=torch.empty(T, D, **f32), dw=torch.empty(V, D, **f32))
    finally:
        b.muon_debug_set_head_codes(before)
    for p, q in zip(d, (ref.dx, ref.dw)):
        assert float((p - q).norm()) <= 4e-3 * float(q.norm())
    assert not d.dx[::11].any()
