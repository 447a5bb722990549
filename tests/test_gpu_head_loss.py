"""GPU parity of the LM-head losses (muon_head_xent, muon_head_distill) with the
fp64 oracle.

Tolerances, derived from the arithmetic the header states.  A logit is an fp32 sum
of exact products in steps of 16 (D/16 additions, each within 2^-23 of a partial
sum that sum |x_i w_i| bounds), so it is within
    e_l = (D/16 + 8) 2^-23 A,   A = max over tokens and entries of sum |x_i w_i|
(times the scale of the logits; the 8 covers scaling, exponent and logarithm).
lse and loss are each within 2 e_l plus (V/256 + 64) 2^-24 relative for the sums.
The gradient of a logit is rounded to bf16 once (2^-8 relative) and q carries the
relative error 2 e_l; the products are fp32 sums.  With |G| |W| and |G|^T |X| formed
from absolute values, every element of dx and dw is within
    (2^-8 + 4 e_l + 2^-12 + steps 2^-23) bound + (bf16 output: 2^-8 |value|);
the 2^-12 is that of logits kept as codes of 2^-11 steps, whose smallest values
(2^-32 of their row's largest) become 0.
The gradient at a sparse entry is a difference c q - p of fp32 values: it adds
4 e_l + 2^-20 of the coefficient, through |W| or |X| of that entry; covered by
adding that to every |G| at an entry before the absolute products are formed."""

import numpy as np
import pytest
import torch

from oracle import head_oracle as ho

pytestmark = pytest.mark.gpu


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def make(T, D, V, seed, offset_x=0, offset_w=0, pad_x=0, pad_w=0, gain=3.0):
    gen = torch.Generator().manual_seed(seed)

    def matrix(rows, cols, std, offset, pad):
        flat = torch.zeros(offset + rows * (cols + pad), dtype=torch.bfloat16)
        m = flat[offset:].view(rows, cols + pad)[:, :cols]
        m.copy_((torch.randn(rows, cols, generator=gen) * std).to(torch.bfloat16))
        d = flat.cuda()
        return d[offset:].view(rows, cols + pad)[:, :cols]

    return matrix(T, D, 1.0, offset_x, pad_x), matrix(V, D, gain / D ** 0.5, offset_w, pad_w), gen


def check(r, ref, x, w, rows, a, dx_dtype, dw_dtype, coef):
    T, D = x.shape
    V = w.shape[0]
    xs = np.where(ref["counts"][:, None], np.abs(x), 0.0)
    e_l = a * (D / 16 + 8) * 2.0 ** -23 * (float((xs @ np.abs(w).T).max()) if T else 0.0)
    rel = (V / 256 + 64) * 2.0 ** -24
    for name in ("loss", "lse"):
        got, want = f64(getattr(r, name)), ref[name]
        scale_e = 2 * e_l + rel * (1 + np.abs(ref["lse"])) * (1 + 2 * abs(coef["z"]) * np.abs(ref["lse"]))
        scale_e = scale_e * (1 + 2 * abs(coef["z"]) * np.abs(ref["lse"]))
        assert got.shape == want.shape and np.all(np.abs(got - want) <= scale_e + 1e-30), (name, np.abs(got - want).max())
        assert np.all(got[~ref["counts"]] == 0.0)
    g = coef["g"]
    assert abs(float(r.total[0]) - ref["total"]) <= float((np.abs(g) * (scale_e + 2.0 ** -20 * np.abs(ref["loss"]))).sum()) + 1e-30
    ids, p, usable = rows
    absg = np.abs(ref["g"])
    slack = np.repeat(np.abs(g * a)[:, None] * 2.0 ** -31, V, 1)
    for t in np.flatnonzero(ref["counts"]):
        np.add.at(slack[t], ids[t][usable[t]], np.abs(g[t] * a) * (4 * e_l + 2.0 ** -20))
    for name, dtype, like, steps in (("dx", dx_dtype, np.abs(w), V / 16 + 64), ("dw", dw_dtype, xs, T / 16 + 16)):
        got = getattr(r, name)
        if dtype is None:
            assert got is None
            continue
        assert got.dtype == dtype
        pick = (lambda m: m @ like) if name == "dx" else (lambda m: m.T @ like)
        bound = (2.0 ** -8 + 4 * e_l + 2.0 ** -12 + steps * 2.0 ** -23) * pick(absg) + 1.01 * pick(slack)
        if dtype == torch.bfloat16:
            bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref[name])
        err = np.abs(f64(got) - ref[name])
        assert np.all(err <= bound + 1e-30), (name, float((err / (bound + 1e-30)).max()))


def coefficients(counts, weight, mean, scale, z):
    wt = np.ones(len(counts)) if weight is None else f64(weight)
    g = np.where(counts, scale * wt, 0.0)
    if mean:
        n = wt[counts].sum()
        g = g / n if n else g * 0
    return {"g": g, "z": z}


BF, FP = torch.bfloat16, torch.float32


@pytest.mark.parametrize("T,D,V,masked,opts", [
    (1, 64, 300, 0.0, {}),
    (1, 2048, 5000, 0.0, dict(z_loss=1e-3)),
    (2, 8, 1, 0.0, {}),                                  # one vocabulary entry: loss 0, no gradient
    (7, 1, 3, 0.0, {}),                                  # one dimension: rows TMA cannot address
    (130, 72, 257, 0.3, dict(weights=True)),             # an entry past a tile
    (256, 128, 512, 0.0, dict(dx=FP, dw=FP)),
    (257, 129, 1000, 0.5, dict(weights=True, mean=False, scale=0.25)),
    (513, 200, 1031, 0.1, dict(logit_scale=0.5, z_loss=1e-2)),
    (300, 320, 2049, 1.0, {}),                           # every token masked
    (64, 1000, 777, 0.2, dict(dx=None)),
    (640, 96, 1500, 0.2, dict(dw=None)),
    (200, 264, 4096, 0.0, dict(pad_x=3, pad_w=8, offset_x=1, offset_w=8)),
    (200, 264, 900, 0.2, dict(offset_w=1, pad_w=1, dw=FP)),
    (1100, 520, 3001, 0.4, {}),
    (20011, 24, 300, 0.6, dict(weights=True)),           # tokens counted in runs first
    (1200, 776, 9100, 0.3, dict(dx=FP)),
])
def test_cross_entropy_matches_the_oracle(T, D, V, masked, opts):
    from paper_2502_16982_b200 import binding as b

    o = dict(opts)
    x, w, gen = make(T, D, V, 1000 * T + D, **{k: o.pop(k) for k in list(o) if k.startswith(("pad", "offset"))})
    targets = torch.randint(0, V, (T,), generator=gen)
    hide = torch.rand(T, generator=gen) < masked
    targets[hide] = torch.tensor([-100, -1, V, 1 << 40])[torch.randint(0, 4, (int(hide.sum()),), generator=gen)]
    weight = (torch.rand(T, generator=gen) + 0.5).cuda() if o.pop("weights", False) else None
    x[hide.cuda()] = float("nan")  # what a masked token holds reaches nothing
    if hide.any():
        x[int(hide.nonzero()[0])] = float("inf")
    dxt, dwt = o.pop("dx", BF), o.pop("dw", BF)
    dx = None if dxt is None else torch.full((T, D), 7.0, dtype=dxt, device="cuda")
    dw = None if dwt is None else torch.full((V, D), 7.0, dtype=dwt, device="cuda")
    ws = torch.full((b.muon_head_workspace_bytes(T, D, V, packed_head=False),), 255, dtype=torch.uint8, device="cuda")
    r = b.muon_head_xent(x, w, targets.cuda(), weight=weight, dx=dx, dw=dw, workspace=ws, **o)
    assert b.muon_head_status(ws) == 0
    rows = ho.target_rows(targets.numpy(), V)
    xr, wr = f64(x), f64(w)
    ref = ho.head_loss(np.where(rows[2].any(1)[:, None], xr, 0.0), wr, rows, weight=None if weight is None else f64(weight), **o)
    coef = coefficients(ref["counts"], weight, o.get("mean", True), o.get("scale", 1.0), o.get("z_loss", 0.0))
    check(r, ref, np.where(ref["counts"][:, None], xr, 0.0), wr, rows, o.get("logit_scale", 1.0), dxt, dwt, coef)


@pytest.mark.parametrize("T,D,V,K,opts", [
    (1, 64, 300, 1, {}),
    (5, 40, 128, 128, {}),                               # every entry of the vocabulary
    (130, 72, 700, 33, dict(temperature=2.0, masked=0.3)),
    (257, 128, 1500, 64, dict(tail=True, weights=True)),
    (300, 203, 2100, 20, dict(twice=True, dw=FP)),
    (512, 256, 3000, 100, dict(z_bf16=True, strided=True, temperature=0.7, scale=0.49, mean=False)),
    (60, 320, 900, 8, dict(neg_inf=True, logit_scale=0.5)),
    (90, 64, 600, 8, dict(masked=1.0)),
    (700, 512, 2600, 5, dict(dx=None, tail=True, temperature=3.0)),
    (900, 768, 12000, 40, dict(masked=0.2)),
    (16384, 16, 260, 3, dict(masked=0.5)),
])
def test_distillation_matches_the_oracle(T, D, V, K, opts):
    from paper_2502_16982_b200 import binding as b

    o = dict(opts)
    x, w, gen = make(T, D, V, 77 * T + K)
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
    ids[some] = -5                                        # entries that are not there
    if o.pop("neg_inf", False):
        z[torch.rand(T, K, generator=gen) < 0.3] = -float("inf")
        z[3] = -float("inf")                              # nothing left: masked
    weight = (torch.rand(T, generator=gen) + 0.5).cuda() if o.pop("weights", False) else None
    tlse = None
    if o.pop("tail", False):
        tlse = (torch.logsumexp(z.double() / tau, 1) + 0.3).float().cuda()
    hidden = torch.tensor(~ho.teacher_rows(ids.numpy(), f64(z), V, tau)[2].any(1))
    x[hidden.cuda()] = float("nan")
    dxt, dwt = o.pop("dx", BF), o.pop("dw", BF)
    ids_d, z_d = ids.cuda(), z.cuda()
    if o.pop("strided", False):
        ids_d = torch.cat([ids_d, ids_d[:, :3] * 0 - 9], 1)[:, :K]
        z_d = torch.cat([z_d, z_d[:, :1] * 0 + 99], 1)[:, :K]
        assert ids_d.stride(0) == K + 3 and z_d.stride(0) == K + 1
    dx = None if dxt is None else torch.full((T, D), 7.0, dtype=dxt, device="cuda")
    dw = None if dwt is None else torch.full((V, D), 7.0, dtype=dwt, device="cuda")
    ws = torch.full((b.muon_head_workspace_bytes(T, D, V, top=K, packed_head=False),), 255, dtype=torch.uint8, device="cuda")
    r = b.muon_head_distill(x, w, ids_d, z_d, teacher_lse=tlse, weight=weight, dx=dx, dw=dw, workspace=ws, **o)
    assert b.muon_head_status(ws) == 0
    rows = ho.teacher_rows(ids.numpy(), f64(z), V, tau, None if tlse is None else f64(tlse))
    xr, wr = np.where(rows[2].any(1)[:, None], f64(x), 0.0), f64(w)
    ref = ho.head_loss(xr, wr, rows, weight=None if weight is None else f64(weight), **o)
    coef = coefficients(ref["counts"], weight, o.get("mean", True), o.get("scale", 1.0), 0.0)
    check(r, ref, xr, wr, rows, o.get("logit_scale", 1.0) / tau, dxt, dwt, coef)


@pytest.fixture
def knobs():
    from paper_2502_16982_b200 import binding as b

    before = b.muon_debug_set_head_piece_bytes(0), b.muon_debug_set_head_codes(-1)
    yield b
    b.muon_debug_set_head_piece_bytes(before[0])
    b.muon_debug_set_head_codes(before[1])


@pytest.mark.parametrize("codes,room", [(1, "full"), (2, "full"), (2, "least"), (2, "between")])
@pytest.mark.parametrize("top", [0, 40])
def test_vocabulary_in_pieces(knobs, codes, room, top):
    """Three tiles of the vocabulary a piece: all of it computed twice, all of it kept
    as codes, one piece kept, two of four."""
    b = knobs
    T, D, V = 390, 72, 2500
    x, w, gen = make(T, D, V, 21)
    b.muon_debug_set_head_piece_bytes(390 * 256 * 2 * 3)
    b.muon_debug_set_head_codes(codes)
    full = b.muon_head_workspace_bytes(T, D, V, top=top)
    least = b.muon_head_workspace_bytes(T, D, V, top=top, least=True)
    piece = 390 * 256 * 2 * 3
    assert full - least == (3 * piece if codes == 2 else 0)
    ws = torch.full(({"full": full, "least": least, "between": least + piece}[room],), 255, dtype=torch.uint8, device="cuda")
    if top:
        ids = torch.stack([torch.randperm(V, generator=gen)[:top] for _ in range(T)])
        ids[7] = -1
        z = torch.randn(T, top, generator=gen)
        r = b.muon_head_distill(x, w, ids.cuda(), z.cuda(), dx=True, dw=True, workspace=ws)
        rows = ho.teacher_rows(ids.numpy(), f64(z), V, 1.0)
    else:
        t = torch.randint(0, V, (T,), generator=gen)
        t[::5] = -100
        r = b.muon_head_xent(x, w, t.cuda(), dx=True, dw=True, workspace=ws)
        rows = ho.target_rows(t.numpy(), V)
    assert b.muon_head_status(ws) == 0
    ref = ho.head_loss(f64(x), f64(w), rows)
    check(r, ref, f64(x), f64(w), rows, 1.0, BF, BF, coefficients(ref["counts"], None, True, 1.0, 0.0))
    with pytest.raises(b.MuonError):
        b.muon_head_xent(x, w, torch.zeros(T, dtype=torch.int64, device="cuda"), dx=True, dw=True,
                         workspace=torch.empty(piece, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("codes", [1, 2])
def test_wide_range_of_logits(knobs, codes):
    """Logits of several hundred: most of a row lies below what a code holds."""
    b = knobs
    b.muon_debug_set_head_codes(codes)
    x, w, gen = make(70, 64, 1500, 31, gain=100.0)
    t = torch.randint(0, 1500, (70,), generator=gen)
    r = b.muon_head_xent(x, w, t.cuda(), dx=True, dw=True)
    rows = ho.target_rows(t.numpy(), 1500)
    ref = ho.head_loss(f64(x), f64(w), rows)
    check(r, ref, f64(x), f64(w), rows, 1.0, BF, BF, coefficients(ref["counts"], None, True, 1.0, 0.0))


def test_no_tokens():
    from paper_2502_16982_b200 import binding as b

    w = torch.randn(300, 64, device="cuda").to(BF)
    dw = torch.full((300, 64), 3.0, dtype=BF, device="cuda")
    r = b.muon_head_xent(torch.empty(0, 64, dtype=BF, device="cuda"), w, torch.empty(0, dtype=torch.int64, device="cuda"),
                         dx=True, dw=dw)
    assert float(r.total[0]) == 0.0 and r.loss.numel() == 0 and r.dx.shape == (0, 64) and not dw.any()


def test_large_logits_stay_finite_and_a_nan_shows():
    from paper_2502_16982_b200 import binding as b

    x, w, gen = make(64, 64, 700, 5, gain=60.0)  # logits up to a few hundred
    t = torch.randint(0, 700, (64,), generator=gen).cuda()
    r = b.muon_head_xent(x, w, t, dx=True, dw=True)
    rows = ho.target_rows(t.cpu().numpy(), 700)
    ref = ho.head_loss(f64(x), f64(w), rows)
    check(r, ref, f64(x), f64(w), rows, 1.0, BF, BF, coefficients(ref["counts"], None, True, 1.0, 0.0))
    x[5, 3] = float("nan")
    r = b.muon_head_xent(x, w, t, dx=True, dw=True)
    ok = torch.arange(64) != 5
    assert torch.isnan(r.loss[5]) and torch.isnan(r.total[0]) and torch.isnan(r.dx[5]).all()
    assert torch.isfinite(r.loss.cpu()[ok]).all() and torch.isfinite(r.dx.cpu()[ok].float()).all()


@pytest.mark.parametrize("dtype", [BF, FP])
def test_gradients_of_micro_batches_add_up(knobs, dtype):
    b = knobs
    b.muon_debug_set_head_codes(1)  # by default the size decides; here both sides form the gradient the same way
    x, w, gen = make(192, 136, 900, 6)
    t = torch.randint(0, 900, (192,), generator=gen).cuda()
    one = b.muon_head_xent(x, w, t, dw=torch.empty(900, 136, dtype=FP, device="cuda"), mean=False, scale=1 / 192)
    acc = torch.full((900, 136), 0.5, dtype=dtype, device="cuda")
    for i in range(0, 192, 64):
        b.muon_head_xent(x[i:i + 64], w, t[i:i + 64], dw=acc, mean=False, scale=1 / 192, accumulate_dw=True)
    err = np.abs(f64(acc) - 0.5 - f64(one.dw))
    rows = ho.target_rows(t.cpu().numpy(), 900)
    ref = ho.head_loss(f64(x), f64(w), rows)
    # both sides round the same gradients of logits; fp32: the order of sums and the 0.5; bf16: three roundings near 0.5
    assert np.all(err <= 64 * 2.0 ** -24 * (0.5 + ref["bound_dw"]) + (3 * 2.0 ** -8 * 0.6 if dtype == BF else 0.0))


def test_results_are_the_same_bits_again_and_on_another_stream():
    from paper_2502_16982_b200 import binding as b

    x, w, gen = make(900, 256, 5000, 8)
    ids = torch.stack([torch.randperm(5000, generator=gen)[:16] for _ in range(900)]).cuda()
    z = torch.randn(900, 16, generator=gen).cuda()
    a = b.muon_head_distill(x, w, ids, z, dx=True, dw=True)
    ws = torch.full((b.muon_head_workspace_bytes(900, 256, 5000, top=16),), 255, dtype=torch.uint8, device="cuda")
    again = b.muon_head_distill(x, w, ids, z, dx=True, dw=True, workspace=ws)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = b.muon_head_distill(x, w, ids, z, dx=True, dw=True, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    for k in ("loss", "lse", "total", "dx", "dw"):
        assert torch.equal(getattr(a, k), getattr(again, k)) and torch.equal(getattr(a, k), getattr(other, k)), k


def test_capture_into_a_graph():
    from paper_2502_16982_b200 import binding as b

    x, w, gen = make(300, 128, 2000, 9)
    t = torch.randint(0, 2000, (300,), generator=gen).cuda()
    eager = b.muon_head_xent(x, w, t, dx=True, dw=True)
    ws = torch.empty(b.muon_head_workspace_bytes(300, 128, 2000), dtype=torch.uint8, device="cuda")
    out = dict(loss=torch.empty(300, device="cuda"), lse=torch.empty(300, device="cuda"), total=torch.empty(1, device="cuda"),
               dx=torch.empty_like(x), dw=torch.empty_like(w))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.muon_head_xent(x, w, t, workspace=ws, **out)
    for v in out.values():
        v.fill_(9.0)
    graph.replay()
    torch.cuda.synchronize()
    for k, v in out.items():
        assert torch.equal(v, getattr(eager, k)), k


def test_margins_are_not_written():
    from paper_2502_16982_b200 import binding as b

    T, D, V = 200, 100, 600
    x, w, gen = make(T, D, V, 11)
    t = torch.randint(0, V, (T,), generator=gen).cuda()
    for dt in (BF, FP):
        dx = torch.full((T + 2, D + 12), 5.0, dtype=dt, device="cuda")
        dw = torch.full((V + 2, D + 12), 5.0, dtype=dt, device="cuda")
        need = b.muon_head_workspace_bytes(T, D, V, packed_head=False)
        ws = torch.full((need + 4096,), 77, dtype=torch.uint8, device="cuda")
        r = b.muon_head_xent(x, w, t, dx=dx[1:-1, 4:-8], dw=dw[1:-1, 4:-8], workspace=ws[:need])
        ref = b.muon_head_xent(x, w, t, dx=torch.empty(T, D, dtype=dt, device="cuda"), dw=torch.empty(V, D, dtype=dt, device="cuda"))
        assert torch.equal(r.dx, ref.dx) and torch.equal(r.dw, ref.dw) and bool((ws[need:] == 77).all())
        for m in (dx, dw):
            m[1:-1, 4:-8] = 5.0
            assert bool((m == 5.0).all())


def test_rows_far_apart():
    """Row strides that put the last rows past 2^31 elements, for w, dw and x, dx."""
    from paper_2502_16982_b200 import binding as b

    T, D, V, ld = 270, 64, 66000, 32768
    x, w, gen = make(T, D, V, 12)
    t = torch.randint(0, V, (T,), generator=gen).cuda()
    t[-1] = V - 1
    near = b.muon_head_xent(x, w, t, dx=True, dw=True)
    far_w, far_dw = (torch.empty(V, ld, dtype=BF, device="cuda")[:, 64:64 + D] for _ in range(2))
    far_w.copy_(w)
    far = b.muon_head_xent(x, far_w, t, dx=True, dw=far_dw)
    for k in ("loss", "lse", "total", "dx", "dw"):
        assert torch.equal(getattr(near, k), getattr(far, k)), k
    del far_w, far_dw, far
    ld = (1 << 31) // (T - 1) // 8 * 8 + 8
    far_x, far_dx = (torch.empty(T, ld, dtype=BF, device="cuda")[:, :D] for _ in range(2))
    far_x.copy_(x)
    far = b.muon_head_xent(far_x, w, t, dx=far_dx, dw=True)
    for k in ("loss", "lse", "total", "dx", "dw"):
        assert torch.equal(getattr(near, k), getattr(far, k)), k


@pytest.mark.parametrize("T", [40, 400])
def test_status_word(T):
    """A status left by an earlier call is reported once and cleared by the next call."""
    from paper_2502_16982_b200 import binding as b

    x, w, gen = make(T, 64, 500, 13)
    t = torch.randint(0, 500, (T,), generator=gen).cuda()
    ws = torch.zeros(b.muon_head_workspace_bytes(T, 64, 500), dtype=torch.uint8, device="cuda")
    at = -ws.data_ptr() % 1024
    ws[at:at + 4].view(torch.int32).fill_(b.MUON_ERR_TIMEOUT)
    assert b.muon_head_status(ws) == b.MUON_ERR_TIMEOUT
    b.muon_head_xent(x, w, t, dx=True, dw=True, workspace=ws)
    assert b.muon_head_status(ws) == 0


def test_refusals_of_the_binding():
    from paper_2502_16982_b200 import binding as b

    x, w, _ = make(4, 16, 50, 1)
    t = torch.zeros(4, dtype=torch.int64, device="cuda")
    ids, z = torch.zeros(4, 3, dtype=torch.int64, device="cuda"), torch.zeros(4, 3, device="cuda")
    bad = [
        lambda: b.muon_head_xent(x.float(), w, t), lambda: b.muon_head_xent(x, w.half(), t),
        lambda: b.muon_head_xent(x, w[:, :8], t), lambda: b.muon_head_xent(x, w, t.int()),
        lambda: b.muon_head_xent(x, w, t[:3]), lambda: b.muon_head_xent(x.t(), w, t),
        lambda: b.muon_head_xent(x.cpu(), w.cpu(), t.cpu()), lambda: b.muon_head_xent(x, w, t, dx=torch.empty_like(w)),
        lambda: b.muon_head_xent(x, w, t, weight=torch.ones(3, device="cuda")),
        lambda: b.muon_head_xent(x, w, t, accumulate_dw=True), lambda: b.muon_head_xent(x, w, t, logit_scale=0.0),
        lambda: b.muon_head_xent(x, w, t, workspace=torch.empty(64, dtype=torch.uint8, device="cuda")),
        lambda: b.muon_head_distill(x, w, ids, z[:, :2]), lambda: b.muon_head_distill(x, w, ids.int(), z),
        lambda: b.muon_head_distill(x, w, ids, z.half()), lambda: b.muon_head_distill(x, w, ids, z, temperature=-1.0),
        lambda: b.muon_head_distill(x, w, ids[:, :0], z[:, :0]),
        lambda: b.muon_head_distill(x, w, ids.repeat(1, 50), z.repeat(1, 50)),
    ]
    for f in bad:
        with pytest.raises(b.MuonError):
            f()
