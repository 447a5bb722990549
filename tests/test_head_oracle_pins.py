"""Pins of the LM-head loss oracle: values worked out by hand, closed forms and
differences, none of which calls the oracle for its expectation; and what the
library refuses or plans on the host, without a GPU."""

import math

import numpy as np
import pytest

from oracle import head_oracle as ho


def test_two_entries_by_hand():
    # one token, x = 1, w = (ln 3, 0): q = (3/4, 1/4); target 1: loss = ln 4, dl = (3/4, -3/4)
    x, w = np.array([[1.0]]), np.array([[math.log(3.0)], [0.0]])
    r = ho.head_loss(x, w, ho.target_rows([1], 2))
    assert abs(r["loss"][0] - math.log(4.0)) < 1e-15 and abs(r["lse"][0] - math.log(4.0)) < 1e-15
    assert np.allclose(r["g"], [[0.75, -0.75]], atol=1e-15)
    assert np.allclose(r["dx"], [[0.75 * math.log(3.0)]], atol=1e-15)
    assert np.allclose(r["dw"], [[0.75], [-0.75]], atol=1e-15)


def test_equal_logits_give_log_vocab():
    x, w = np.ones((3, 4)), np.full((7, 4), 0.3)
    r = ho.head_loss(x, w, ho.target_rows([0, 6, -100], 7), z_loss=0.5)
    lse = math.log(7.0) + 1.2
    assert np.allclose(r["loss"][:2], math.log(7.0) + 0.5 * lse * lse, atol=1e-13) and r["loss"][2] == 0.0
    assert np.allclose(r["lse"], [lse, lse, 0.0], atol=1e-13)


def test_distillation_from_itself_is_zero_and_has_no_gradient():
    rng = np.random.default_rng(3)
    x, w = rng.standard_normal((4, 5)), rng.standard_normal((6, 5))
    ids = np.tile(np.arange(6), (4, 1))
    r = ho.head_loss(x, w, ho.teacher_rows(ids, x @ w.T, 6, 2.0), temperature=2.0)
    assert np.abs(r["loss"]).max() < 1e-14 and np.abs(r["g"]).max() < 1e-15


def test_one_entry_is_cross_entropy_and_a_twice_listed_entry_is_one():
    rng = np.random.default_rng(4)
    x, w = rng.standard_normal((5, 3)), rng.standard_normal((9, 3))
    t = np.array([0, 8, 3, -1, 9])
    a = ho.head_loss(x, w, ho.target_rows(t, 9))
    b = ho.head_loss(x, w, ho.teacher_rows(t[:, None], np.full((5, 1), -7.5), 9, 1.0))
    c = ho.head_loss(x, w, ho.teacher_rows(np.stack([t, t], 1), np.zeros((5, 2)), 9, 1.0))
    for k in ("lse", "dx", "dw"):
        assert np.allclose(a[k], b[k], atol=1e-14) and np.allclose(a[k], c[k], atol=1e-14)
    assert np.allclose(a["loss"], b["loss"], atol=1e-14)
    assert np.allclose(c["loss"], a["loss"] - math.log(2.0) * (a["loss"] != 0), atol=1e-14)  # its own entropy


@pytest.mark.parametrize("kind", ["xent", "distill", "tail"])
def test_gradients_are_the_differences(kind):
    rng = np.random.default_rng(5)
    T, D, V, K = 4, 3, 8, 3
    x, w = rng.standard_normal((T, D)), rng.standard_normal((V, D))
    weight = rng.random(T) + 0.5
    kw = dict(weight=weight, scale=1.7, logit_scale=0.6)
    if kind == "xent":
        rows = ho.target_rows([1, -100, 7, 2], V)
        kw["z_loss"] = 0.03
    else:
        ids = np.stack([rng.permutation(V)[:K] for _ in range(T)])
        ids[2] = [5, -1, 99]
        z = rng.standard_normal((T, K))
        lse = np.logaddexp.reduce(z / 1.5, axis=1) + 0.2 if kind == "tail" else None
        rows = ho.teacher_rows(ids, z, V, 1.5, lse)
        kw["temperature"] = 1.5
    r = ho.head_loss(x, w, rows, **kw)
    e = 1e-5
    for name, at in (("dx", x), ("dw", w)):
        num = np.zeros_like(at)
        for i in np.ndindex(at.shape):
            keep = at[i]
            at[i] = keep + e
            up = ho.head_loss(x, w, rows, grads=False, **kw)["total"]
            at[i] = keep - e
            num[i] = (up - ho.head_loss(x, w, rows, grads=False, **kw)["total"]) / (2 * e)
            at[i] = keep
        # central differences: e^2 times a third derivative of a few units, and 1e-16 / e of rounding
        assert np.abs(num - r[name]).max() < 2e-9, name


def test_masked_tokens_reach_nothing():
    rng = np.random.default_rng(6)
    x, w = rng.standard_normal((3, 4)), rng.standard_normal((5, 4))
    x[1] = np.nan
    r = ho.head_loss(x, w, ho.target_rows([2, -100, 0], 5))
    s = ho.head_loss(x[[0, 2]], w, ho.target_rows([2, 0], 5))
    assert r["total"] == s["total"] and np.array_equal(r["dw"], s["dw"]) and np.array_equal(r["dx"][[0, 2]], s["dx"])
    none = ho.head_loss(x, w, ho.target_rows([-1, -1, 5], 5))
    assert none["total"] == 0.0 and not none["dx"].any() and not none["dw"].any()


def _args(b, **kw):
    a = b.muon_head_args(16, 64, 1000, 1, 1 << 20, 1 << 20, 64, 64, b.MUON_DTYPE_BF16, b.MUON_DTYPE_BF16, None, 1.0, 1.0,
                         1 << 20, 1 << 20, 1 << 20, 1 << 20, 1 << 20, 64, 64)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("change,code", [
    (dict(dim=0), "INVALID_ARG"), (dict(vocab=-1), "INVALID_ARG"), (dict(tokens=-1), "INVALID_ARG"),
    (dict(x=None), "INVALID_ARG"), (dict(w=None), "INVALID_ARG"), (dict(loss=None), "INVALID_ARG"),
    (dict(ld_x=63), "INVALID_ARG"), (dict(ld_w=63), "INVALID_ARG"), (dict(ld_dx=1), "INVALID_ARG"),
    (dict(ld_dw=1), "INVALID_ARG"), (dict(scale=math.inf), "INVALID_ARG"), (dict(logit_scale=0.0), "INVALID_ARG"),
    (dict(logit_scale=-1.0), "INVALID_ARG"), (dict(logit_scale=math.nan), "INVALID_ARG"),
    (dict(x_dtype=1), "UNSUPPORTED"), (dict(w_dtype=1), "UNSUPPORTED"), (dict(dx_dtype=2), "UNSUPPORTED"),
    (dict(dw_dtype=-1), "UNSUPPORTED"), (dict(vocab=(1 << 24) + 1), "UNSUPPORTED"),
    (dict(x=(1 << 20) + 1), "ALIGNMENT"), (dict(loss=(1 << 20) + 2), "ALIGNMENT"),
    (dict(dw=(1 << 20) + 2, dw_dtype=1), "ALIGNMENT"), (dict(), "WORKSPACE"),
])
def test_refusals_of_both_losses(change, code):
    """Refused before anything is launched (the addresses are never read)."""
    import ctypes as C

    from paper_2502_16982_b200 import binding as b

    L, a = b.lib(), _args(b, **change)
    t = b.muon_head_teacher(1 << 20, 1 << 20, 8, 8, None, 8, b.MUON_DTYPE_FP32, 1.0, 0)
    want = getattr(b, "MUON_ERR_" + code)
    assert L.muon_head_xent(C.byref(a), 1 << 20, 0.0, None, 0, 0, None) == want
    assert b.muon_last_error()
    assert L.muon_head_distill(C.byref(a), C.byref(t), None, 0, 0, None) == want


def test_refusals_of_targets_and_teachers():
    import ctypes as C

    from paper_2502_16982_b200 import binding as b

    L, a = b.lib(), _args(b)
    assert L.muon_head_xent(C.byref(a), None, 0.0, None, 0, 0, None) == b.MUON_ERR_INVALID_ARG
    assert L.muon_head_xent(C.byref(a), (1 << 20) + 4, 0.0, None, 0, 0, None) == b.MUON_ERR_ALIGNMENT
    assert L.muon_head_xent(C.byref(a), 1 << 20, math.nan, None, 0, 0, None) == b.MUON_ERR_INVALID_ARG
    assert L.muon_head_xent(None, 1 << 20, 0.0, None, 0, 0, None) == b.MUON_ERR_INVALID_ARG
    assert L.muon_head_distill(C.byref(a), None, None, 0, 0, None) == b.MUON_ERR_INVALID_ARG

    def distill(**kw):
        t = b.muon_head_teacher(1 << 20, 1 << 20, 8, 8, None, 8, b.MUON_DTYPE_FP32, 1.0, 0)
        for k, v in kw.items():
            setattr(t, k, v)
        return L.muon_head_distill(C.byref(a), C.byref(t), None, 0, 0, None)

    assert distill(top=0) == b.MUON_ERR_UNSUPPORTED and distill(top=129) == b.MUON_ERR_UNSUPPORTED
    assert distill(top_ids=None) == b.MUON_ERR_INVALID_ARG and distill(top_logits=None) == b.MUON_ERR_INVALID_ARG
    assert distill(ld_ids=7) == b.MUON_ERR_INVALID_ARG and distill(ld_logits=7) == b.MUON_ERR_INVALID_ARG
    assert distill(temperature=0.0) == b.MUON_ERR_INVALID_ARG and distill(temperature=math.inf) == b.MUON_ERR_INVALID_ARG
    assert distill(logits_dtype=5) == b.MUON_ERR_UNSUPPORTED
    assert distill(top_ids=(1 << 20) + 1) == b.MUON_ERR_ALIGNMENT


def test_workspace_stays_bounded_on_the_host():
    """The workspace must not grow with tokens x vocab: the gradient of the logits is
    kept for one piece of the vocabulary only."""
    from paper_2502_16982_b200 import binding as b

    full = b.muon_head_workspace_bytes(65536, 2048, 163840)
    least = b.muon_head_workspace_bytes(65536, 2048, 163840, least=True)
    logits = 65536 * 163840 * 2
    assert least < full < logits / 4 and least < logits / 10
    # without gradients: a copy of x, one byte of statistics for eight logits, a few words a token
    assert b.muon_head_workspace_bytes(8192, 2048, 163840, dx=False, dw=False) < 8192 * (2 * 2048 + 163840 // 8) + (1 << 20)
    assert b.muon_head_workspace_bytes(0, 64, 1000) > 0
    with pytest.raises(b.MuonError):
        b.muon_head_workspace_bytes(16, 64, 1000, top=129)
