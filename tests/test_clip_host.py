"""Refusals of the gradient norm and clipping that the host side checks; no GPU."""

import ctypes as C

import pytest

P = 1 << 20  # an address that no call here reaches


def _tensor(b, **more):
    t = dict(g=P, out=None, numel=100, g_dtype=b.MUON_DTYPE_FP32, out_dtype=b.MUON_DTYPE_FP32)
    t.update(more)
    return b.muon_grad_tensor(t["g"], t["out"], t["numel"], t["g_dtype"], t["out_dtype"])


def _norm(b, tensors, n=None, max_norm=1.0, eps=1e-6, sum_sq=P, norm=P, coef=P, workspace=P, nbytes=16384):
    arr = (b.muon_grad_tensor * max(1, len(tensors)))(*tensors)
    return b.lib().muon_grad_norm(arr, len(tensors) if n is None else n, max_norm, eps, sum_sq, norm, coef, workspace, nbytes, 0, None)


def _clip(b, tensors, n=None, max_norm=1.0, eps=1e-6, sum_sq=P, norm=P, coef=P):
    arr = (b.muon_grad_tensor * max(1, len(tensors)))(*tensors)
    return b.lib().muon_clip_grads(arr, len(tensors) if n is None else n, sum_sq, max_norm, eps, norm, coef, 0, None)


@pytest.mark.parametrize("code,more", [
    ("INVALID_ARG", dict(g=None)), ("INVALID_ARG", dict(numel=-1)), ("UNSUPPORTED", dict(numel=1 << 42)),
    ("UNSUPPORTED", dict(g_dtype=2)), ("ALIGNMENT", dict(g=P + 2)), ("ALIGNMENT", dict(g=P + 1, g_dtype=0, out_dtype=0)),
])
def test_tensors_that_are_refused(code, more):
    from paper_2502_16982_b200 import binding as b

    for call in (_norm, _clip):
        assert call(b, [_tensor(b), _tensor(b, **more)]) == getattr(b, "MUON_ERR_" + code)


@pytest.mark.parametrize("code,more", [
    ("UNSUPPORTED", dict(out=P * 2, out_dtype=7)), ("ALIGNMENT", dict(out=P * 2 + 2)),
    ("INVALID_ARG", dict(out=P, out_dtype=0)),
])
def test_outputs_that_are_refused(code, more):
    from paper_2502_16982_b200 import binding as b

    assert _clip(b, [_tensor(b, **more)]) == getattr(b, "MUON_ERR_" + code)


@pytest.mark.parametrize("more", [dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(eps=-1.0), dict(eps=float("nan")),
                                  dict(eps=float("inf")), dict(n=-1)])
def test_limits_that_are_refused(more):
    from paper_2502_16982_b200 import binding as b

    for call in (_norm, _clip):
        assert call(b, [_tensor(b)], **more) == b.MUON_ERR_INVALID_ARG


def test_other_refusals():
    from paper_2502_16982_b200 import binding as b

    assert _norm(b, [_tensor(b)], sum_sq=None, norm=None, coef=None) == b.MUON_ERR_INVALID_ARG
    assert _norm(b, [_tensor(b)], sum_sq=P + 4) == b.MUON_ERR_ALIGNMENT
    assert _norm(b, [_tensor(b)], norm=P + 2) == b.MUON_ERR_ALIGNMENT
    assert _norm(b, [_tensor(b)], workspace=None) == b.MUON_ERR_WORKSPACE
    assert _norm(b, [_tensor(b)], nbytes=b.MUON_GRAD_NORM_WORKSPACE_BYTES - 1) == b.MUON_ERR_WORKSPACE
    assert _norm(b, [_tensor(b)], workspace=P + 4) == b.MUON_ERR_WORKSPACE
    assert _clip(b, [_tensor(b)], sum_sq=None) == b.MUON_ERR_INVALID_ARG
    hp = b.muon_adamw_hparams(1e-3, 0.0, 0.9, 0.95, 1e-8, 1)
    t = (b.muon_adamw_tensor * 1)(b.muon_adamw_tensor(P, P, P, P, 4, 1, 1))
    assert b.lib().muon_adamw_step_clipped(t, 1, C.byref(hp), None, 0, None) == b.MUON_ERR_INVALID_ARG
    assert b.lib().muon_adamw_step_clipped(t, 1, C.byref(hp), P + 2, 0, None) == b.MUON_ERR_ALIGNMENT


def test_adamw_lists(monkeypatch):
    """Any iterables, of which the parameters' number counts; shorter ones are refused."""
    torch = pytest.importorskip("torch")
    from paper_2502_16982_b200 import binding as b

    seen = []

    class Lib:
        @staticmethod
        def muon_adamw_step(arr, n, hp, dev, stream):
            seen.append(list((C.c_int64 * (6 * n)).from_address(arr)))
            return 0

    monkeypatch.setattr(b, "lib", lambda: Lib)
    monkeypatch.setattr(b, "_raw_stream", lambda stream, dev: None)
    p, m, v = ([torch.zeros(k + 1) for k in range(3)] for _ in range(3))
    g = [torch.zeros(k + 1, dtype=torch.bfloat16 if k else torch.float32) for k in range(4)]
    b.muon_adamw_step(p, iter(g), tuple(m), (x for x in v), 1, 1e-3, 0.0)
    words = [w for k in range(3) for w in (p[k].data_ptr(), g[k].data_ptr(), m[k].data_ptr(), v[k].data_ptr(), k + 1,
                                           b.MUON_DTYPE_FP32 | (b.MUON_DTYPE_BF16 if k else b.MUON_DTYPE_FP32) << 32)]
    assert seen == [words]
    for bad in ((p, g, m[:2], v), ([], [], [], []), (p, g[:2], m, v), (p, g, v[::-1], m), (p, g, [x.half() for x in m], v),
                ([x.half() for x in p], g, m, v)):
        with pytest.raises(b.MuonError):
            b.muon_adamw_step(*bad, 1, 1e-3, 0.0)
    assert len(seen) == 1
