"""Refusals and workspace sizes of the log probabilities at the head that need no GPU."""

import ctypes as C

import pytest

P = 1 << 20  # an address that no call here reaches


def _args(b, **more):
    a = b.muon_logprob_args(16, 64, 1000, 0, P, P, 64, 64, b.MUON_DTYPE_BF16, b.MUON_DTYPE_BF16, P, 1.0, 0, P, P, P)
    for k, v in more.items():
        setattr(a, k, v)
    return a


def _grads(b, **more):
    d = b.muon_logprob_grads(P, P, P, P, 64, 64, b.MUON_DTYPE_BF16, b.MUON_DTYPE_FP32, 0, 0)
    for k, v in more.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("code,more", [
    ("INVALID_ARG", dict(tokens=-1)), ("INVALID_ARG", dict(dim=0)), ("INVALID_ARG", dict(vocab=0)),
    ("UNSUPPORTED", dict(tokens=(1 << 24) + 1)), ("UNSUPPORTED", dict(vocab=(1 << 24) + 1)), ("UNSUPPORTED", dict(dim=(1 << 20) + 1)),
    ("UNSUPPORTED", dict(x_dtype=1)), ("UNSUPPORTED", dict(w_dtype=1)), ("INVALID_ARG", dict(x=None)), ("INVALID_ARG", dict(w=None)),
    ("INVALID_ARG", dict(logprob=None)), ("INVALID_ARG", dict(targets=None)), ("INVALID_ARG", dict(ld_x=63)),
    ("INVALID_ARG", dict(ld_w=63)), ("INVALID_ARG", dict(logit_scale=0.0)), ("INVALID_ARG", dict(logit_scale=float("nan"))),
    ("INVALID_ARG", dict(logit_scale=3e38)), ("ALIGNMENT", dict(x=P + 1)), ("ALIGNMENT", dict(w=P + 1)),
    ("ALIGNMENT", dict(targets=P + 4)), ("ALIGNMENT", dict(entropy=P + 2)), ("ALIGNMENT", dict(lse=P + 2)), ("ALIGNMENT", dict(logprob=P + 2)),
])
def test_arguments_that_are_refused(code, more):
    from paper_2502_16982_b200 import binding as b

    a, d, want = _args(b, **more), _grads(b), getattr(b, "MUON_ERR_" + code)
    assert b.lib().muon_head_logprob(C.byref(a), None, 0, 0, None) == want
    assert b.lib().muon_head_logprob_grad(C.byref(a), C.byref(d), None, 0, 0, None) == want


@pytest.mark.parametrize("code,args,more", [
    ("INVALID_ARG", dict(lse=None), {}), ("INVALID_ARG", dict(entropy=None), {}), ("INVALID_ARG", {}, dict(dx=None, dw=None)),
    ("INVALID_ARG", {}, dict(ld_dx=63)), ("INVALID_ARG", {}, dict(ld_dw=63)), ("UNSUPPORTED", {}, dict(dx_dtype=2)),
    ("UNSUPPORTED", {}, dict(dw_dtype=2)), ("ALIGNMENT", {}, dict(g_logprob=P + 2)), ("ALIGNMENT", {}, dict(g_entropy=P + 2)),
    ("ALIGNMENT", {}, dict(dx=P + 1)), ("ALIGNMENT", {}, dict(dw=P + 2)),
])
def test_gradients_that_are_refused(code, args, more):
    from paper_2502_16982_b200 import binding as b

    a, d = _args(b, **args), _grads(b, **more)
    assert b.lib().muon_head_logprob_grad(C.byref(a), C.byref(d), None, 0, 0, None) == getattr(b, "MUON_ERR_" + code)


def test_workspace_is_checked_and_holds_no_logits_of_more_than_a_piece():
    from paper_2502_16982_b200 import binding as b

    L = b.lib()
    a, d = _args(b), _grads(b)
    assert L.muon_head_logprob(C.byref(a), None, 0, 0, None) == b.MUON_ERR_WORKSPACE
    assert L.muon_head_logprob(C.byref(a), P, 512, 0, None) == b.MUON_ERR_WORKSPACE
    assert L.muon_head_logprob(C.byref(a), P + 8, 1 << 30, 0, None) == b.MUON_ERR_WORKSPACE
    assert L.muon_head_logprob_grad(C.byref(a), C.byref(d), None, 0, 0, None) == b.MUON_ERR_WORKSPACE
    assert L.muon_head_logprob(None, P, 1 << 30, 0, None) == b.MUON_ERR_INVALID_ARG
    assert L.muon_head_logprob_grad(C.byref(a), None, P, 1 << 30, 0, None) == b.MUON_ERR_INVALID_ARG
    assert L.muon_head_logprob_workspace_bytes(None, None, None) == b.MUON_ERR_INVALID_ARG
    for T in (8, 1024, 8192, 65536):
        rows = T * (2 * 2048 + 64) + (1 << 20)
        stats = T * 640 * 4 * 8
        n = b.muon_head_logprob_workspace_bytes(T, 2048, 163840, grads=False)
        assert stats + stats // 2 <= n <= stats + stats // 2 + rows
        assert b.muon_head_logprob_workspace_bytes(T, 2048, 163840, grads=False, entropy=False) <= stats + rows
        part = T * 2048 * 4
        assert b.muon_head_logprob_workspace_bytes(T, 2048, 163840, grads=True) <= rows + 2 * max(256 << 20, part)


@pytest.mark.parametrize("size", [dict(tokens=1 << 32), dict(dim=(1 << 32) + 64), dict(vocab=(1 << 31) + 1)])
def test_sizes_past_32_bits_are_refused(size):
    import torch
    from paper_2502_16982_b200 import binding as b

    args = dict(dict(tokens=16, dim=64, vocab=1000), **size)
    with pytest.raises(b.MuonError) as e:
        b.muon_head_logprob_workspace_bytes(grads=True, **args)
    assert e.value.code == b.MUON_ERR_UNSUPPORTED
    x, w = (torch.empty(n, args["dim"], dtype=torch.bfloat16, device="meta") for n in (args["tokens"], args["vocab"]))
    with pytest.raises(b.MuonError) as e:
        b.muon_head_logprob(x, w, torch.empty(args["tokens"], dtype=torch.int64, device="meta"))
    assert e.value.code == b.MUON_ERR_UNSUPPORTED
