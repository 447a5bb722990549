"""Workspaces of a pass that kept its logits, as the gradient's call checks them; no GPU."""

import ctypes as C

import pytest

P = 1 << 30  # an address that no call here reaches
T, D, V = 300, 64, 1000


def _call(b, workspace, kept, kept_bytes=None):
    a = b.muon_logprob_args(T, D, V, 0, 1 << 20, 1 << 20, D, D, b.MUON_DTYPE_BF16, b.MUON_DTYPE_BF16, 1 << 20, 1.0, 0, 1 << 20, 1 << 20, 1 << 20)
    d = b.muon_logprob_grads(1 << 20, 1 << 20, 1 << 20, 1 << 20, D, D, b.MUON_DTYPE_BF16, b.MUON_DTYPE_BF16, 0, 0, kept,
                             (1 << 28) if kept_bytes is None else kept_bytes)
    return b.lib().muon_head_logprob_grad(C.byref(a), C.byref(d), workspace, 1 << 28, 0, None)


def _sizes(b):
    kept = b.muon_head_logprob_workspace_bytes(T, D, V, grads=False, entropy=False, keep=True) - 1024
    own = b.muon_head_logprob_workspace_bytes(T, D, V, grads=True, keep=True) - 1024
    return kept, own


def test_a_workspace_that_overlaps_what_was_kept_is_refused():
    from paper_2502_16982_b200 import binding as b

    kept, own = _sizes(b)
    assert kept % 1024 == 0 and own % 1024 == 0
    for workspace in (P, P + 1024, P + kept - 1024, P - own + 1024):
        assert _call(b, workspace, P) == b.MUON_ERR_WORKSPACE
        assert b.muon_last_error() == "workspace and kept overlap"


def test_what_was_kept_is_whole_and_aligned():
    from paper_2502_16982_b200 import binding as b

    kept, own = _sizes(b)
    assert _call(b, P + (1 << 29), P, kept - 1) == b.MUON_ERR_WORKSPACE
    assert _call(b, P + (1 << 29), P + 512) == b.MUON_ERR_WORKSPACE
    assert _call(b, P + (1 << 29), P, 0) == b.MUON_ERR_WORKSPACE
