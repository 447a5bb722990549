"""The coefficient on its way to the step, and what the C entries refuse; no GPU."""

import ctypes as C

import torch


def test_null_and_misaligned_coefficients_are_refused():
    from paper_2502_16982_b200 import binding as b

    L, hp = b.lib(), b.Hyper().to_c()
    for coef, want in ((None, b.MUON_ERR_INVALID_ARG), (4098, b.MUON_ERR_ALIGNMENT), (4096, b.MUON_ERR_INVALID_ARG)):  # the last: no context
        assert L.muon_step_clipped(None, C.byref(hp), coef, None) == want
        assert L.muon_step_bucket_clipped(None, C.byref(hp), 0, coef, None) == want


def test_the_owner_computes_step_passes_it_on():
    from paper_2502_16982_b200.distributed import DistributedMuon

    seen = []
    m = DistributedMuon([(8, 12, 2, torch.float32, torch.float32)], "cpu", step_fn=lambda mats, hp, *coef: seen.append(coef))
    coef = torch.ones(1)
    m.step(None)
    m.step(None, coef=coef)
    assert seen == [(), (coef,)]
