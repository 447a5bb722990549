"""Refusals of the log probabilities over stored logits that the host side checks; no GPU."""

import ctypes as C

import pytest

P = 1 << 20  # an address that no call here reaches


def _args(b, **more):
    a = b.muon_logits_args(4, 100, P, 100, b.MUON_DTYPE_BF16, 8, 1.0, 0, P, P, P, P, P, P, P)
    for k, v in more.items():
        setattr(a, k, v)
    return a


BAD = [
    ("INVALID_ARG", dict(tokens=-1)), ("INVALID_ARG", dict(vocab=0)), ("INVALID_ARG", dict(vocab=-5)),
    ("UNSUPPORTED", dict(tokens=(1 << 24) + 1)), ("UNSUPPORTED", dict(vocab=(1 << 24) + 1, ld=1 << 25)),
    ("UNSUPPORTED", dict(dtype=2)), ("UNSUPPORTED", dict(top=129)), ("UNSUPPORTED", dict(top=-1)), ("INVALID_ARG", dict(top=101)),
    ("INVALID_ARG", dict(logit_scale=0.0)), ("INVALID_ARG", dict(logit_scale=-1.0)), ("INVALID_ARG", dict(logit_scale=float("inf"))),
    ("INVALID_ARG", dict(logit_scale=float("nan"))), ("INVALID_ARG", dict(logit_scale=3e38)),  # times log2(e)
    ("INVALID_ARG", dict(logits=None)), ("INVALID_ARG", dict(ld=99)), ("ALIGNMENT", dict(logits=P + 1)),
    ("ALIGNMENT", dict(dtype=1, logits=P + 2)), ("ALIGNMENT", dict(targets=P + 4)), ("ALIGNMENT", dict(lse=P + 2)),
    ("ALIGNMENT", dict(top_ids=P + 4)), ("ALIGNMENT", dict(top_logprob=P + 1)),
]


@pytest.mark.parametrize("code,more", BAD)
def test_arguments_that_are_refused(code, more):
    from paper_2502_16982_b200 import binding as b

    a = _args(b, **more)
    assert b.lib().muon_logits_logprob(C.byref(a), 0, None) == getattr(b, "MUON_ERR_" + code)
    assert b.lib().muon_logits_logprob_grad(C.byref(a), P, P, 2 * P, 1 << 25, 0, None) == getattr(b, "MUON_ERR_" + code)


def test_what_only_one_of_them_refuses():
    from paper_2502_16982_b200 import binding as b

    L = b.lib()
    bad = b.MUON_ERR_INVALID_ARG
    assert L.muon_logits_logprob(None, 0, None) == bad
    assert L.muon_logits_logprob(C.byref(_args(b, targets=None)), 0, None) == bad  # logprob without targets
    nothing = _args(b, logprob=None, entropy=None, lse=None, top_ids=None, top_logits=None, top_logprob=None)
    assert L.muon_logits_logprob(C.byref(nothing), 0, None) == bad
    grad = lambda a, r=P, h=P, d=2 * P, ld=100: L.muon_logits_logprob_grad(C.byref(a), r, h, d, ld, 0, None)
    assert grad(_args(b, lse=None)) == bad
    assert grad(_args(b, entropy=None)) == bad
    assert grad(_args(b, targets=None)) == bad
    assert grad(_args(b), d=None) == bad
    assert grad(_args(b), ld=99) == bad
    assert grad(_args(b, ld=120), d=P) == bad  # in place with another stride
    assert grad(_args(b), r=P + 2) == b.MUON_ERR_ALIGNMENT
    assert grad(_args(b), h=P + 2) == b.MUON_ERR_ALIGNMENT
    assert grad(_args(b), d=2 * P + 1) == b.MUON_ERR_ALIGNMENT
    # no tokens: nothing to do
    assert L.muon_logits_logprob(C.byref(_args(b, tokens=0, logits=None)), 0, None) == b.MUON_OK
    assert grad(_args(b, tokens=0, logits=None)) == b.MUON_OK


@pytest.mark.parametrize("size", [dict(shape=((1 << 31) + 4, 10)), dict(shape=(4, (1 << 31) + 10)), dict(top=1 << 32)])
def test_sizes_past_32_bits_are_refused(size):
    import torch
    from paper_2502_16982_b200 import binding as b

    class Fake:  # stands for a tensor on a device: only shapes are looked at before the refusal
        device = torch.device("cuda", 0)

        def __init__(self, shape):
            self.shape = shape

        def dim(self):
            return 2

        def stride(self, i):
            return (self.shape[1], 1)[i]

    with pytest.raises(b.MuonError) as e:
        b.muon_logits_logprob(Fake(size.get("shape", (4, 10))), top=size.get("top", 0))
    assert e.value.code == b.MUON_ERR_UNSUPPORTED


def test_structs_as_bytes_are_the_structs():
    from paper_2502_16982_b200 import binding as b

    v = (1, 2, 3, 4, 5, 6, 0.5, 8, 9, 10, 11, 12, 13, 14, 15)
    assert bytes(b.muon_logits_args(*v)) == b._pack_logits_args(*v)
    v = (1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 0.5, 13, 14, 15, 16)
    assert bytes(b.muon_logprob_args(*v)) == b._pack_logprob_args(*v)
