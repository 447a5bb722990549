"""Limits of the LM-head losses that the host side checks; no GPU."""

import ctypes as C

import pytest
import torch


def _call(b, logit_scale=1.0, temperature=None):
    """Error code of a call that lacks nothing but its workspace."""
    a = b.muon_head_args(16, 64, 1000, 1, 1 << 20, 1 << 20, 64, 64, b.MUON_DTYPE_BF16, b.MUON_DTYPE_BF16, None, 1.0,
                         logit_scale, 1 << 20, None, None, None, None, 64, 64, b.MUON_DTYPE_BF16, b.MUON_DTYPE_BF16)
    if temperature is None:
        return b.lib().muon_head_xent(C.byref(a), 1 << 20, 0.0, None, 0, 0, None)
    t = b.muon_head_teacher(1 << 20, 1 << 20, 8, 8, None, 8, b.MUON_DTYPE_FP32, temperature, 0)
    return b.lib().muon_head_distill(C.byref(a), C.byref(t), None, 0, 0, None)


@pytest.mark.parametrize("logit_scale,temperature", [
    (3e38, None),      # times log2(e): infinite
    (1e-45, 1e30),     # the quotient is 0
    (1e30, 1e-30),     # the quotient is infinite
    (1.0, 1e-40),      # 1 / temperature is infinite
])
def test_a_scale_that_fp32_cannot_hold_is_refused(logit_scale, temperature):
    from paper_2502_16982_b200 import binding as b

    assert _call(b, logit_scale, temperature) == b.MUON_ERR_INVALID_ARG
    assert b"scale" in b.lib().muon_last_error() or b"temperature" in b.lib().muon_last_error()


@pytest.mark.parametrize("logit_scale,temperature", [(1.0, None), (2e38, None), (2e-38, None), (1.0, 1e-6), (1.0, 1e6), (1e20, 1e20), (1e-40, None),
                                                     (1.0, 3e38)])
def test_scales_that_it_can_are_not(logit_scale, temperature):
    from paper_2502_16982_b200 import binding as b

    assert _call(b, logit_scale, temperature) == b.MUON_ERR_WORKSPACE


@pytest.mark.parametrize("size", [dict(tokens=(1 << 32) + 4), dict(dim=(1 << 32) + 64), dict(vocab=(1 << 32) + 100), dict(top=(1 << 32) + 1),
                                  dict(tokens=-(1 << 32) + 4)])
def test_sizes_past_32_bits_are_refused(size):
    """They must not be cut to their low 32 bits on the way into the library."""
    from paper_2502_16982_b200 import binding as b

    args = dict(dict(tokens=16, dim=64, vocab=1000, top=8), **size)
    with pytest.raises(b.MuonError) as e:
        b.muon_head_workspace_bytes(**args)
    assert e.value.code == b.MUON_ERR_UNSUPPORTED
    if "top" not in size and args["tokens"] > 0:
        x, w = (torch.empty(n, args["dim"], dtype=torch.bfloat16, device="meta") for n in (args["tokens"], args["vocab"]))
        with pytest.raises(b.MuonError) as e:
            b.muon_head_xent(x, w, torch.empty(args["tokens"], dtype=torch.int64, device="meta"), dx=True, dw=True)
        assert e.value.code == b.MUON_ERR_UNSUPPORTED


def test_workspace_against_an_array_of_logits():
    """What the header says of both sizes: the recommended one may hold every logit as 16
    bits, the least one a piece of 256 MiB; without gradients no logits at all."""
    from paper_2502_16982_b200 import binding as b

    for T in (1024, 4096, 8192, 65536):
        logits = T * 163840 * 2
        stats, rest = logits // 16, T * (2 * 2048 + 64) + (1 << 20)  # a copy of x, words per token
        part = T * 2048 * 4
        full, least, forward = (b.muon_head_workspace_bytes(T, 2048, 163840, **k)
                                for k in ({}, dict(least=True), dict(dx=False, dw=False)))
        assert least <= stats + rest + max(256 << 20, part) + (256 << 20)
        assert full <= min(logits, 3 << 30) + stats + rest + max(256 << 20, part)
        assert forward <= stats + rest
        assert full >= min(logits, (3 << 30) - (256 << 20) - stats)


@pytest.mark.parametrize("tokens,dim,vocab,top,packed,dx,dw", [
    (8192, 2048, 163840, 0, True, True, True), (333, 203, 5003, 0, False, True, True), (4096, 2048, 163840, 64, True, True, True),
    (1000, 64, 30000, 0, True, True, False), (2000, 1024, 20000, 33, False, False, True), (100, 2048, 163840, 0, False, True, True),
    (300, 2560, 1000, 5, True, True, True), (4096, 2048, 163840, 0, True, False, False), (70000, 64, 5000, 8, True, False, False),
])
def test_least_workspace_is_the_sum_that_the_header_gives(tokens, dim, vocab, top, packed, dx, dw):
    from paper_2502_16982_b200 import binding as b

    def up(v, to):
        return (v + to - 1) // to * to

    entries, tiles, rows = tokens * max(top, 1), up(vocab, 256) // 256, up(dim, 8)
    stats = up(tokens * tiles * 32, 1024)
    least = up(tokens * rows * 2, 1024) + stats + tokens * 16 + entries * 12
    if top:
        least += tokens * (9 + tiles + 1) + entries * 4
    if not packed:
        least += up(vocab * rows * 2, 1024)
    got = b.muon_head_workspace_bytes(tokens, dim, vocab, top=top, dx=dx, dw=dw, packed_head=packed, least=True)
    slack = 16 * 1024 + tokens // 64  # arrays rounded up, the control block, tokens counted in runs
    if not (dx or dw):
        assert least <= got <= least + slack
        return
    # a piece: whole tiles, spread evenly over the pieces, so between half of the most and the most
    most = max((256 << 20) // (tokens * 512), 1)
    pieces = -(-tiles // min(most, tiles))
    least += tokens * 512 * -(-tiles // pieces)
    part = tokens * rows * 4
    upto = max(256 << 20, part) if dx and stats < max(256 << 20, part) else 0
    assert least <= got <= least + slack + upto
    if dx and stats < part:
        assert got >= least + part
