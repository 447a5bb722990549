"""Launches of muon_head_logprob overlap; what comes after the call in the stream does not
overlap with them."""

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("masked", ["all", "all_but_one", "none"])
@pytest.mark.parametrize("T,D,V", [(24, 2048, 163840), (256, 512, 100000), (1, 64, 3000)])
def test_the_workspace_is_free_when_the_call_has_ended(T, D, V, masked):
    from paper_2502_16982_b200 import binding as b

    gen = torch.Generator(device="cuda").manual_seed(61)
    x = torch.randn(T, D, generator=gen, device="cuda").to(torch.bfloat16)
    w = torch.randn(V, D, generator=gen, device="cuda").to(torch.bfloat16)
    y = torch.randint(0, V, (T,), generator=gen, device="cuda")
    if masked != "none":
        y[0 if masked == "all" else 1:] = -100
    ws = torch.empty(b.muon_head_logprob_workspace_bytes(T, D, V, grads=False), dtype=torch.uint8, device="cuda")
    want = b.muon_head_logprob(x, w, y, keep=False)
    torch.cuda.synchronize()
    for i in range(20):
        r = b.muon_head_logprob(x, w, y, keep=False, workspace=ws)
        ws.fill_(i + 1)  # the next user of this memory
        found = (ws == i + 1).all()
        assert bool(found), i
        assert all(torch.equal(p, q) for p, q in zip(r, want))
    if masked == "all":
        assert not any(t.any() for t in want)
