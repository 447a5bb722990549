"""The example's stage on its own samples: it runs, clipped, and the gradients are right."""

import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


def test_policy_stage_runs_and_its_gradients_are_those_of_the_objective():
    """Clipped steps on the model's own samples; the head's gradient against differences of the
    objective in fp64."""
    import torch

    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_and_distill.py")
    spec = importlib.util.spec_from_file_location("train_and_distill", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    r = example.main(["--steps", "3", "--dim", "64", "--vocab", "300", "--rows", "8", "--clip", "0.5", "--policy-steps", "3"])
    assert len(r["reward"]) == 3 and all(0.0 <= v <= 1.0 for v in r["reward"])
    mb = example.mb
    gen = torch.Generator().manual_seed(1)
    x, w = torch.randn(50, 64, generator=gen).bfloat16().cuda(), (torch.randn(300, 64, generator=gen) * 0.2).bfloat16().cuda()
    y = torch.randint(0, 300, (50,), generator=gen).cuda()
    g, h = torch.randn(50, generator=gen).cuda() / 50, torch.full((50,), -0.01 / 50, device="cuda")
    out = mb.muon_head_logprob(x, w, y)
    d = mb.muon_head_logprob_grad(x, w, y, out, g_logprob=g, g_entropy=h, dw=torch.empty(300, 64, device="cuda"))
    w64 = w.double().requires_grad_()
    l = x.double() @ w64.t()
    l.retain_grad()
    lq = torch.log_softmax(l, dim=1)
    (g.double() * lq.gather(1, y[:, None])[:, 0] - h.double() * (lq.exp() * lq).sum(1)).sum().backward()
    # every gradient of a logit is rounded to bf16 once, 2^-8; twice that covers the rest
    bound = 2.0 ** -7 * (l.grad.abs().t() @ x.double().abs())
    assert bool(((d.dw.double() - w64.grad).abs() <= bound).all())
