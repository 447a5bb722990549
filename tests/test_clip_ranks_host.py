"""Clipping over data-parallel ranks (DistributedMuon.clip_grads) on CPU ranks (gloo), with
plain stand-ins for the library calls: every rank scales its own matrices by the
coefficient of all, a rank without matrices takes part, and others' squares count once."""

import math
import os
import socket
import sys

import pytest
import torch
import torch.distributed as dist
import torch.multiprocessing as mp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def _free_port():
    s = socket.socket()
    s.bind(("127.0.0.1", 0))
    port = s.getsockname()[1]
    s.close()
    return port


def _clip(grads, max_norm, eps, sum_sq):
    if sum_sq is None:
        return sum((g.double() ** 2).sum() for g in grads).reshape(1) if grads else torch.zeros(1, dtype=torch.float64)
    norm = sum_sq.sqrt()
    coef = (max_norm / (norm + eps)).clamp(max=1.0).float()
    for g in grads:
        g.mul_(coef)
    return norm, coef


def _worker(rank, world, port, out, count):
    os.environ["MASTER_ADDR"] = "127.0.0.1"
    os.environ["MASTER_PORT"] = str(port)
    dist.init_process_group("gloo", rank=rank, world_size=world)
    from paper_2502_16982_b200.distributed import DistributedMuon

    m = DistributedMuon([(8, 12, count, torch.float32, torch.float32)], "cpu", dist, step_fn=lambda mats, hp: None, clip_fn=_clip)
    gen = torch.Generator().manual_seed(5 + rank)
    mine = [torch.randn(8, 12, generator=gen) for _ in range(count)]
    for g, v in zip(m.grads[0], mine):
        g.copy_(v)
    norm, coef = m.clip_grads(2.0, others=torch.tensor([9.0 + rank], dtype=torch.float64), reduce_grads=True)
    owned = {i: m.grads[0][i].clone() for i in m.owned}
    torch.save({"mine": mine, "owned": owned, "norm": float(norm), "coef": float(coef)}, "%s.%d" % (out, rank))
    dist.barrier()
    dist.destroy_process_group()


@pytest.mark.timeout(600)
@pytest.mark.parametrize("count", [5, 1])  # one matrix: the other rank owns nothing
def test_two_cpu_ranks_clip_by_the_norm_of_all(tmp_path, count):
    out = str(tmp_path / "r")
    mp.spawn(_worker, args=(2, _free_port(), out, count), nprocs=2, join=True)
    r = [torch.load("%s.%d" % (out, k)) for k in range(2)]
    total = [a + b for a, b in zip(r[0]["mine"], r[1]["mine"])]
    want = math.sqrt(float(sum((g.double() ** 2).sum() for g in total)) + 9.0 + 10.0)
    coef = 2.0 / (want + 1e-6)
    seen = {}
    for k in r:
        assert abs(k["norm"] - want) <= 1e-6 * want and abs(k["coef"] - coef) <= 1e-6 * coef
        seen.update(k["owned"])
    assert sorted(seen) == list(range(count))
    for i, g in seen.items():
        assert torch.allclose(g, total[i] * coef, rtol=1e-5, atol=1e-7)
