"""Workloads of the losses at the LM head: softmax cross entropy over a large
vocabulary and distillation from a teacher's top logits, each alone (evaluation)
and with the gradients of the hidden states and of the head (training).

``own = False`` computes them in elementary torch operations in 32 bits; ``own =
True`` makes the calls a training program makes of this package.
"""

import math

import torch

own = False

# Sizes: hidden 2048 and vocabulary 163840 are the embedding / LM head of the
# package's largest parameter set, hidden 1536 - 2560 its dense models; the other
# vocabularies are of usual and of odd sizes.


def listed():
    def xent(name, tokens, dim, vocab, **more):
        return dict(dict(name=name, op="xent", tokens=tokens, dim=dim, vocab=vocab, grads=True, masked=0.0,
                         weights=False, z_loss=0.0), **more)

    def distill(name, tokens, dim, vocab, top, **more):
        return dict(dict(name=name, op="distill", tokens=tokens, dim=dim, vocab=vocab, top=top, grads=True, masked=0.0,
                         temperature=1.0, tail=False), **more)

    return [
        # one training micro-batch of the largest set: two sequences of 4096 tokens
        xent("xent_train_8192", 8192, 2048, 163840),
        # fine-tuning: more than half of the tokens are prompt and carry no loss; per-token weights
        xent("xent_masked_prompts", 6000, 2048, 163840, masked=0.6, weights=True),
        # a dense model with a mid-sized vocabulary of odd size and the z-loss term
        xent("xent_odd_vocab_zloss", 4097, 1536, 50021, masked=0.05, z_loss=1e-4),
        # evaluation (perplexity): no gradients
        xent("xent_eval", 4096, 2048, 163840, grads=False),
        # a short ragged batch on the full vocabulary: the head's traffic counts, not the products
        xent("xent_short_batch", 100, 2048, 163840, masked=0.1),
        # one token of a small model: latency
        xent("xent_one_token", 1, 512, 8192),
        # a small experiment: odd row length, so that no row but the first is aligned
        xent("xent_small_odd_rows", 333, 203, 5003, masked=0.2, weights=True),
        # distillation step from 64 stored teacher logits a token
        distill("distill_train_4096", 4096, 2048, 163840, 64, masked=0.1),
        # temperature 2, odd sizes, 20 entries a token, some rows without a teacher
        distill("distill_odd_t2", 1777, 1792, 32003, 20, masked=0.3, temperature=2.0),
        # the teacher's full normaliser is known, 8 entries a token
        distill("distill_tail_mass", 1024, 2560, 65536, 8, tail=True),
        # evaluation of a student
        distill("distill_eval", 2000, 2048, 100000, 32, grads=False),
        # a few tokens of a small model: latency
        distill("distill_few_tokens", 24, 256, 4096, 16),
    ]


#: T * D * V of the largest listed case
_MOST = 8192 * 2048 * 163840


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        tokens, vocab = spread(1, 8192), spread(1000, 163840)
        dim = rng.choice([64, 128, 256, 512, 1000, 1024, 1408, 1536, 1792, 2048, 2304, 2560, rng.randint(64, 2560)])
        if tokens * dim * vocab <= _MOST:
            break
    grads, masked = rng.random() < 0.75, rng.choice([0.0, 0.0, 0.1, 0.5])
    if rng.random() < 0.5:
        return dict(op="xent", tokens=tokens, dim=dim, vocab=vocab, grads=grads, masked=masked,
                    weights=rng.random() < 0.3, z_loss=rng.choice([0.0, 0.0, 1e-4]))
    return dict(op="distill", tokens=tokens, dim=dim, vocab=vocab, top=rng.choice([1, 5, 8, 16, 20, 32, 50, 64, 100, 128]),
                grads=grads, masked=masked, temperature=rng.choice([1.0, 1.0, 2.0]), tail=rng.random() < 0.3)


def prepare(case, seed):
    """Hidden states, the head and the targets of one call.  The hidden states lean
    towards their targets' rows of the head, as after some training: the losses are
    a few nats and part of the tokens are predicted with confidence."""
    T, D, V = case["tokens"], case["dim"], case["vocab"]
    gen = torch.Generator(device="cuda").manual_seed(int(seed))

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def rand(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    w = (randn(V, D) * 0.02).to(torch.bfloat16)
    noise = randn(T, D)
    # frequent tokens have low ids
    first = (rand(T).double().square() * V).long().clamp_(max=V - 1)
    # push[t]: by how much the target's logit is lifted over the others
    push = math.log(V) * (0.2 + 1.2 * rand(T))
    norm2 = 0.02 * 0.02 * D
    masked = rand(T) < case["masked"]
    s = {"case": case, "w": w}
    if case["op"] == "xent":
        s["x"] = (noise + (push / norm2)[:, None] * w[first].float()).to(torch.bfloat16)
        s["targets"] = torch.where(masked, torch.full_like(first, -100), first)
        s["weight"] = rand(T) + 0.5 if case["weights"] else None
    else:
        K = case["top"]
        # K different entries a token: the first one and others at an odd stride from it
        step = 1 + (rand(T) * (V // K - 1)).long()
        ids = (first[:, None] + step[:, None] * torch.arange(K, device="cuda")) % V
        # the teacher's logits fall with the rank
        z = math.log(V) * 1.2 - 1.1 * torch.log1p(torch.arange(K, device="cuda", dtype=torch.float32)) + 0.3 * randn(T, K)
        z = z.sort(dim=1, descending=True).values
        lift = torch.softmax(z, dim=1)
        lean = torch.zeros(T, D, device="cuda")
        for k in range(min(K, 4)):  # the student leans towards the teacher's first entries
            lean += lift[:, k : k + 1] * w[ids[:, k]].float()
        s["x"] = (noise + (push / norm2)[:, None] * lean).to(torch.bfloat16)
        s["top_ids"] = torch.where(masked[:, None], torch.full_like(ids, -1), ids)
        s["top_logits"] = z
        # a full normaliser of the teacher that leaves 2 - 20 % for the entries that were not kept
        kept = torch.logsumexp(z / case["temperature"], dim=1)
        s["teacher_lse"] = kept - torch.log1p(-(0.02 + 0.18 * rand(T))) if case["tail"] else None
    return s


def run(s):
    c = s["case"]
    if own:
        from paper_2502_16982_b200 import binding

        want = True if c["grads"] else None
        if c["op"] == "xent":
            r = binding.muon_head_xent(s["x"], s["w"], s["targets"], weight=s["weight"], z_loss=c["z_loss"], dx=want,
                                       dw=want)
        else:
            r = binding.muon_head_distill(s["x"], s["w"], s["top_ids"], s["top_logits"], temperature=c["temperature"],
                                          teacher_lse=s["teacher_lse"], dx=want, dw=want)
        return {"loss": r.loss, "lse": r.lse, "total": r.total, "dx": r.dx, "dw": r.dw}
    return _plain_xent(s, c) if c["op"] == "xent" else _plain_distill(s, c)


def _softmax_of(x, w, valid, inv_t):
    """Logits of the tokens that count, exponentials, their sums and logarithms of the sums."""
    x = torch.where(valid[:, None], x.float(), 0.0)
    logits = x @ w.t()
    if inv_t != 1.0:
        logits = logits * inv_t
    top = logits.amax(dim=1, keepdim=True)
    e = torch.exp(logits - top)
    total = e.sum(dim=1, keepdim=True)
    return x, logits, e, total, (top + torch.log(total))[:, 0]


def _outputs(x, w, dlogits, loss, lse, coef, valid):
    loss, lse = torch.where(valid, loss, 0.0), torch.where(valid, lse, 0.0)
    out = {"loss": loss, "lse": lse, "total": (coef * loss).sum().reshape(1), "dx": None, "dw": None}
    if dlogits is not None:
        out["dx"] = (dlogits @ w).to(torch.bfloat16)
        out["dw"] = (dlogits.t() @ x).to(torch.bfloat16)
    return out


def _plain_xent(s, c):
    valid = (s["targets"] >= 0) & (s["targets"] < c["vocab"])
    target = torch.where(valid, s["targets"], 0)[:, None]
    w = s["w"].float()
    x, logits, e, total, lse = _softmax_of(s["x"], w, valid, 1.0)
    loss = lse - logits.gather(1, target)[:, 0]
    weight = valid.float() if s["weight"] is None else torch.where(valid, s["weight"], 0.0)
    coef = weight / weight.sum().clamp_min(1e-30)
    more = 1.0
    if c["z_loss"]:
        loss = loss + c["z_loss"] * lse * lse
        more = 1.0 + 2.0 * c["z_loss"] * lse
    d = None
    if c["grads"]:
        d = e.mul_((more / total[:, 0])[:, None])
        d.scatter_add_(1, target, torch.full_like(target, -1, dtype=torch.float32))
        d.mul_(coef[:, None])
    return _outputs(x, w, d, loss, lse, coef, valid)


def _plain_distill(s, c):
    here = (s["top_ids"] >= 0) & (s["top_ids"] < c["vocab"])
    ids = torch.where(here, s["top_ids"], 0)
    valid = here.any(dim=1)
    z = torch.where(here, s["top_logits"] / c["temperature"], -math.inf)
    if s["teacher_lse"] is None:
        z = torch.where(valid[:, None], z, 0.0)
        e = torch.exp(z - z.amax(dim=1, keepdim=True))
        p = e / e.sum(dim=1, keepdim=True)
    else:
        p = torch.exp(z - s["teacher_lse"][:, None])
    p = torch.where(here, p, 0.0)
    w = s["w"].float()
    x, logits, e, total, lse = _softmax_of(s["x"], w, valid, 1.0 / c["temperature"])
    log_p = torch.where(p > 0, torch.log(p), 0.0)
    loss = (p * (log_p - (logits.gather(1, ids) - lse[:, None]))).sum(dim=1)
    weight = valid.float()
    coef = weight / weight.sum().clamp_min(1e-30)
    d = None
    if c["grads"]:
        d = e.mul_((p.sum(dim=1) / total[:, 0])[:, None])
        d.scatter_add_(1, ids, -p)
        d.mul_((coef / c["temperature"])[:, None])
    return _outputs(x, w, d, loss, lse, coef, valid)


def exact(case, seed):
    """The definitions in 64 bits, some tokens at a time."""
    s = prepare(case, seed)
    T, D, V = case["tokens"], case["dim"], case["vocab"]
    w, tau = s["w"].double(), case.get("temperature", 1.0)
    distill = case["op"] == "distill"
    ids = s["top_ids"] if distill else s["targets"][:, None]
    usable = (ids >= 0) & (ids < V)
    counts = usable.any(1)
    if distill:
        z = s["top_logits"].double() / tau
        z[~usable] = -math.inf
        ref = s["teacher_lse"].double() if case["tail"] else torch.logsumexp(z, 1)
        p = torch.exp(z - ref[:, None])
        p[~usable] = 0.0
    else:
        p = usable.double()
    weight = torch.ones(T, dtype=torch.float64, device=w.device)
    if s.get("weight") is not None:
        weight = s["weight"].double()
    weight = weight * counts
    g = weight / weight.sum() if bool(counts.any()) else weight
    loss = torch.zeros(T, dtype=torch.float64, device=w.device)
    lse = torch.zeros_like(loss)
    dx = torch.zeros(T, D, dtype=torch.float64, device=w.device)
    dw = torch.zeros(V, D, dtype=torch.float64, device=w.device) if case["grads"] else None
    for rows in counts.nonzero()[:, 0].split(512):
        x = s["x"][rows].double()
        l = (x @ w.t()) / tau
        norm = torch.logsumexp(l, 1)
        log_q = l - norm[:, None]
        pr, ir = p[rows], ids[rows].clamp(0, V - 1)
        lse[rows] = norm
        loss[rows] = (torch.xlogy(pr, pr) - pr * log_q.gather(1, ir)).sum(1)
        c = pr.sum(1)
        if not distill and case["z_loss"]:
            loss[rows] += case["z_loss"] * norm**2
            c = c + 2 * case["z_loss"] * norm
        if case["grads"]:
            d = torch.exp(log_q) * c[:, None]
            d.scatter_add_(1, ir, -pr)
            d *= (g[rows] / tau)[:, None]
            dx[rows] = d @ w
            dw.addmm_(d.t(), x)
    return {"loss": loss, "lse": lse, "total": (g * loss).sum().reshape(1), "dx": dx if case["grads"] else None, "dw": dw}


def work(case):
    T, D, V = case["tokens"], case["dim"], case["vocab"]
    counted = max(1.0, T * (1.0 - case["masked"]))
    targets = 8 * T if case["op"] == "xent" else 12 * T * case["top"]
    nbytes = 2 * T * D + 2 * V * D + targets + 8 * T
    flops = 2.0 * counted * D * V
    if case["grads"]:
        nbytes += 2 * T * D + 2 * V * D
        flops *= 3
    return {"bytes": float(nbytes), "flops": flops}
