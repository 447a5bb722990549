"""Workloads of the operators around policy training and around the update: log
probabilities of given tokens with their entropy, at the LM head and over stored
logits (there with the best alternatives), each with its gradients; the global
gradient norm with clipping, alone and inside the AdamW step.

``own = False`` computes them in elementary torch operations in 32 bits; ``own =
True`` makes the calls a training program makes of this package.
"""

import math

import torch

own = False

# Sizes: hidden 2048 and vocabulary 163840 are the embedding / LM head of the
# package's largest parameter set, hidden 1536 - 2560 its dense models, 2048 x 1408
# its experts; the other vocabularies are of usual and of odd sizes.


def listed():
    def head(name, tokens, dim, vocab, **more):
        return dict(dict(name=name, op="head", tokens=tokens, dim=dim, vocab=vocab, grads=True, masked=0.0, scale=1.0), **more)

    def logits(name, tokens, vocab, **more):
        return dict(dict(name=name, op="logits", tokens=tokens, vocab=vocab, fp32=False, top=0, grads=False, masked=0.0,
                         scale=1.0), **more)

    def clip(name, tensors, **more):
        return dict(dict(name=name, op="clip", tensors=tensors, fp32=False, out_fp32=False, adamw=False, ratio=0.4), **more)

    return [
        # policy training, one micro-batch of the largest set: log probabilities, entropies, then the gradients
        head("head_policy_8192", 8192, 2048, 163840),
        # scoring rollouts under the policy of before (or a reference): forward only; half the tokens are prompt
        head("head_score_masked", 6000, 2048, 163840, grads=False, masked=0.5),
        # a dense model, odd vocabulary, sampled at temperature 1 / 0.8
        head("head_policy_odd", 1777, 1536, 50021, masked=0.1, scale=0.8),
        # a few tokens of a small model with gradients: latency
        head("head_few_tokens", 24, 512, 8192),
        # a teacher's logits on their way into distillation: 64 alternatives a token
        logits("logits_teacher_top64", 4096, 163840, top=64),
        # a server's log probabilities for 32 sequences, a token each, fp32 logits of a sampler at temperature 1 / 1.25
        logits("logits_decode_32", 32, 163840, fp32=True, top=20, scale=1.25),
        # one token of a small model: latency
        logits("logits_one_token", 1, 8192, top=5),
        # policy training over stored logits: gradients as well, odd rows, padding masked
        logits("logits_policy_grads", 4000, 50021, grads=True, masked=0.15),
        # the expert bucket's gradients of one layer, clipped into a second set of buffers
        clip("clip_experts", "198x2883584"),
        # gains, biases and small matrices: many tensors, fp32, of odd sizes; kept below the limit, so only the norm counts
        clip("clip_many_small", "96x2048,64x577,48x131072,30x1,40x33333", fp32=True, out_fp32=True, ratio=1.7),
        # embedding, head and gains: clipped inside the AdamW step, fp32 master weights, bf16 gradients
        clip("clip_adamw_head", "2x335544320,55x2048", adamw=True),
        # one small parameter group: latency
        clip("clip_adamw_small", "3x1408,1x65536", fp32=True, adamw=True),
    ]


_MOST = 8192 * 2048 * 163840
_MOST_LOGITS = 4096 * 163840
_MOST_GRADS = 500_000_000


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["head", "logits", "clip"])
    if op == "head":
        while True:
            tokens, vocab = spread(1, 8192), spread(1000, 163840)
            dim = rng.choice([64, 256, 512, 1000, 1024, 1408, 1536, 1792, 2048, 2304, 2560, rng.randint(64, 2560)])
            if tokens * dim * vocab <= _MOST:
                break
        return dict(op=op, tokens=tokens, dim=dim, vocab=vocab, grads=rng.random() < 0.6,
                    masked=rng.choice([0.0, 0.1, 0.5]) if tokens >= 32 else 0.0, scale=rng.choice([1.0, 1.0, 0.7]))
    if op == "logits":
        while True:
            tokens, vocab = spread(1, 8192), spread(1000, 163840)
            if tokens * vocab <= _MOST_LOGITS:
                break
        top = rng.choice([0, 1, 5, 20, 50, 64, 100, 128])
        return dict(op=op, tokens=tokens, vocab=vocab, fp32=rng.random() < 0.4 and tokens * vocab <= _MOST_LOGITS // 2, top=top,
                    grads=rng.random() < 0.4, masked=rng.choice([0.0, 0.1, 0.5]) if top == 0 and tokens >= 32 else 0.0,
                    scale=rng.choice([1.0, 1.0, 0.7]))
    kinds, left = [], _MOST_GRADS
    for _ in range(rng.randint(1, 5)):
        numel, count = spread(1, 20_000_000), spread(1, 300)
        count = max(1, min(count, left // numel))
        if count * numel <= left:
            kinds.append("%dx%d" % (count, numel))
            left -= count * numel
    return dict(op=op, tensors=",".join(kinds), fp32=rng.random() < 0.5, out_fp32=rng.random() < 0.5, adamw=rng.random() < 0.5,
                ratio=rng.choice([0.1, 0.5, 1.7]))


_STD = 1e-3  # of a gradient's elements, before the scale of its tensor
_HYPER = dict(lr=1e-3, wd=0.1, beta1=0.9, beta2=0.95, eps=1e-8)
_STEP = 10
_NORM_EPS = 1e-6


def _sizes(case):
    out = []
    for kind in case["tensors"].split(","):
        count, numel = kind.split("x")
        out += [int(numel)] * int(count)
    return out


def _flat(sizes, dtype, fill=None):
    """One buffer for all tensors, each at a multiple of 64 elements, and the views of it."""
    starts, end = [], 0
    for n in sizes:
        starts.append(end)
        end += (n + 63) // 64 * 64
    buffer = torch.zeros(end, dtype=dtype, device="cuda")
    views = [buffer[a : a + n] for a, n in zip(starts, sizes)]
    if fill is not None:
        for i, t in enumerate(views):
            t.copy_(fill(i, t.numel()))
    return buffer, views


def prepare(case, seed):
    """What a training program holds before the call."""
    gen = torch.Generator(device="cuda").manual_seed(int(seed))

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def rand(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    s = {"case": case}
    if case["op"] == "clip":
        sizes = _sizes(case)
        g_type = torch.float32 if case["fp32"] else torch.bfloat16
        # some tensors' gradients are several times larger than others'
        level = torch.exp(0.5 * randn(len(sizes))).tolist()
        _, s["grads"] = _flat(sizes, g_type, lambda i, n: randn(n) * (_STD * level[i]))
        s["max_norm"] = case["ratio"] * _STD * math.sqrt(sum(n * a * a for n, a in zip(sizes, level)))
        if case["adamw"]:
            s["params_flat"], s["params"] = _flat(sizes, torch.float32, lambda i, n: randn(n) * 0.02)
            s["m_flat"], s["m"] = _flat(sizes, torch.float32, lambda i, n: randn(n) * (0.3 * _STD))
            s["v_flat"], s["v"] = _flat(sizes, torch.float32, lambda i, n: (rand(n) + 0.1) * _STD**2)
        else:
            s["out_flat"], s["out"] = _flat(sizes, torch.float32 if case["out_fp32"] else torch.bfloat16)
        if own:  # the handle that a program keeps beside its gradients
            from paper_2502_16982_b200 import binding

            s["handle"] = binding.MuonGrads(s["grads"], out=s.get("out"))
        return s

    T, V = case["tokens"], case["vocab"]
    # frequent tokens have low ids
    first = (rand(T).double().square() * V).long().clamp_(max=V - 1)
    # push[t]: by how much the token's logit is lifted over the others
    push = math.log(V) * (0.2 + 1.2 * rand(T))
    masked = rand(T) < case["masked"]
    s["targets"] = torch.where(masked, torch.full_like(first, -100), first)
    if case["op"] == "head":
        D = case["dim"]
        s["w"] = (randn(V, D) * 0.02).to(torch.bfloat16)
        s["x"] = (randn(T, D) + (push / (0.02 * 0.02 * D))[:, None] * s["w"][first].float()).to(torch.bfloat16)
    else:
        # a body of logits, and eight entries a token that stand out beside the given one
        z = randn(T, V).mul_(1.5)
        more = (rand(T, 8) * V).long().clamp_(max=V - 1)
        for k in range(8):  # one entry a row at a time: a sum whose order is fixed
            z.scatter_add_(1, more[:, k : k + 1], math.log(V) * rand(T, 1))
        z.scatter_add_(1, first[:, None], push[:, None])
        s["logits"] = z if case["fp32"] else z.to(torch.bfloat16)
    if case["grads"]:
        # gradient of a mean over tokens: minus the advantages, and a bonus on the entropy
        s["g_logprob"] = -randn(T) / T
        s["g_entropy"] = torch.full((T,), -0.01 / T, device="cuda")
    return s


def run(s):
    c = s["case"]
    if not own:
        return {"head": _plain_head, "logits": _plain_logits, "clip": _plain_clip}[c["op"]](s, c)
    from paper_2502_16982_b200 import binding

    if c["op"] == "clip":
        if not c["adamw"]:
            r = s["handle"].muon_clip_grads(s["max_norm"], eps=_NORM_EPS)
            return {"norm": r.norm, "coef": r.coef, "grads": s["out_flat"]}
        r = s["handle"].muon_grad_norm(s["max_norm"], eps=_NORM_EPS)
        binding.muon_adamw_step(s["params"], s["grads"], s["m"], s["v"], _STEP, coef=r.coef, **_HYPER)
        return {"norm": r.norm, "coef": r.coef, "params": s["params_flat"], "m": s["m_flat"], "v": s["v_flat"]}
    if c["op"] == "head":
        r = binding.muon_head_logprob(s["x"], s["w"], s["targets"], logit_scale=c["scale"])
        out = {"logprob": r.logprob, "entropy": r.entropy, "lse": r.lse, "dx": None, "dw": None}
        if c["grads"]:
            d = binding.muon_head_logprob_grad(s["x"], s["w"], s["targets"], r, g_logprob=s["g_logprob"],
                                               g_entropy=s["g_entropy"], logit_scale=c["scale"], dx=True, dw=True)
            out["dx"], out["dw"] = d.dx, d.dw
        return out
    r = binding.muon_logits_logprob(s["logits"], s["targets"], top=c["top"], logit_scale=c["scale"])
    out = {"logprob": r.logprob, "entropy": r.entropy, "lse": r.lse, "top_ids": r.top_ids, "top_logits": r.top_logits,
           "top_logprob": r.top_logprob, "dlogits": None}
    if c["grads"]:
        out["dlogits"] = binding.muon_logits_logprob_grad(s["logits"], s["targets"], r, g_logprob=s["g_logprob"],
                                                          g_entropy=s["g_entropy"], logit_scale=c["scale"])
    return out


def _plain_statistics(l, targets, V):
    """Log-sum-exp, log probability of the token and entropy of rows of scaled logits;
    what a masked token gives is 0."""
    valid = (targets >= 0) & (targets < V)
    target = torch.where(valid, targets, 0)[:, None]
    top = l.amax(dim=1, keepdim=True)
    y = l - top
    e = torch.exp(y)
    total = e.sum(dim=1)
    log_total = torch.log(total)
    logprob = y.gather(1, target)[:, 0] - log_total
    entropy = log_total - (e * y).sum(dim=1) / total
    lse = top[:, 0] + log_total
    zero = torch.zeros_like(lse)
    return valid, target, torch.where(valid, logprob, zero), torch.where(valid, entropy, zero), torch.where(valid, lse, zero)


def _plain_dlogits(s, c, l, valid, target, entropy, lse):
    log_q = l.sub_(lse[:, None])
    q = torch.exp(log_q)
    r, h = torch.where(valid, s["g_logprob"], 0.0), torch.where(valid, s["g_entropy"], 0.0)
    d = q * (-(r + h * entropy)[:, None] - h[:, None] * log_q)
    d.scatter_add_(1, target, r[:, None])
    d = d.mul_(c["scale"])
    return torch.where(valid[:, None], d, 0.0)


def _plain_head(s, c):
    valid = (s["targets"] >= 0) & (s["targets"] < c["vocab"])
    x, w = torch.where(valid[:, None], s["x"].float(), 0.0), s["w"].float()
    l = (x @ w.t()).mul_(c["scale"])
    valid, target, logprob, entropy, lse = _plain_statistics(l, s["targets"], c["vocab"])
    out = {"logprob": logprob, "entropy": entropy, "lse": lse, "dx": None, "dw": None}
    if c["grads"]:
        d = _plain_dlogits(s, c, l, valid, target, entropy, lse)
        out["dx"], out["dw"] = (d @ w).to(torch.bfloat16), (d.t() @ x).to(torch.bfloat16)
    return out


def _plain_logits(s, c):
    V = c["vocab"]
    raw = s["logits"].float()
    l = raw * c["scale"]
    valid, target, logprob, entropy, lse = _plain_statistics(l, s["targets"], V)
    out = {"logprob": logprob, "entropy": entropy, "lse": lse, "top_ids": None, "top_logits": None, "top_logprob": None,
           "dlogits": None}
    if c["top"]:
        # equal logits: the lowest index first.  One whole number orders both: the bits of a
        # float, made ascending, above the index counted down
        bits = (raw + 0.0).view(torch.int32).long()
        key = torch.where(bits >= 0, bits, -2147483648 - bits) * V + torch.arange(V - 1, -1, -1, device=raw.device)
        ids = V - 1 - key.topk(c["top"], dim=1).values.remainder(V)
        out["top_ids"], out["top_logits"] = ids, raw.gather(1, ids)
        out["top_logprob"] = out["top_logits"] * c["scale"] - lse[:, None]
    if c["grads"]:
        out["dlogits"] = _plain_dlogits(s, c, l, valid, target, entropy, lse).to(s["logits"].dtype)
    return out


def _plain_clip(s, c):
    total = torch.zeros((), dtype=torch.float64, device="cuda")
    for g in s["grads"]:
        total += g.float().square().sum(dtype=torch.float64)
    norm = total.sqrt()
    coef = (s["max_norm"] / (norm + _NORM_EPS)).clamp(max=1.0).float().reshape(1)
    out = {"norm": norm.float().reshape(1), "coef": coef}
    if not c["adamw"]:
        for g, o in zip(s["grads"], s["out"]):
            o.copy_(g.float() * coef)
        out["grads"] = s["out_flat"]
        return out
    h = _HYPER
    bias1, bias2 = 1.0 - h["beta1"] ** _STEP, 1.0 - h["beta2"] ** _STEP
    for p, g, m, v in zip(s["params"], s["grads"], s["m"], s["v"]):
        g = g.float() * coef
        m.mul_(h["beta1"]).add_(g * (1.0 - h["beta1"]))
        v.mul_(h["beta2"]).add_(g * g * (1.0 - h["beta2"]))
        p.sub_(((m / bias1) / ((v / bias2).sqrt() + h["eps"]) + p * h["wd"]) * h["lr"])
    out.update(params=s["params_flat"], m=s["m_flat"], v=s["v_flat"])
    return out


def exact(case, seed):
    """The definitions in 64 bits, some tokens (tensors) at a time."""
    s = prepare(case, seed)
    if case["op"] == "clip":
        norm = math.sqrt(math.fsum(float(torch.dot(g.double(), g.double())) for g in s["grads"]))
        coef = min(1.0, s["max_norm"] / (norm + _NORM_EPS))
        as64 = {"dtype": torch.float64, "device": "cuda"}
        out = {"norm": torch.tensor([norm], **as64), "coef": torch.tensor([coef], **as64)}
        if not case["adamw"]:
            out["grads"], _ = _flat(_sizes(case), torch.float64, lambda i, n: s["grads"][i].double() * coef)
            return out
        out["params"], params = _flat(_sizes(case), torch.float64)
        out["m"], ms = _flat(_sizes(case), torch.float64)
        out["v"], vs = _flat(_sizes(case), torch.float64)
        for i, (p, g, m, v) in enumerate(zip(s["params"], s["grads"], s["m"], s["v"])):
            g = g.double() * coef
            m = _HYPER["beta1"] * m.double() + (1 - _HYPER["beta1"]) * g
            v = _HYPER["beta2"] * v.double() + (1 - _HYPER["beta2"]) * g**2
            step = m / (1 - _HYPER["beta1"] ** _STEP) / (torch.sqrt(v / (1 - _HYPER["beta2"] ** _STEP)) + _HYPER["eps"])
            params[i].copy_(p.double() - _HYPER["lr"] * (step + _HYPER["wd"] * p.double()))
            ms[i].copy_(m)
            vs[i].copy_(v)
        return out

    T, V, scale, top = case["tokens"], case["vocab"], case["scale"], case.get("top", 0)
    as64 = {"dtype": torch.float64, "device": "cuda"}
    at_head = case["op"] == "head"
    out = {k: torch.zeros(T, **as64) for k in ("logprob", "entropy", "lse")}
    if at_head:
        w = s["w"].double()
        out["dx"] = torch.zeros(T, case["dim"], **as64) if case["grads"] else None
        out["dw"] = torch.zeros(V, case["dim"], **as64) if case["grads"] else None
    else:
        out["top_ids"] = torch.zeros(T, top, dtype=torch.int64, device="cuda") if top else None
        out["top_logits"] = torch.zeros(T, top, **as64) if top else None
        out["top_logprob"] = torch.zeros(T, top, **as64) if top else None
        out["dlogits"] = torch.zeros(T, V, **as64) if case["grads"] else None
    counted = ((s["targets"] >= 0) & (s["targets"] < V)).nonzero()[:, 0]
    for rows in counted.split(512):
        raw = s["x"][rows].double() @ w.t() if at_head else s["logits"][rows].double()
        log_q = torch.log_softmax(raw * scale, dim=1)
        y = s["targets"][rows][:, None]
        lp = log_q.gather(1, y)
        ent = -(torch.exp(log_q) * log_q).sum(1)
        out["logprob"][rows] = lp[:, 0]
        out["entropy"][rows] = ent
        out["lse"][rows] = (raw.gather(1, y) * scale - lp)[:, 0]
        if top:
            order = raw.sort(dim=1, descending=True, stable=True).indices[:, :top]
            out["top_ids"][rows] = order
            out["top_logits"][rows] = raw.gather(1, order)
            out["top_logprob"][rows] = log_q.gather(1, order)
        if case["grads"]:
            r, h = s["g_logprob"][rows].double(), s["g_entropy"][rows].double()
            q = torch.exp(log_q)
            d = -r[:, None] * q - h[:, None] * q * (log_q + ent[:, None])
            d[torch.arange(len(rows), device="cuda"), y[:, 0]] += r
            d *= scale
            if at_head:
                out["dx"][rows] = d @ w
                out["dw"].addmm_(d.t(), s["x"][rows].double())
            else:
                out["dlogits"][rows] = d
    return out


def work(case):
    if case["op"] == "clip":
        n = sum(_sizes(case))
        g = 4 if case["fp32"] else 2
        if case["adamw"]:  # weights and both moments read and written
            return {"bytes": float(n * (g + 24)), "flops": 18.0 * n}
        return {"bytes": float(n * (g + (4 if case["out_fp32"] else 2))), "flops": 3.0 * n}
    T, V = case["tokens"], case["vocab"]
    counted = max(1.0, T * (1.0 - case["masked"]))
    if case["op"] == "head":
        D = case["dim"]
        nbytes, flops = 2 * T * D + 2 * V * D + 20 * T, 2.0 * counted * D * V
        if case["grads"]:
            nbytes += 2 * T * D + 2 * V * D + 8 * T
            flops *= 3
        return {"bytes": float(nbytes), "flops": flops}
    size = 4 if case["fp32"] else 2
    nbytes, flops = counted * V * size + 20 * T + 16 * T * case["top"], 6.0 * counted * V
    if case["grads"]:
        nbytes += T * V * size + 8 * T
        flops *= 2
    return {"bytes": float(nbytes), "flops": flops}
