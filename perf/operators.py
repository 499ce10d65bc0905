"""The update-side operators that stand between a rollout's logits and a clipped gradient step, as
they are timed and compared: each in a plain form of elementary torch operations, and as the calls
that a user makes of `paper_2309_00754_gb300.hydra`.

  stats  of every sampled token's row of logits: the token's log-probability, the entropy, the
         (max, log-sum) pair that normalises the row, and the k likeliest tokens
  grad   the gradient of those log-probabilities and entropies with respect to the logits
  clip   the global norm of many gradient tensors, and the tensors scaled down to a largest norm

Sizes are those of experience scoring and updates with a Llama-7B-shaped actor (vocabulary 32000,
d 4096, SwiGLU 11008, LoRA on q/v/gate/up/down) and odd ones around them. Rows of logits may stand
further apart than the vocabulary, sequences end before their slots do, and a vocabulary may be
masked with -inf or with the type's lowest value."""
import math

import torch

own = False  # the framework's entry points in place of the plain forms

DEV = "cuda"
EPS = 1e-6  # of the clipping coefficient max_norm / (norm + EPS)
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one decode step of one sequence: the drawn token's log-probability and five alternatives
        {"name": "stats_1x32000_f32_k5", "op": "stats", "s": 1, "l": 1, "v": 32000, "ld": 32000,
         "type": "f32", "k": 5, "mask": "none"},
        # one decode step of 64 sequences, with the twenty alternatives that serving offers
        {"name": "stats_64x32000_f32_k20", "op": "stats", "s": 64, "l": 1, "v": 32000, "ld": 32000,
         "type": "f32", "k": 20, "mask": "none"},
        # an update batch of four ragged 400-token completions, for losses and entropy alone
        {"name": "stats_4x400x32000_f32", "op": "stats", "s": 4, "l": 400, "v": 32000, "ld": 32000,
         "type": "f32", "k": 0, "mask": "none"},
        # constrained decoding: forbidden tokens at -inf, an odd vocabulary, rows at odd strides
        {"name": "stats_37x9x50001_masked_k20", "op": "stats", "s": 37, "l": 9, "v": 50001,
         "ld": 50003, "type": "bf16", "k": 20, "mask": "inf"},
        # a large scored batch in bf16, with alternatives kept for each token
        {"name": "stats_8x1024x32000_bf16_k8", "op": "stats", "s": 8, "l": 1024, "v": 32000,
         "ld": 32000, "type": "bf16", "k": 8, "mask": "none"},
        # the gradient of a small ragged minibatch, odd sizes: latency counts
        {"name": "grad_3x7x1001_bf16", "op": "grad", "s": 3, "l": 7, "v": 1001, "ld": 1001,
         "type": "bf16", "out": "bf16", "mask": "none", "entropy": True},
        # the update batch above: fp32 logits, bf16 gradients for the head's backward product
        {"name": "grad_4x400x32000_f32_bf16", "op": "grad", "s": 4, "l": 400, "v": 32000,
         "ld": 32000, "type": "f32", "out": "bf16", "mask": "none", "entropy": True},
        # a full minibatch at 512 tokens, with a masked vocabulary, all in fp32
        {"name": "grad_8x512x32000_f32", "op": "grad", "s": 8, "l": 512, "v": 32000, "ld": 32000,
         "type": "f32", "out": "f32", "mask": "lowest", "entropy": True},
        # the gradients of a two-layer toy actor's LoRA set
        {"name": "clip_toy_f32", "op": "clip", "layers": 2, "d": 256, "ffn": 512, "r": 8,
         "type": "f32", "bucket": False, "odd": 0, "max_norm": 0.05, "first": True},
        # LoRA gradients of odd sizes that lie back to back in one bucket, both types
        {"name": "clip_bucket_mixed", "op": "clip", "layers": 13, "d": 1024, "ffn": 2752, "r": 8,
         "type": "mixed", "bucket": True, "odd": 3, "max_norm": 1.0, "first": False},
        # the LoRA set of the 7B-shaped actor, rank 16
        {"name": "clip_7b_r16_f32", "op": "clip", "layers": 32, "d": 4096, "ffn": 11008, "r": 16,
         "type": "f32", "bucket": False, "odd": 0, "max_norm": 1.0, "first": False},
        # the same in bf16 at rank 64
        {"name": "clip_7b_r64_bf16", "op": "clip", "layers": 32, "d": 4096, "ffn": 11008, "r": 64,
         "type": "bf16", "bucket": False, "odd": 0, "max_norm": 1.0, "first": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["stats", "stats", "grad", "clip"])
    if op == "clip":
        while True:
            c = {"op": op, "layers": _log(rng, 1, 40), "d": 8 * _log(rng, 16, 640),
                 "ffn": 8 * _log(rng, 32, 1760), "r": 8 * _log(rng, 1, 16),
                 "type": rng.choice(["f32", "bf16", "mixed"]), "bucket": rng.random() < 0.5,
                 "odd": rng.choice([0, 0, 1, 3, 5]), "max_norm": rng.choice([0.05, 1.0, 1e6]),
                 "first": rng.random() < 0.3}
            if work(c)["bytes"] <= 800e6:
                return c
    while True:
        v = rng.choice([32000, _log(rng, 1000, 152000), 8 * _log(rng, 125, 19000)])
        c = {"op": op, "s": _log(rng, 1, 64), "l": _log(rng, 1, 1024), "v": v,
             "ld": v + rng.choice([0, 0, rng.randint(1, 9), 64]), "type": rng.choice(["f32", "bf16"]),
             "mask": rng.choice(["none", "none", "inf", "lowest"])}
        if op == "stats":
            c["k"] = rng.choice([0, 1, rng.randint(2, 32), 20])
        else:
            c["out"] = rng.choice([c["type"], "f32", "bf16"])
            c["entropy"] = rng.random() < 0.6
        if work(c)["bytes"] <= (320e6 if op == "stats" else 800e6):
            return c


# --------------------------------------------------------------------------- inputs


def _lengths(case):
    """A quarter of the slots to all of them; which sequence has which is up to the seed. One-token
    calls are decode steps: every row is live."""
    s, l = case["s"], case["l"]
    if l == 1 or s == 1:
        return [l] * s
    return [max(1, round(l * (0.25 + 0.75 * i / (s - 1)))) for i in range(s)]


def _numels(case):
    """Elements of the gradient tensors: per layer A and B of q/v, gate/up and down in the fused
    layouts, then the reward head and its bias. `odd` is added to every width."""
    d, f, r = case["d"] + case["odd"], case["ffn"] + case["odd"], case["r"]
    layer = [2 * r * d, 3 * d * 2 * r, 2 * r * d, 2 * f * 2 * r, r * f, d * r]
    return layer * case["layers"] + [d, 1]


def _kinds(case):
    """Which of the gradient tensors are in which type."""
    n = len(_numels(case))
    return [case["type"] if case["type"] != "mixed" else ("f32", "bf16")[i % 3 == 0] for i in range(n)]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    t = {"case": case}
    if case["op"] == "clip":
        sizes, kinds = _numels(case), _kinds(case)
        # tensors of a step have scales of their own; in a first step A's gradients are zero (B is)
        std = (10 ** (torch.rand(len(sizes), device=DEV, generator=g) * 2 - 4)).tolist()
        t["grads"] = []
        t["flat"] = {}
        for kind in sorted(set(kinds)):
            mine = [i for i, x in enumerate(kinds) if x == kind]
            flat = torch.randn(sum(sizes[i] for i in mine), device=DEV, generator=g)
            parts = flat.split([sizes[i] for i in mine])
            for i, p in zip(mine, parts):
                p.mul_(0.0 if case["first"] and i % 2 == 0 and i < len(sizes) - 2 else std[i])
            flat = flat.to(TYPES[kind])
            parts = flat.split([sizes[i] for i in mine])
            t["grads"] += [(i, p if case["bucket"] else p.clone()) for i, p in zip(mine, parts)]
            t["flat"][kind] = torch.full_like(flat, math.nan)  # where the clipped gradients go
        t["outs"] = []
        for kind in sorted(set(kinds)):
            mine = [i for i, x in enumerate(kinds) if x == kind]
            t["outs"] += list(zip(mine, t["flat"][kind].split([sizes[i] for i in mine])))
        t["grads"] = [p for _, p in sorted(t["grads"], key=lambda x: x[0])]
        t["outs"] = [p for _, p in sorted(t["outs"], key=lambda x: x[0])]
        t["kinds"] = kinds
        t["norm"] = torch.zeros(2, device=DEV)
        return t
    s, l, v, ld = case["s"], case["l"], case["v"], case["ld"]
    rows, dt = s * l, TYPES[case["type"]]
    # some rows nearly certain of a token, others nearly uniform
    scale = 10 ** (torch.rand(rows, 1, device=DEV, generator=g) * 1.2 - 0.6)
    z = torch.randn(rows, v, device=DEV, generator=g) * scale
    z -= 2.0 * torch.log(1e-3 + torch.rand(1, v, device=DEV, generator=g))  # common tokens
    if case["mask"] != "none":
        keep = 10 ** (torch.rand(rows, 1, device=DEV, generator=g) * -3.5)  # shares that stay allowed
        z.masked_fill_(torch.rand(rows, v, device=DEV, generator=g) > keep,
                       -math.inf if case["mask"] == "inf" else torch.finfo(dt).min)
        if rows > 5:
            z[5] = -math.inf if case["mask"] == "inf" else torch.finfo(dt).min  # nothing is left
    u = torch.rand(rows, v, device=DEV, generator=g).clamp_(1e-20, 1 - 1e-7)
    t["ids"] = (z - torch.log(-torch.log(u))).argmax(1).int()
    del u
    whole = torch.zeros(rows, ld, dtype=dt, device=DEV)
    whole[:, :v] = z
    t["logits"] = whole[:, :v]
    t["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device=DEV)[
        torch.randperm(s, device=DEV, generator=g)]
    if case["op"] == "stats":
        k = case["k"]
        t["logp"], t["entropy"] = (torch.full((rows,), math.nan, device=DEV) for _ in range(2))
        t["norm"] = torch.full((rows, 2), math.nan, device=DEV)
        t["top_ids"] = torch.full((rows, k), -7, dtype=torch.int32, device=DEV) if k else None
        t["top_logp"] = torch.full((rows, k), math.nan, device=DEV) if k else None
        return t
    # what the forward pass left, and the gradients that the losses give
    t["norm"], t["entropy"] = torch.empty(rows, 2, device=DEV), torch.empty(rows, device=DEV)
    for at in range(0, rows, 512):
        y = t["logits"][at:at + 512].double()
        m = y.amax(1, keepdim=True)
        y = torch.where(m == -math.inf, -math.inf, y - m)
        total = y.exp().sum(1, keepdim=True)
        y = y - torch.where(total > 0, total.log(), 0)
        t["norm"][at:at + 512] = torch.cat([m, torch.where(total > 0, total.log(), 0)], 1).float()
        t["entropy"][at:at + 512] = -torch.where(y == -math.inf, 0, y * y.exp()).sum(1).float()
    live = torch.arange(l, device=DEV)[None] < t["lengths"][:, None]
    n = sum(_lengths(case))
    t["grad_logp"] = torch.where(live.reshape(-1), torch.randn(rows, device=DEV, generator=g) / n, 0)
    t["grad_entropy"] = (torch.where(live.reshape(-1), -0.05 / n, 0.0).float() if case["entropy"]
                         else None)
    t["dlogits"] = torch.full((rows, ld), math.nan, dtype=TYPES[case["out"]], device=DEV)[:, :v]
    return t


# --------------------------------------------------------------------------- one pass


def run(t):
    op = t["case"]["op"]
    if op == "stats":
        return _stats_own(t) if own else _stats(t)
    if op == "grad":
        return _grad_own(t) if own else _grad(t)
    return _clip_own(t) if own else _clip(t)


def _stats_own(t):
    from paper_2309_00754_gb300 import hydra as H

    c = t["case"]
    H.hydra_token_logprobs_entropy(t["logits"], t["ids"], t["lengths"], c["s"], c["l"], t["logp"],
                                   t["entropy"], t["norm"], t["top_ids"], t["top_logp"])
    out = {k: t[k] for k in ("logp", "entropy", "norm")}
    return out | ({"top_ids": t["top_ids"], "top_logp": t["top_logp"]} if c["k"] else {})


def _grad_own(t):
    from paper_2309_00754_gb300 import hydra as H

    c = t["case"]
    H.hydra_token_logprobs_entropy_grad(t["logits"], t["ids"], t["lengths"], c["s"], c["l"], t["norm"],
                                        t["entropy"], t["grad_logp"], t["grad_entropy"], t["dlogits"])
    return t["dlogits"]


def _clip_own(t):
    from paper_2309_00754_gb300 import hydra as H

    if "list" not in t:  # a program keeps the list and the workspace as long as its gradients' buffers
        t["list"] = H.GradList(t["grads"], t["outs"])
        t["ws"] = torch.empty(H.grad_norm_workspace_size(), dtype=torch.uint8, device=DEV)
    H.hydra_clip_grad_norm(t["list"], t["case"]["max_norm"], t["norm"], t["ws"])
    return t["flat"] | {"norm": t["norm"]}


def _live(t):
    c = t["case"]
    return (torch.arange(c["l"], device=DEV)[None] < t["lengths"][:, None]).reshape(-1)


def _stats(t):
    live, k = _live(t), t["case"]["k"]
    z = t["logits"].float()
    m = z.amax(1, keepdim=True)
    d = z - torch.where(m == -math.inf, 0.0, m)
    e = d.exp()
    total = e.sum(1, keepdim=True)
    log_total = torch.where(total > 0, total.log(), 0.0)
    lp = d - log_total
    entropy = -torch.where(e > 0, e / total * lp, 0.0).sum(1)
    out = {"logp": torch.where(live, lp.gather(1, t["ids"].long()[:, None])[:, 0], 0.0),
           "entropy": torch.where(live, entropy, 0.0),
           "norm": torch.where(live[:, None], torch.cat([m, log_total], 1), 0.0)}
    if k:
        # the value's order in the upper half, the lower index first in the lower
        bits = (z + 0.0).view(torch.int32)
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() << 32
        last = 0x7FFFFFFF
        order += last - torch.arange(z.shape[1], device=DEV)
        ids = last - (order.topk(k, 1).values & last)
        out["top_ids"] = torch.where(live[:, None], ids, -1).int()
        out["top_logp"] = torch.where(live[:, None], lp.gather(1, ids), 0.0)
    return out


def _grad(t):
    z, norm = t["logits"].float(), t["norm"]
    m = norm[:, :1]
    lp = z - torch.where(m == -math.inf, 0.0, m) - norm[:, 1:]
    p = lp.exp()
    weight = t["grad_logp"][:, None]
    if t["grad_entropy"] is not None:
        weight = weight + t["grad_entropy"][:, None] * (lp + t["entropy"][:, None])
    d = torch.where(p > 0, -p * weight, 0.0)
    hit = torch.arange(z.shape[1], device=DEV)[None] == t["ids"][:, None]
    d = torch.where(hit, d + t["grad_logp"][:, None], d)
    live = _live(t)[:, None] & (m > -math.inf)
    return torch.where(live, d, 0.0).to(t["dlogits"].dtype)


def _clip(t):
    sums = [g.float().square().sum() for g in t["grads"]]
    norm = torch.stack(sums).double().sum().sqrt()
    coef = (t["case"]["max_norm"] / (norm + EPS)).clamp(max=1.0)
    clipped = [(g.float() * coef.float()).to(g.dtype) for g in t["grads"]]
    out = {kind: torch.cat([g for g, x in zip(clipped, t["kinds"]) if x == kind]) for kind in t["flat"]}
    return out | {"norm": torch.stack([norm, coef]).float()}


# --------------------------------------------------------------------------- work


def work(case):
    if case["op"] == "clip":
        n = [0, 0]
        for size, kind in zip(_numels(case), _kinds(case)):
            n[kind == "bf16"] += size
        return {"bytes": 2 * (4 * n[0] + 2 * n[1]) + 8, "flops": 3 * sum(n)}
    live, rows, v = sum(_lengths(case)), case["s"] * case["l"], case["v"]
    size = {"f32": 4, "bf16": 2}
    read = live * v * size[case["type"]] + 4 * (live + case["s"])
    if case["op"] == "stats":
        return {"bytes": read + rows * (16 + 8 * case["k"]), "flops": 6 * live * v}
    return {"bytes": read + rows * v * size[case["out"]] + live * (20 if case["entropy"] else 12),
            "flops": 6 * live * v}


# --------------------------------------------------------------------------- 64 bits


def exact(case, seed):
    t = prepare(case, seed)
    if case["op"] == "clip":
        square = sum(float(g.double().pow(2).sum()) for g in t["grads"])
        norm = math.sqrt(square)
        coef = min(1.0, case["max_norm"] / (norm + EPS))
        out = {kind: torch.cat([g.double() * coef for g in t["grads"] if g.dtype == TYPES[kind]])
               for kind in t["flat"]}
        return out | {"norm": torch.tensor([norm, coef], dtype=torch.float64)}
    rows, v = t["logits"].shape
    live = torch.cat([torch.arange(case["l"], device=DEV) < n for n in t["lengths"].tolist()])
    blocks = range(0, rows, 256)
    if case["op"] == "stats":
        got = [_exact_stats(t["logits"][a:a + 256].double(), t["ids"][a:a + 256].long(), case["k"])
               for a in blocks]
        out = {k: torch.cat([x[k] for x in got]) for k in got[0]}
        for k in out:
            out[k][~live] = -1 if k == "top_ids" else 0
        return out
    out = torch.empty(rows, v, dtype=torch.float64, device=DEV)
    for a in blocks:
        out[a:a + 256] = _exact_grad(t["logits"][a:a + 256].double(), t["ids"][a:a + 256].long(),
                                     t["grad_logp"][a:a + 256].double(),
                                     t["grad_entropy"][a:a + 256].double() if case["entropy"] else None)
    out[~live] = 0
    return out


def _log_softmax(z):
    """(log-probabilities, max, log of the sum); a row of nothing but -inf has -inf everywhere."""
    m = z.max(1, keepdim=True).values
    empty = torch.isinf(m)
    shifted = (z - m).masked_fill(empty, -math.inf)
    log_sum = torch.logsumexp(shifted, 1, keepdim=True).masked_fill(empty, 0.0)
    return shifted - log_sum, m, log_sum


def _exact_stats(z, ids, k):
    lp, m, log_sum = _log_softmax(z)
    p = lp.exp()
    out = {"logp": lp[torch.arange(len(ids), device=DEV), ids],
           "entropy": -(p * lp.clamp(min=-1e4)).sum(1), "norm": torch.cat([m, log_sum], 1)}
    if k:
        at = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :k]
        out["top_ids"], out["top_logp"] = at.int(), lp.gather(1, at)
    return out


def _exact_grad(z, ids, grad_logp, grad_entropy):
    lp, m, _ = _log_softmax(z)
    p = lp.exp()
    d = -p * grad_logp[:, None]
    d[torch.arange(len(ids), device=DEV), ids] += grad_logp
    if grad_entropy is not None:
        lp = lp.clamp(min=-1e4)
        entropy = -(p * lp).sum(1, keepdim=True)
        d -= p * (lp + entropy) * grad_entropy[:, None]
    return d.masked_fill(torch.isinf(m), 0.0)
