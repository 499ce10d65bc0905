"""The operators of decoding with drafted tokens over a paged key/value cache, as they are timed and
compared: each in a plain form of elementary torch operations, and as the calls that a user makes of
`paper_2309_00754_gb300.hydra`.

  append  new tokens' keys and values rotated, held in 4 bits or bf16 and written to their pages, the
          queries rotated beside them; then the appended rows read back dense, as the cache holds them
  attend  attention of each sequence's new tokens over its cached ones, through the page table
  verify  drafted tokens accepted or refused by the target's probabilities from given random
          numbers, and the token that follows them

Sizes are those of generation with a Llama-7B-shaped actor (32 heads of 128, vocabulary 32000, some
hundred tokens a sequence) and generic ones around them: grouped heads, heads of 64, long contexts,
odd batches. Sequences have lengths of their own, and pages lie in any order.

A page holds, for each key/value head, tiles of 16 tokens. In 4 bits a token's head is held in groups
of 64 channels, each with a scale and a zero point: scale (code - zero). Tile of 16 tokens x D:
  codes of keys    [token][t 4][group][16 channels], channel = 64 group + 16 t + ..., low nibble first
  codes of values  [p 2][g 8][t 4][group][m 2][b 2][4 channels], token = 8 p + 2 t + b,
                   channel = 64 group + 8 g + 4 m + ...
  scales, bf16     [g 8][h 2][key, value][group], token = 8 h + g
  zeros of keys    [g 8][h 2][group], 16 bits each, 17 times the zero point
  zeros of values  [t 4][p 2][group][b 2], the same
and in bf16
  keys             [channel / 32][token][32]
  values           [p 2][channel / 32][g 8][t 4][4 channels][b 2], channel = 32 .. + 4 g + ..."""
import math

import torch

own = False  # the framework's entry points in place of the plain forms

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
GROUP = 64   # channels that share a scale
TILE = 16    # tokens of a tile


def listed():
    return [
        # one decode step's token of one sequence
        {"name": "append_1x1_int4", "op": "append", "kind": "int4", "s": 1, "l": 1, "heads": 32, "kv": 32,
         "dh": 128, "page": 16, "cached": 300},
        # drafted tokens of an odd batch with grouped heads of 64, unquantised
        {"name": "append_37x5_bf16", "op": "append", "kind": "bf16", "s": 37, "l": 5, "heads": 12, "kv": 4,
         "dh": 64, "page": 32, "cached": 1000},
        # the prompts of a batch, ragged
        {"name": "append_8x512_int4", "op": "append", "kind": "int4", "s": 8, "l": 512, "heads": 32, "kv": 32,
         "dh": 128, "page": 64, "cached": 0},
        # one decode step of one short sequence: latency
        {"name": "attend_1x1_300_int4", "op": "attend", "kind": "int4", "s": 1, "l": 1, "heads": 32, "kv": 32,
         "dh": 128, "page": 16, "ctx": 300},
        # a decode step of a rollout batch of both streams, prompt and completion up to 800 tokens
        {"name": "attend_64x1_800_int4", "op": "attend", "kind": "int4", "s": 64, "l": 1, "heads": 32, "kv": 32,
         "dh": 128, "page": 16, "ctx": 800},
        # four drafts and the token before them over grouped heads
        {"name": "attend_16x5_4096_int4", "op": "attend", "kind": "int4", "s": 16, "l": 5, "heads": 32, "kv": 8,
         "dh": 128, "page": 64, "ctx": 4096},
        # few sequences with very long contexts
        {"name": "attend_3x1_131072_int4", "op": "attend", "kind": "int4", "s": 3, "l": 1, "heads": 32, "kv": 8,
         "dh": 128, "page": 128, "ctx": 131072},
        # an odd batch of drafted tokens with heads of 64 over an unquantised cache
        {"name": "attend_13x7_2000_bf16", "op": "attend", "kind": "bf16", "s": 13, "l": 7, "heads": 12, "kv": 4,
         "dh": 64, "page": 32, "ctx": 2000},
        # one sequence's four drafts
        {"name": "verify_1x4x32000_f32", "op": "verify", "s": 1, "d": 4, "v": 32000, "ld": 32000, "type": "f32",
         "mode": "draft", "mask": "none"},
        # a batch's drafts
        {"name": "verify_64x4x32000_f32", "op": "verify", "s": 64, "d": 4, "v": 32000, "ld": 32000, "type": "f32",
         "mode": "draft", "mask": "none"},
        # constrained decoding: forbidden tokens at -inf, an odd vocabulary, rows at odd strides
        {"name": "verify_37x7x50001_bf16", "op": "verify", "s": 37, "d": 7, "v": 50001, "ld": 50003, "type": "bf16",
         "mode": "draft", "mask": "inf"},
        # drafts copied from earlier text, greedy decoding, a large vocabulary
        {"name": "verify_24x8x128000_greedy", "op": "verify", "s": 24, "d": 8, "v": 128000, "ld": 128000,
         "type": "bf16", "mode": "greedy", "mask": "none"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "verify"])
    while True:
        if op == "verify":
            v = rng.choice([32000, _log(rng, 1000, 152000), 8 * _log(rng, 125, 19000)])
            c = {"op": op, "s": _log(rng, 1, 128), "d": rng.randint(1, 8), "v": v,
                 "ld": v + rng.choice([0, 0, rng.randint(1, 9), 64]), "type": rng.choice(["f32", "bf16"]),
                 "mode": rng.choice(["draft", "draft", "given", "greedy"]),
                 "mask": rng.choice(["none", "none", "inf", "lowest"])}
            if work(c)["bytes"] <= 45e6:
                return c
            continue
        kv = rng.choice([1, 2, 4, 8, 8, 32, rng.randint(1, 32)])
        c = {"op": op, "kind": rng.choice(["int4", "int4", "bf16"]), "s": _log(rng, 1, 128),
             "l": rng.choice([1, 1, rng.randint(2, 8), rng.randint(2, 16)]) if op == "attend" else
             rng.choice([1, rng.randint(2, 8), _log(rng, 8, 700)]),
             "heads": kv * (1 if kv > 16 else rng.choice([1, 2, 4, rng.randint(1, 8)])), "kv": kv,
             "dh": rng.choice([64, 128, 128]), "page": rng.choice([16, 32, 64, 128])}
        c["cached" if op == "append" else "ctx"] = _log(rng, c["l"], 30000)
        w = work(c)
        if w["bytes"] <= (100e6 if op == "append" else 200e6) and w["flops"] <= 4e9:
            if c["s"] * c.get("ctx", c.get("cached", 0)) * kv * c["dh"] <= 3e8:
                return c


# --------------------------------------------------------------------------- inputs


def _spread(s, n, least=0.25):
    """A quarter of n to all of it over the sequences."""
    return [n] if s == 1 else [max(1, round(n * (least + (1 - least) * i / (s - 1)))) for i in range(s)]


def _counts(case):
    """(tokens in the cache before the call, new tokens) of each sequence; which has which is up to the seed."""
    s, l = case["s"], case["l"]
    new = _spread(s, l, 0.0)
    if s > 6:
        new[s // 2] = 0  # a sequence that has ended
    if case["op"] == "append":
        return [0] * s if case["cached"] == 0 else _spread(s, case["cached"]), new
    return [max(0, n - m) for n, m in zip(_spread(s, case["ctx"]), new)], new


def _drafts(case):
    return [case["d"]] if case["s"] == 1 else [round(case["d"] * i / (case["s"] - 1)) for i in range(case["s"])]


def _tile_bytes(case):
    d = case["dh"]
    return TILE * (d + 8 * d // GROUP) if case["kind"] == "int4" else TILE * 4 * d


def _quantise(x):
    """(codes, scales, zeros) of fp32 [..., D]: one scale and zero point for each group of channels."""
    x = x.unflatten(-1, (-1, GROUP))
    lo, hi = x.amin(-1, keepdim=True).clamp(max=0), x.amax(-1, keepdim=True).clamp(min=0)
    scale = ((hi * 0.5 - lo * 0.5) * torch.tensor(2 / 15, device=DEV)).bfloat16().float()
    some = scale > 0
    by = torch.where(some, scale, 1.0)
    zero = torch.where(some, (-lo / by).round().clamp(0, 15), 0.0)
    codes = torch.where(some, ((x / by).round() + zero).clamp(0, 15), 0.0)
    return codes, scale, zero


def _bytes(x):
    return x.contiguous().view(torch.uint8).flatten(3)


def _pack(k, v, kind):
    """The bytes [pages, heads, ...] of values [pages, heads, page, D] (4 bits: quantised here)."""
    pages, heads, page, d = k.shape
    k, v = (x.reshape(pages, heads, page // TILE, TILE, d) for x in (k, v))
    if kind == "bf16":
        k = k.bfloat16().unflatten(-1, (-1, 32)).transpose(3, 4)
        v = v.bfloat16().unflatten(4, (-1, 8, 4)).unflatten(3, (2, 4, 2)).permute(0, 1, 2, 3, 6, 7, 4, 8, 5)
        return torch.cat([_bytes(k), _bytes(v)], 3).flatten(2)
    (kc, ks, kz), (vc, vs, vz) = _quantise(k.float()), _quantise(v.float())
    # [pages, heads, tiles, token, group, channel]
    kc = kc.byte().unflatten(-1, (4, 8, 2)).permute(0, 1, 2, 3, 5, 4, 6, 7)
    kc = kc[..., 0] | kc[..., 1] << 4
    vc = vc.byte().unflatten(-1, (8, 2, 2, 2)).unflatten(3, (2, 4, 2)).permute(0, 1, 2, 3, 7, 4, 6, 8, 5, 9, 10)
    vc = vc[..., 0] | vc[..., 1] << 4
    scales = torch.stack([ks[..., 0], vs[..., 0]], 4).bfloat16().unflatten(3, (2, 8)).transpose(3, 4)
    kz, vz = ((x[..., 0] * 17).short() for x in (kz, vz))
    kz = kz.unflatten(3, (2, 8)).transpose(3, 4)
    vz = vz.unflatten(3, (2, 4, 2)).permute(0, 1, 2, 4, 3, 6, 5)
    return torch.cat([_bytes(x) for x in (kc, vc, scales, kz, vz)], 3).flatten(2)


def _values(raw, case):
    """fp32 keys and values [..., page, D] of a cache's bytes [..., bytes of a page's head]."""
    d, groups, lead = case["dh"], case["dh"] // GROUP, raw.shape[:-1]
    raw = raw.reshape(-1, _tile_bytes(case))
    if case["kind"] == "bf16":
        k, v = raw.view(torch.bfloat16).float().split(TILE * d, 1)
        k = k.reshape(-1, d // 32, TILE, 32).transpose(1, 2)
        v = v.reshape(-1, 2, d // 32, 8, 4, 4, 2).permute(0, 1, 4, 6, 2, 3, 5)
        return tuple(x.reshape(*lead, -1, d) for x in (k, v))
    kc, vc, scales, kz, vz = raw.split([TILE * d // 2] * 2 + [TILE * 4 * groups] + [TILE * 2 * groups] * 2, 1)
    kc, vc = (torch.stack([x & 15, x >> 4], -1).float() for x in (kc, vc))
    kc = kc.reshape(-1, TILE, 4, groups, 16).transpose(2, 3).reshape(-1, TILE, groups, GROUP)
    vc = vc.reshape(-1, 2, 8, 4, groups, 2, 2, 4).permute(0, 1, 3, 6, 4, 2, 5, 7).reshape(-1, TILE, groups, GROUP)
    scales = scales.contiguous().view(torch.bfloat16).float().reshape(-1, 8, 2, 2, groups).transpose(1, 2)
    ks, vs = scales.reshape(-1, TILE, 2, groups).unbind(2)
    kz, vz = (x.contiguous().view(torch.int16).float() / 17 for x in (kz, vz))
    kz = kz.reshape(-1, 8, 2, groups).transpose(1, 2).reshape(-1, TILE, groups)
    vz = vz.reshape(-1, 4, 2, groups, 2).permute(0, 2, 1, 4, 3).reshape(-1, TILE, groups)
    k, v = ((c - z[..., None]) * s[..., None] for c, z, s in ((kc, kz, ks), (vc, vz, vs)))
    return tuple(x.reshape(*lead, -1, d) for x in (k, v))


def _rope(positions, d):
    """(cos, sin) of every position and pair of channels."""
    angle = torch.arange(positions, device=DEV, dtype=torch.float64)[:, None] * 10000.0 ** (
        -torch.arange(0, d, 2, device=DEV, dtype=torch.float64) / d)
    return torch.stack([angle.cos(), angle.sin()], -1).float()


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    if case["op"] == "verify":
        return _prepare_verify(case, g)
    t = {"case": case}
    s, l, heads, kv, d, page = (case[k] for k in ("s", "l", "heads", "kv", "dh", "page"))
    order = torch.randperm(s, device=DEV, generator=g)
    cached, new = (torch.tensor(x, dtype=torch.int32, device=DEV)[order] for x in _counts(case))
    t["cached"], t["new"] = cached, new
    used = (cached + new + page - 1) // page
    width = -(-(max(a + b for a, b in zip(*_counts(case)))) // page) + 1
    n_pages = sum(-(-(a + b) // page) for a, b in zip(*_counts(case))) + 3
    column = torch.arange(width, device=DEV)[None]
    at = (used.cumsum(0) - used)[:, None] + column
    shuffled = torch.randperm(n_pages, device=DEV, generator=g).int()
    t["table"] = torch.where(column < used[:, None], shuffled[at.clamp(max=n_pages - 1)], -1).int()
    size = _tile_bytes(case) * (page // TILE)
    qkv = torch.randn(s * l, (heads + 2 * kv) * d, device=DEV, generator=g).bfloat16()
    loud = 0.4 * torch.randn(kv, 1, d, device=DEV, generator=g)  # channels of keys have scales of their own
    if case["op"] == "append":
        qkv.unflatten(1, (-1, d))[:, heads:heads + kv] *= loud.exp()[:, 0]
        t["raw"] = torch.full((n_pages, kv, size), 255, dtype=torch.uint8, device=DEV)
        t["rope"] = _rope(int(max(a + b for a, b in zip(*_counts(case)))), d)
        t["k"], t["v"] = qkv[:, heads * d:(heads + kv) * d], qkv[:, (heads + kv) * d:]
        t["k_out"], t["v_out"] = torch.empty(2, s * l, kv * d, dtype=torch.bfloat16, device=DEV)
    else:
        k = torch.randn(n_pages, kv, page, d, device=DEV, generator=g).mul_(loud.exp())
        v = torch.randn(n_pages, kv, page, d, device=DEV, generator=g)
        v *= 10 ** (torch.rand(n_pages, kv, page, 1, device=DEV, generator=g) * 0.6 - 0.3)
        t["raw"] = _pack(k, v, case["kind"])
    t["q"] = qkv[:, :heads * d]
    t["out"] = torch.empty(s * l, heads * d, dtype=torch.bfloat16, device=DEV)
    return t


def _prepare_verify(case, g):
    t = {"case": case}
    s, d, v, ld, dt = (case[k] for k in ("s", "d", "v", "ld", "type"))
    scale = 10 ** (torch.rand(s, 1, 1, device=DEV, generator=g) * 0.8 - 0.4)
    z = torch.randn(s, d + 1, v, device=DEV, generator=g) * scale
    z -= 2.0 * torch.log(1e-3 + torch.rand(1, 1, v, device=DEV, generator=g))  # common tokens
    w = z[:, :d] + 0.4 * torch.randn(s, d, v, device=DEV, generator=g)         # a draft model near the target
    if case["mask"] != "none":
        low = -math.inf if case["mask"] == "inf" else torch.finfo(TYPES[dt]).min
        z.masked_fill_(torch.rand(s, d + 1, v, device=DEV, generator=g) < 0.7, low)
        # the draft model knows most of the forbidden tokens
        w.masked_fill_((z[:, :d] == low) & (torch.rand(s, d, v, device=DEV, generator=g) < 0.9999), low)
    if case["mode"] == "greedy":
        ids = z[:, :d].argmax(2)
        other = torch.randint(0, v, (s, d), device=DEV, generator=g)
        ids = torch.where(torch.rand(s, d, device=DEV, generator=g) < 0.8, ids, other)
    else:
        u = torch.rand(s, d, v, device=DEV, generator=g).clamp_(1e-20, 1 - 1e-7)
        ids = (w - torch.log(-torch.log(u))).argmax(2)
    t["ids"] = ids.int()
    for name, x in (("z", z), ("w", w)):
        whole = torch.zeros(x.shape[0] * x.shape[1], ld, dtype=TYPES[dt], device=DEV)
        whole[:, :v] = x.flatten(0, 1)
        t[name] = whole[:, :v]
    if case["mode"] != "draft":
        t["w"] = None
    t["drafts"] = torch.tensor(_drafts(case), dtype=torch.int32, device=DEV)[
        torch.randperm(s, device=DEV, generator=g)]
    t["u"] = t["noise"] = None
    if case["mode"] != "greedy":
        t["u"] = torch.rand(s, d, device=DEV, generator=g)
        t["noise"] = -torch.log(-torch.log(torch.rand(s, v, device=DEV, generator=g).clamp_(1e-20, 1 - 1e-7)))
    t["tokens"] = torch.full((s, d + 1), -7, dtype=torch.int32, device=DEV)
    t["accepted"] = torch.full((s,), -7, dtype=torch.int32, device=DEV)
    t["logp"] = torch.full((s, d + 1), math.nan, device=DEV)
    t["accept"] = torch.full((s, d), math.nan, device=DEV)
    return t


# --------------------------------------------------------------------------- one pass


def run(t):
    op = t["case"]["op"]
    if op == "append":
        return _append_own(t) if own else _append(t)
    if op == "attend":
        return _attend_own(t) if own else _attend(t)
    return _verify_own(t) if own else _verify(t)


def _cache(t):
    from paper_2309_00754_gb300 import hydra as H

    if "cache" not in t:  # a program keeps the cache's handle
        c = t["case"]
        kind = H.HYDRA_KV_INT4 if c["kind"] == "int4" else H.HYDRA_KV_BF16
        t["cache"] = H.KvCache(kind, t["raw"].shape[0], c["page"], c["kv"], c["dh"], data=t["raw"])
    return t["cache"]


def _append_own(t):
    from paper_2309_00754_gb300 import hydra as H

    c, cache = t["case"], _cache(t)
    H.hydra_kv_append(cache, t["table"], t["cached"], t["new"], c["s"], c["l"], t["q"], t["k"], t["v"], t["rope"],
                      t["out"])
    H.hydra_kv_read(cache, t["table"], t["cached"], t["new"], c["s"], c["l"], t["k_out"], t["v_out"])
    return {"q": t["out"], "k": t["k_out"], "v": t["v_out"]}


def _attend_own(t):
    from paper_2309_00754_gb300 import hydra as H

    c, cache = t["case"], _cache(t)
    if "ws" not in t:
        n = H.paged_attention_workspace_size(c["s"], c["l"], c["heads"], c["kv"], c["dh"])
        t["ws"] = torch.empty(n, dtype=torch.uint8, device=DEV)
    H.hydra_paged_attention(cache, t["table"], t["cached"], t["new"], c["s"], c["l"], t["q"], t["out"],
                            c["dh"] ** -0.5, t["ws"])
    return t["out"]


def _verify_own(t):
    from paper_2309_00754_gb300 import hydra as H

    c = t["case"]
    H.hydra_verify_drafts(t["z"], t["w"], t["ids"], t["drafts"], t["u"], t["noise"], c["s"], c["d"], t["tokens"],
                          t["accepted"], t["logp"], t["accept"])
    return {k: t[k] for k in ("tokens", "accepted", "logp", "accept")}


def _positions(t):
    """The position of every slot [S, L], and whether a token stands there."""
    slot = torch.arange(t["case"]["l"], device=DEV)[None]
    return t["cached"][:, None] + slot, slot < t["new"][:, None]


def _append(t):
    c = t["case"]
    s, l, d, kv = c["s"], c["l"], c["dh"], c["kv"]
    at, live = _positions(t)
    q, k, v = (t[x].reshape(s, l, -1, d).float() for x in ("q", "k", "v"))
    cos, sin = t["rope"][at.clamp(max=len(t["rope"]) - 1)][:, :, None].unbind(-1)

    def turn(x):
        a, b = x.chunk(2, -1)
        return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)

    q, k = turn(q), turn(k)
    if c["kind"] == "int4":
        k, v = (((codes - zero) * scale).flatten(-2) for codes, scale, zero in (_quantise(k), _quantise(v)))
    rows = t["raw"].shape[0] * c["page"]
    if "pool" not in t:  # a row more, for the slots without a token
        t["pool"] = torch.full((2, rows + 1, kv, d), math.nan, dtype=torch.bfloat16, device=DEV)
    page = t["table"].gather(1, (at // c["page"]).clamp(max=t["table"].shape[1] - 1).long())
    row = torch.where(live, page * c["page"] + at % c["page"], rows).long()
    t["pool"][0, row.flatten()] = k.bfloat16().flatten(0, 1)
    t["pool"][1, row.flatten()] = v.bfloat16().flatten(0, 1)
    k, v = (torch.where(live[..., None, None], x[row], 0.0).reshape(s * l, -1) for x in t["pool"])
    return {"q": torch.where(live[..., None, None], q, 0.0).bfloat16().reshape(s * l, -1), "k": k, "v": v}


def _attend(t):
    c = t["case"]
    s, l, d, kv = c["s"], c["l"], c["dh"], c["kv"]
    at, live = _positions(t)
    raw = t["raw"][t["table"].clamp(min=0).long()]
    k, v = (x.transpose(1, 2).reshape(s, kv, -1, d) for x in _values(raw, c))
    seen = torch.arange(k.shape[2], device=DEV)
    # nothing of what lies behind a sequence's end is used
    inside = (seen[None] < (t["cached"] + t["new"])[:, None])[:, None, :, None]
    k, v = (torch.where(inside, x, 0.0) for x in (k, v))
    q = t["q"].reshape(s, l, kv, -1, d).float().permute(0, 2, 3, 1, 4)  # [S, Hk, G, L, D]
    scores = (q.flatten(2, 3) @ k.transpose(2, 3) * d ** -0.5).unflatten(2, (-1, l))
    scores = scores.masked_fill((seen[None, None] > at[..., None])[:, None, None], -math.inf)
    e = (scores - scores.amax(-1, keepdim=True)).exp()
    p = e / e.sum(-1, keepdim=True)
    o = (p.flatten(2, 3) @ v).unflatten(2, (-1, l)).permute(0, 3, 1, 2, 4).reshape(s * l, -1)
    return torch.where(live.reshape(-1, 1), o, 0.0).bfloat16()


def _verify(t):
    c = t["case"]
    s, d, v = c["s"], c["d"], c["v"]
    step = torch.arange(d, device=DEV)[None]
    inside = step < t["drafts"][:, None]
    z = t["z"].reshape(s, d + 1, v).double()
    lp = z - z.amax(2, keepdim=True)
    lp = lp - lp.exp().sum(2, keepdim=True).log()
    ids = t["ids"].long()
    hit = lp[:, :d].gather(2, ids[..., None])[..., 0]
    if c["mode"] == "greedy":
        accept = (z[:, :d].argmax(2) == ids).double()
        go = accept > 0.5
    else:
        if t["w"] is None:
            accept = hit.exp()
        else:
            w = t["w"].reshape(s, d, v).double()
            lq = w - w.amax(2, keepdim=True)
            lq = lq - lq.exp().sum(2, keepdim=True).log()
            chance = lq.gather(2, ids[..., None])[..., 0]
            accept = torch.where(hit == -math.inf, 0.0, (hit - chance).exp().clamp(max=1.0))
        go = t["u"] < accept.float()
    n = (inside & go).long().cumprod(1).sum(1)
    last = z[torch.arange(s, device=DEV), n]
    score = last.float()
    if c["mode"] != "greedy":
        refused = (n < t["drafts"])[:, None]
        at = n.clamp(max=d - 1)
        row = torch.arange(s, device=DEV)
        if t["w"] is None:
            rest = torch.where(torch.arange(v, device=DEV)[None] == ids[row, at][:, None], -math.inf, last.float())
        else:
            rest = (lp[row, at].exp() - lq[row, at].exp()).clamp(min=0).log().float()
        some = (rest > -math.inf).any(1, keepdim=True)
        score = torch.where(refused & some, rest, score) + t["noise"]
    then = score.argmax(1)
    slot = torch.arange(d + 1, device=DEV)[None]
    tokens = torch.where(slot < n[:, None], torch.cat([ids, ids[:, :1]], 1), then[:, None])
    logp = lp.gather(2, tokens[..., None])[..., 0]
    there = slot <= n[:, None]
    return {"tokens": torch.where(there, tokens, -1).int(), "accepted": n.int(),
            "logp": torch.where(there, logp, 0.0).float(), "accept": torch.where(inside, accept, 0.0).float()}


# --------------------------------------------------------------------------- work


def work(case):
    if case["op"] == "verify":
        n, s, v = sum(_drafts(case)), case["s"], case["v"]
        size = 4 if case["type"] == "f32" else 2
        rows = n + s + (n if case["mode"] == "draft" else 0)
        noise = 4 * s * v if case["mode"] != "greedy" else 0
        return {"bytes": rows * v * size + noise + 4 * (3 * s * case["d"] + 2 * s + 2 * s * (case["d"] + 1)),
                "flops": 4 * rows * v}
    s, l, d, heads, kv = (case[k] for k in ("s", "l", "dh", "heads", "kv"))
    cached, new = _counts(case)
    token = kv * _tile_bytes(case) // TILE
    if case["op"] == "append":
        n = sum(new)
        dense = 2 * d * (2 * n * (heads + 2 * kv) + (s * l - n) * (heads + 2 * kv))
        rope = 4 * d * len({a + i for a, b in zip(cached, new) for i in range(b)})
        return {"bytes": dense + rope + 2 * n * token, "flops": n * d * (3 * (heads + kv) + 8 * kv)}
    seen = sum(a + b for a, b in zip(cached, new) if b)
    table = sum(-(-(a + b) // case["page"]) for a, b in zip(cached, new) if b)
    return {"bytes": seen * token + 2 * d * heads * (sum(new) + s * l) + 4 * table + 8 * s,
            "flops": 4 * heads * d * sum(b * a + b * (b + 1) // 2 for a, b in zip(cached, new))}


# --------------------------------------------------------------------------- 64 bits


def exact(case, seed):
    t = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "verify": _exact_verify}[case["op"]](case, t)


def _exact_append(case, t):
    """Rows one sequence at a time, from the definition: angles, groups, codes."""
    s, l, d = case["s"], case["l"], case["dh"]
    out = {x: torch.zeros(s, l, t[x].shape[1] // d, d, dtype=torch.float64, device=DEV) for x in ("q", "k", "v")}
    for i, (first, n) in enumerate(zip(t["cached"].tolist(), t["new"].tolist())):
        if n == 0:
            continue
        turn = torch.view_as_complex(t["rope"][first:first + n].double())[:, None]
        for x in ("q", "k", "v"):
            y = t[x].double().view(s, l, -1, d)[i, :n]
            if x != "v":
                y = torch.complex(y[..., :d // 2], y[..., d // 2:]) * turn
                y = torch.cat([y.real, y.imag], -1)
            if x != "q" and case["kind"] == "int4":
                parts = y.view(n, -1, d // GROUP, GROUP)
                low = parts.min(-1, keepdim=True).values.clamp_max(0)
                high = parts.max(-1, keepdim=True).values.clamp_min(0)
                step = ((high - low) / 15).to(torch.bfloat16).double()
                safe = step.masked_fill(step == 0, 1)
                zero = torch.round(-low / safe).clamp(0, 15)
                code = torch.clamp(torch.round(parts / safe) + zero, 0, 15)
                y = ((code - zero) * step).view(n, -1, d)
            out[x][i, :n] = y
    return {k: x.view(s * l, -1) for k, x in out.items()}


def _held(raw, case):
    """Keys and values [tokens, D] that the pages' bytes of one head stand for, each found by its address."""
    d, groups, size = case["dh"], case["dh"] // GROUP, _tile_bytes(case)
    raw = raw.reshape(-1)
    at = torch.arange(len(raw) // size * TILE, device=DEV)[:, None]
    base, tok, ch = at // TILE * size, at % TILE, torch.arange(d, device=DEV)[None]
    p, t, b = tok // 8, tok % 8 // 2, tok % 2
    if case["kind"] == "bf16":
        held = raw.view(torch.bfloat16).double()
        key = (ch // 32 * TILE + tok) * 32 + ch % 32
        value = TILE * d + (((p * (d // 32) + ch // 32) * 8 + ch % 32 // 4) * 4 + t) * 8 + ch % 4 * 2 + b
        return held[base // 2 + key], held[base // 2 + value]

    def word(where):
        return raw[where].long() + 256 * raw[where + 1].long()

    def scale(where):
        return (word(where) << 16).int().view(torch.float32).double()

    def code(where, n):
        return (raw[where + n // 2].long() >> (n % 2 * 4)) & 15

    grp, inner = ch // GROUP, ch % GROUP
    scales = base + TILE * d
    zeros = scales + TILE * 4 * groups
    by_token = (tok % 8 * 2 + tok // 8) * 2
    key = code(base + tok * (d // 2) + (inner // 16 * groups + grp) * 8, ch % 16)
    lane = (p * 8 + inner // 8) * 4 + t
    value = code(base + TILE * d // 2 + (lane * groups + grp) * 8 + inner % 8 // 4 * 4 + b * 2, ch % 4)
    zero_k = word(zeros + by_token * groups + grp * 2) // 17
    zero_v = word(zeros + TILE * 2 * groups + ((t * 2 + p) * groups + grp) * 4 + b * 2) // 17
    return ((key - zero_k) * scale(scales + by_token * 2 * groups + grp * 2),
            (value - zero_v) * scale(scales + by_token * 2 * groups + (groups + grp) * 2))


def _exact_attend(case, t):
    s, l, d, kv = case["s"], case["l"], case["dh"], case["kv"]
    group = case["heads"] // kv
    out = torch.zeros(s, l, kv, group, d, dtype=torch.float64, device=DEV)
    for i, (first, n) in enumerate(zip(t["cached"].tolist(), t["new"].tolist())):
        if n == 0:
            continue
        pages = t["table"][i, :-(-(first + n) // case["page"])].long()
        for h in range(kv):
            k, v = (x[:first + n] for x in _held(t["raw"][pages, h], case))
            q = t["q"].double().view(s, l, kv, group, d)[i, :n, h].reshape(-1, d)
            logits = torch.einsum("rd,kd->rk", q, k) / math.sqrt(d)
            last = torch.arange(n, device=DEV).repeat_interleave(group) + first
            logits[torch.arange(first + n, device=DEV)[None] > last[:, None]] = -math.inf
            out[i, :n, h] = torch.einsum("rk,kd->rd", torch.softmax(logits, 1), v).view(n, group, d)
    return out.view(s * l, -1)


def _exact_verify(case, t):
    s, d, v = case["s"], case["d"], case["v"]
    out = {"tokens": torch.full((s, d + 1), -1, dtype=torch.int32), "accepted": torch.zeros(s, dtype=torch.int32),
           "logp": torch.zeros(s, d + 1, dtype=torch.float64), "accept": torch.zeros(s, d, dtype=torch.float64)}
    for i, n in enumerate(t["drafts"].tolist()):
        z = t["z"][i * (d + 1):(i + 1) * (d + 1)].double()
        p = torch.log_softmax(z, 1)
        ids = t["ids"][i].tolist()
        q = torch.log_softmax(t["w"][i * d:(i + 1) * d].double(), 1) if t["w"] is not None else None
        going, follow = True, []
        for j in range(n):
            x = ids[j]
            if case["mode"] == "greedy":
                a = float(torch.argmax(z[j]) == x)
            else:
                a = min(1.0, math.exp(float(p[j, x]) - (float(q[j, x]) if q is not None else 0.0)))
            out["accept"][i, j] = a
            if going:
                going = a > 0.5 if case["mode"] == "greedy" else float(t["u"][i, j]) < a
                if going:
                    follow.append(x)
        j = len(follow)
        score = z[j].clone()
        if case["mode"] != "greedy":
            if not going:
                rest = score.index_fill(0, torch.tensor(ids[j], device=DEV), -math.inf) if q is None else torch.log(
                    torch.relu(p[j].exp() - q[j].exp()))
                score = rest if bool((rest > -math.inf).any()) else score
            score = score + t["noise"][i].double()
        follow.append(int(torch.argmax(score)))
        out["accepted"][i] = j
        for at, x in enumerate(follow):
            out["tokens"][i, at] = x
            out["logp"][i, at] = p[at, x]
    return out
