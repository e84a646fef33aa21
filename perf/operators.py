"""Performance cases of the operators around the mixed-precision cache of one attention layer, on one MI355X:

  rotary      rotary positions of a projection's queries and keys, its values converted and laid out with them;
  attend      attention of whole prompts under score rules (tanh cap, distance bias, documents, prefix, window);
  importance  the prompt tokens' H2O scores under the same rules, from the attention's log-sum-exp;
  decode      attention of one new token over a filled mixed-precision cache under the same rules.

Shapes and precisions are those of the package's workloads and of its tests, plus ragged lengths.
"""
from __future__ import annotations

import math

import torch

own = False

D = 128
SCALE = 1.0 / math.sqrt(128.0)
DEV = "cuda"
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


def _rotary(name, batch, tokens, q_heads, kv_heads, x="fp16", y="fp16", rot=128, interleaved=False, scaling="none", factor=1.0,
            original=4096, base=10000.0, first=0, ragged=False, packed=True):
    c = dict(kind="rotary", batch=batch, tokens=tokens, q_heads=q_heads, kv_heads=kv_heads, x=x, y=y, rot=rot,
             interleaved=interleaved, scaling=scaling, factor=factor, original=original, base=base, first=first, ragged=ragged,
             packed=packed)
    return c if name is None else dict(c, name=name)


def _prompt(name, kind, batch, tokens, q_heads, kv_heads, cap=0.0, bias=False, docs=0, prefix=False, window=0, packed=False,
            pad=False):
    c = dict(kind=kind, batch=batch, tokens=tokens, q_heads=q_heads, kv_heads=kv_heads, cap=cap, bias=bias, docs=docs,
             prefix=prefix, window=window, packed=packed, pad=pad)
    return c if name is None else dict(c, name=name)


def _decode(name, batch, q_heads, kv_heads, length, hi=16, lo=2, group=32, num=1, den=10, recent=64, cap=0.0, bias=False,
            begin=False):
    c = dict(kind="decode", batch=batch, q_heads=q_heads, kv_heads=kv_heads, length=length, hi=hi, lo=lo, group=group, num=num,
             den=den, recent=recent, cap=cap, bias=bias, begin=begin)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # One request's next token far into a context that was stretched eight times: launch latency.
        _rotary("rotary_token", 1, 1, 32, 8, scaling="yarn", factor=8.0, first=30011),
        # A batch of prompts of no round length, bf16 projection, half of each head rotated, pairs of neighbours.
        _rotary("rotary_partial", 3, 1531, 40, 40, x="bf16", rot=64, interleaved=True, ragged=True),
        # A served batch's prompts from the projection into the cache's layout (the llama2_7b workload's sizes).
        _rotary("rotary_prompt", 8, 4096, 32, 32, scaling="bands", factor=4.0),
        # A few tokens with four heads: the smallest attention, where launches count.
        _prompt("attend_tiny", "attend", 1, 77, 4, 4, bias=True),
        # Prompts of the llama2_7b workload for a model that caps its scores.
        _prompt("attend_capped", "attend", 8, 4096, 32, 32, cap=50.0),
        # Prompts packed of documents and padded, GQA, straight from the fused projection's rows.
        _prompt("attend_documents", "attend", 16, 2011, 32, 8, docs=6, packed=True, pad=True),
        # A prefix that sees itself both ways and a bias by distance, 13B heads, no round length.
        _prompt("attend_prefix", "attend", 2, 1531, 40, 40, bias=True, prefix=True),
        # One long prompt under GQA with a sliding window (the mistral_7b workload's length).
        _prompt("attend_long", "attend", 1, 16384, 32, 8, window=4096),
        # Scores of a short prompt under a distance bias (the tiny workload's size).
        _prompt("importance_tiny", "importance", 1, 512, 4, 4, bias=True),
        # Scores of a served batch's packed prompts with capped scores, GQA.
        _prompt("importance_documents", "importance", 8, 4096, 32, 8, cap=30.0, docs=3, pad=True),
        # One request being decoded under a distance bias, its first tokens padding: INT3 retained pool, no round length.
        _decode("decode_bias", 1, 40, 40, 5003, hi=16, lo=3, group=64, num=1, den=5, recent=33, bias=True, begin=True),
        # A served batch under GQA with capped scores (the mistral_7b workload).
        _decode("decode_capped", 16, 32, 8, 16384, hi=16, lo=2, group=32, num=1, den=10, recent=128, cap=50.0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: every kind, type, head layout and rule, sizes over the listed range."""
    kind = rng.choice(("rotary", "attend", "attend", "importance", "decode"))
    G = rng.choice((1, 1, 2, 4, 8))
    Hkv = rng.choice((4, 8, 32, 40) if G == 1 else (4, 8))
    Hq = Hkv * G
    if kind == "rotary":
        T = rng.choice((1, _log_int(rng, 2, 8192)))
        B = _log_int(rng, 1, max(1, min(64, (8 * 4096 * 96) // (T * (Hq + 2 * Hkv)))))
        x = rng.choice(("fp16", "bf16", "fp32"))
        scaling = rng.choice(("none", "linear", "ntk", "bands", "yarn"))
        return _rotary(None, B, T, Hq, Hkv, x=x, y=rng.choice(("fp16", x)), rot=rng.choice((128, 128, 96, 64, 32, 20)),
                       interleaved=rng.random() < 0.5, scaling=scaling, factor=1.0 if scaling == "none" else rng.choice((2.0, 4.0, 8.0)),
                       base=rng.choice((10000.0, 500000.0)), first=rng.choice((0, _log_int(rng, 1, 1000000))),
                       ragged=rng.random() < 0.5, packed=rng.random() < 0.7)
    if kind == "decode":
        L = _log_int(rng, 300, 32768)
        B = _log_int(rng, 1, max(1, min(16, (16 * 8 * 16384) // (Hkv * L))))
        hi, lo = rng.choice(((16, 2), (16, 2), (8, 2), (8, 4), (16, 4), (16, 3), (4, 2), (16, 0)))
        return _decode(None, B, Hq, Hkv, L, hi=hi, lo=lo, group=rng.choice((32, 64)), den=rng.choice((4, 5, 10)),
                       recent=rng.choice((32, 33, 64, 128)), cap=rng.choice((0.0, 30.0, 50.0)), bias=rng.random() < 0.5,
                       begin=rng.random() < 0.5)
    T = _log_int(rng, 1, 16384)
    B = _log_int(rng, 1, max(1, min(16, (1 << 32) // (Hq * T * T))))
    if Hq * T * T > 1 << 33:
        T = int(math.sqrt((1 << 33) / Hq))
    docs = rng.choice((0, 0, _log_int(rng, 1, 9)))
    return _prompt(None, kind, B, T, Hq, Hkv, cap=rng.choice((0.0, 0.0, 30.0, 50.0)), bias=rng.random() < 0.35, docs=min(docs, T),
                   prefix=rng.random() < 0.25, window=rng.choice((0, 0, 0, _log_int(rng, 1, 4096))), packed=rng.random() < 0.5,
                   pad=docs > 0 and rng.random() < 0.6)


# -- inputs -----------------------------------------------------------------------------

def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) % (1 << 40)) * 16 + stream)
    return g


def _randn(shape, g, scale=None):
    x = torch.randn(shape, generator=g, device=DEV)
    return x if scale is None else x * scale


def _outliers(heads, g):
    """Factors of the channels of every head: four fixed outlier channels in rotary pairs, as the workloads have them."""
    f = torch.ones(heads, D, device=DEV)
    at = torch.randint(0, D // 2, (heads, 2), generator=g, device=DEV)
    f.scatter_(1, at, 4.0)
    f.scatter_(1, at + D // 2, 4.0)
    return f


def _inverse_frequencies(c):
    """float64 [rot / 2] radians a position, and the factor on the rotated channels."""
    r, base, f, L0 = c["rot"], c["base"], c["factor"], float(c["original"])
    p = torch.arange(r // 2, dtype=torch.float64)
    w, m = base ** (-2.0 * p / r), 1.0
    if c["scaling"] == "linear":
        w = w / f
    elif c["scaling"] == "ntk":
        w = (base * f ** (r / (r - 2.0))) ** (-2.0 * p / r)
    elif c["scaling"] == "bands":
        keep = ((L0 * w / (2 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)
        w = w * keep + w / f * (1.0 - keep)
    elif c["scaling"] == "yarn":
        pair = lambda turns: r * math.log(L0 / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(0.0, math.floor(pair(32.0))), min(r - 1.0, math.ceil(pair(1.0)))
        ramp = ((p - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
        w = w / f * ramp + w * (1.0 - ramp)
        m = 0.1 * math.log(f) + 1.0
    return w, m


def _layout(x, packed):
    """x [B, H, T, 128] as it is, or as a view of [B, T, H, 128] rows."""
    return x.transpose(1, 2).contiguous().transpose(1, 2) if packed else x.contiguous()


def _prepare_rotary(c, seed):
    B, T, Hq, Hkv = c["batch"], c["tokens"], c["q_heads"], c["kv_heads"]
    g = _gen(seed, 0)
    rows = _randn((B, T, (Hq + 2 * Hkv) * D), g).to(TYPES[c["x"]])
    heads = rows.view(B, T, Hq + 2 * Hkv, D).transpose(1, 2)
    xs = [heads[:, :Hq], heads[:, Hq:Hq + Hkv], heads[:, Hq + Hkv:]]
    if not c["packed"]:
        xs = [x.contiguous() for x in xs]
    first = torch.full((B,), c["first"], device=DEV)
    if c["ragged"]:  # every sequence at a position of its own
        first = first + torch.randint(0, 257, (B,), generator=g, device=DEV)
    pos = (first[:, None] + torch.arange(T, device=DEV)).to(torch.int32).contiguous()
    w, m = _inverse_frequencies(c)
    s = dict(case=c, xs=xs, positions=pos, w=w.to(DEV), m=m,
             ys=[torch.empty(B, x.shape[1], T, D, dtype=TYPES[c["y"]], device=DEV) for x in xs])
    if own:
        from paper_2402_18096_amd import mikv
        s["rotary"] = mikv.MikvRotary(c["rot"], c["base"], interleaved=c["interleaved"], scaling=c["scaling"],
                                      factor=c["factor"], original_length=c["original"], device=DEV)
    return s


def _slopes(Hq):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / Hq) for h in range(Hq)], dtype=torch.float32, device=DEV)


def _prepare_prompt(c, seed):
    B, T, Hq, Hkv = c["batch"], c["tokens"], c["q_heads"], c["kv_heads"]
    g = _gen(seed, 1)
    f = _outliers(Hkv, g)
    q = _layout(_randn((B, Hq, T, D), g).half(), c["packed"])
    k = _layout((_randn((B, Hkv, T, D), g) * f[:, None]).half(), c["packed"])
    v = _layout(_randn((B, Hkv, T, D), g).half(), c["packed"])
    s = dict(case=c, q=q, k=k, v=v, slopes=_slopes(Hq) if c["bias"] else None, documents=None, prefix=None)
    if c["docs"]:
        # cuts at places of their own in every sequence; the last document is padding (-1) where the case pads
        n = c["docs"]
        cuts = torch.randint(1, max(2, T), (B, n), generator=g, device=DEV)
        ids = (torch.arange(T, device=DEV)[None, :, None] >= cuts[:, None, :]).sum(-1)
        if c["pad"]:
            ids = torch.where(ids == n, -1, ids)
        s["documents"] = ids.to(torch.int32).contiguous()
    if c["prefix"]:
        s["prefix"] = torch.randint(0, T // 2 + 1, (B,), generator=g, device=DEV).to(torch.int32)
    if c["kind"] == "importance":
        s["lse"] = _plain_attend(s)["lse"]
        s["v"] = None
        s["scores"] = torch.empty(B, Hkv, T, dtype=torch.float32, device=DEV)
    else:
        s["out"] = torch.empty(B, T, Hq, D, dtype=torch.float16, device=DEV).transpose(1, 2)
        s["lse"] = torch.empty(B, Hq, T, dtype=torch.float32, device=DEV)
    if c["docs"] or c["prefix"] or c["window"]:
        s["begin"] = torch.empty(B, T, dtype=torch.int32, device=DEV)
        s["end"] = torch.empty(B, T, dtype=torch.int32, device=DEV)
    if own and c["kind"] == "importance":
        from paper_2402_18096_amd import mikv
        s["ws"] = torch.empty(mikv.mikv_prompt_importance_workspace_size(B, Hq, Hkv, T), dtype=torch.uint8, device=DEV)
    return s


def _quantize(x, bits, group):
    """Codes uint8 [..., 128], scale and zero fp16 [..., 128 / group] of fp16 rows: asymmetric, per row and channel group,
    single precision with a correctly rounded quotient (taken in 64 bits, which rounds the same)."""
    y = x.float().unflatten(-1, (D // group, group))
    lo, hi = y.amin(-1), y.amax(-1)
    top = float((1 << bits) - 1)
    a, b = ((hi - lo).double() / top).float().half(), lo.half()
    af, bf = a.float()[..., None], b.float()[..., None]
    t = torch.where(af == 0, torch.zeros_like(y), ((y - bf).double() / af.double()).float())
    return t.round().clamp(0, top).to(torch.uint8).flatten(-2), a, b


def _prepare_decode(c, seed):
    B, Hq, Hkv, L = c["batch"], c["q_heads"], c["kv_heads"], c["length"]
    g = _gen(seed, 2)
    f = _outliers(Hkv, g)
    k = (_randn((B, Hkv, L, D), g) * f[:, None]).half()
    v = (_randn((B, Hkv, L, D), g) * f[:, None]).half()
    q = _randn((B, Hq, D), g).half()
    # the important tokens of every head: the recent ones and random others, as many in each
    n = min(L, c["recent"] + L * c["num"] // c["den"])
    order = torch.rand(B, Hkv, L, generator=g, device=DEV)
    order[..., L - min(L, c["recent"]):] = 2.0
    mask = torch.zeros(B, Hkv, L, dtype=torch.bool, device=DEV)
    mask.scatter_(2, order.topk(n, dim=-1).indices, True)
    begin = None
    if c["begin"]:
        begin = torch.randint(0, max(1, L // 4), (B,), generator=g, device=DEV).to(torch.int32)
    s = dict(case=c, q=q, slopes=_slopes(Hq) if c["bias"] else None, begin=begin, n=n)
    if own:
        from paper_2402_18096_amd import mikv
        cache = mikv.MikvCache(B, Hq, Hkv, c["group"], c["hi"], c["lo"], n, max(L - n, 1), L, DEV)
        mikv.mikv_quantize_kv(cache, k, v, 0, None, mask.to(torch.uint8))
        s["cache"] = cache
        s["out"] = torch.empty(B, Hq, D, dtype=torch.float32, device=DEV)
        s["probs_hi"] = torch.empty(B, Hq, cache.cap_hi, dtype=torch.float32, device=DEV)
        s["probs_lo"] = torch.empty(B, Hq, cache.cap_lo, dtype=torch.float32, device=DEV) if c["lo"] else None
        s["ws"] = torch.empty(mikv.mikv_decode_workspace_size(cache, L), dtype=torch.uint8, device=DEV)
    else:
        at = torch.arange(L, device=DEV).expand(B, Hkv, L)
        for pool, keep, bits in (("hi", mask, c["hi"]), ("lo", ~mask, c["lo"])):
            if bits == 0:
                continue
            m = int(keep[0, 0].sum())
            pos = at[keep].view(B, Hkv, m)
            rows = [x[keep].view(B, Hkv, m, D) for x in (k, v)]
            s[pool] = (pos, *[(x,) if bits == 16 else _quantize(x, bits, c["group"]) for x in rows])
    return s


def prepare(case, seed):
    if case["kind"] == "rotary":
        return _prepare_rotary(case, seed)
    return _prepare_decode(case, seed) if case["kind"] == "decode" else _prepare_prompt(case, seed)


# -- the plain forms ----------------------------------------------------------------------

def _plain_rotary(s):
    c = s["case"]
    r = c["rot"]
    angle = s["positions"].double()[:, None, :, None] * s["w"]  # [B, 1, T, r / 2]
    cos, sin = (angle.cos() * s["m"]).float(), (angle.sin() * s["m"]).float()

    def turn(x):
        y = x[..., :r].float()
        if c["interleaved"]:
            a, b = y[..., 0::2], y[..., 1::2]
            y = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=-1).flatten(-2)
        else:
            a, b = y[..., :r // 2], y[..., r // 2:]
            y = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)
        return torch.cat((y, x[..., r:].float()), dim=-1).to(TYPES[c["y"]]).contiguous()

    return {"q": turn(s["xs"][0]), "k": turn(s["xs"][1]), "v": s["xs"][2].to(TYPES[c["y"]]).contiguous()}


def _plain_scores(s):
    """Scores fp32 [B, Hkv, G, T, T] under the rules, -inf where query i does not see key j."""
    c, q, k = s["case"], s["q"], s["k"]
    B, T, Hq, Hkv = c["batch"], c["tokens"], c["q_heads"], c["kv_heads"]
    x = q.float().reshape(B, Hkv, Hq // Hkv * T, D) @ k.float().transpose(-1, -2)
    x = x.view(B, Hkv, Hq // Hkv, T, T).mul_(SCALE)
    if c["cap"]:
        x.div_(c["cap"]).tanh_().mul_(c["cap"])
    i, j = torch.arange(T, device=DEV)[:, None], torch.arange(T, device=DEV)[None, :]
    if s["slopes"] is not None:
        x.sub_(s["slopes"].view(Hkv, Hq // Hkv, 1, 1) * (i - j).abs().float())
    seen = (j <= i).expand(B, T, T)
    if s["prefix"] is not None:
        seen = seen | (j < s["prefix"][:, None, None])
    if c["window"]:
        seen = seen & (j > i - c["window"])
    if s["documents"] is not None:
        ids = s["documents"]
        seen = seen & (ids[:, :, None] == ids[:, None, :]) & (ids >= 0)[:, :, None]
    return x.masked_fill_(~seen[:, None, None], -math.inf)


def _plain_attend(s):
    c = s["case"]
    B, T, Hq, Hkv = c["batch"], c["tokens"], c["q_heads"], c["kv_heads"]
    x = _plain_scores(s)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)  # a row that sees nothing
    x = x.sub_(m).exp_()
    l = x.sum(-1, keepdim=True)
    o = x.view(B, Hkv, Hq // Hkv * T, T) @ s["v"].float()
    o = (o.view(B, Hq, T, D) / torch.where(l == 0, 1.0, l).view(B, Hq, T, 1)).half()
    return {"out": o, "lse": (l.log() + m).view(B, Hq, T)}


def _plain_importance(s):
    c = s["case"]
    B, T, Hq, Hkv = c["batch"], c["tokens"], c["q_heads"], c["kv_heads"]
    lse = s["lse"].view(B, Hkv, Hq // Hkv, T, 1)
    x = _plain_scores(s).sub_(torch.where(lse == -math.inf, 0.0, lse)).exp_()
    return {"scores": x.sum((2, 3))}


def _plain_decode(s):
    c = s["case"]
    B, Hq, Hkv, L = c["batch"], c["q_heads"], c["kv_heads"], c["length"]
    G, group = Hq // Hkv, c["group"]

    def rows(r):
        if len(r) == 1:
            return r[0].float()
        code, a, b = r
        return (code.float().unflatten(-1, (D // group, group)) * a.float()[..., None] + b.float()[..., None]).flatten(-2)

    pools = [s["hi"], s["lo"]] if "lo" in s else [s["hi"]]
    pos = torch.cat([p[0] for p in pools], dim=2)
    k = torch.cat([rows(p[1]) for p in pools], dim=2)
    v = torch.cat([rows(p[2]) for p in pools], dim=2)
    x = s["q"].float().view(B, Hkv, G, D) @ k.transpose(-1, -2) * SCALE
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    if s["slopes"] is not None:
        x = x - s["slopes"].view(Hkv, G, 1) * (L - 1 - pos).float()[:, :, None]
    if s["begin"] is not None:
        x = x.masked_fill((pos < s["begin"][:, None, None])[:, :, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - m)
    l = e.sum(-1, keepdim=True)
    p = (e / l).view(B, Hq, -1)
    out = {"out": ((e @ v) / l).view(B, Hq, D), "probs_hi": p[..., :s["n"]].contiguous()}
    if "lo" in s:
        out["probs_lo"] = p[..., s["n"]:].contiguous()
    return out


def run(s):
    c = s["case"]
    kind = c["kind"]
    if not own:
        return {"rotary": _plain_rotary, "attend": _plain_attend, "importance": _plain_importance,
                "decode": _plain_decode}[kind](s)
    from paper_2402_18096_amd import mikv
    if kind == "rotary":
        mikv.mikv_rotary(s["rotary"], s["xs"], s["ys"], positions=s["positions"], rotate=(True, True, False))
        return {"q": s["ys"][0], "k": s["ys"][1], "v": s["ys"][2]}
    if kind == "decode":
        rules = mikv.ScoreRules(cap=c["cap"], slopes=s["slopes"], begin=s["begin"])
        mikv.mikv_decode_attention_scored(s["cache"], c["length"], s["q"], s["out"], s["probs_hi"], s["probs_lo"],
                                          rules=rules, scale=SCALE, workspace=s["ws"])
        out = {"out": s["out"], "probs_hi": s["probs_hi"]}
        if c["lo"]:
            out["probs_lo"] = s["probs_lo"][..., :c["length"] - s["n"]]
        return out
    if "begin" in s:
        mikv.mikv_mask_spans(s["begin"], s["end"], documents=s["documents"], prefix=s["prefix"], window=c["window"])
    rules = mikv.ScoreRules(cap=c["cap"], slopes=s["slopes"], begin=s.get("begin"), end=s.get("end"))
    if kind == "importance":
        mikv.mikv_prompt_importance(s["q"], s["k"], s["lse"], s["scores"], rules=rules, scale=SCALE, workspace=s["ws"])
        return {"scores": s["scores"]}
    mikv.mikv_prompt_attention(s["q"], s["k"], s["v"], s["out"], lse=s["lse"], rules=rules, scale=SCALE)
    return {"out": s["out"], "lse": s["lse"]}


# -- what a pass cannot do without ------------------------------------------------------------

def _pairs(c):
    """(query, key) pairs that see each other, per sequence and query head: documents as long as their mean."""
    T = c["tokens"]
    n = c["docs"] + 1 if c["docs"] else 1
    used = T * c["docs"] / n if c["pad"] else T
    t = T / n
    seen = t * (t + 1) / 2 if not c["window"] or c["window"] >= t else c["window"] * t - c["window"] * (c["window"] - 1) / 2
    if c["prefix"] and not c["docs"]:
        seen += (T / 4) * (T / 4) / 2
    return used / t * seen


def work(case):
    c = case
    B, Hq, Hkv = c["batch"], c["q_heads"], c["kv_heads"]
    size = lambda t: TYPES[t].itemsize  # noqa: E731
    if c["kind"] == "rotary":
        n = B * c["tokens"] * (Hq + 2 * Hkv) * D
        return {"bytes": n * (size(c["x"]) + size(c["y"])) + 4 * B * c["tokens"],
                "flops": 3 * B * c["tokens"] * (Hq + Hkv) * c["rot"]}
    if c["kind"] == "decode":
        def token(bits):
            return 0 if bits == 0 else 4 * D if bits == 16 else 2 * (D * bits // 8 + 4 * (D // c["group"]))
        L = c["length"]
        n = min(L, c["recent"] + L * c["num"] // c["den"])
        seen = L if c["lo"] else n
        share = 0.875 if c["begin"] else 1.0  # tokens before the first position have to be neither read nor multiplied
        kv = B * Hkv * share * (n * token(c["hi"]) + (L - n) * token(c["lo"]) + (4 * seen if c["bias"] or c["begin"] else 0))
        return {"bytes": kv + 4 * B * Hq * seen + 6 * B * Hq * D, "flops": 4 * D * B * Hq * seen * share}
    T, pairs = c["tokens"], _pairs(c)
    masks = 4 * B * T if c["docs"] else 0
    if c["kind"] == "importance":
        return {"bytes": 2 * D * B * T * (Hq + Hkv) + 4 * B * T * (Hq + Hkv) + masks, "flops": 2 * D * B * Hq * pairs}
    return {"bytes": 2 * D * B * T * (2 * Hq + 2 * Hkv) + 4 * B * Hq * T + masks, "flops": 4 * D * B * Hq * pairs}


# -- in 64 bits -------------------------------------------------------------------------------

def _exact_rotary(s):
    c = s["case"]
    r = c["rot"]
    theta = s["positions"].double()[..., None] * s["w"]
    z = torch.polar(torch.full_like(theta, s["m"]), theta)[:, None]  # [B, 1, T, r / 2]
    out = {}
    for name, x in zip("qkv", s["xs"]):
        y = x.double().contiguous()
        if name != "v":
            if c["interleaved"]:
                w = torch.view_as_complex(y[..., :r].unflatten(-1, (r // 2, 2)).contiguous()) * z
                y[..., :r] = torch.view_as_real(w).flatten(-2)
            else:
                w = torch.complex(y[..., :r // 2], y[..., r // 2:r]) * z
                y[..., :r // 2], y[..., r // 2:r] = w.real, w.imag
        out[name] = y
    return out


def _exact_prompt(s, seen_by_key):
    """Head by head: {"out", "lse"}, or with `seen_by_key` {"scores"} from the state's log-sum-exp."""
    c = s["case"]
    B, T, Hq, Hkv = c["batch"], c["tokens"], c["q_heads"], c["kv_heads"]
    G = Hq // Hkv
    i = torch.arange(T, device=DEV).view(T, 1)
    j = i.view(1, T)
    out = torch.zeros(B, Hq, T, D, dtype=torch.float64, device=DEV) if not seen_by_key else None
    lse = torch.full((B, Hq, T), -math.inf, dtype=torch.float64, device=DEV)
    scores = torch.zeros(B, Hkv, T, dtype=torch.float64, device=DEV)
    for b in range(B):
        last = i.expand(T, T)  # the last key that a query sees
        if s["prefix"] is not None:
            last = torch.maximum(last, s["prefix"][b].long() - 1)
        hidden = j > last
        if c["window"]:
            hidden = hidden | (i - j >= c["window"])
        if s["documents"] is not None:
            d = s["documents"][b]
            hidden = hidden | (d.view(T, 1) != d.view(1, T)) | (d.view(T, 1) < 0)
        some = ~hidden.all(1)
        for h in range(Hq):
            t = SCALE * (s["q"][b, h].double() @ s["k"][b, h // G].double().T.contiguous())
            if c["cap"]:
                t = torch.tanh(t / c["cap"]) * c["cap"]
            if s["slopes"] is not None:
                t = t - s["slopes"][h].double() * torch.abs(i - j)
            t[hidden] = -math.inf
            if seen_by_key:
                p = torch.exp(t[some] - s["lse"][b, h].double()[some].view(-1, 1))
                scores[b, h // G] += p.sum(0)
            else:
                z = torch.logsumexp(t[some], 1)
                lse[b, h, some] = z
                out[b, h, some] = torch.exp(t[some] - z.view(-1, 1)) @ s["v"][b, h // G].double()
    return {"scores": scores} if seen_by_key else {"out": out, "lse": lse}


def _exact_decode(s):
    c = s["case"]
    B, Hq, Hkv, L = c["batch"], c["q_heads"], c["kv_heads"], c["length"]
    G, n = Hq // Hkv, s["n"]
    pools = [p for p in ("hi", "lo") if p in s]
    out = torch.empty(B, Hq, D, dtype=torch.float64, device=DEV)
    probs = []

    def value(r, b, h):
        if len(r) == 1:
            return r[0][b, h].double()
        code, a, z = (x[b, h].double() for x in r)
        wide = lambda x: x.repeat_interleave(c["group"], dim=-1)  # noqa: E731
        return wide(a) * code + wide(z)

    for b in range(B):
        for h in range(Hkv):
            at = torch.cat([s[p][0][b, h] for p in pools])
            key, val = (torch.cat([value(s[p][w], b, h) for p in pools]) for w in (1, 2))
            t = SCALE * (key @ s["q"][b, h * G:(h + 1) * G].double().T.contiguous())  # [tokens, G]
            if c["cap"]:
                t = torch.tanh(t / c["cap"]) * c["cap"]
            if s["slopes"] is not None:
                t = t - (L - 1 - at).double()[:, None] * s["slopes"][h * G:(h + 1) * G].double()
            if s["begin"] is not None:
                t[at < s["begin"][b]] = -math.inf
            p = torch.softmax(t, 0).T
            out[b, h * G:(h + 1) * G] = p @ val
            probs.append(p)
    probs = torch.stack(probs).view(B, Hq, -1)
    r = {"out": out, "probs_hi": probs[..., :n].contiguous()}
    if "lo" in s:
        r["probs_lo"] = probs[..., n:].contiguous()
    return r


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rotary":
        return _exact_rotary(s)
    if case["kind"] == "decode":
        return _exact_decode(s)
    return _exact_prompt(s, case["kind"] == "importance")
